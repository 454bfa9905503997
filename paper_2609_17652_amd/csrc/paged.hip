// fathom_paged_map and fathom_paged_write: block tables, slot maps and the new
// rows of a paged cache.
//
// Map.  All that a request needs of the others are three prefix sums over the
// requests: of its new rows, of the pages it takes and of those it returns.  A
// workgroup computes them in registers (up to 4 requests a thread, wave scans
// joined through LDS) and keeps them in LDS, where every slot and every moved
// page finds its request by binary search; so slots and pages are spread over
// threads evenly however uneven the requests are.  The ring is read at its front
// and written behind its end, the table's read and written entries are disjoint,
// so nothing waits for anything.  A small call is one workgroup and one launch;
// a large one spreads slots and pages over workgroups that each recompute the
// sums (16 bytes a request from L2); the first of them writes lengths and state, or, where
// the caller's are in place and the others still read them, a second launch does.  Bound by
// latency: launch, lengths, sums, then a search and two trips to memory a slot; 64 requests' one
// token 4.4 us, 450000 slots of 512 requests 15.9 (two launches and slots one request after
// another: 13 and 23; pages moved by the threads that have slots: 18).
//
// Write.  A copy of rows: 16 lanes take a row's 256 bytes of output, the row's
// slot gives the page.  Bound by bytes where they are many (139315 tokens of 8 heads, fp32 to
// bf16, 1.7 GB: 0.33 ms, 5.2 TB/s) and by one trip to memory after another (slot and row, store)
// where they are few.
#include "paged.hpp"

namespace fathom {

// Threads of a workgroup and requests of a thread: up to 256 requests of a small call 256 and 1
// (its 4 waves meet sooner), up to 1024 requests 1024 and 1, up to the limit 1024 and 4.
constexpr int kMapThreads = 1024;
constexpr int kMapFew = 256;
static_assert(kMaxSeqs % kMapThreads == 0, "requests divide over the threads");

struct MapArgs {
  const int64_t *n_old, *n;
  int S, H, shift;
  int32_t* table;
  int64_t ld_table;
  int32_t* ring;
  int64_t P;
  const int64_t* state;
  int64_t* slots;
  int64_t T;
  int64_t *start, *n_now, *n_unit, *state_out;
  uint32_t* st;
};

// Inclusive sums of three values over the workgroup (each thread's own sum given).
template <int THREADS>
__device__ __forceinline__ void block_scan3(int64_t (&v)[3], int64_t (&part)[3][THREADS / kWave]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t x = __shfl_up(v[i], o, kWave);
      if (lane >= o) v[i] += x;
    }
    if (lane == 63) part[i][wave] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    int64_t before = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) before += w < wave ? part[i][w] : 0;
    v[i] += before;
  }
}

// The last of `count` non-decreasing entries that is at most x (the first is).
__device__ __forceinline__ int last_at_most(const int32_t* a, int count, int32_t x) {
  int lo = 0, len = count;
  while (len > 1) {
    const int half = len >> 1;
    if (a[lo + half] <= x) {
      lo += half;
      len -= half;
    } else {
      len = half;
    }
  }
  return lo;
}

__device__ __forceinline__ int32_t clip31(int64_t x) { return (int32_t)(x < 0x7fffffff ? x : 0x7fffffff); }

// FILL: slots, table and ring.  FINISH: start, lengths and state, after every read.
template <int THREADS, int kPer, bool FILL, bool FINISH>
__global__ __launch_bounds__(THREADS) void paged_map_kernel(MapArgs a) {
  extern __shared__ int32_t sm[];
  __shared__ int64_t part[3][THREADS / kWave];
  __shared__ int64_t tot[4];  // rows, pages returned; pages taken by those served
  const int S = a.S, tid = threadIdx.x;
  int32_t* s_start = sm;        // [S] first new row
  int32_t* s_taken = sm + S;    // [S] pages taken before
  int32_t* s_back = sm + 2 * S; // [S] pages returned before
  int32_t* s_old = sm + 3 * S;  // [S] old length; ~old where the request is not served
  int32_t* s_after = sm + 4 * S;  // [S] pages after
  const int64_t cap = a.ld_table << a.shift, rnd = (1 << a.shift) - 1;
  int64_t head = a.state[0], count = a.state[1];
  uint32_t flags = 0;
  const bool bad_state = head < 0 || head >= a.P || count < 0 || count > a.P;
  if (bad_state) {
    flags |= FATHOM_DEV_BAD_PAGE;
    count = 0;
  }
  if (tid == 0) tot[2] = 0;
  int64_t no[kPer], nn[kPer], sum[3] = {0, 0, 0};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = tid * kPer + i;
    no[i] = s < S ? a.n_old[s] : 0;
    nn[i] = s < S ? a.n[s] : 0;
  }
  int64_t add[kPer][3];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool ok = no[i] >= 0 && no[i] <= cap && nn[i] >= 0 && nn[i] <= cap;
    const int64_t before = (no[i] + rnd) >> a.shift, after = (nn[i] + rnd) >> a.shift;
    add[i][0] = ok && nn[i] > no[i] ? nn[i] - no[i] : 0;
    add[i][1] = ok && after > before ? after - before : 0;
    add[i][2] = ok && before > after ? before - after : 0;
#pragma unroll
    for (int x = 0; x < 3; ++x) sum[x] += add[i][x];
  }
  int64_t inc[3] = {sum[0], sum[1], sum[2]};
  block_scan3<THREADS>(inc, part);
  if (tid == THREADS - 1) {
    tot[0] = inc[0];
    tot[1] = inc[2];
  }
  int64_t at[3] = {inc[0] - sum[0], inc[1] - sum[1], inc[2] - sum[2]}, mine = 0;
  int64_t first[kPer];
  bool served[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int s = tid * kPer + i;
    const bool ok_old = no[i] >= 0 && no[i] <= cap, ok = ok_old && nn[i] >= 0 && nn[i] <= cap;
    first[i] = at[0];
    const bool fits = add[i][0] == 0 || at[0] + add[i][0] <= a.T, pages = add[i][1] == 0 || at[1] + add[i][1] <= count;
    served[i] = ok && fits && pages;
    if (s < S) {
      if (!ok || !fits) flags |= FATHOM_DEV_BAD_N;
      else if (!pages) flags |= FATHOM_DEV_PAGES_SHORT;
      s_start[s] = clip31(at[0]);
      s_taken[s] = clip31(at[1]);
      s_back[s] = clip31(at[2]);
      s_old[s] = served[i] ? (int32_t)no[i] : -1;
      s_after[s] = ok ? (int32_t)((nn[i] + rnd) >> a.shift) : 0;
      if (served[i]) mine += add[i][1];
    }
    if (!ok_old) no[i] = 0;
#pragma unroll
    for (int x = 0; x < 3; ++x) at[x] += add[i][x];
  }
  __syncthreads();
  if (mine) atomicAdd((unsigned long long*)&tot[2], (unsigned long long)mine);  // whole numbers: any order
  __syncthreads();
  const int64_t taken = tot[2], rows = tot[0];
  int64_t back = tot[1];
  if (bad_state) back = 0;
  if (count + back > a.P) {
    flags |= FATHOM_DEV_BAD_PAGE;
    back = 0;
  }
  if constexpr (FILL) {
    const int64_t gt = (int64_t)blockIdx.x * THREADS + tid, step = (int64_t)gridDim.x * THREADS;
#pragma unroll 4
    for (int64_t t = gt; t < a.T; t += step) {
      int64_t slot = -1;
      if (t < rows) {
        const int s = last_at_most(s_start, S, (int32_t)t);
        const int32_t old = s_old[s];
        if (old >= 0) {
          const int32_t p = old + (int32_t)(t - s_start[s]), before = (int32_t)(((int64_t)old + rnd) >> a.shift);
          const int32_t e = p >> a.shift;
          int32_t id;
          if (e >= before) {
            int64_t r = head + s_taken[s] + (e - before);
            if (r >= a.P) r -= a.P;
            id = a.ring[r];
          } else {
            id = a.table[(int64_t)s * a.ld_table + e];
          }
          if (id >= 0 && id < a.P) slot = ((int64_t)id << a.shift) + (p & rnd);
          else flags |= FATHOM_DEV_BAD_PAGE;
        }
      }
      a.slots[t] = slot;
    }
    // pages that move, from the other end: the last threads have no slot
#pragma unroll 2
    for (int64_t m = step - 1 - gt; m < taken + back; m += step) {
      const bool take = m < taken;
      const int64_t j = take ? m : m - taken;
      const int s = last_at_most(take ? s_taken : s_back, S, (int32_t)j);
      int64_t r = head + (take ? j : count + j);
      while (r >= a.P) r -= a.P;
      int32_t *ring = a.ring + r, *entry = a.table + (int64_t)s * a.ld_table;
      if (take) entry += (((int64_t)s_old[s] + rnd) >> a.shift) + (j - s_taken[s]);
      else entry += s_after[s] + (j - s_back[s]);
      const int32_t id = *(take ? ring : entry);
      if (id < 0 || id >= a.P) flags |= FATHOM_DEV_BAD_PAGE;
      *(take ? entry : ring) = id;
    }
  }
  if constexpr (FINISH) {
    if (blockIdx.x == 0) {
      __syncthreads();  // s_back is done with: it takes the lengths, for stores in order
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int s = tid * kPer + i;
        if (s >= S) break;
        const int64_t now = served[i] ? nn[i] : no[i];
        a.start[s] = first[i];
        a.n_now[s] = now;
        s_back[s] = (int32_t)now;
      }
      if (tid == 0) {
        a.start[S] = rows;
        const int64_t h1 = head + taken;
        const int64_t c0 = bad_state ? a.state[1] : count - taken + back;
        a.state_out[0] = bad_state ? head : h1 >= a.P ? h1 - a.P : h1;
        a.state_out[1] = c0;
      }
      if (a.n_unit) {
        __syncthreads();
        for (int u = tid; u < S * a.H; u += THREADS) a.n_unit[u] = s_back[(uint32_t)u / (uint32_t)a.H];
      }
    }
  }
  if (flags) set_status(a.st, flags);
}

// Lengths and state with the slots, or (in place, several workgroups) in a launch of their own.
template <int THREADS, int PER>
static void launch_map(const MapArgs& a, int64_t wgs, bool apart, hipStream_t s) {
  const size_t lds = (size_t)5 * a.S * sizeof(int32_t);
  const dim3 grid((unsigned)(wgs < 1 ? 1 : wgs < 512 ? wgs : 512)), threads(THREADS);
  if (apart || wgs <= 1) {
    hipLaunchKernelGGL((paged_map_kernel<THREADS, PER, true, true>), grid, threads, lds, s, a);
  } else {
    hipLaunchKernelGGL((paged_map_kernel<THREADS, PER, true, false>), grid, threads, lds, s, a);
    hipLaunchKernelGGL((paged_map_kernel<THREADS, PER, false, true>), dim3(1), threads, lds, s, a);
  }
}

fathom_status launch_paged_map(const int64_t* n_old, const int64_t* n, int S, int H, int shift, int32_t* table,
                               int64_t ld_table, int32_t* ring, int64_t P, const int64_t* state, int64_t* slots,
                               int64_t T, int64_t* start, int64_t* n_now, int64_t* n_unit, int64_t* state_out,
                               uint32_t* st, hipStream_t s) {
  const MapArgs a = {n_old, n,     S, H,     shift, table, ld_table, ring, P,
                     state, slots, T, start, n_now, n_unit, state_out, st};
  // A step that moves few tokens is one small workgroup (launch after launch: 64 requests' one
  // token 4.8 us, 6.7 in a large one; 462 tokens 6.7 and 7.2; 538 8.7 and 7.9); else a slot a thread, over two
  // workgroups a CU at most, all writing what they find (1811 tokens 7.5 us, 13.6 in one
  // workgroup).  (Pages taken are bounded by the new tokens; pages that come back are not, but a
  // workgroup moves 1000 in about a microsecond.)
  const bool apart = n_now != n_old && n_now != n && state_out != state;
  // in place: one workgroup, or a launch of its own for lengths and state (about 4 us); else a
  // quarter more than the slots need, which has the pages that move
  const int64_t wgs = !apart && T <= 2 * kMapThreads ? 1 : (T + T / 4 + kMapThreads - 1) / kMapThreads;
  if (T <= 2 * kMapFew && S <= kMapFew) launch_map<kMapFew, 1>(a, 1, apart, s);
  else if (S <= kMapThreads) launch_map<kMapThreads, 1>(a, wgs, apart, s);
  else launch_map<kMapThreads, kMaxSeqs / kMapThreads>(a, wgs, apart, s);
  FATHOM_LAUNCH_CHECK();
  return FATHOM_OK;
}

// ---------------------------------------------------------------- write
constexpr int kWriteThreads = 256;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct WriteArgs {
  const void *K, *V;
  int64_t ldk_tok, ldk_head, ldv_tok, ldv_head;
  const int64_t* slots;
  uint32_t rows;  // T*H
  uint16_t *Kp, *Vp;
  int H, shift;
  int64_t cap;  // slots of the pool
  int64_t ld_page, ld_head, ld_tok;
  uint32_t* st;
};

__device__ __forceinline__ uint32_t pack_pair(float a, float b, bool bf) {
  if (bf) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const b2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  const h2 v = {(_Float16)a, (_Float16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// F32: fp32 rows, rounded; otherwise a copy.  A row per 16 lanes (four, their loads in flight at
// once, are slower at every size: 512 rows 3.6 us against 2.8, 524288 rows 107 against 101).
template <bool F32, bool BF>
__global__ __launch_bounds__(kWriteThreads) void paged_write_kernel(WriteArgs a) {
  const int x = threadIdx.x & 15, g = threadIdx.x >> 4;
  const bool v_side = blockIdx.y != 0;
  const void* src = v_side ? a.V : a.K;
  uint16_t* dst = v_side ? a.Vp : a.Kp;
  const int64_t ls_tok = v_side ? a.ldv_tok : a.ldk_tok, ls_head = v_side ? a.ldv_head : a.ldk_head;
  const uint32_t r = (blockIdx.z * gridDim.x + blockIdx.x) * (uint32_t)(kWriteThreads / 16) + g;
  if (r >= a.rows) return;
  const uint32_t t = r / (uint32_t)a.H, h = r - t * (uint32_t)a.H;
  const int64_t slot = a.slots[t], o = (int64_t)t * ls_tok + (int64_t)h * ls_head + 8 * x;
  u32x4 v;
  if constexpr (F32) {
    const u32x4* p = reinterpret_cast<const u32x4*>(reinterpret_cast<const float*>(src) + o);
    const u32x4 lo = p[0], hi = p[1];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      v[e] = pack_pair(__uint_as_float(lo[2 * e]), __uint_as_float(lo[2 * e + 1]), BF);
      v[2 + e] = pack_pair(__uint_as_float(hi[2 * e]), __uint_as_float(hi[2 * e + 1]), BF);
    }
  } else {
    v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(src) + o);
  }
  if (slot < 0) return;
  if (slot >= a.cap) {
    if (x == 0) set_status(a.st, FATHOM_DEV_BAD_PAGE);
    return;
  }
  *reinterpret_cast<u32x4*>(dst + (slot >> a.shift) * a.ld_page + (int64_t)h * a.ld_head +
                            (slot & ((1 << a.shift) - 1)) * a.ld_tok + 8 * x) = v;
}

fathom_status launch_paged_write(const void* K, const void* V, fathom_dtype sdt, int64_t ldk_tok, int64_t ldk_head,
                                 int64_t ldv_tok, int64_t ldv_head, const int64_t* slots, int64_t T,
                                 const fathom_pages& p, uint32_t* st, hipStream_t s) {
  const int shift = __builtin_ctz((unsigned)p.page);
  const WriteArgs a = {K, V, ldk_tok, ldk_head, ldv_tok, ldv_head, slots, (uint32_t)(T * p.H),
                       reinterpret_cast<uint16_t*>(p.K), reinterpret_cast<uint16_t*>(p.V), p.H, shift, p.P << shift,
                       p.ld_page, p.ld_head, p.ld_tok, st};
  // an axis of a grid has fewer than 2^32 threads: beyond 2^22 groups of rows a second one goes on
  const uint32_t groups = (a.rows + kWriteThreads / 16 - 1) / (kWriteThreads / 16), wide = 1u << 22;
  const uint32_t deep = (groups + wide - 1) / wide;
  const dim3 grid(deep > 1 ? wide : groups, 2, deep), threads(kWriteThreads);
  if (sdt != FATHOM_F32) hipLaunchKernelGGL((paged_write_kernel<false, false>), grid, threads, 0, s, a);
  else if (p.dt == FATHOM_BF16) hipLaunchKernelGGL((paged_write_kernel<true, true>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((paged_write_kernel<true, false>), grid, threads, 0, s, a);
  FATHOM_LAUNCH_CHECK();
  return FATHOM_OK;
}

}  // namespace fathom
