// fathom_paged_attn: dense attention of new tokens over a paged cache.
//
// The query rows of a (request, KV head) are its new tokens' G heads, row r =
// token*G + g, so the G heads share every K and V row that is loaded.  Scores are
// computed transposed, S^T = K Q^T: an accumulator lane then holds scores of ONE
// query row, so the softmax of a row needs one exchange between lane groups, and
// the lane's probabilities are already the B operand of O^T = V^T P^T, with the
// keys of a 16-key step in the order that the accumulator holds them; V^T is
// read from row-major LDS rows by transposing loads in the same key order.  The
// running maximum and sum and both products are fp32.
//
// K and V rows go from the pages to LDS without registers, 1 KB (4 rows) an
// instruction; 16 rows from a multiple of 16 lie in one page, so a page number is
// uniform and comes over the scalar path.  LDS rows are 256 bytes (every bank
// once); 16-byte chunks are permuted by the row so that the 16 rows of a K
// fragment (chunk ^ row) and the 4 rows of a V read (chunk ^ 4 row) spread over
// the banks.
//
// Two kernels.  attn_few_kernel takes requests of at most 32 query rows (decode,
// drafted tokens): bound by reading the cache, so the 32-key blocks of all
// requests and heads are cut into equal shares, one per wave, whatever the
// lengths are; each wave runs its share through two private LDS stages without
// meeting the others, and pieces of a request join in attn_join_kernel.
// attn_many_kernel takes the others, and a request that is the only one of a call whose bounds
// allow more rows, 128 query rows a workgroup, bound by issue and power; keys are
// split over workgroups where the tiles are few.
//
// Rows that a query must not see get a probability of 0, but 0 * Inf is not 0:
// V rows behind the end are cleared in LDS, and in steps with masked places
// the non-finite values of V are taken out of the product and added for the rows
// that see them.  Elsewhere they go into the product as they are: they change their own
// channel only, which is made up anew at the end of a piece or tile where it is not finite
// (nothing in the loops, 0.3 us a call where latency counts; with one such value 2048 tokens
// over 65536 take 9.0 ms instead of 2.3, 32 ragged single tokens 1.2 instead of 0.6).
#include <type_traits>

#include "paged.hpp"

namespace fathom {

#define LDS_PTR(T) __attribute__((address_space(3))) T*
// 32-bit LDS offsets as pointers
#define LDS_AT(T, at) ((LDS_PTR(T))(uintptr_t)(at))
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowBytes = 2 * kD;
constexpr int kFewRows = 32;      // query rows of a request and head that attn_few_kernel takes
constexpr int kFewKeys = 32;      // keys a step of a wave
constexpr int kFewWaves = 4;
constexpr int kFewWorkers = 1024; // waves: one workgroup of 128 KB of LDS on each of 256 CUs
constexpr int kFewStage = 2 * kFewKeys * kRowBytes;
constexpr int kManyRows = 128;    // attn_many_kernel: query rows of a workgroup, 32 a wave
constexpr int kBlock = 32;        // keys of a block
constexpr int kBlockBytes = kBlock * kRowBytes;
constexpr int kManyStages = 4;    // blocks in each of the rings of K and V
constexpr int kManyLds = 2 * kManyStages * kBlockBytes;
constexpr int kManyKeys = 64;     // keys are divided among workgroups by these

struct TileRecord;
struct PagedAttnArgs {
  const uint16_t* q;
  int64_t ldq_tok, ldq_head;
  Paged c;
  const int64_t *start, *n;
  int S, G, few;        // few: query rows up to which a request goes to attn_few_kernel
  int64_t T, max_new;
  float sm_scale, softcap;
  const float* slopes;
  const int64_t *prefix, *first;
  uint16_t* out;
  float *part_o, *part_ml;  // partial results: rows of kD sums, and (maximum, sum) of each
  int nsplit, part_units;   // attn_many_kernel: parts of a tile's keys at most, units of 64 keys of a part at least
  bool all_parts;           // as many as there may be, or one
  TileRecord* tiles;        // its tiles, of more than 64 requests
  int64_t ntiles;
  uint32_t* st;
};

// What no kernel of a call writes, over the scalar path where the index is uniform (a
// vector load in the loop would wait for every load in flight).
template <typename T>
__device__ __forceinline__ T fixed(const T* p, int64_t i) {
  return ((const __attribute__((address_space(4))) T*)p)[i];
}
__device__ __forceinline__ int page_uniform(const Paged& c, int s, int e) {
  return fixed(c.table + (int64_t)s * c.ld_table, e);
}

// New tokens of request s, their first row in *a and its tokens in *n; 0 (with
// BAD_N) where the lengths do not fit together.
__device__ __forceinline__ int request_rows(const PagedAttnArgs& p, int s, int64_t* a, int64_t* n, uint32_t& flags) {
  const int64_t b = fixed(p.start, s), e = fixed(p.start, s + 1), m = fixed(p.n, s);
  *a = b;
  *n = m;
  const bool ok = b >= 0 && e >= b && e <= p.T && m >= 0 && m <= (p.c.ld_table << p.c.shift) && e - b <= m &&
                  e - b <= p.max_new;
  if (!ok) {
    flags |= FATHOM_DEV_BAD_N;
    return 0;
  }
  return (int)(e - b);
}

// What a query token sees: [lo, hi).
__device__ __forceinline__ void token_range(const PagedAttnArgs& p, int s, int64_t row, int pos, int n, int* lo,
                                            int* hi) {
  *lo = 0;
  *hi = pos + 1;
  if (p.prefix) {
    const int64_t v = fixed(p.prefix, s), x = v < n ? v : n;
    if (x > *hi) *hi = (int)x;
  }
  if (p.first) {
    const int64_t x = p.first[row];
    *lo = x < 0 ? 0 : x > n ? n : (int)x;
  }
}

// ---------------------------------------------------------------- tools
// Rows, four of 64 lanes x 16 bytes at a time, 2 or 4 times: rows 4y .. 4y + 3 from base +
// 1024 y + off[y] (a lane's) to LDS at `lds` + 1024 y + 16 lane; an instruction's offset counts
// on both sides.  The wait is the caller's (vmcnt); no register is written.
template <int N>
__device__ __forceinline__ void load_to_lds(uint32_t lds, const void* from, const uint32_t (&off)[N]) {
  const uint64_t at = reinterpret_cast<uint64_t>(from);
  const uint64_t base = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32) |
                        (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
  lds = __builtin_amdgcn_readfirstlane((int)lds);
  if constexpr (N == 4) {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:1024\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:3*1024" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base)
        : "memory");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(lds),
        "v"(off[0]), "v"(off[1]), "s"(base)
        : "memory");
  }
}

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 16-byte chunk of an LDS row of K or V where the row's chunk `c` is kept.
__device__ __forceinline__ int k_chunk(int row, int c) { return c ^ (row & 15); }
__device__ __forceinline__ int v_chunk(int row, int c) { return c ^ ((row & 3) << 2); }

template <bool BF>
struct Mx;
template <>
struct Mx<false> {
  typedef f16x8 v8;
  typedef _Float16 v2 __attribute__((ext_vector_type(2)));
  typedef _Float16 t;
  static constexpr uint16_t kInf = 0x7C00, kOne = 0x3C00;
  static constexpr float kShift = 8.0f;  // probabilities are kept times 2^8: no subnormals down to 2^-22
  static __device__ __forceinline__ f32x4 mfma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  // sum + a[0] + a[1], in 32 bits
  static __device__ __forceinline__ float add_pair(v2 a, float sum) {
    const v2 one = {(_Float16)1.0f, (_Float16)1.0f};
    return __builtin_amdgcn_fdot2(a, one, sum, false);
  }
  static __device__ __forceinline__ float add_zeros(v2 a, float sum) {
    const v2 zero = {(_Float16)0.0f, (_Float16)0.0f};
    return __builtin_amdgcn_fdot2(a, zero, sum, false);
  }
};
template <>
struct Mx<true> {
  typedef bf16x8 v8;
  typedef __bf16 v2 __attribute__((ext_vector_type(2)));
  typedef __bf16 t;
  static constexpr uint16_t kInf = 0x7F80, kOne = 0x3F80;
  static constexpr float kShift = 0.0f;
  static __device__ __forceinline__ f32x4 mfma16(v8 a, v8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(v8 a, v8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float add_pair(v2 a, float sum) {
    const v2 one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(a, one, sum, false);
  }
  static __device__ __forceinline__ float add_zeros(v2 a, float sum) {
    const v2 zero = {(__bf16)0.0f, (__bf16)0.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(a, zero, sum, false);
  }
};

// f(integral_constant<int, i>) for i = A .. B - 1: indices known to the compiler whatever a loop's size
template <int A, int B, class Fn>
__device__ __forceinline__ void static_for(Fn f) {
  if constexpr (A < B) {
    f(std::integral_constant<int, A>());
    static_for<A + 1, B>(f);
  }
}

template <class V8>
__device__ __forceinline__ V8 lds_v8(uint32_t at) {
  return *LDS_AT(const V8, at);
}
// Four rows' values of a lane's channel: rows and channels as the callers' lanes give them.
__device__ __forceinline__ s16x4 lds_tr(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_AT(s16x4, at));
}
template <class V8>
__device__ __forceinline__ V8 join4(s16x4 a, s16x4 b) {
  return __builtin_bit_cast(V8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Whether BYTES (a multiple of 1024) of V, from `mine` - 16 lane on, hold a value that is not
// finite; uniform.
// (Zero times such a value is no zero: a sum of products with zeros shows it.)
template <bool BF, int BYTES>
__device__ __forceinline__ bool any_nonfinite(uint32_t mine) {
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < BYTES; i += 1024) {
    const u32x4 w = *LDS_AT(const u32x4, mine + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = Mx<BF>::add_zeros(__builtin_bit_cast(typename Mx<BF>::v2, (uint32_t)w[e]), sum[e]);
  }
  return __ballot((sum[0] + sum[1]) + (sum[2] + sum[3]) != 0.0f) != 0;  // NaN
}

// Such values leave the product, and are added (as they are: Inf and NaN do what the sum
// would) to the four sums of a lane's channels where its query sees their key.
template <bool BF>
__device__ __forceinline__ bool nonfinite_bits(short x) {
  return ((uint16_t)x & Mx<BF>::kInf) == Mx<BF>::kInf;
}
template <bool BF>
__device__ __forceinline__ s16x8 finite_part(s16x8 v) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (nonfinite_bits<BF>(v[e])) v[e] = 0;
  return v;
}
template <bool BF>
__device__ __forceinline__ float nonfinite_part(short x) {
  return nonfinite_bits<BF>(x) ? (float)__builtin_bit_cast(typename Mx<BF>::t, x) : 0.0f;
}

// A channel of O that a value which is not finite came into may be NaN where the sum is
// infinite: probabilities below 2^-149 (of 16 bits, below their last place) are 0, and 0 * Inf is
// NaN, as is Inf - Inf where a probability is a sum of two values.  Such channels are made up
// anew, from the rows of V that hold such values: what follows finds them among keys [k0, k1), k0 a
// multiple of 16, in the pages, 16 at a time, and visits each.  A wave by itself.
template <bool BF, class Fn>
__device__ __forceinline__ void nonfinite_rows(const PagedAttnArgs& p, int s, int h, int k0, int k1, Fn visit) {
  const int lane = threadIdx.x & 63, quad = lane >> 4;
#pragma unroll 1
  for (int k = k0; k < k1; k += 16) {
    const int id = page_uniform(p.c, s, k >> p.c.shift);
    if ((uint32_t)id >= (uint32_t)p.c.P) continue;
    const uint16_t* row0 = p.c.V + (int64_t)id * p.c.ld_page + (int64_t)h * p.c.ld_head +
                           (int64_t)(k & ((1 << p.c.shift) - 1)) * p.c.ld_tok;
    s16x8 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * i + quad;
      v[i] = (s16x8){};
      if (k + row < k1) v[i] = *reinterpret_cast<const s16x8*>(row0 + row * p.c.ld_tok + 8 * (lane & 15));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) bad |= nonfinite_bits<BF>(v[i][e]);
      const uint64_t lanes = __ballot(bad);
#pragma unroll 1
      for (int j = 0; j < 4; ++j)
        if (lanes >> (16 * j) & 0xFFFF) visit(k + 4 * i + j, row0 + (4 * i + j) * p.c.ld_tok);
    }
  }
}
// Element `bit` of a lane's part of O with a seen value x: the first that is not finite takes the
// place of what is there, the others are added.
template <bool BF>
__device__ __forceinline__ float with_nonfinite(float o, short x, uint64_t& found, int bit) {
  if (!nonfinite_bits<BF>(x)) return o;
  const float y = nonfinite_part<BF>(x);
  const bool more = found >> bit & 1;
  found |= 1ull << bit;
  return more ? o + y : y;
}
// Four channels of the sum of a row's parts at(c), c = first, first + step .. below count (-1: not
// there), against the maximum M; where `o`, that sum, is not finite the parts are added again,
// and what is not finite in a part is kept where its weight is 0.
template <class At>
__device__ __forceinline__ f32x4 parts_sum(const PagedAttnArgs& p, f32x4 o, int first, int step, int count, float M,
                                           At at) {
  const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f}, z = o * zero;
  if ((z[0] + z[1]) + (z[2] + z[3]) == 0.0f) return o;
  o = zero;
#pragma unroll 1
  for (int c = first; c < count; c += step) {
    const int64_t row = at(c);
    if (row < 0 || p.part_ml[2 * row] == -__builtin_huge_valf()) continue;
    const float w = __builtin_amdgcn_exp2f(p.part_ml[2 * row] - M);
    const f32x4 v = *reinterpret_cast<const f32x4*>(p.part_o + row * kD + 4 * (threadIdx.x & 31));
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += w == 0.0f && v[e] - v[e] != 0.0f ? v[e] : w * v[e];
  }
  return o;
}

// z in units of log2: the scaled score, capped, less the distance's bias.
struct ScoreMap {
  float c1;   // sm_scale log2e, or 2 log2e sm_scale / softcap
  float cap;  // softcap log2e, 0: none
};
template <bool CAP>
__device__ __forceinline__ float mapped(const ScoreMap& m, float slope, float s, int dist) {
  float z = s * m.c1;
  if constexpr (CAP) {  // tanh x = 1 - 2 / (e^2x + 1)
    const float t = __builtin_amdgcn_exp2f(z);
    z = __builtin_fmaf(__builtin_amdgcn_rcpf(t + 1.0f), -2.0f * m.cap, m.cap);
  }
  return __builtin_fmaf(-slope, fabsf((float)dist), z);  // the row's slope times log2e
}
__device__ __forceinline__ ScoreMap score_map(const PagedAttnArgs& p) {
  ScoreMap m;
  const float c1 = p.softcap > 0.0f ? 2.0f * kLog2e * (p.sm_scale / p.softcap) : p.sm_scale * kLog2e;
  m.c1 = fminf(fmaxf(c1, -3.4e38f), 3.4e38f);  // a score of 0 stays 0
  m.cap = p.softcap > 0.0f ? p.softcap * kLog2e : 0.0f;
  return m;
}

// The first and last of the keys that any new token of a request may see, as [lo, n)
// with lo a multiple of 32 (few tokens: attn_few_kernel).
__device__ __forceinline__ int few_lo(const PagedAttnArgs& p, int64_t a, int rows, int64_t n) {
  if (!p.first) return 0;
  int64_t lo = n;
  for (int i = 0; i < rows; ++i) {
    const int64_t x = p.first[a + i];
    lo = x < lo ? x : lo;
  }
  lo = lo < 0 ? 0 : lo;
  return (int)(lo & ~(int64_t)(kFewKeys - 1));
}

__device__ __forceinline__ int few_blocks(const PagedAttnArgs& p, int s, uint32_t& flags) {
  int64_t a, n;
  const int rows = request_rows(p, s, &a, &n, flags);
  if (rows == 0 || rows * p.G > p.few) return 0;  // else one block at least, for rows that see nothing
  return max(((int)n - few_lo(p, a, rows, n) + kFewKeys - 1) / kFewKeys, 1);
}
__device__ __forceinline__ int scan_add(int v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(v, o, kWave);
    if ((int)(threadIdx.x & 63) >= o) v += x;
  }
  return v;
}
// before[s] = the sum of count(r) over r < s, s <= S; every thread, `part` one entry a wave.
template <class Fn>
__device__ __forceinline__ void sums_before(int S, int* before, int* part, Fn count) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 63, wave = tid >> 6, per = (S + nt - 1) / nt;
  for (int s = tid; s < S; s += nt) before[s] = count(s);
  __syncthreads();
  int sum = 0;
  for (int s = tid * per; s < min((tid + 1) * per, S); ++s) sum += before[s];
  const int inc = scan_add(sum);
  if (lane == 63) part[wave] = inc;
  __syncthreads();
  int base = inc - sum;
  for (int w = 0; w < wave; ++w) base += part[w];
  for (int s = tid * per; s < min((tid + 1) * per, S); ++s) {
    const int x = before[s];
    before[s] = base;
    base += x;
  }
  if (tid == nt - 1) before[S] = base;
  __syncthreads();
}
// Blocks of 32 keys of the requests: before[s] those of the requests before s (of one
// head), before[S] all.  Every thread of the workgroup.  Up to 64 requests every wave writes
// the same by itself, a lane a request, without a barrier.
__device__ __forceinline__ void few_plan(const PagedAttnArgs& p, int* before, int* part, uint32_t& flags) {
  const int lane = threadIdx.x & 63;
  if (p.S <= kWave) {
    const int nb = lane < p.S ? few_blocks(p, lane, flags) : 0, inc = scan_add(nb);
    if (lane < p.S) before[lane] = inc - nb;
    if (lane == kWave - 1) before[p.S] = inc;
    return;
  }
  sums_before(p.S, before, part, [&](int s) { return few_blocks(p, s, flags); });
}

// The last s with before[s] <= x (x < before[S]): the request of block x.
__device__ __forceinline__ int request_of(const int* before, int S, int x) {
  int lo = 0, len = S;
  while (len > 1) {
    const int half = len >> 1;
    const bool up = before[lo + half] <= x;
    lo += up ? half : 0;
    len = up ? len - half : half;
  }
  return lo;
}

// a / b of non-negative values (a 64-bit division takes some 150 instructions)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// Share of worker w: blocks [share(w), share(w + 1)) of W.
__device__ __forceinline__ int64_t share(int64_t w, int64_t W) { return (int64_t)((uint64_t)(w * W) / kFewWorkers); }
__device__ __forceinline__ int worker_of(int64_t g, int64_t W) {
  return (int)quotient((g + 1) * kFewWorkers - 1, W);
}

// A wave's place in the blocks of all requests and heads.
struct Place {
  int s, h, b, nb, lo, n;  // request, head, block of nb, the request's first key and tokens
};

template <bool BF, int CT>
__global__ __launch_bounds__(kFewWaves * kWave, 1) void attn_few_kernel(PagedAttnArgs p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef typename Mx<BF>::v8 v8;
  constexpr int R = 16 * CT;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  int* before = reinterpret_cast<int*>(smem + kFewWaves * 2 * kFewStage);
  int* part = before + p.S + 1;
  uint32_t flags = 0;
  few_plan(p, before, part, flags);
  if (flags && blockIdx.x == 0) set_status(p.st, flags);
  flags = 0;
  const int S = p.S, H = p.c.H, G = p.G;
  const bool capped = p.softcap > 0.0f;
  const ScoreMap sm = score_map(p);
  const int64_t W = (int64_t)before[S] * H;
  const int worker = uniform((int)blockIdx.x * kFewWaves + wave);
  const int64_t g0 = share(worker, W), g1 = share(worker + 1, W);
  if (g0 >= g1) return;
  const int steps = uniform((int)(g1 - g0));
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))smem + wave * 2 * kFewStage;
  const int quad = lane >> 4, lr = lane & 15;
  // a lane's place in an instruction's four rows of the pages (K and V chunks permuted)
  const uint32_t row_step = (uint32_t)p.c.ld_tok * 2;
  uint32_t koff[4], voff[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * i + quad;
    koff[i] = row * row_step + 16 * k_chunk(row, lr) - 1024 * i;  // 4 rows are 1024 bytes at least
    voff[i] = row * row_step + 16 * v_chunk(row, lr) - 1024 * i;
  }
  auto lowest = [&](int s) -> int {  // few_lo of request s, by the wave
    if (!p.first) return 0;
    const int64_t a = fixed(p.start, s), e = fixed(p.start, s + 1), n = fixed(p.n, s);
    int64_t lo = a + lane < e ? p.first[a + lane] : n;
    lo = lo < 0 ? 0 : lo > n ? n : lo;
    int x = (int)lo;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x = min(x, __shfl_xor(x, o, kWave));
    return uniform(x & ~(kFewKeys - 1));
  };
  auto place = [&](int64_t g) {
    Place x;
    x.s = uniform(request_of(before, S, (int)quotient(g, H)));
    const int first = uniform(before[x.s]);
    x.nb = uniform(before[x.s + 1]) - first;
    const int64_t rem = g - (int64_t)first * H;
    x.h = uniform((int)quotient(rem, x.nb));
    x.b = uniform((int)(rem - (int64_t)x.h * x.nb));
    x.lo = lowest(x.s);
    x.n = uniform((int)fixed(p.n, x.s));
    return x;
  };
  auto next = [&](Place& x) {  // the next block; not past the last of all
    if (++x.b < x.nb) return;
    x.b = 0;
    if (++x.h < H) return;
    x.h = 0;
    do {
      ++x.s;
      x.nb = x.s < S ? uniform(before[x.s + 1] - before[x.s]) : 1;
    } while (x.nb == 0);
    if (x.s < S) {
      x.lo = lowest(x.s);
      x.n = uniform((int)fixed(p.n, x.s));
    }
  };
  // page numbers of the 16-key groups of a place's block (-1 behind the end)
  auto pages = [&](const Place& x, int (&id)[2]) {
    const int key = x.lo + kFewKeys * x.b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int k = key + 16 * i;
      id[i] = k < x.n ? page_uniform(p.c, x.s, k >> p.c.shift) : -1;
    }
  };
  auto issue = [&](const Place& x, const int (&id)[2], int stage) {
    const uint32_t at = lds0 + stage * kFewStage;
    const int key = x.lo + kFewKeys * x.b;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bool ok = (uint32_t)id[i] < (uint32_t)p.c.P;
      const int64_t o = (int64_t)(ok ? id[i] : 0) * p.c.ld_page + (int64_t)x.h * p.c.ld_head +
                        (int64_t)((key + 16 * i) & ((1 << p.c.shift) - 1)) * p.c.ld_tok;
      const void *kb = p.c.K + o, *vb = p.c.V + o;  // absent: rows of page 0, which no one uses
      load_to_lds(at + i * 4096, kb, koff);
      load_to_lds(at + kFewStage / 2 + i * 4096, vb, voff);
    }
  };

  Place now = place(g0), ahead = now;
  int id[3][2];  // page numbers of this step, the next and the one after
  pages(ahead, id[0]);
  issue(ahead, id[0], 0);
  if (steps > 1) {
    next(ahead);
    pages(ahead, id[1]);
    issue(ahead, id[1], 1);
  }
  // ---- a piece of a request and head at a time ----
  int step = 0;
  while (step < steps) {
    const int s = now.s, h = now.h, b_first = now.b, b_end = uniform(min(now.nb, now.b + steps - step));
    const int64_t a = fixed(p.start, s);
    const int n = now.n, rows = uniform((int)(fixed(p.start, s + 1) - a)) * G, lo_key = now.lo;
    v8 qf[CT][4];
    int pos[CT], lo[CT], hi[CT], lo_max = 0, hi_min = n;
    float slope[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int r = 16 * t + lr, tok = r / G, g = r - tok * G;
      pos[t] = 0;
      lo[t] = 0;
      hi[t] = n;
      slope[t] = 0.0f;
      s16x8 z = {};
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) qf[t][kk] = __builtin_bit_cast(v8, z);
      if (r < rows) {
        pos[t] = n - rows / G + tok;
        token_range(p, s, a + tok, pos[t], n, &lo[t], &hi[t]);
        if (p.slopes) slope[t] = p.slopes[h * G + g] * kLog2e;
        const uint16_t* qp = p.q + (a + tok) * p.ldq_tok + (int64_t)(h * G + g) * p.ldq_head + 8 * quad;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) qf[t][kk] = *reinterpret_cast<const v8*>(qp + 32 * kk);
      }
      lo_max = max(lo_max, lo[t]);
      hi_min = min(hi_min, hi[t]);
    }
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) {
      lo_max = max(lo_max, __shfl_xor(lo_max, o, kWave));
      hi_min = min(hi_min, __shfl_xor(hi_min, o, kWave));
    }
    lo_max = uniform(lo_max);
    hi_min = uniform(hi_min);
    f32x4 o[CT][8];
    float m[CT], l[CT];
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      m[t] = -__builtin_huge_valf();
      l[t] = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c) o[t][c] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (int b = b_first; b < b_end; ++b, ++step) {
      const int stage = step & 1;
      const uint32_t at = lds0 + stage * kFewStage, vat = at + kFewStage / 2;
      if (step + 2 < steps) {  // its page numbers arrive during this step
        next(ahead);
        pages(ahead, id[2]);
      }
      if (step + 1 < steps) wait_vm<16>();
      else wait_vm<0>();
      const int key = lo_key + kFewKeys * b;
      const int cur0 = id[0][0], cur1 = id[0][1];
      const bool in0 = (uint32_t)cur0 < (uint32_t)p.c.P, in1 = (uint32_t)cur1 < (uint32_t)p.c.P;
      if ((!in0 && key < n) || (!in1 && key + 16 < n)) flags |= FATHOM_DEV_BAD_PAGE;
      const bool masked = key < lo_max || key + kFewKeys > hi_min || !in0 || !in1;
      if (masked && (key + kFewKeys > n || !in0 || !in1)) {  // rows that are not there: V is cleared
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int row = 4 * y + quad;
          if (key + row >= n || !(row < 16 ? in0 : in1))
            *LDS_AT(u32x4, vat + row * kRowBytes + 16 * lr) = (u32x4){0u, 0u, 0u, 0u};
        }
      }
      // ---- S^T: two groups of 16 keys ----
      f32x4 sc[CT][2];
#pragma unroll
      for (int gk = 0; gk < 2; ++gk) {
        v8 kf[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          kf[kk] = lds_v8<v8>(at + (16 * gk + lr) * kRowBytes + 16 * k_chunk(lr, 4 * kk + quad));
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
          if (16 * t < rows) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) x = Mx<BF>::mfma16(kf[kk], qf[t][kk], x);
          }
          sc[t][gk] = x;
        }
      }
      // ---- softmax, probabilities as two values of the pages' type ----
      v8 ph[CT], pl[CT];
#pragma unroll
      for (int t = 0; t < CT; ++t) {
        if (16 * t >= rows) continue;
        float z[8], mx = -__builtin_huge_valf();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int k = key + 16 * (e >> 2) + 4 * quad + (e & 3);
          z[e] = capped ? mapped<true>(sm, slope[t], sc[t][e >> 2][e & 3], pos[t] - k)
                        : mapped<false>(sm, slope[t], sc[t][e >> 2][e & 3], pos[t] - k);
          if (masked) {
            if (!(k >= lo[t] && k < hi[t] && (e < 4 ? in0 : in1))) z[e] = -__builtin_huge_valf();
          }
          mx = fmaxf(mx, z[e]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        if (__ballot(mx > m[t])) {
          const float mn = fmaxf(m[t], mx);
          const float f = mn == -__builtin_huge_valf() ? 1.0f : __builtin_amdgcn_exp2f(m[t] - mn);
          m[t] = mn;
          l[t] *= f;
#pragma unroll
          for (int c = 0; c < 8; ++c) o[t][c] *= f;
        }
        const float ref = m[t] == -__builtin_huge_valf() ? 0.0f : m[t];
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          // (the shift after the difference: m less the shift would be rounded, by 8 and more of large scores)
          const float x = __builtin_amdgcn_exp2f((z[e] - ref) + Mx<BF>::kShift);
          sum += x;
          const typename Mx<BF>::t xh = (typename Mx<BF>::t)x;
          ph[t][e] = xh;
          pl[t][e] = (typename Mx<BF>::t)(x - (float)xh);
        }
        l[t] += sum;
      }
      // ---- O^T += V^T P^T, 16 channels at a time ----
      const int r0 = 4 * quad + (lr >> 2);  // row and 8-byte piece that this lane names
      auto v_at = [&](int c) -> s16x8 {
        const uint32_t va = vat + r0 * kRowBytes + 16 * v_chunk(r0, 2 * c + ((lr & 3) >> 1)) + 8 * (lr & 1);
        return __builtin_shufflevector(lds_tr(va), lds_tr(va + 16 * kRowBytes), 0, 1, 2, 3, 4, 5, 6, 7);
      };
      const bool clean = masked && any_nonfinite<BF, kFewStage / 2>(vat + 16 * lane);
      if (clean) {
#pragma unroll 1
        for (int row = 0; row < kFewKeys; ++row) {
          const int k = key + row;
          const bool in = row < 16 ? in0 : in1;
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const s16x4 x = *LDS_AT(const s16x4, vat + row * kRowBytes + 16 * v_chunk(row, 2 * c + (quad >> 1)) + 8 * (quad & 1));
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int t = 0; t < CT; ++t)
                if (in && k >= lo[t] && k < hi[t]) o[t][c][e] += nonfinite_part<BF>(x[e]);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        s16x8 x = v_at(c);
        if (clean) x = finite_part<BF>(x);
        const v8 vf = __builtin_bit_cast(v8, x);
#pragma unroll
        for (int t = 0; t < CT; ++t) {
          if (16 * t >= rows) continue;
          o[t][c] = Mx<BF>::mfma16(vf, ph[t], o[t][c]);
          o[t][c] = Mx<BF>::mfma16(vf, pl[t], o[t][c]);
        }
      }
      // this stage is read: its next block
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        id[0][i] = id[1][i];
        id[1][i] = id[2][i];
      }
      if (step + 2 < steps) issue(ahead, id[1], stage);
    }
    // ---- the piece's result: the output where it is the whole, or a part ----
    const bool whole = b_first == 0 && b_end == now.nb;
    const int slot = step - (b_end - b_first) == 0 ? 0 : 1;
    const int64_t pr = ((int64_t)worker * 2 + slot) * R;
    float sum[CT], zeros[4] = {};  // zeros: NaN where O is not finite and the sum is
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      sum[t] = l[t];
      sum[t] += __shfl_xor(sum[t], 16, kWave);
      sum[t] += __shfl_xor(sum[t], 32, kWave);
      if (16 * t + lr < rows && sum[t] - sum[t] == 0.0f) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) zeros[e] = __builtin_fmaf(o[t][c][e], 0.0f, zeros[e]);
      }
    }
    if (__ballot((zeros[0] + zeros[1]) + (zeros[2] + zeros[3]) != 0.0f)) {
      uint64_t found = 0;
      const int key = lo_key + kFewKeys * b_first;
      nonfinite_rows<BF>(p, s, h, key, min(n, lo_key + kFewKeys * b_end), [&](int k, const uint16_t* row) {
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const s16x4 x = *reinterpret_cast<const s16x4*>(row + 16 * c + 4 * quad);
#pragma unroll
          for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (k >= lo[t] && k < hi[t])
                o[t][c][e] = with_nonfinite<BF>(o[t][c][e], x[e], found, 32 * t + 4 * c + e);
        }
      });
    }
#pragma unroll
    for (int t = 0; t < CT; ++t) {
      const int r = 16 * t + lr;
      const float lt = sum[t];
      if (r >= rows) continue;
      if (whole) {
        const int tok = r / G, g = r - tok * G;
        uint16_t* op = p.out + ((a + tok) * H * G + h * G + g) * kD + 4 * quad;
        const float f = lt > 0.0f || lt != lt ? 1.0f / lt : 0.0f;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          typename Mx<BF>::t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (typename Mx<BF>::t)(lt == 0.0f ? 0.0f : o[t][c][e] * f);
          *reinterpret_cast<u32x2*>(op + 16 * c) = *reinterpret_cast<u32x2*>(y);
        }
      } else {
        float* op = p.part_o + (pr + r) * kD + 4 * quad;
#pragma unroll
        for (int c = 0; c < 8; ++c) *reinterpret_cast<f32x4*>(op + 16 * c) = o[t][c];
        if (quad == 0) {
          // (a sum without a maximum is NaN, of NaN scores, and must not be taken for an empty part)
          p.part_ml[(pr + r) * 2] = m[t] == -__builtin_huge_valf() && lt != 0.0f ? 0.0f : m[t];
          p.part_ml[(pr + r) * 2 + 1] = lt;
        }
      }
    }
    const int taken = b_end - b_first;
    now.b += taken - 1;
    if (step < steps) next(now);
  }
  if (flags && lane == 0) set_status(p.st, flags);
}

// The requests and heads of attn_few_kernel whose blocks went to more than one wave:
// out = sum_c 2^(m_c - M) o_c / sum_c 2^(m_c - M) l_c over a row's parts, in a fixed order.
// Block counts are recomputed from the lengths.  Bound by trips to memory: one for the lengths,
// one for every part's (m, l), a thread a part, and one for eight parts' sums at a time, 32
// threads and 4 channels a thread each (one part after another: 14 us for 128 parts, where this
// takes 6).  Of at most eight parts, eight rows at a time take one trip for all (64 requests of
// 32 rows 146 us with attention, this way 117).  blockIdx.x is the request and head or, where
// these are more than the waves' bounds, the bound: the first inside of a request and head joins
// it (4000 requests 10.3 ms with attention, 0.47).
constexpr int kJoinGroups = 8, kJoinBatch = 8;
template <bool BF, bool LOOP>
__global__ __launch_bounds__(256) void attn_join_kernel(PagedAttnArgs p, int R) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ float weight[kFewWorkers], red_m[4], red_l[4];
  __shared__ f32x4 acc[kJoinGroups][32];
  int* before = reinterpret_cast<int*>(smem);
  const int H = p.c.H, G = p.G;
  const bool bounds = p.S * H >= kFewWorkers;
  uint32_t flags = 0;
  few_plan(p, before, before + p.S + 1, flags);
  const int64_t W = (int64_t)uniform(before[p.S]) * H;
  const int64_t at = share(blockIdx.x + 1, W), last = share(blockIdx.x, W);
  if (bounds && (at == last || at >= W)) return;
  const int s = bounds ? uniform(request_of(before, p.S, (int)quotient(at, H))) : blockIdx.x / H;
  const int nb = uniform(before[s + 1] - before[s]);
  if (nb == 0) return;
  const int64_t a = fixed(p.start, s);
  const int rows = (int)(fixed(p.start, s + 1) - a) * G;
  const int h = bounds ? (int)quotient(at - (int64_t)uniform(before[s]) * H, nb) : blockIdx.x % H;
  const int64_t g0 = (int64_t)uniform(before[s]) * H + (int64_t)h * nb;
  const int w0 = worker_of(g0, W), count = worker_of(g0 + nb - 1, W) - w0 + 1;
  if (count == 1 || (bounds && (at == g0 || last > g0))) return;
  const int tid = threadIdx.x, x = tid & 31, g = tid >> 5;
  auto store = [&](int r, f32x4 o, float l) {  // the 4 channels from 4 x
    const int tok = r / G;
    typename Mx<BF>::t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (typename Mx<BF>::t)(l == 0.0f ? 0.0f : o[e] / l);
    *reinterpret_cast<u32x2*>(p.out + ((a + tok) * H * G + h * G + (r - tok * G)) * kD + 4 * x) =
        *reinterpret_cast<u32x2*>(y);
  };
  // a part is its wave's first piece, but for a wave that begins in an earlier request or head
  const int64_t step = 2 * R, late = share(w0, W) < g0 ? R : 0;
  auto part_of = [&](int r) {
    return [=](int c) -> int64_t {
      return share(w0 + c, W) == share(w0 + c + 1, W) ? -1 : w0 * step + r + c * step + (c == 0 ? late : 0);
    };
  };
  if (count <= kJoinBatch) {
    for (int r = blockIdx.y * kJoinGroups + g; r < rows; r += gridDim.y * kJoinGroups) {
      const int64_t row0 = w0 * step + r;
      float m[kJoinBatch], lp[kJoinBatch], M = -__builtin_huge_valf(), l = 0.0f;
      f32x4 v[kJoinBatch], o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < kJoinBatch; ++c) {  // (behind the last part: that one again, unused)
        const int64_t at = row0 + min(c, count - 1) * step + (c == 0 ? late : 0);
        m[c] = p.part_ml[2 * at];
        lp[c] = p.part_ml[2 * at + 1];
        v[c] = *reinterpret_cast<const f32x4*>(p.part_o + at * kD + 4 * x);
      }
#pragma unroll
      for (int c = 0; c < kJoinBatch; ++c) {
        if (c >= count || share(w0 + c, W) == share(w0 + c + 1, W)) m[c] = -__builtin_huge_valf();
        M = fmaxf(M, m[c]);
      }
#pragma unroll
      for (int c = 0; c < kJoinBatch; ++c) {
        if (m[c] == -__builtin_huge_valf()) continue;
        const float w = __builtin_amdgcn_exp2f(m[c] - M);
        l += w * lp[c];
        o += w * v[c];
      }
      store(r, parts_sum(p, o, 0, 1, count, M, part_of(r)), l);
    }
    return;
  }
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    const int64_t row0 = w0 * step + r;
    float M = -__builtin_huge_valf(), l = 0.0f;
    for (int c = tid; c < count; c += 256) {
      float m = -__builtin_huge_valf();
      if (share(w0 + c, W) < share(w0 + c + 1, W)) m = p.part_ml[2 * (row0 + c * step + (c == 0 ? late : 0))];
      weight[c] = m;
      M = fmaxf(M, m);
    }
    M = wave_max(M);
    if ((tid & 63) == 0) red_m[tid >> 6] = M;
    __syncthreads();
    M = fmaxf(fmaxf(red_m[0], red_m[1]), fmaxf(red_m[2], red_m[3]));
    for (int c = tid; c < count; c += 256) {
      const float m = weight[c];
      const float w = m == -__builtin_huge_valf() ? -1.0f : __builtin_amdgcn_exp2f(m - M);
      weight[c] = w;  // -1: none, the part may not be there
      if (m != -__builtin_huge_valf()) l += w * p.part_ml[2 * (row0 + c * step + (c == 0 ? late : 0)) + 1];
    }
    l = wave_sum(l);
    if ((tid & 63) == 0) red_l[tid >> 6] = l;
    __syncthreads();
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = g; c0 < count; c0 += kJoinGroups * kJoinBatch) {
      f32x4 v[kJoinBatch];
      float w[kJoinBatch];
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i) {
        const int c = c0 + i * kJoinGroups;
        const int cc = min(c, count - 1);  // (behind the last: that one again, unused)
        w[i] = c < count ? weight[cc] : -1.0f;
        v[i] = *reinterpret_cast<const f32x4*>(p.part_o + (row0 + cc * step + (cc == 0 ? late : 0)) * kD + 4 * x);
      }
#pragma unroll
      for (int i = 0; i < kJoinBatch; ++i) {
        const f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
        o += w[i] < 0.0f ? z : w[i] * v[i];
      }
    }
    acc[g][x] = parts_sum(p, o, g, kJoinGroups, count, M, part_of(r));
    __syncthreads();
    if (tid >= 32) {
      if constexpr (LOOP) continue;
      return;
    }
    const float den = (red_l[0] + red_l[1]) + (red_l[2] + red_l[3]);
    f32x4 sum = acc[0][tid];
#pragma unroll
    for (int i = 1; i < kJoinGroups; ++i) sum += acc[i][tid];
    store(r, sum, den);
    if constexpr (!LOOP) return;
  }
}

// ---------------------------------------------------------------- many query rows
// A workgroup's share: a tile of at most 128 / G new tokens of one request and head.
struct ManyTile {
  int s, h, tok0, toks, total, n;  // tokens of the tile and of the request, new and all
  int lo, hi;                      // the union of their ranges
  int lo_max, hi_min;              // and what all of them see (up to the first token's own position)
  int64_t a;                       // the request's first row
};

// The tile that is taken as the i-th of n (each by `times` workgroups): later ones, which see
// more, first.  Where all workgroups run at once, two a CU, the second half goes the other way
// up, so that long and short ones share a CU (2048 new tokens 61 us -> 56, 2 x 1024 48 -> 40).
__device__ __forceinline__ int tile_order(int n, int i, int times) {
  const int first = (n + 1) / 2;
  return i >= first && i < n && n * times <= 512 ? i - first : n - 1 - i;
}

// A tile as attn_tiles_kernel writes it; request -1: none.
struct TileRecord {
  int s, tok0, total, n;
  int64_t a;
};

// Tiles of more than 64 requests with more than `few` query rows each, tm tokens a tile, in the
// order in which workgroups take them: every workgroup sums over all requests, a thread takes a
// tile.  (Sums in each of attn_many_kernel's workgroups: 4000 requests of 40 query rows 2.3 ms,
// this way 1.0.)
__global__ __launch_bounds__(256) void attn_tiles_kernel(PagedAttnArgs p, int tm) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  int *before = reinterpret_cast<int*>(smem), *part = before + p.S + 1;
  const int tid = threadIdx.x;
  uint32_t flags = 0;
  sums_before(p.S, before, part, [&](int s) {
    int64_t a, n;
    const int rows = request_rows(p, s, &a, &n, flags);
    return rows * p.G > p.few ? (rows + tm - 1) / tm : 0;
  });
  if (flags && blockIdx.x == 0) set_status(p.st, flags);
  const int64_t tile = (int64_t)blockIdx.x * 256 + tid;
  if (tile >= p.ntiles) return;
  const int x = tile_order(before[p.S], (int)tile, p.c.H * p.nsplit);
  TileRecord t = {-1, 0, 0, 0, 0};
  if (x >= 0) {
    t.s = request_of(before, p.S, x);
    t.tok0 = (x - before[t.s]) * tm;
    t.a = p.start[t.s];
    t.total = (int)(p.start[t.s + 1] - t.a);
    t.n = (int)p.n[t.s];
  }
  p.tiles[tile] = t;
}

// Lanes' requests in the order of their lengths, to an eighth: longer ones, taken first, leave
// short ones for the end (64 requests of 100 to 16000 tokens 1.50 ms -> 1.27).  Returns the
// lane that each came from.
__device__ __forceinline__ int by_length(int length, int& tiles, int& rows, int64_t& n, int64_t& a) {
  const int lane = threadIdx.x & 63;
  const int key = length > 0 ? ((int)__float_as_uint((float)length) - (127 << 23)) >> 20 : 0;  // 8 bits
  const uint64_t live = __ballot(length > 0);
  if (live == 0 || !__ballot(length > 0 && key != __builtin_amdgcn_readlane(key, __builtin_ctzll(live)))) return lane;
  uint64_t same = ~0ull;  // lanes whose key is the lane's own, as far as it is looked at
  int rank = 0;           // lanes whose key is below
#pragma unroll
  for (int b = 7; b >= 0; --b) {
    const bool one = (key >> b) & 1;
    const uint64_t ones = __ballot(one);
    rank += one ? __builtin_popcountll(same & ~ones) : 0;
    same &= one ? ones : ~ones;
  }
  rank += __builtin_popcountll(same & ((1ull << lane) - 1));
  tiles = __builtin_amdgcn_ds_permute(4 * rank, tiles);
  rows = __builtin_amdgcn_ds_permute(4 * rank, rows);
  n = __builtin_amdgcn_ds_permute(4 * rank, (int)n);
  a = __builtin_amdgcn_ds_permute(4 * rank, (int)a);
  return __builtin_amdgcn_ds_permute(4 * rank, lane);
}

// Tile `tile` of those of all requests with more than `few` query rows, tm tokens each; false
// where there are fewer.  Up to 64 requests a wave finds it by itself, a lane a request; of more
// it is read.  Every thread of 256; red[12] is LDS.
__device__ __forceinline__ bool many_tile(const PagedAttnArgs& p, int tm, int tile, int h, int* red, ManyTile* t,
                                          uint32_t& flags) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  t->h = h;
  if (p.S <= kWave) {
    int64_t a = 0, n = 0;
    int rows = 0, tiles = 0;
    if (lane < p.S) {
      rows = request_rows(p, lane, &a, &n, flags);
      if (rows * p.G > p.few) tiles = (rows + tm - 1) / tm;
    }
    const int sid = by_length(tiles > 0 ? (int)n : 0, tiles, rows, n, a);
    const int inc = scan_add(tiles);
    const int x = tile_order(__builtin_amdgcn_readlane(inc, kWave - 1), tile, p.c.H * p.nsplit);
    if (x < 0) return false;
    t->s = uniform(__builtin_popcountll(__ballot(inc <= x)));  // requests that end before tile x
    t->tok0 = (x - __builtin_amdgcn_readlane(inc - tiles, t->s)) * tm;
    t->total = __builtin_amdgcn_readlane(rows, t->s);
    t->n = __builtin_amdgcn_readlane((int)n, t->s);
    t->a = __builtin_amdgcn_readlane((int)a, t->s);  // (below 2^30)
    t->s = __builtin_amdgcn_readlane(sid, t->s);
  } else {
    const TileRecord* r = p.tiles + tile;
    t->s = fixed(&r->s, 0);
    if (t->s < 0) return false;
    t->tok0 = fixed(&r->tok0, 0);
    t->total = fixed(&r->total, 0);
    t->n = fixed(&r->n, 0);
    t->a = fixed(&r->a, 0);
  }
  t->toks = min(tm, t->total - t->tok0);
  t->hi_min = t->n - t->total + t->tok0 + 1;
  if (!p.first && !p.prefix) {
    t->lo = t->lo_max = 0;
    t->hi = t->n - t->total + t->tok0 + t->toks;
    return true;
  }
  int lo = t->n, hi = 0, lo_max = 0;
  if (tid < t->toks) {
    token_range(p, t->s, t->a + t->tok0 + tid, t->n - t->total + t->tok0 + tid, t->n, &lo, &hi);
    lo_max = lo;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o, kWave));
    hi = max(hi, __shfl_xor(hi, o, kWave));
    lo_max = max(lo_max, __shfl_xor(lo_max, o, kWave));
  }
  __syncthreads();  // red is free
  if (lane == 0) {
    red[wave] = lo;
    red[4 + wave] = hi;
    red[8 + wave] = lo_max;
  }
  __syncthreads();
  t->lo = uniform(min(min(red[0], red[1]), min(red[2], red[3]))) & ~(kManyKeys - 1);
  t->hi = uniform(max(max(red[4], red[5]), max(red[6], red[7])));
  t->lo_max = uniform(max(max(red[8], red[9]), max(red[10], red[11])));
  __syncthreads();
  return true;
}

// The keys of a tile in units of 64 (one where no query sees any: a loop that may not run costs
// the kernel spilled registers), and the parts that they are cut into.
__device__ __forceinline__ int units_of(const ManyTile& t) { return max((t.hi - t.lo + kManyKeys - 1) / kManyKeys, 1); }
__device__ __forceinline__ int parts_of(const PagedAttnArgs& p, int units) {
  const int most = units / p.part_units;
  return most >= p.nsplit ? p.nsplit : p.all_parts ? 1 : max(most, 1);
}

// Keys go by in blocks of 32.  While the matrix cores form the scores of the next block and
// add the last block's product with V, the vector unit takes the exponentials of this one:
// three blocks are under way at a time, in registers S (two), P (two) and O, 190 and no more
// than 256 of them, so that two workgroups share a CU and one computes while the other
// begins, waits or ends.  The maximum that the exponentials are taken against is raised only
// when a score exceeds it by more than kSlack (a factor of 2^kSlack is no loss in 32-bit
// sums, and Mx::kShift leaves room for it in the probabilities), so the sums are rarely
// rescaled.
//
// Probabilities are rounded to the pages' type once (attn_few_kernel keeps them as a sum of two):
// what is lost would take a second product with V, half as many matrix instructions again.
// Against 64 bits the bf16 output is off by 2.0e-3 of its size there, and by 1.7e-3, its own
// rounding, with probabilities of 32 bits.
//
// Bound by the power that the card allows and by issue: 2048 tokens over 65536 take 2.0 to 2.3
// ms (as cards differ), 0.96 to 1.1 PFLOP/s, where a large matrix product of this type reaches
// 1.2.  The clock falls to 1.7 GHz (2.2 and more where the matrix cores are mostly idle); in its
// cycles the matrix cores are busy to 51 % and vector instructions issue in 47 %.  With
// neither exponentials nor LDS reads the same instructions take 1.75 ms.  64 rows a wave and
// one workgroup a CU need half of the LDS reads and are up to 5 % faster there, and slower where
// tiles are short (6 requests of documents 303 us against 188).
constexpr float kSlack = 6.0f;

// A block's scores between two steps: as the matrix instructions leave them, or, mapped, as
// values of their own (values put back into an accumulator cost copies of all of it).
struct Scores16 {
  float v[16];
  __device__ __forceinline__ float& operator[](int i) { return v[i]; }
  __device__ __forceinline__ float operator[](int i) const { return v[i]; }
};

#define INLINE __attribute__((always_inline))

// MAP: 0 the scaled score, 1 with a bias (and for scales that are not above 0), 2 capped.
template <bool BF, int MAP>
__global__ __launch_bounds__(256, 2) void attn_many_kernel(PagedAttnArgs p) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  typedef typename Mx<BF>::v8 v8;
  typedef typename Mx<BF>::t vt;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), half = lane >> 5, lr = lane & 31;
  const int H = p.c.H, G = p.G;
  const int bid = blockIdx.x, h = bid % H, part = (bid / H) % p.nsplit, tile = bid / H / p.nsplit;
  int* red = reinterpret_cast<int*>(smem + kManyLds);
  ManyTile t;
  {
    uint32_t flags = 0;
    const bool some = many_tile(p, kManyRows / G, tile, h, red, &t, flags);
    if (flags && blockIdx.x == 0) set_status(p.st, flags);
    if (!some) return;
  }
  const int units = units_of(t), parts = parts_of(p, units);
  if (part >= parts) return;
  const int unit0 = (int)((int64_t)units * part / parts), unit1 = (int)((int64_t)units * (part + 1) / parts);
  // blocks, an even number
  const int nb = (unit1 - unit0) * (kManyKeys / kBlock), key0 = t.lo + unit0 * kManyKeys, n = t.n;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(LDS_PTR(char))smem;
  const int rows = t.toks * G;

  bool absent = false;
  // whether key k's page is there
  auto there = [&](int k) INLINE -> bool {
    return !absent || (uint32_t)page_of(p.c, t.s, min(k, n - 1) >> p.c.shift) < (uint32_t)p.c.P;
  };

  // ---- loads: wave w takes keys 8w .. 8w + 7 of a block ----
  const uint32_t row_step = (uint32_t)p.c.ld_tok * 2;
  uint32_t koff[2], voff[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = 4 * i + (lane >> 4), at = 8 * wave + row;
    koff[i] = row * row_step + 16 * k_chunk(at, lane & 15) - 1024 * i;  // 4 rows are 1024 bytes at least
    voff[i] = row * row_step + 16 * v_chunk(at, lane & 15) - 1024 * i;
  }
  // Where the wave's keys of block b begin in a pool; page 0 where there is none.
  const uint16_t *Kh = p.c.K + (int64_t)h * p.c.ld_head, *Vh = p.c.V + (int64_t)h * p.c.ld_head;
  auto page = [&](int b) INLINE -> int {
    const int k = key0 + b * kBlock + 8 * wave;
    return b < nb && k < n ? page_uniform(p.c, t.s, k >> p.c.shift) : 0;
  };
  auto place = [&](int b, int id) INLINE -> int64_t {
    const int k = key0 + b * kBlock + 8 * wave;
    return (int64_t)((uint32_t)id < (uint32_t)p.c.P ? id : 0) * p.c.ld_page +
           (int64_t)(k & ((1 << p.c.shift) - 1)) * p.c.ld_tok;
  };
  auto stage = [](int b) INLINE -> uint32_t { return (uint32_t)(b % kManyStages) * kBlockBytes; };
  constexpr uint32_t kVRing = kManyLds / 2;  // V's stages behind K's
  const uint32_t mine = lds0 + wave * (kBlockBytes / 4);
  // `advance(b)` issues K of block b + 4 and V of block b + 2, in stages that are read by then.
  // Blocks behind the last are loaded from page 0 and not used, so that the number of loads in
  // flight is always the same.
  int64_t from0 = place(0, page(0)), from1 = place(1, page(1)), from2 = place(2, page(2)), from3 = place(3, page(3));
  load_to_lds(mine + stage(0), Kh + from0, koff);
  load_to_lds(mine + stage(1), Kh + from1, koff);
  load_to_lds(mine + stage(2), Kh + from2, koff);
  load_to_lds(mine + kVRing + stage(0), Vh + from0, voff);
  load_to_lds(mine + stage(3), Kh + from3, koff);
  load_to_lds(mine + kVRing + stage(1), Vh + from1, voff);
  int id_next = page(4);

  // ---- the wave's 32 query rows, two lanes each ----
  v8 qf[8];
  int pos = 0, lo = 0, hi = n, lo_max = 0, hi_min = n;
  float slope = 0.0f;
  const ScoreMap sm = score_map(p);
  {
    const int r = wave * 32 + lr, tok = r / G, g = r - tok * G;
    const s16x8 zero = {};
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) qf[kk] = __builtin_bit_cast(v8, zero);
    if (r < rows) {
      const int64_t row = t.a + t.tok0 + tok;
      pos = n - t.total + t.tok0 + tok;
      token_range(p, t.s, row, pos, n, &lo, &hi);
      if (p.slopes) slope = p.slopes[h * G + g] * kLog2e;
      const uint16_t* qp = p.q + row * p.ldq_tok + (int64_t)(h * G + g) * p.ldq_head + 8 * half;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) qf[kk] = *reinterpret_cast<const v8*>(qp + 16 * kk);
      lo_max = lo;
      hi_min = MAP != 0 ? min(hi, pos + 1) : hi;  // (map_seen)
    }
  }
  if (!p.prefix && !p.first) {  // the wave's first token
    hi_min = wave * 32 < rows ? n - t.total + t.tok0 + wave * 32 / G + 1 : n;
  } else {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) {
      lo_max = max(lo_max, __shfl_xor(lo_max, o, kWave));
      hi_min = min(hi_min, __shfl_xor(hi_min, o, kWave));
    }
  }
  lo_max = uniform(lo_max);
  hi_min = uniform(hi_min);
  // ---- absent pages among the keys: all blocks count as masked then ----
  {
    const uint32_t e1 = min(key0 + nb * kBlock, n);  // (a step behind it may pass 2^31)
    for (uint32_t k = (uint32_t)key0 + 16u * (uint32_t)tid; k < e1; k += 16 * 256)
      absent |= (uint32_t)page_of(p.c, t.s, k >> p.c.shift) >= (uint32_t)p.c.P;
    const bool any = __ballot(absent) != 0;
    if (lane == 0) red[wave] = any;
    __syncthreads();
    absent = uniform(red[0] | red[1] | red[2] | red[3]) != 0;
    if (absent && tid == 0) set_status(p.st, FATHOM_DEV_BAD_PAGE);
  }
  const float c1 = MAP != 0 ? 1.0f : sm.c1;

  // LDS places of a lane's part of K fragments (of key lr, channels 8 half ..: chunk
  // `half`, permuted) and of V^T fragments (groups of 16 lanes name channels 0..15 and 16..31
  // and keys 4 half ..); channels 16 kk and 32 d on, the chunk differs in bits of its own
  uint32_t kaddr = lds0 + lr * kRowBytes + 16 * k_chunk(lr, half), vaddr;
  {
    const int r0 = 4 * half + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    vaddr = lds0 + kVRing + r0 * kRowBytes + 16 * v_chunk(r0, ch) + 8 * (lane & 1);
  }
  auto k_frag = [&](uint32_t at, int kk) INLINE { return lds_v8<v8>((kaddr ^ (32 * kk)) + at); };
  auto v_frag = [&](uint32_t at, int j) INLINE {  // keys 16 (j >> 2) .., channels 32 (j & 3) ..
    const uint32_t va = (vaddr ^ (64 * (j & 3))) + at + 16 * (j >> 2) * kRowBytes;
    return join4<v8>(lds_tr(va), lds_tr(va + 8 * kRowBytes));
  };

  typedef std::conditional_t<MAP == 0, f32x16, Scores16> Sv;
  f32x16 o[4];      // O^T: channels 32 d + 8 (e >> 2) + 4 half + (e & 3)
  Sv sa, sb;        // S^T: keys 8 (e >> 2) + 4 half + (e & 3)
  u32x4 pa[2], pb[2];
  // l: the sum of the probabilities; nr: kShift less the reference that they are taken against
  // (in log2; at first a reference that every score raises and against which -Inf gives 0)
  float nr = 1e37f, l = 0.0f, mx;  // mx: the lane's maximum of a block's scores
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;

  // S^T of the block at byte `at` of K's ring
  auto scores = [&](uint32_t at, Sv& s) INLINE {
    f32x16 acc = {};
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) acc = Mx<BF>::mfma32(k_frag(at, kk), qf[kk], acc);
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = acc[e];
  };
  // O^T += V^T P^T of the block at byte `at` of V's ring
  auto product = [&](uint32_t at, const u32x4(&pr)[2]) INLINE {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j & 3] = Mx<BF>::mfma32(v_frag(at, j), __builtin_bit_cast(v8, pr[j >> 2]), o[j & 3]);
  };
  auto exponentials = [&](const Sv& s, u32x4(&pr)[2]) INLINE {
#pragma unroll
    for (int e = 0; e < 16; e += 2) {
      const float x0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c1, nr));
      const float x1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e + 1], c1, nr));
      const typename Mx<BF>::v2 pair = {(vt)x0, (vt)x1};
      l = Mx<BF>::add_pair(pair, l);
      pr[e >> 3][(e & 7) >> 1] = __builtin_bit_cast(uint32_t, pair);
    }
  };
  // The mapped score of element e of a block, with a bias linear in the key: it is the bias for
  // keys up to the row's own (mask_block has the others).
  auto bias_base = [&](int key) INLINE { return slope * (float)(key + 4 * half - pos); };
  auto map_seen = [&](float s, int e, float base) INLINE -> float {
    const float bias = __builtin_fmaf(slope, (float)(8 * (e >> 2) + (e & 3)), base);
    if constexpr (MAP == 1) return __builtin_fmaf(s, sm.c1, bias);
    return mapped<true>(sm, 0.0f, s, 0) + bias;
  };
  auto maximum = [&](const Sv& s) INLINE {
    mx = fmaxf(s[0], s[1]);
#pragma unroll
    for (int e = 2; e < 16; e += 2) mx = fmaxf(fmaxf(mx, s[e]), s[e + 1]);
  };
  auto map_block = [&](Sv& s, int key) INLINE {
    if constexpr (MAP != 0) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = map_seen(s[e], e, bias_base(key));
    }
    maximum(s);
  };
  // What the rows of the wave do not see of the block at `key` takes no part; `mx` again.
  auto mask_block = [&](Sv& s, int key) INLINE {
    if (key >= lo_max && key + kBlock <= hi_min && !absent) return;
    if (MAP != 0 && p.prefix) {  // keys behind the row's own: slope * distance was added, not taken off
#pragma unroll
      for (int e = 0; e < 16; ++e)
        s[e] = __builtin_fmaf(-2.0f * slope, (float)max(key + 8 * (e >> 2) + 4 * half + (e & 3) - pos, 0), s[e]);
    }
    const uint32_t from = lo - key - 4 * half, count = max(hi - lo, 0);
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if ((uint32_t)(8 * (e >> 2) + (e & 3)) - from >= count) s[e] = -__builtin_huge_valf();
    if (absent) {
      const bool in0 = there(key), in1 = there(key + 16);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (!(e < 8 ? in0 : in1)) s[e] = -__builtin_huge_valf();
    }
    maximum(s);
  };
  // Where `mx` exceeds the reference by kSlack: the reference becomes the maximum of the row's
  // scores, l follows, and f is the factor for O.
  auto raise = [&](float& f) INLINE -> bool {
    if (!__ballot(__builtin_fmaf(mx, c1, nr) > kSlack + Mx<BF>::kShift)) return false;
    const float top = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    // scores far from 0 round it: downwards, or the probabilities taken against it overflow
    const float at = __builtin_fmaf(-top, c1, Mx<BF>::kShift);
    const float to = fminf(nr, __builtin_fmaf(fabsf(at), -0x1p-23f, at));
    f = __builtin_amdgcn_exp2f(to - nr);
    nr = to;
    l *= f;
    return true;
  };
  auto rescale = [&](float f) INLINE {
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] *= f;
  };
  // Block b is begun: its V, the next block's K and that of the block after, of which the first
  // fragments are read ahead, are in LDS once all but what the last call issued is; K of block
  // b and V of block b - 2 are read, by every wave.
  auto advance = [&](int b) INLINE {
    wait_vm<4>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int64_t from4 = place(b + 4, id_next);
    id_next = page(b + 5);
    load_to_lds(mine + stage(b + 4), Kh + from4, koff);
    load_to_lds(mine + kVRing + stage(b + 2), Vh + from2, voff);
    from2 = from3;
    from3 = from4;
  };
  // A block that not every query of the workgroup sees whole: V's rows that are not there are
  // cleared, and of values that are not finite the product takes none: they go to O of the
  // queries that see them before the block's V is cleared of them.
  auto prepare = [&](int b) INLINE {
    const int key_b = key0 + b * kBlock;
    if (key_b >= t.lo_max && key_b + kBlock <= t.hi_min && !absent) return;
    int x = lane;
    asm volatile("" : "+v"(x));  // (else what follows from the lane stays in registers throughout)
    const uint32_t v0 = lds0 + kVRing + stage(b), own = v0 + wave * (kBlockBytes / 4);
    const int key_w = key_b + 8 * wave;
    const bool in = there(key_w);
    if (key_w + 8 > n || !in) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int row = 4 * y + (x >> 4);
        if (key_w + row >= n || !in)
          *LDS_AT(u32x4, own + row * kRowBytes + 16 * (x & 15)) = (u32x4){0u, 0u, 0u, 0u};
      }
    }
    const bool bad = any_nonfinite<BF, kBlockBytes / 4>(own + 16 * x);
    if (x == 0) red[wave] = bad;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (!uniform(red[0] | red[1] | red[2] | red[3])) return;
#pragma unroll 1
    for (int row = 0; row < kBlock; ++row) {
      const int k = key_b + row;
      const bool sees = k >= lo && k < hi && there(k);
#pragma unroll
      for (int y = 0; y < 16; ++y) {  // channels 8 y + 4 half ..
        const s16x4 v = *LDS_AT(const s16x4, v0 + row * kRowBytes + 16 * v_chunk(row, y) + 8 * (x >> 5));
#pragma unroll
        for (int e = 0; e < 4; ++e) o[y >> 2][4 * (y & 3) + e] += sees ? nonfinite_part<BF>(v[e]) : 0.0f;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const uint32_t at = own + y * 1024 + 16 * x;
      *LDS_AT(s16x8, at) = finite_part<BF>(*LDS_AT(const s16x8, at));
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // A step: the exponentials of `s` to P, the scores of the next block (K at byte `kat`) to `sn`
  // and their maximum, the product of the last block (P in `pp`, V at byte `vat`).  16 pieces
  // of one matrix instruction with its LDS fragment, read two pieces ahead (the last two, in
  // `ka` and `kb`, for the step after, K at `kafter`), and of one exponential with what
  // belongs to it.
  auto step = [&](const Sv& s, u32x4(&pr)[2], uint32_t kat, Sv& sn, int key_next, uint32_t vat, const u32x4(&pp)[2],
                  v8& ka, v8& kb, uint32_t kafter) INLINE {
    v8 fr[18];
    f32x16 acc;
    float base = 0.0f, even = 0.0f;
    asm volatile("" : "+v"(kaddr), "+v"(vaddr));  // (else twelve addresses stay in registers)
    fr[0] = ka;
    fr[1] = kb;
    static_for<0, 16>([&](auto piece) INLINE {
      constexpr int j = decltype(piece)::value;
      if constexpr (j < 6) fr[j + 2] = k_frag(kat, j + 2);
      else if constexpr (j < 14) fr[j + 2] = v_frag(vat, j - 6);
      else fr[j + 2] = k_frag(kafter, j - 14);
      const f32x16 zero = {};
      if constexpr (j < 8) acc = Mx<BF>::mfma32(fr[j], qf[j], j == 0 ? zero : acc);
      else o[j & 3] = Mx<BF>::mfma32(fr[j], __builtin_bit_cast(v8, pp[(j - 8) >> 2]), o[j & 3]);
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], c1, nr));
      if constexpr (j % 2 == 0) {
        even = x;
      } else {
        const typename Mx<BF>::v2 pair = {(vt)even, (vt)x};
        l = Mx<BF>::add_pair(pair, l);
        // pinned: the compiler would move it to where it is used, behind the branch
        uint32_t word = __builtin_bit_cast(uint32_t, pair);
        asm volatile("" : "+v"(word), "+v"(l));
        pr[j >> 3][(j & 7) >> 1] = word;
      }
      // once the scores are complete: map them, and the maximum, a pair or two at a time
      if constexpr (j >= 10) {
        constexpr int first = j < 14 ? j - 10 : 4 + 2 * (j - 14), last = j < 14 ? first + 1 : first + 2;
        static_for<first, last>([&](auto two) INLINE {
          constexpr int e = 2 * decltype(two)::value;
          if constexpr (MAP == 0) {
            mx = e == 0 ? fmaxf(acc[0], acc[1]) : fmaxf(fmaxf(mx, acc[e]), acc[e + 1]);
          } else {
            if constexpr (e == 0) base = bias_base(key_next);
            sn[e] = map_seen(acc[e], e, base);
            sn[e + 1] = map_seen(acc[e + 1], e + 1, base);
            mx = e == 0 ? fmaxf(sn[0], sn[1]) : fmaxf(fmaxf(mx, sn[e]), sn[e + 1]);
          }
          asm volatile("" : "+v"(mx));
        });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (MAP == 0) sn = acc;
    ka = fr[16];
    kb = fr[17];
  };

  float f;
  wait_vm<4>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  scores(stage(0), sa);  // before K of block 4 takes its stage
  advance(0);
  prepare(0);
  map_block(sa, key0);
  mask_block(sa, key0);
  raise(f);  // (O is 0, or not finite)
  scores(stage(1), sb);
  exponentials(sa, pa);
  map_block(sb, key0 + kBlock);
  mask_block(sb, key0 + kBlock);
  // where it is raised, the product that is still to come is in the old scale: O follows after it
  bool up = raise(f);
  v8 ka = k_frag(stage(2), 0), kb = k_frag(stage(2), 1);
  int b = 1;
#pragma unroll 1
  for (; b + 1 < nb; b += 2) {  // blocks b and b + 1
    advance(b);
    prepare(b);
    step(sb, pb, stage(b + 1), sa, key0 + kBlock * (b + 1), stage(b - 1), pa, ka, kb, stage(b + 2));
    if (up) rescale(f);
    mask_block(sa, key0 + kBlock * (b + 1));
    up = raise(f);
    advance(b + 1);
    prepare(b + 1);
    step(sa, pa, stage(b + 2), sb, key0 + kBlock * (b + 2), stage(b), pb, ka, kb, stage(b + 3));
    if (up) rescale(f);
    mask_block(sb, key0 + kBlock * (b + 2));
    up = raise(f);
  }
  advance(b);
  prepare(b);
  product(stage(b - 1), pa);
  if (up) rescale(f);
  exponentials(sb, pb);
  product(stage(b), pb);

  // ---- the output, or a part of it ----
  wait_vm<0>();
  const int r = wave * 32 + lr;
  l += __shfl_xor(l, 32, kWave);
  {
    float zeros[4] = {};
    if (r < rows && l - l == 0.0f) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) zeros[e & 3] = __builtin_fmaf(o[d][e], 0.0f, zeros[e & 3]);
    }
    if (__ballot((zeros[0] + zeros[1]) + (zeros[2] + zeros[3]) != 0.0f)) {
      uint64_t found = 0;
      nonfinite_rows<BF>(p, t.s, h, key0, min(n, key0 + nb * kBlock), [&](int k, const uint16_t* row) INLINE {
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          const s16x4 x = *reinterpret_cast<const s16x4*>(row + 8 * y + 4 * half);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * (y & 3) + e;
            if (k >= lo && k < hi) o[y >> 2][i] = with_nonfinite<BF>(o[y >> 2][i], x[e], found, 4 * y + e);
          }
        }
      });
    }
  }
  if (r >= rows) return;
  if (parts == 1) {
    const int tok = r / G, g = r - tok * G;
    uint16_t* op = p.out + ((t.a + t.tok0 + tok) * H * G + h * G + g) * kD + 4 * half;
    const float f = 1.0f / l;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        vt y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = (vt)(l == 0.0f ? 0.0f : o[d][e + i] * f);
        *reinterpret_cast<u32x2*>(op + 32 * d + 2 * e) = *reinterpret_cast<u32x2*>(y);
      }
  } else {
    const int64_t pr = (((int64_t)tile * H + h) * p.nsplit + part) * kManyRows + r;
    float* op = p.part_o + pr * kD + 4 * half;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<f32x4*>(op + 32 * d + 2 * e) = (f32x4){o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]};
    if (half == 0) {
      p.part_ml[pr * 2] = Mx<BF>::kShift - nr;
      p.part_ml[pr * 2 + 1] = l;
    }
  }
}

// The tiles whose keys were split, a workgroup 16 query rows, 8 at a time, 32 threads and 4
// channels a thread each.  Bound by reading the parts: four parts' loads are on their way at
// once, whatever the number is (behind the last: that one again, unused; loads that depend on it
// came one after another).
constexpr int kManyJoin = 16, kMaxSplit = 8, kManyBatch = 4;
template <bool BF>
__global__ __launch_bounds__(256) void attn_many_join_kernel(PagedAttnArgs p) {
  __shared__ int red[12];
  uint32_t flags = 0;
  const int H = p.c.H, G = p.G, tile = blockIdx.x / H, h = blockIdx.x % H;
  ManyTile t;
  if (!many_tile(p, kManyRows / G, tile, h, red, &t, flags)) return;
  const int parts = parts_of(p, units_of(t)), rows = t.toks * G;
  if (parts == 1) return;
  const int64_t base = ((int64_t)tile * H + h) * p.nsplit * kManyRows;
  const int x = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < kManyJoin; i += 8) {
    const int r = blockIdx.y * kManyJoin + i + (threadIdx.x >> 5);
    if (r >= rows) return;
    float M = -__builtin_huge_valf(), l = 0.0f;  // (a part's maximum is a number: the reference it was taken against)
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < parts; c0 += kManyBatch) {
      float m[kManyBatch], lp[kManyBatch], top = M;
      f32x4 v[kManyBatch];
#pragma unroll
      for (int c = 0; c < kManyBatch; ++c) {
        const int64_t pr = base + (int64_t)min(c0 + c, parts - 1) * kManyRows + r;
        m[c] = p.part_ml[2 * pr];
        lp[c] = p.part_ml[2 * pr + 1];
        v[c] = *reinterpret_cast<const f32x4*>(p.part_o + pr * kD + 4 * x);
      }
#pragma unroll
      for (int c = 0; c < kManyBatch; ++c) top = fmaxf(top, m[c]);
      const float f = c0 == 0 ? 1.0f : __builtin_amdgcn_exp2f(M - top);
      M = top;
      l *= f;
      o *= f;
#pragma unroll
      for (int c = 0; c < kManyBatch; ++c) {
        if (c0 + c >= parts) continue;
        const float w = __builtin_amdgcn_exp2f(m[c] - M);
        l += w * lp[c];
        o += w * v[c];
      }
    }
    o = parts_sum(p, o, 0, 1, parts, M, [&](int c) { return base + (int64_t)c * kManyRows + r; });
    const int tok = r / G;
    typename Mx<BF>::t y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (typename Mx<BF>::t)(l == 0.0f ? 0.0f : o[e] / l);
    *reinterpret_cast<u32x2*>(p.out + ((t.a + t.tok0 + tok) * H * G + h * G + (r - tok * G)) * kD + 4 * x) =
        *reinterpret_cast<u32x2*>(y);
  }
}

// ---------------------------------------------------------------- launches
struct PagedAttnPlan {
  int few, R, rows;   // rows up to which a request goes to attn_few_kernel, that it is built for, that there can be
  bool run_few, run_many;
  int64_t tiles;      // bound on attn_many_kernel's row tiles
  int nsplit, part_units;  // parts of a tile's keys at most, units of 64 keys of a part at least
  bool all_parts;          // that many or one
  int64_t part_rows;  // rows of partial results
  int64_t records;    // tiles that attn_tiles_kernel writes
};

static PagedAttnPlan attn_plan(int64_t T, int S, int H, int G, int64_t max_new) {
  PagedAttnPlan a = {};
  const int64_t most = (max_new < T ? max_new : T) * G;  // query rows of a request and head, at most
  a.R = most <= 16 ? 16 : kFewRows;
  a.rows = (int)(most < kFewRows ? most : kFewRows);
  a.run_many = most > kFewRows;
  // T and max_new are bounds, so what may be large may also be small.  Of several requests both
  // kernels take theirs; one request, which is most often as large as its bounds, is
  // attn_many_kernel's whatever it has (attn_few_kernel and its join without rows cost 8 us, a
  // third of a prompt of 500 tokens).
  a.run_few = !a.run_many || S > 1;
  a.few = a.run_few ? kFewRows : 0;
  const int tm = kManyRows / G;
  a.nsplit = a.part_units = 1;
  if (a.run_many) {
    // requests that attn_many_kernel can have (of one, T is more than kFewRows / G)
    const int64_t large = T / (kFewRows / G + 1) < S ? T / (kFewRows / G + 1) : S;
    a.tiles = T / tm + large;
    // two workgroups on each of 256 CUs: the parts that leave the fewest places idle in the last
    // round, the first that leave at most a tenth.  A part costs its sums' way to memory and back,
    // so it has some keys at least: where the tiles alone fill few of the CUs 4 units (64 tokens
    // over 4000 24 us, 39 with 16), then 8 and 16 (1024 over none 35 and 30, over 1000 49 and 60;
    // 1500 over none 47 and 42), and where they fill all, 32 in each of the parts or none are made
    // (2336 over none to 2000 177 us, 224 in one or two parts; over 8000 407, 482 in one).
    const int64_t wgs = ((T + tm - 1) / tm + large / 2) * H;
    a.all_parts = wgs >= 512;
    a.part_units = wgs >= 512 ? 32 : wgs > 256 ? 16 : wgs >= 64 ? 8 : 4;
    double best = 0.0;
    for (int ns = 1; ns <= kMaxSplit && best < 0.9; ++ns) {
      const int64_t rounds = (wgs * ns + 511) / 512;
      const double used = (double)(wgs * ns) / (double)(rounds * 512);
      if (used <= best || (ns > 1 && wgs * ns > 2048)) continue;
      best = used;
      a.nsplit = ns;
    }
  }
  const int64_t few_rows = a.run_few ? (int64_t)kFewWorkers * 2 * a.R : 0;
  const int64_t many_part = a.run_many && a.nsplit > 1 ? a.tiles * H * a.nsplit * kManyRows : 0;
  a.part_rows = few_rows > many_part ? few_rows : many_part;
  a.records = S > kWave ? a.tiles : 0;
  return a;
}

size_t paged_attn_ws_bytes(int64_t T, int S, int H, int G, int64_t max_new) {
  const PagedAttnPlan a = attn_plan(T, S, H, G, max_new);
  return (size_t)a.part_rows * (kD + 2) * sizeof(float) + (size_t)a.records * sizeof(TileRecord) + 1024;
}

template <bool BF>
static void launch_attn(PagedAttnArgs p, const PagedAttnPlan& a, hipStream_t s) {
  const size_t plan = (size_t)(p.S + 1 + 4) * sizeof(int);
  const int64_t most = (p.c.ld_table << p.c.shift) / kManyKeys / a.part_units;  // parts of the longest request
  p.nsplit = (int)(most >= a.nsplit ? a.nsplit : a.all_parts || most < 1 ? 1 : most);
  p.part_units = a.part_units;
  p.all_parts = a.all_parts;
  p.few = a.few;
  if (a.run_many) {
    const dim3 grid((unsigned)(a.tiles * p.nsplit * p.c.H)), threads(256);
    const size_t lds = kManyLds + 12 * sizeof(int);
    if (a.records > 0)
      hipLaunchKernelGGL(attn_tiles_kernel, dim3((unsigned)((a.records + 255) / 256)), threads, plan, s, p, kManyRows / p.G);
    if (p.softcap > 0.0f) hipLaunchKernelGGL((attn_many_kernel<BF, 2>), grid, threads, lds, s, p);
    else if (p.slopes || !(p.sm_scale > 0.0f)) hipLaunchKernelGGL((attn_many_kernel<BF, 1>), grid, threads, lds, s, p);
    else hipLaunchKernelGGL((attn_many_kernel<BF, 0>), grid, threads, lds, s, p);
    if (p.nsplit > 1)
      hipLaunchKernelGGL((attn_many_join_kernel<BF>), dim3((unsigned)(a.tiles * p.c.H), kManyRows / kManyJoin), threads,
                         0, s, p);
  }
  if (a.run_few) {
    const dim3 grid(kFewWorkers / kFewWaves), threads(kFewWaves * kWave);
    const size_t lds = (size_t)kFewWaves * 2 * kFewStage + plan;
    if (a.R == 16) hipLaunchKernelGGL((attn_few_kernel<BF, 1>), grid, threads, lds, s, p);
    else hipLaunchKernelGGL((attn_few_kernel<BF, kFewRows / 16>), grid, threads, lds, s, p);
    // A request and head of more than eight parts is joined a workgroup a row where these are few,
    // and where they are many, so that most have few parts, by a few workgroups that go over the rows.
    const int pairs = p.S * p.c.H, units = pairs < kFewWorkers ? pairs : kFewWorkers - 1;
    const int y = a.run_many || pairs >= 128 ? (a.rows < 4 ? a.rows : 4) : a.rows;
    if (y < a.rows) hipLaunchKernelGGL((attn_join_kernel<BF, true>), dim3(units, y), dim3(256), plan, s, p, a.R);
    else hipLaunchKernelGGL((attn_join_kernel<BF, false>), dim3(units, y), dim3(256), plan, s, p, a.R);
  }
}

fathom_status launch_paged_attn(const void* q, int64_t ldq_tok, int64_t ldq_head, const Paged& c, bool bf16,
                                const int64_t* start, const int64_t* n, int S, int64_t T, int64_t max_new, int G,
                                float sm_scale, float softcap, const float* slopes, const int64_t* prefix,
                                const int64_t* first, void* out, void* ws, uint32_t* st, hipStream_t s) {
  const PagedAttnPlan a = attn_plan(T, S, c.H, G, max_new);
  PagedAttnArgs p = {};
  p.q = reinterpret_cast<const uint16_t*>(q);
  p.ldq_tok = ldq_tok;
  p.ldq_head = ldq_head;
  p.c = c;
  p.start = start;
  p.n = n;
  p.S = S;
  p.G = G;
  p.T = T;
  p.max_new = max_new;
  p.sm_scale = sm_scale;
  p.softcap = softcap;
  p.slopes = slopes;
  p.prefix = prefix;
  p.first = first;
  p.out = reinterpret_cast<uint16_t*>(out);
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = p.part_o + a.part_rows * kD;
  p.tiles = reinterpret_cast<TileRecord*>(p.part_ml + a.part_rows * 2);
  p.ntiles = a.records;
  p.st = st;
  if (bf16) launch_attn<true>(p, a, s);
  else launch_attn<false>(p, a, s);
  FATHOM_LAUNCH_CHECK();
  return FATHOM_OK;
}

}  // namespace fathom
