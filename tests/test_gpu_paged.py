"""The paged cache's calls on the GPU against oracle/paged.py (64 bits) and against the contiguous calls.

Pools are filled with NaN before the rows of the requests go in: what a call reads beyond them shows.

Tolerance of attention, per value, from the arithmetic that the header states.  With A = sum_j p_j |V_j|: the output is
rounded to its type (eps/2 of the value); probabilities of more than 32 query rows are rounded to it once (eps/2 each, so
eps/2 A); a score is a sum of 128 products in fp32, off by at most (128 + 8) 2^-24 times its sum of magnitudes `top`
(the 8: the scale, the cap's exp, divide and product, the bias), which moves a probability by that relative amount and
the sum of all by as much again; sums over n keys in fp32 and the joins of parts are within 64 2^-24 A (the partial sums
of a tree of at most 64 joins).  The cap multiplies an error of a few 2^-24 of 1 by softcap."""
import numpy as np
import pytest
import torch

import paper_2609_17652_amd as F
from oracle import paged as O

pytestmark = pytest.mark.gpu

DEV, D = "cuda", 128
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    F.lib()


def pools(rng, lengths, H, page, dt, major="head", spare=3, fill=float("nan"), scale=1.0):
    """Tables, K and V pools holding random rows of the lengths (everything else `fill`), and the rows [S][H][n][D]."""
    need = [O.pages_of(n, page) for n in lengths]
    P, L = sum(need) + spare, max(max(need), 1)
    order = rng.permutation(P).astype(np.int32)
    table = np.full((len(lengths), L), -1, np.int32)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    shape = (P, H, page, D) if major == "head" else (P, page, H, D)
    out, rows = [], []
    for _ in range(2):
        pool = torch.full(shape, fill, dtype=dt)
        view = pool if major == "head" else pool.transpose(1, 2)
        mine = []
        for s, n in enumerate(lengths):
            x = torch.from_numpy(rng.standard_normal((H, n, D)).astype(np.float32) * scale).to(dt)
            for j in range(need[s]):
                part = x[:, j * page:(j + 1) * page]
                view[table[s, j], :, :part.shape[1]] = part
            mine.append(x)
        dev = pool.to(DEV)
        out.append(dev if major == "head" else dev.transpose(1, 2))
        rows.append(mine)
    return torch.from_numpy(table).to(DEV), out[0], out[1], rows[0], rows[1]


def i64(x):
    return torch.tensor(x, dtype=torch.int64, device=DEV)


def status(st):
    return int(st.item())


# ---------------------------------------------------------------- map
def run_map(n_old, n, page, table, ring, state, T, H, in_place=False):
    t, r = torch.from_numpy(table.copy()).to(DEV), torch.from_numpy(ring.copy()).to(DEV)
    st, a, b, s0 = F.new_status(), i64(n_old), i64(n), i64(state)
    kw = dict(n_now=a, state_out=s0) if in_place else {}
    out = F.fathom_paged_map(a, b, page, t, r, s0, T, H, dev_status=st, **kw)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, r, *out)] + [status(st)]


def random_map(rng, S, page, L, T_extra, spare, P_extra=0):
    n_old = rng.integers(0, L * page + 1, S)
    n = np.where(rng.random(S) < 0.3, rng.integers(0, L * page + 1, S), np.minimum(n_old + 1, L * page))
    n_old[rng.random(S) < 0.1] = 0
    held = [(int(x) + page - 1) // page for x in n_old]
    grow = sum(max((int(b) + page - 1) // page - h, 0) for b, h in zip(n, held))
    P = sum(held) + max(grow + spare, 1) + P_extra
    order = rng.permutation(P).astype(np.int32)
    table, at = np.full((S, L), -1, np.int32), 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    head = int(rng.integers(0, P))
    ring = np.full(P, -1, np.int32)
    count = max(min(grow + spare, P - at), 0)
    for i in range(count):
        ring[(head + i) % P] = order[at + i]
    T = int(np.maximum(n - n_old, 0).sum()) + T_extra
    return n_old, n, table, ring, [head, count], max(T, 0)


def check_map(args, page, H, in_place=False):
    n_old, n, table, ring, state, T = args
    got = run_map(n_old, n, page, table, ring, state, T, H, in_place)
    want = O.paged_map(n_old, n, page, table, ring, state, T, H)
    names = ("table", "ring", "slots", "start", "n_now", "n_unit", "state")
    for name, g, w in zip(names, got, want):
        assert np.array_equal(g, w), name
    flags = (F.FATHOM_DEV_PAGES_SHORT if want[7] else 0) | (F.FATHOM_DEV_BAD_N if want[8] else 0)
    assert got[7] == flags


@pytest.mark.parametrize("S,page,L,H", [(1, 16, 3, 1), (2, 64, 5, 8), (64, 32, 9, 2), (65, 16, 40, 3), (300, 64, 30, 1),
                                        (1023, 16, 7, 1), (4096, 16, 12, 2)])
def test_map_random(S, page, L, H):
    rng = np.random.default_rng(S)
    check_map(random_map(rng, S, page, L, 4, 5), page, H)
    check_map(random_map(rng, S, page, L, 0, 0), page, H, in_place=True)
    check_map(random_map(rng, S, page, L, 2, -4), page, H)  # too few pages for the last ones
    if S > 1:
        check_map(random_map(rng, S, page, L, -3, 5), page, H)  # too few rows for the last ones


def test_map_bad_lengths_and_empty_calls():
    table, ring = np.full((5, 4), -1, np.int32), np.arange(20, dtype=np.int32)
    check_map(([-1, 0, 65, 5, 0], [4, 65, 3, -2, 20], table, ring, [3, 20], 20), 16, 1)
    check_map(([0] * 3, [0] * 3, table[:3], ring, [0, 20], 4), 16, 2)  # nothing moves
    out = run_map([], [], 16, np.zeros((0, 4), np.int32), ring, [7, 9], 3, 1)
    assert out[2].tolist() == [-1] * 3 and out[3].tolist() == [0] and out[6].tolist() == [7, 9] and out[7] == 0


def test_map_ends_requests_behind_rows_that_do_not_fit():
    """A request without new rows is served wherever it stands: the pages it returns are no longer its own."""
    table = np.array([[-1, -1], [4, 2], [3, -1]], np.int32)
    args = [0, 30, 16], [20, 0, 5], 16, table, np.array([0, 1, 5, -1, -1, -1], np.int32), [0, 3], 10
    out = run_map(*args, 1)
    for got, want in zip(out[:7], O.paged_map(*args, 1)):
        assert np.array_equal(got, want)
    assert out[4].tolist() == [0, 0, 5] and out[1].tolist() == [0, 1, 5, 4, 2, -1] and out[6].tolist() == [0, 5]
    assert out[7] == F.FATHOM_DEV_BAD_N


def test_map_bad_state_and_pages():
    table, ring = np.array([[9, -1], [-5, -1]], np.int32), np.array([1, 2, 3, 99], np.int32)
    for state in ([4, 1], [-1, 1], [0, 5], [0, -1]):  # nothing is taken
        out = run_map([0, 0], [4, 0], 16, table, ring, state, 4, 1)
        assert out[7] & F.FATHOM_DEV_BAD_PAGE and out[7] & F.FATHOM_DEV_PAGES_SHORT
        assert np.array_equal(out[0], table) and np.array_equal(out[1], ring) and out[6].tolist() == state
        assert out[2].tolist() == [-1] * 4 and out[4].tolist() == [0, 0]
    out = run_map([3, 3], [5, 5], 16, table, ring, [0, 3], 4, 1)  # entries outside the pool: no slots
    assert out[7] == F.FATHOM_DEV_BAD_PAGE and out[2].tolist() == [-1] * 4
    out = run_map([0, 0], [0, 3], 16, table, ring, [3, 1], 3, 1)  # the ring holds a page outside the pool
    assert out[7] == F.FATHOM_DEV_BAD_PAGE and out[2].tolist() == [-1] * 3
    out = run_map([16, 16], [0, 0], 16, table, ring, [0, 3], 3, 1)  # more come back than there is room for
    assert out[7] == F.FATHOM_DEV_BAD_PAGE and np.array_equal(out[1], ring) and out[6].tolist() == [0, 3]


# ---------------------------------------------------------------- write
@pytest.mark.parametrize("T,H,page,dt,src,major", [(1, 1, 16, "f16", "f16", "head"), (3, 8, 64, "bf16", "f32", "token"),
                                                   (67, 2, 32, "bf16", "bf16", "head"), (130, 3, 16, "f16", "f32", "head"),
                                                   (2500, 8, 128, "f16", "f16", "token")])
def test_write(T, H, page, dt, src, major):
    rng = np.random.default_rng(T)
    P = T // page + 4
    t, sdt = TYPES[dt], torch.float32 if src == "f32" else TYPES[dt]
    shape = (P, H, page, D) if major == "head" else (P, page, H, D)
    pools_ = [torch.full(shape, 7.0, dtype=t, device=DEV) for _ in range(2)]
    K, V = (x if major == "head" else x.transpose(1, 2) for x in pools_)
    rows = torch.from_numpy(rng.standard_normal((T, 3 * H + 1, D)).astype(np.float32) * 3).to(sdt).to(DEV)
    Kn, Vn = rows[:, 1:H + 1], rows[:, 2 * H:3 * H]  # strided views of a fused projection
    slots = rng.permutation(P * page)[:T].astype(np.int64)
    slots[rng.random(T) < 0.1] = -1
    st = F.new_status()
    F.fathom_paged_write(Kn, Vn, torch.from_numpy(slots).to(DEV), K, V, dev_status=st)
    for got, new in ((K, Kn), (V, Vn)):
        want = torch.full((P, H, page, D), 7.0, dtype=t)
        for i, s in enumerate(slots):
            if s >= 0:
                want[s // page, :, s % page] = new[i].cpu().to(t)
        assert torch.equal(got.cpu(), want)
    assert status(st) == 0


def test_write_slot_outside_the_pool_and_special_values():
    K, V = (torch.zeros((2, 1, 16, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    x = torch.zeros((3, 1, D), device=DEV)
    x[1, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.4e38])
    st = F.new_status()
    F.fathom_paged_write(x + 1, x, i64([32, 5, 1 << 40]), K, V, dev_status=st)
    assert status(st) == F.FATHOM_DEV_BAD_PAGE
    assert float(K[0, 0, 5, 9]) == 1.0 and float(K.float().nan_to_num(0, 0, 0).sum()) == D - 4
    v = V[0, 0, 5, :4].float().cpu()
    assert v[0] == float("inf") and v[1] == float("-inf") and v[2] != v[2] and v[3] == float("inf")
    F.fathom_paged_write(x[:0], x[:0], i64([]), K, V)


# ---------------------------------------------------------------- pack
@pytest.mark.parametrize("lengths,H,page,dt,major", [([1], 1, 16, "f16", "head"), ([63, 0, 64, 65], 2, 32, "bf16", "token"),
                                                     ([700, 129, 1000], 3, 16, "bf16", "head"),
                                                     ([33000, 20001], 8, 64, "f16", "head"),
                                                     ([40000], 8, 1024, "bf16", "token")])
def test_pack_equals_contiguous(lengths, H, page, dt, major):
    rng = np.random.default_rng(len(lengths))
    table, K, _, Kr, _ = pools(rng, lengths, H, page, TYPES[dt], major)
    S, cap = len(lengths), max(lengths)
    flat = torch.zeros((S * H, cap, D), dtype=torch.float32)
    for s, n in enumerate(lengths):
        flat[s * H:(s + 1) * H, :n] = Kr[s].float()
    flat = flat.to(DEV)
    nb = (cap + 63) // 64 + 1
    n = i64(lengths)
    st = F.new_status()
    planes = torch.full((S * H, D, 4, nb), -1, dtype=torch.int64, device=DEV)
    scales = torch.full((S * H, D, nb), -1, dtype=torch.int16, device=DEV)
    F.fathom_paged_pack(K, table, n, planes, scales, dev_status=st)
    want = F.fathom_pack(flat, n.repeat_interleave(H), nb)
    assert torch.equal(planes, want[0]) and torch.equal(scales, want[1]) and status(st) == 0
    # grown from a shorter prefix, by one token and by more
    for back in (1, 150):
        old = torch.clamp(n - back, min=0)
        p, s = F.fathom_pack(flat, old.repeat_interleave(H), nb)
        F.fathom_paged_pack(K, table, n, p, s, old, back, dev_status=st)
        assert torch.equal(p, want[0]) and torch.equal(s, want[1]) and status(st) == 0


def test_pack_absent_pages_and_bad_lengths():
    rng = np.random.default_rng(5)
    table, K, _, Kr, _ = pools(rng, [100, 200], 1, 64, torch.float16)
    table[0, 1] = 77
    planes = torch.zeros((2, D, 4, 4), dtype=torch.int64, device=DEV)
    scales = torch.zeros((2, D, 4), dtype=torch.int16, device=DEV)
    st = F.new_status()
    F.fathom_paged_pack(K, table, i64([100, 257]), planes, scales, dev_status=st)  # 257 > 4 pages: empty
    assert status(st) == F.FATHOM_DEV_BAD_PAGE | F.FATHOM_DEV_BAD_N
    flat = torch.zeros((2, 100, D))
    flat[0, :64] = Kr[0][0, :64].float()  # tokens of the absent page count as zeros
    want = F.fathom_pack(flat.to(DEV), i64([100, 0]), 4)
    assert torch.equal(planes, want[0]) and torch.equal(scales, want[1])


# ---------------------------------------------------------------- sparse attention
@pytest.mark.parametrize("lengths,H,G,page,k,sink,local,major", [([300], 1, 1, 16, 5, 0, 0, "head"),
                                                                ([900, 40, 0], 2, 4, 64, 100, 4, 32, "token"),
                                                                ([5000, 3500], 8, 4, 128, 1000, 4, 32, "head"),
                                                                ([77], 1, 8, 16, 0, 2, 9, "head")])
@pytest.mark.parametrize("qdt", [torch.float32, torch.float16])
def test_sparse_equals_contiguous(lengths, H, G, page, k, sink, local, major, qdt):
    rng = np.random.default_rng(k + 1)
    table, K, V, Kr, Vr = pools(rng, lengths, H, page, torch.float16, major)
    S, U, cap = len(lengths), len(lengths) * H, max(lengths)
    flat = [torch.zeros((U, cap, D), dtype=torch.float16) for _ in range(2)]
    for s, n in enumerate(lengths):
        for f, r in zip(flat, (Kr, Vr)):
            f[s * H:(s + 1) * H, :n] = r[s]
    q = torch.from_numpy(rng.standard_normal((U, G, D)).astype(np.float32)).to(qdt).to(DEV)
    idx = torch.from_numpy(rng.integers(-2, cap + 3, (U, G, k)).astype(np.int32)).to(DEV)  # some outside
    n, st = i64(lengths), F.new_status()
    got = F.fathom_paged_sparse_attn(q, K, V, table, n, idx if k else None, sink, local, dev_status=st)
    want = F.fathom_sparse_attn(q, flat[0].to(DEV), flat[1].to(DEV), n.repeat_interleave(H), idx if k else idx, sink, local)
    assert torch.equal(got, want) and status(st) == 0


def test_sparse_bf16_against_64_bits_and_absent_pages():
    rng = np.random.default_rng(9)
    n, k = 500, 60
    table, K, V, Kr, Vr = pools(rng, [n], 2, 32, torch.bfloat16)
    q = torch.from_numpy(rng.standard_normal((2, 3, D)).astype(np.float32)).bfloat16().to(DEV)
    idx = torch.stack([torch.from_numpy(rng.permutation(n)[:k].astype(np.int32)) for _ in range(6)]).view(2, 3, k).to(DEV)

    def expect(skip):
        out = np.zeros((2, 3, D))
        for h in range(2):
            for g in range(3):
                r = [i for i in idx[h, g].tolist() if not skip(i)]
                z = Kr[0][h, r].double().numpy() @ q[h, g].double().cpu().numpy() / np.sqrt(D)
                w = np.exp(z - z.max())
                out[h, g] = (w / w.sum()) @ Vr[0][h, r].double().numpy()
        return out

    st = F.new_status()
    got = F.fathom_paged_sparse_attn(q, K, V, table, i64([n]), idx, dev_status=st).cpu().numpy()
    assert np.abs(got - expect(lambda i: False)).max() < 1e-5 and status(st) == 0  # 32-bit sums of 60 rows
    table[0, 3] = -7
    got = F.fathom_paged_sparse_attn(q, K, V, table, i64([n]), idx, dev_status=st).cpu().numpy()
    assert np.abs(got - expect(lambda i: i // 32 == 3)).max() < 1e-5 and status(st) == F.FATHOM_DEV_BAD_PAGE
    st = F.new_status()
    got = F.fathom_paged_sparse_attn(q, K, V, table, i64([513]), idx, dev_status=st)  # 513 > 16 pages: empty
    assert (got == 0).all() and status(st) == F.FATHOM_DEV_BAD_N


# ---------------------------------------------------------------- attention
def attn_case(seed, reqs, H, G, page, dt, major="head", softcap=0.0, bias=False, prefix=None, docs=None, scale=None,
              pad=0, qs=2.0, lead=0):
    """Runs the call for requests (n, new) and checks it against the oracle; returns what was made."""
    rng = np.random.default_rng(seed)
    t = TYPES[dt]
    lengths, news = [r[0] for r in reqs], [r[1] for r in reqs]
    table, K, V, Kr, Vr = pools(rng, lengths, H, page, t, major)
    T = lead + sum(news) + pad
    HG = H * G
    fused = torch.from_numpy(rng.standard_normal((T, HG + 2, D)).astype(np.float32) * qs).to(t)
    q = fused.to(DEV)[:, 1:HG + 1]  # a view of a fused projection
    start = np.concatenate([[0], np.cumsum(news)]) + lead
    slopes = torch.tensor([2.0 ** -(1 + i % 8) for i in range(HG)], dtype=torch.float32) if bias else None
    pre = i64(prefix) if prefix is not None else None
    first = None
    if docs is not None:
        first = np.zeros(T, np.int64)
        for s, (n, new) in enumerate(reqs):
            pos = n - new + np.arange(new)
            first[start[s]:start[s + 1]] = docs(s, pos)
    out = torch.full((T, HG, D), 5.0, dtype=t, device=DEV)
    st = F.new_status()
    F.fathom_paged_attn(q, K, V, table, i64(start.tolist()), i64(lengths), max(news), scale, softcap,
                        None if slopes is None else slopes.to(DEV), pre, None if first is None else i64(first.tolist()),
                        out, dev_status=st)
    assert status(st) == 0
    got = out.double().cpu().numpy()
    qd = fused[:, 1:HG + 1].double().numpy()
    eps = torch.finfo(t).eps
    sm = 1 / np.sqrt(D) if scale is None else scale
    for s, (n, new) in enumerate(reqs):
        a = start[s]
        for h in range(H):
            ref, mag, top = O.paged_attn(qd[a:a + new, h * G:(h + 1) * G], Kr[s][h].double().numpy(),
                                         Vr[s][h].double().numpy(), n, G, sm, softcap,
                                         None if slopes is None else slopes[h * G:(h + 1) * G].double().numpy(),
                                         None if prefix is None else prefix[s],
                                         None if first is None else first[a:a + new])
            dz = (D + 8) * 2.0 ** -24 * top + 8 * 2.0 ** -24 * softcap + (2.0 ** -22 * n if bias else 0)
            p = eps / 2 if new * G > 32 else eps * eps
            tol = eps / 2 * np.abs(ref) + mag * (p + 2 * dz[..., None] + 64 * 2.0 ** -24) * (1 + eps)
            err = np.abs(got[a:a + new, h * G:(h + 1) * G] - ref)
            worst = (err / np.maximum(tol, 1e-30)).max() if new else 0.0
            assert (err <= tol + 1e-30).all(), (s, h, worst)
    assert (got[:lead] == 5.0).all() and (got[lead + sum(news):] == 5.0).all()  # rows of no request
    return K, V, table, q, out


FEW = [  # decode and drafted tokens: at most 32 query rows a request and head
    ([(1, 1)], 1, 1, 16, "f16"), ([(2, 1)], 1, 8, 16, "bf16"), ([(31, 1), (32, 1), (33, 1), (16, 1)], 2, 4, 16, "f16"),
    ([(4096, 1)], 8, 4, 64, "f16"), ([(5000, 1), (1, 1), (129, 1), (777, 1)], 3, 5, 32, "bf16"),
    ([(1000, 4), (4, 4), (65, 2)], 2, 4, 64, "bf16"), ([(300, 8), (8, 8), (31, 5)], 2, 4, 128, "f16"),
    ([(640, 10), (35, 3)], 1, 3, 16, "bf16"), ([(2000, 1)] * 40 + [(40, 0), (0, 0)], 1, 2, 256, "f16"),
]


@pytest.mark.parametrize("i", range(len(FEW)))
def test_attn_few_rows(i):
    reqs, H, G, page, dt = FEW[i]
    attn_case(i, reqs, H, G, page, dt, "head" if i % 2 else "token", pad=i % 3, lead=i % 2)


MANY = [  # chunks of prompts
    ([(33, 33)], 1, 1, 16, "f16"), ([(64, 64)], 2, 4, 64, "bf16"), ([(65, 65), (200, 130)], 1, 4, 16, "f16"),
    ([(700, 300)], 2, 8, 32, "bf16"), ([(1030, 257), (513, 513)], 1, 2, 128, "f16"),
    ([(90, 90), (1000, 11), (61, 60)], 2, 3, 64, "bf16"), ([(1500, 1), (800, 333), (64, 16), (2, 1)], 2, 4, 64, "f16"),
    ([(500, 120)], 1, 7, 1024, "f16"), ([(2600, 70)], 8, 1, 16, "bf16"),
]


@pytest.mark.parametrize("i", range(len(MANY)))
def test_attn_many_rows(i):
    reqs, H, G, page, dt = MANY[i]
    attn_case(100 + i, reqs, H, G, page, dt, "head" if i % 2 else "token", pad=i % 3, lead=i % 2)


CROWDS = [  # more requests than a wave has lanes, than a workgroup has threads, and more (request, head) than waves
    ([(3000, 1)] + [(20 + i, 1) for i in range(69)], 1, 4, 16, "f16"),
    ([(1 + 5 * (i % 7), 1 + (i % 7)) for i in range(330)] + [(900, 2)], 1, 3, 16, "bf16"),
    ([(33 + i % 5, i % 3) for i in range(150)] + [(2500, 4), (600, 1)], 8, 2, 32, "bf16"),
    ([(40 + i, 1 + (i % 3) * 20) for i in range(66)] + [(700, 500), (0, 0)], 2, 4, 32, "f16"),
    ([(64, 33 if i % 90 == 7 else 1) for i in range(300)], 4, 1, 64, "bf16"),
]


@pytest.mark.parametrize("i", range(len(CROWDS)))
@pytest.mark.parametrize("docs", [False, True])
def test_attn_many_requests(i, docs):
    reqs, H, G, page, dt = CROWDS[i]
    attn_case(200 + i, reqs, H, G, page, dt, "head" if i % 2 else "token",
              docs=(lambda s, pos: pos // 50 * 50 + (s % 3 == 0) * 7) if docs else None)


def test_attn_bad_lengths_among_many_requests():
    """One of 70 requests does not fit together, of few rows or of many: BAD_N, its rows are left, the others served."""
    rng = np.random.default_rng(21)
    G, S, bad = 2, 70, 33
    for new in (1, 20):
        news, lengths = [new] * S, [30 + i for i in range(S)]
        table, K, V, Kr, Vr = pools(rng, lengths, 1, 16, torch.float16)
        q = torch.from_numpy(rng.standard_normal((new * S, G, D)).astype(np.float32)).half()
        start = [new * i for i in range(S + 1)]
        said = list(lengths)
        said[bad] = -1 if new == 1 else 10 ** 12
        st = F.new_status()
        out = torch.full((new * S, G, D), 5.0, dtype=torch.float16, device=DEV)
        F.fathom_paged_attn(q.to(DEV), K, V, table, i64(start), i64(said), new, out=out, dev_status=st)
        assert status(st) == F.FATHOM_DEV_BAD_N
        out = out.double().cpu().numpy()
        for s in range(S):
            rows = slice(new * s, new * (s + 1))
            if s == bad:
                assert (out[rows] == 5.0).all()
                continue
            ref, mag, _ = O.paged_attn(q[rows].double().numpy(), Kr[s][0].double().numpy(), Vr[s][0].double().numpy(),
                                       lengths[s], G, 1 / np.sqrt(D))
            assert (np.abs(out[rows] - ref) <= 2.0 ** -11 * np.abs(ref) + mag * (2.0 ** -11 + 1e-4)).all()


@pytest.mark.parametrize("new", [1, 40])
def test_attn_page_numbers_of_every_kind(new):
    """A request of nothing but absent pages gives 0 and BAD_PAGE, whatever the numbers are."""
    rng = np.random.default_rng(22)
    table, K, V, _, _ = pools(rng, [64], 1, 16, torch.bfloat16)
    q = torch.from_numpy(rng.standard_normal((new, 2, D)).astype(np.float32)).bfloat16().to(DEV)
    for bad in (-1, -(1 << 30), -(1 << 31), (1 << 31) - 1, 1 << 30, K.shape[0]):
        table.fill_(bad)
        st = F.new_status()
        out = F.fathom_paged_attn(q, K, V, table, i64([0, new]), i64([64]), new, dev_status=st)
        assert status(st) == F.FATHOM_DEV_BAD_PAGE and (out == 0).all(), bad


@pytest.mark.parametrize("kw", [dict(scale=0.0), dict(scale=0.0, softcap=2.0), dict(softcap=2.0 ** -10), dict(softcap=1024.0),
                                dict(scale=-0.3, softcap=5.0), dict(scale=0.02, bias=True)])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_attn_scales_and_caps(kw, dt):
    attn_case(23, [(300, 1), (200, 70), (64, 6)], 2, 4, 16, dt, **kw)


MIXED = [(400, 1), (300, 150), (90, 5), (129, 64), (40, 40), (700, 2)]


@pytest.mark.parametrize("opt", ["cap", "bias", "prefix", "docs", "all", "scale"])
@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_attn_options(opt, dt):
    kw = {}
    if opt in ("cap", "all"):
        kw["softcap"] = 3.0
    if opt in ("bias", "all"):
        kw["bias"] = True
    if opt in ("prefix", "all"):
        kw["prefix"] = [0, 280, 10, 5000, -3, 699]
    if opt in ("docs", "all"):
        kw["docs"] = lambda s, pos: pos // (37 + 20 * s) * (37 + 20 * s)
    if opt == "scale":
        kw["scale"] = -0.05
    attn_case(7, MIXED, 2, 4, 32, dt, **kw)


@pytest.mark.parametrize("reqs", [[(100, 3), (64, 1), (40, 8)], [(300, 100), (128, 64), (50, 50)]])
def test_attn_rows_that_see_nothing(reqs):
    """first behind the token: an empty row gives 0; first below 0 is 0; the others are as they were."""
    K, V, table, q, out = attn_case(3, reqs, 2, 4, 16, "f16",
                                    docs=lambda s, pos: np.where(pos % 3 == 0, pos + 1 + 10 ** 6 * (pos % 2), -5))
    pos = np.concatenate([n - new + np.arange(new) for n, new in reqs])
    assert (out[torch.from_numpy(pos % 3 == 0).to(DEV)] == 0).all()


@pytest.mark.parametrize("new,n,dt", [(2, 70, "f16"), (1, 45, "bf16"), (60, 150, "bf16"), (100, 100, "f16")])
def test_attn_infinities_in_masked_places(new, n, dt):
    """Values that are not finite, in K and V, reach the rows that see them and no others."""
    rng = np.random.default_rng(11)
    G, t = 4, TYPES[dt]
    table, K, V, Kr, Vr = pools(rng, [n], 1, 16, t)
    place = {"inf": n - 1, "nan": n // 2}
    q = torch.from_numpy(rng.standard_normal((new, G, D)).astype(np.float32)).to(t)
    pg = lambda pool, i: pool[int(table[0, i // 16]), 0, i % 16]  # noqa: E731
    pg(V, place["inf"])[3] = float("inf")
    pg(V, place["inf"])[77] = float("-inf")
    pg(V, place["nan"])[5] = float("nan")
    pg(K, place["nan"])[0] = float("nan")
    pg(K, place["inf"])[1] = float("inf")
    # documents: half of the tokens begin behind the NaN
    first = np.where(np.arange(new) % 2 == 0, place["nan"] + 1, 0)
    out = F.fathom_paged_attn(q.to(DEV), K, V, table, i64([0, new]), i64([n]), new, first=i64(first.tolist())).cpu()
    clean = out[(first > place["nan"]) & (np.arange(new) < new - 1)]
    seen = n - new + np.arange(new)
    for i in range(new):
        ok = first[i] > place["nan"] and i < new - 1 or (seen[i] < place["nan"])
        if ok and first[i] <= seen[i]:
            assert torch.isfinite(out[i]).all(), i
        elif place["nan"] >= first[i] and seen[i] >= place["nan"]:
            assert torch.isnan(out[i]).all(), i  # a NaN score
    assert torch.isfinite(clean).all()
    # V alone: the last token's values are infinite in two channels where its probability is not 0
    pg(K, place["inf"])[1] = 0.0
    out = F.fathom_paged_attn(q.to(DEV), K, V, table, i64([0, new]), i64([n]), new,
                              first=i64([place["nan"] + 1] * new)).cpu().float()
    live = seen > place["nan"]
    assert torch.isfinite(out[:new - 1][live[:-1]]).all()
    last = out[new - 1]
    assert (last[:, 3] == float("inf")).all() and (last[:, 77] == float("-inf")).all()
    assert torch.isfinite(last[:, :3]).all() and torch.isfinite(last[:, 78:]).all()


@pytest.mark.parametrize("new", [2, 50])
def test_attn_absent_pages_are_masked(new):
    rng = np.random.default_rng(12)
    n, G, page = 200, 4, 32
    table, K, V, Kr, Vr = pools(rng, [n, 64], 1, page, torch.float16)
    q = torch.from_numpy(rng.standard_normal((new + 1, G, D)).astype(np.float32)).half()
    for bad in (-1, 10 ** 6, K.shape[0]):
        t = table.clone()
        t[0, 2] = bad
        st = F.new_status()
        out = F.fathom_paged_attn(q.to(DEV), K, V, t, i64([0, new, new + 1]), i64([n, 64]), new, dev_status=st).double().cpu()
        assert status(st) == F.FATHOM_DEV_BAD_PAGE
        keep = np.r_[0:64, 96:n]
        for i in range(new):
            j = keep[keep <= n - new + i]
            for g in range(G):
                z = Kr[0][0, j].double().numpy() @ q[i, g].double().numpy() / np.sqrt(D)
                w = np.exp(z - z.max())
                ref = (w / w.sum()) @ Vr[0][0, j].double().numpy()
                # fp16 rounding of the value and of probabilities around 1, |V| below 5
                assert np.abs(out[i, g].numpy() - ref).max() < 2.0 ** -11 * 10


def test_attn_bad_lengths_leave_rows():
    """A request whose lengths do not fit together is left out with BAD_N; the others are served."""
    rng = np.random.default_rng(13)
    table, K, V, Kr, Vr = pools(rng, [100, 100, 100], 1, 16, torch.float16)
    q = torch.from_numpy(rng.standard_normal((9, 4, D)).astype(np.float32)).half().to(DEV)
    good = F.fathom_paged_attn(q, K, V, table, i64([0, 3, 6, 9]), i64([100, 100, 100]), 3)
    for start, n in (([0, 3, 6, 9], [100, 113, 100]), ([0, 3, 6, 9], [100, -1, 100]), ([0, 3, 6, 9], [100, 2, 100])):
        st = F.new_status()
        out = torch.full((9, 4, D), 5.0, dtype=torch.float16, device=DEV)
        F.fathom_paged_attn(q, K, V, table, i64(start), i64(n), 3, out=out, dev_status=st)
        assert status(st) == F.FATHOM_DEV_BAD_N
        # where the keys are cut depends on all lengths, so the fp32 sums may differ (64 2^-24 of sum p |V| each, |V| < 5),
        # and the values that they round to by one step
        for part in (slice(0, 3), slice(6, 9)):
            x, y = out[part].float(), good[part].float()
            assert ((x - y).abs() <= 2.0 ** -10 * y.abs() + 2 * 64 * 2.0 ** -24 * 5 + 2.0 ** -24).all()
        assert (out[3:6] == 5.0).all()
    for start in ([0, 3, 7, 9], [0, 4, 6, 9]):  # more rows than max_new
        st = F.new_status()
        F.fathom_paged_attn(q, K, V, table, i64(start), i64([100] * 3), 3, dev_status=st)
        assert status(st) == F.FATHOM_DEV_BAD_N
    for start in ([0, 3, 6, 10], [-1, 2, 4, 6], [0, 3, 2, 9]):  # outside the rows, out of order
        st = F.new_status()
        F.fathom_paged_attn(q, K, V, table, i64(start), i64([100] * 3), 9, dev_status=st)
        assert status(st) == F.FATHOM_DEV_BAD_N


def test_attn_offsets_past_32_bits():
    """Pages behind 2^32 bytes and 2^31 elements of the pool, and a long table."""
    P, H, page = 2400, 8, 1024
    K = torch.empty((P, H, page, D), dtype=torch.float16, device=DEV)  # 5 GB
    V = torch.empty_like(K)
    rng = np.random.default_rng(14)
    n = 70
    rows = [torch.from_numpy(rng.standard_normal((H, n, D)).astype(np.float32)).half() for _ in range(2)]
    for pool, r in ((K, rows[0]), (V, rows[1])):
        pool[P - 1].fill_(float("nan"))
        pool[P - 1, :, :n] = r.to(DEV)
    table = torch.full((1, 2000), P - 1, dtype=torch.int32, device=DEV)
    for new in (1, 40):
        q = torch.from_numpy(rng.standard_normal((new, H, D)).astype(np.float32)).half()
        out = F.fathom_paged_attn(q.to(DEV), K, V, table, i64([0, new]), i64([n]), new).double().cpu().numpy()
        for h in range(H):
            ref, mag, _ = O.paged_attn(q[:, h:h + 1].double().numpy(), rows[0][h].double().numpy(),
                                       rows[1][h].double().numpy(), n, 1, 1 / np.sqrt(D))
            assert (np.abs(out[:, h:h + 1] - ref) <= 2.0 ** -11 * np.abs(ref) + mag * (2.0 ** -11 + 1e-4)).all()
    x = torch.ones((1, H, D), dtype=torch.float16, device=DEV)
    F.fathom_paged_write(x, 2 * x, i64([(P - 1) * page + 999]), K, V)
    assert (K[P - 1, :, 999] == 1).all() and (V[P - 1, :, 999] == 2).all()


def test_attn_repeats_bit_for_bit_and_long_split():
    """One long request: its keys are cut over every wave and joined in a fixed order; chunks likewise."""
    for new in (1, 40):
        K, V, table, q, out = attn_case(15, [(9000 + new, new)], 2, 2, 64, "f16")
        again = F.fathom_paged_attn(q, K, V, table, i64([0, new]), i64([9000 + new]), new)
        assert torch.equal(out, again)


@pytest.mark.parametrize("H,G,new,n", [(64, 8, 130, 6300), (64, 8, 130, 700), (24, 8, 100, 1200), (1, 8, 60, 5000)])
def test_attn_splits_of_many_rows(H, G, new, n):
    """Tiles that fill the card, half of it or little, keys cut into parts or not: heads at both ends against 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(24)
    page = 64
    P = O.pages_of(n, page)
    K, V = (torch.randn((P, H, page, D), generator=gen, device=DEV).half() for _ in range(2))
    table = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)[None]
    q = torch.randn((new, H * G, D), generator=gen, device=DEV).half()
    out = F.fathom_paged_attn(q, K, V, table, i64([0, new]), i64([n]), new).double().cpu().numpy()
    for h in {0, H - 1}:
        rows = [x[table[0].long(), h].reshape(-1, D)[:n].double().cpu().numpy() for x in (K, V)]
        mine = slice(h * G, (h + 1) * G)
        ref, mag, top = O.paged_attn(q[:, mine].double().cpu().numpy(), *rows, n, G, 1 / np.sqrt(D))
        tol = 2.0 ** -11 * np.abs(ref) + mag * (2.0 ** -11 + 2 * (D + 8) * 2.0 ** -24 * top[..., None] + 64 * 2.0 ** -24) * 1.001
        assert (np.abs(out[:, mine] - ref) <= tol).all(), h


# ---------------------------------------------------------------- together
class Serving:
    """A serving loop over the paged calls: map, write, attention over all rows; the bit-plane store alongside and
    sparse attention over what its scan selects."""

    def __init__(self, S, H, G, page, L, P, dt=torch.float16):
        self.H, self.G, self.page = H, G, page
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table, self.ring = torch.full((S, L), -1, **i32), torch.arange(P, **i32)
        self.state, self.n = i64([0, P]), i64([0] * S)
        self.K, self.V = (torch.full((P, H, page, D), float("nan"), dtype=dt, device=DEV) for _ in range(2))
        nb = (L * page + 63) // 64
        self.planes = torch.zeros((S * H, D, 4, nb), dtype=torch.int64, device=DEV)
        self.scales = torch.zeros((S * H, D, nb), dtype=torch.int16, device=DEV)
        self.var = torch.ones((S * H, D), device=DEV)
        self.st = F.new_status()

    def step(self, n_new, q, K, V, max_new, k=0):
        H, G, S = self.H, self.G, self.n.numel()
        old = self.n.clone()
        slots, start, self.n, unit, self.state = F.fathom_paged_map(old, n_new, self.page, self.table, self.ring, self.state,
                                                                    q.shape[0], H, dev_status=self.st)
        F.fathom_paged_write(K, V, slots, self.K, self.V, dev_status=self.st)
        out = F.fathom_paged_attn(q, self.K, self.V, self.table, start, self.n, max_new, dev_status=self.st)
        F.fathom_paged_pack(self.K, self.table, self.n, self.planes, self.scales, torch.minimum(old, self.n), max_new,
                            dev_status=self.st)
        if not k:
            return out, None, None
        qu = q.reshape(S, H, G, D).reshape(S * H, G, D).contiguous()
        dep, _ = F.fathom_alloc_depths(qu, self.var, F.FATHOM_WATERFILL, 48, dev_status=self.st)
        idx, _ = F.fathom_scan_topk(self.planes, self.scales, unit, qu, dep, k, 4, 8, dev_status=self.st, max_unit_bits=48)
        return out, idx, F.fathom_paged_sparse_attn(qu, self.K, self.V, self.table, self.n, idx, 4, 8, dev_status=self.st)


def test_serving_loop_equals_contiguous():
    """Prompts of uneven length, decode steps, one request ends and another takes its place: the paged calls give what the
    contiguous ones give over the same rows."""
    rng = np.random.default_rng(16)
    S, H, G, page, L = 3, 2, 4, 16, 30
    sv = Serving(S, H, G, page, L, 70)
    kept = [[torch.zeros((H, 0, D), dtype=torch.float16) for _ in range(2)] for _ in range(S)]

    def step(news, k, ends=()):
        for s in ends:
            kept[s] = [torch.zeros((H, 0, D), dtype=torch.float16) for _ in range(2)]
        T = sum(news)
        rows = [torch.from_numpy(rng.standard_normal((T, m, D)).astype(np.float32)).half() for m in (H * G, H, H)]
        at = 0
        for s, m in enumerate(news):
            for i in range(2):
                kept[s][i] = torch.cat([kept[s][i], rows[1 + i][at:at + m].transpose(0, 1)], 1)
            at += m
        n = [x[0].shape[1] for x in kept]
        out, idx, sparse = sv.step(i64(n), *(r.to(DEV) for r in rows), max(news), k)
        assert status(sv.st) & ~F.FATHOM_DEV_TOPK_FALLBACK == 0 and sv.n.tolist() == n
        at = 0
        for s, m in enumerate(news):
            for h in range(H):
                ref, mag, _ = O.paged_attn(rows[0][at:at + m, h * G:(h + 1) * G].double().numpy(),
                                           kept[s][0][h].double().numpy(), kept[s][1][h].double().numpy(), n[s], G,
                                           1 / np.sqrt(D))
                err = np.abs(out[at:at + m, h * G:(h + 1) * G].double().cpu().numpy() - ref)
                assert (err <= 2.0 ** -11 * np.abs(ref) + mag * (2.0 ** -11 + 1e-4)).all()
            at += m
        cap = max(n)
        flat = [torch.zeros((S * H, cap, D), dtype=torch.float16) for _ in range(2)]
        for s in range(S):
            for i in range(2):
                flat[i][s * H:(s + 1) * H, :n[s]] = kept[s][i]
        Kf, Vf = (f.to(DEV) for f in flat)
        nu = i64(n).repeat_interleave(H)
        planes, scales = F.fathom_pack(Kf, nu, sv.scales.shape[-1])
        for u in range(S * H):
            nb = (n[u // H] + 63) // 64
            assert torch.equal(planes[u, :, :, :nb], sv.planes[u, :, :, :nb])
            assert torch.equal(scales[u, :, :nb], sv.scales[u, :, :nb])
        if k:
            qu = rows[0].view(S * H, G, D).to(DEV)
            dep, _ = F.fathom_alloc_depths(qu, sv.var, F.FATHOM_WATERFILL, 48)
            wi, _ = F.fathom_scan_topk(planes, scales, nu, qu, dep, k, 4, 8, max_unit_bits=48)
            assert torch.equal(wi, idx)
            assert torch.equal(F.fathom_sparse_attn(qu, Kf, Vf, nu, wi, 4, 8), sparse)

    step([130, 63, 64], 0)
    for _ in range(3):
        step([1, 1, 1], 20)
    # request 1 ends: its pages go back, and the next call may take them
    old = sv.n.clone()
    _, _, sv.n, _, sv.state = F.fathom_paged_map(old, i64([old[0], 0, old[2]]), page, sv.table, sv.ring, sv.state, 0, H,
                                                 dev_status=sv.st)
    kept[1] = [torch.zeros((H, 0, D), dtype=torch.float16) for _ in range(2)]
    step([1, 200, 30], 0)
    for _ in range(2):
        step([1, 1, 1], 20)


def test_two_graphs_and_two_streams():
    """Decode steps captured into two graphs that share one workspace, replayed several times with other work between;
    and calls on two streams at once, each with its own workspace."""
    rng = np.random.default_rng(17)
    H, G, page = 2, 4, 32
    sets = []
    for lengths in ([500, 90, 1300], [64, 2000, 33]):
        table, K, V, _, _ = pools(rng, lengths, H, page, torch.float16)
        q = torch.zeros((3, H * G, D), dtype=torch.float16, device=DEV)
        out = torch.zeros_like(q)
        sets.append(dict(q=q, K=K, V=V, table=table, start=i64([0, 1, 2, 3]), n=i64(lengths), out=out))
    ws = torch.empty((F.fathom_paged_attn_workspace_size(3, 3, H, G, 1),), dtype=torch.uint8, device=DEV)

    def call(s, ws, stream=None):
        return F.fathom_paged_attn(s["q"], s["K"], s["V"], s["table"], s["start"], s["n"], 1, out=s["out"], ws=ws,
                                   stream=stream)

    graphs = []
    for s in sets:
        call(s, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(s, ws)
        graphs.append(g)
    for rep in range(3):
        want = []
        for s in sets:
            s["q"].copy_(torch.from_numpy(rng.standard_normal(s["q"].shape).astype(np.float32)).half())
            call(s, torch.empty_like(ws))
            want.append(s["out"].clone())
            s["out"].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(sets, want):
            assert torch.equal(s["out"], w)
    streams = [torch.cuda.Stream() for _ in sets]
    own = [torch.empty_like(ws) for _ in sets]
    for s in sets:
        s["out"].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for s, w, x in zip(sets, own, streams):
            call(s, w, stream=x)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        assert torch.equal(s["out"], w)


def test_a_step_of_all_calls_in_a_graph():
    """Map, write, attention, pack and sparse attention captured together; lengths and rows change between replays, a
    request ends and begins again.  Every replay gives what the same calls give eagerly on a state of their own."""
    rng = np.random.default_rng(25)
    S, H, G, page, L, P, k = 3, 2, 4, 16, 20, 60, 30
    i32 = dict(dtype=torch.int32, device=DEV)
    half = dict(dtype=torch.float16, device=DEV)
    idx = torch.from_numpy(rng.integers(0, 200, (S * H, G, k)).astype(np.int32)).to(DEV)

    def state():
        nb = (L * page + 63) // 64
        return dict(table=torch.full((S, L), -1, **i32), ring=torch.arange(P, **i32), head=i64([0, P]), n=i64([0] * S),
                    to=i64([0] * S), K=torch.zeros((P, H, page, D), **half), V=torch.zeros((P, H, page, D), **half),
                    planes=torch.zeros((S * H, D, 4, nb), dtype=torch.int64, device=DEV),
                    scales=torch.zeros((S * H, D, nb), dtype=torch.int16, device=DEV), st=F.new_status())

    def step(x, rows, max_new):
        slots, start, now, unit, _ = F.fathom_paged_map(x["n"], x["to"], page, x["table"], x["ring"], x["head"],
                                                        rows["q"].shape[0], H, state_out=x["head"], dev_status=x["st"])
        F.fathom_paged_write(rows["K"], rows["V"], slots, x["K"], x["V"], dev_status=x["st"])
        out = torch.zeros_like(rows["q"])
        F.fathom_paged_attn(rows["q"], x["K"], x["V"], x["table"], start, now, max_new, out=out, dev_status=x["st"])
        F.fathom_paged_pack(x["K"], x["table"], now, x["planes"], x["scales"], torch.minimum(x["n"], now), max_new,
                            dev_status=x["st"])
        sparse = F.fathom_paged_sparse_attn(rows["qs"], x["K"], x["V"], x["table"], now, idx, 2, 5, dev_status=x["st"])
        torch.add(now, 0, out=x["n"])
        return out, sparse, unit

    def new_rows(T):
        r = {m: torch.from_numpy(rng.standard_normal((T, c, D)).astype(np.float32)).half().to(DEV)
             for m, c in (("q", H * G), ("K", H), ("V", H))}
        r["qs"] = torch.from_numpy(rng.standard_normal((S * H, G, D)).astype(np.float32)).to(DEV)
        return r

    a, b = state(), state()
    prompts = new_rows(130 + 63 + 64)
    for x in (a, b):
        x["to"].copy_(i64([130, 63, 64]))
        step(x, prompts, 130)
    rows = new_rows(S)
    torch.cuda.synchronize()
    kept = {m: x.clone() for m, x in b.items()}  # the capture's warm-up below moves it
    b["to"].copy_(b["n"] + 1)
    step(b, rows, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(b, rows, 1)
    for m, x in kept.items():
        b[m].copy_(x)
    n = [130, 63, 64]
    for i in range(6):
        n = [n[0] + 1, 0 if i == 2 else n[1] + 1, n[2] + (i != 4)]
        fresh = new_rows(S)
        for m in rows:
            rows[m].copy_(fresh[m])
        for x in (a, b):
            x["to"].copy_(i64(n))
        want = step(a, rows, 1)
        graph.replay()
        torch.cuda.synchronize()
        assert b["n"].tolist() == n and status(a["st"]) == status(b["st"]) == 0, i
        for w, g in zip(want, got):
            assert torch.equal(w, g), i
        for m in ("table", "ring", "head", "K", "V", "planes", "scales"):
            assert torch.equal(a[m], b[m]), (i, m)


@pytest.mark.parametrize("new", [1, 30])
def test_interleaved_pools_and_shared_pages(new):
    """K and V in one buffer (strides of their own), and two requests that begin with the same pages."""
    rng = np.random.default_rng(26)
    H, G, page, n = 2, 3, 16, 90
    buf = torch.full((20, 2, H, page, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    K, V = buf[:, 0], buf[:, 1]
    table = torch.tensor([[3, 9, 1, 4, 12, 7], [3, 9, 1, 15, 2, 6]], dtype=torch.int32, device=DEV)
    slots = lambda s, lo, hi: i64([int(table[s, p // page]) * page + p % page for p in range(lo, hi)])  # noqa: E731
    kv = [torch.from_numpy(rng.standard_normal((n, H, D)).astype(np.float32)).bfloat16() for _ in range(4)]
    for s in range(2):  # the first 48 rows are request 0's for both
        lo = 0 if s == 0 else 48
        F.fathom_paged_write(kv[2 * s][lo:].to(DEV), kv[2 * s + 1][lo:].to(DEV), slots(s, lo, n), K, V)
    for i in (2, 3):
        kv[i][:48] = kv[i - 2][:48]
    q = torch.from_numpy(rng.standard_normal((2 * new, H * G, D)).astype(np.float32)).bfloat16()
    out = F.fathom_paged_attn(q.to(DEV), K, V, table, i64([0, new, 2 * new]), i64([n, n]), new).double().cpu().numpy()
    eps = 2.0 ** -8
    for s in range(2):
        for h in range(H):
            mine = slice(s * new, (s + 1) * new), slice(h * G, (h + 1) * G)
            ref, mag, _ = O.paged_attn(q[mine].double().numpy(), kv[2 * s][:, h].double().numpy(),
                                       kv[2 * s + 1][:, h].double().numpy(), n, G, 1 / np.sqrt(D))
            assert (np.abs(out[mine] - ref) <= eps * np.abs(ref) + mag * (eps + 1e-4)).all()
    nn = i64([n, n])
    planes = torch.empty((2 * H, D, 4, 2), dtype=torch.int64, device=DEV)
    scales = torch.empty((2 * H, D, 2), dtype=torch.int16, device=DEV)
    F.fathom_paged_pack(K, table, nn, planes, scales)
    flat = [torch.stack([kv[2 * s + i][:, h] for s in range(2) for h in range(H)]).to(DEV) for i in range(2)]
    want = F.fathom_pack(flat[0].float(), nn.repeat_interleave(H), 2)
    assert torch.equal(planes, want[0]) and torch.equal(scales, want[1])


# ---------------------------------------------------------------- one request under loose bounds
def close(got, q, K, V, n, G, chunk, sm=1 / np.sqrt(D)):
    """Whether the rows [new][G][D] of one request and head are within the tolerance above; chunk: probabilities are
    rounded once.  Outputs below the type's normal numbers are off by half of their step."""
    t = q.dtype
    eps = torch.finfo(t).eps
    ref, mag, top = O.paged_attn(q.double().numpy(), K.double().numpy(), V.double().numpy(), n, G, sm)
    dz = (D + 8) * 2.0 ** -24 * top[..., None]
    tol = eps / 2 * np.abs(ref) + mag * ((eps / 2 if chunk else eps * eps) + 2 * dz + 64 * 2.0 ** -24) * (1 + eps)
    return (np.abs(got.double().cpu().numpy() - ref) <= tol + torch.finfo(t).smallest_normal * eps / 2).all()


@pytest.mark.parametrize("new", [0, 1, "few", "more"])
@pytest.mark.parametrize("H,G,n,T,max_new,lead,dt", [(2, 4, 150, 16, 16, 0, "f16"), (2, 4, 3000, 64, 64, 3, "bf16"),
                                                     (8, 4, 200, 2048, 2048, 5, "f16"), (1, 8, 100, 40, 33, 3, "bf16"),
                                                     (2, 1, 90, 100, 64, 1, "f16"), (1, 3, 5000, 300, 1 << 40, 7, "bf16")])
def test_attn_one_request_below_its_bounds(H, G, n, T, max_new, lead, dt, new):
    """max_new and T are bounds: one request may have any number of tokens below them, few query rows among them."""
    new = {"few": 32 // G, "more": 32 // G + 1}.get(new, new)
    rng = np.random.default_rng(31)
    table, K, V, Kr, Vr = pools(rng, [n], H, 32, TYPES[dt])
    q = torch.from_numpy(rng.standard_normal((T, H * G, D)).astype(np.float32) * 2).to(TYPES[dt])
    out, st = torch.full((T, H * G, D), 5.0, dtype=TYPES[dt], device=DEV), F.new_status()
    F.fathom_paged_attn(q.to(DEV), K, V, table, i64([lead, lead + new]), i64([n]), max_new, out=out, dev_status=st)
    assert status(st) == 0
    mine = slice(lead, lead + new)
    for h in range(H if new else 0):
        heads = slice(h * G, (h + 1) * G)
        assert close(out[mine, heads], q[mine, heads], Kr[0][h], Vr[0][h], n, G, True), h
    out[mine] = 5.0
    assert (out == 5.0).all()


def test_attn_one_request_in_a_graph_with_other_lengths():
    """A call captured for up to 16 tokens, replayed with fewer, none and all of them."""
    rng = np.random.default_rng(32)
    H, G, T, n = 2, 4, 16, 300
    table, K, V, Kr, Vr = pools(rng, [n], H, 16, torch.float16)
    q = torch.from_numpy(rng.standard_normal((T, H * G, D)).astype(np.float32) * 2).half()
    qd, start, out = q.to(DEV), i64([0, T]), torch.zeros((T, H * G, D), dtype=torch.float16, device=DEV)
    ws = torch.empty((F.fathom_paged_attn_workspace_size(T, 1, H, G, T),), dtype=torch.uint8, device=DEV)

    def call():
        return F.fathom_paged_attn(qd, K, V, table, start, i64n, T, out=out, ws=ws)

    i64n = i64([n])
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for a, b in ((0, 16), (0, 1), (3, 11), (5, 5), (7, 16), (15, 16)):
        start.copy_(i64([a, b]))
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        for h in range(H if b > a else 0):
            heads = slice(h * G, (h + 1) * G)
            assert close(out[a:b, heads], q[a:b, heads], Kr[0][h], Vr[0][h], n, G, True), (a, b)
        assert (out[:a] == 5.0).all() and (out[b:] == 5.0).all()


# ---------------------------------------------------------------- streams
def pool_of(stream):
    """Address ranges of the memory that the allocator keeps for a stream."""
    return [(x["address"], x["address"] + x["total_size"]) for x in torch.cuda.memory_snapshot()
            if x["stream"] == stream.cuda_stream]


def test_what_a_call_makes_is_of_its_stream():
    """With stream= given, outputs and workspaces made by a call lie in that stream's memory (the current stream's may be
    handed out again while the call runs), for the paged calls and those over contiguous rows."""
    rng = np.random.default_rng(35)
    H, G, n = 2, 4, 500
    table, K, V, _, _ = pools(rng, [n], H, 16, torch.float16, fill=0.0)
    q = torch.from_numpy(rng.standard_normal((1, H * G, D)).astype(np.float32)).half().to(DEV)
    qu, flat = q.view(H, G, D), torch.randn((H, n, D), device=DEV)
    rows = flat.half()
    nn, nu, var = i64([n]), i64([n] * H), torch.ones((H, D), device=DEV)
    idx = torch.arange(60, dtype=torch.int32, device=DEV).expand(H, G, 60).contiguous()
    torch.cuda.synchronize()
    x = torch.cuda.Stream()
    kw = dict(stream=x)
    made = [F.fathom_paged_attn(q, K, V, table, i64([0, 1]), nn, 1, **kw)]
    need = F.fathom_paged_attn_workspace_size(1, 1, H, G, 1)
    assert sum(b - a for a, b in pool_of(x)) >= need  # the workspace was there
    made += F.fathom_paged_map(nn, nn + 1, 16, table.clone(), torch.arange(8, dtype=torch.int32, device=DEV), i64([0, 8]), 1,
                               H, **kw)
    made += [F.fathom_paged_sparse_attn(qu, K, V, table, nn, idx, **kw), F.fathom_sparse_attn(qu, rows, rows, nu, idx, **kw)]
    planes, scales = F.fathom_pack(flat, nu, **kw)
    dep, th = F.fathom_alloc_depths(qu, var, **kw)
    scores = F.fathom_scan(planes, scales, nu, qu, dep, **kw)
    made += [planes, scales, dep, th, scores, *F.fathom_topk(scores, nu, 30, **kw)]
    made += F.fathom_scan_topk(planes, scales, nu, qu, dep, 30, **kw)
    mu, basis, lam = F.fathom_klt_calibrate(flat, nu, **kw)
    made += [mu, basis, lam, F.fathom_klt_rotate_keys(flat, nu, mu, basis, **kw), F.fathom_klt_rotate_q(qu, basis, **kw)]
    torch.cuda.synchronize()
    ranges = pool_of(x)
    for i, t in enumerate(made):
        assert any(a <= t.data_ptr() < b for a, b in ranges), (i, t.shape)


def test_calls_on_two_streams_make_their_own_workspaces():
    """Calls on two streams in turn, each with a workspace and an output of its own making."""
    rng = np.random.default_rng(36)
    H, G = 2, 4
    cases = []
    for lengths, new in (([3000, 90], 1), ([64, 5000], 1), ([700, 400], 90), ([9000, 20], 8)):
        table, K, V, _, _ = pools(rng, lengths, H, 32, torch.float16)
        news = [min(new, m) for m in lengths]
        q = torch.from_numpy(rng.standard_normal((sum(news), H * G, D)).astype(np.float32)).half().to(DEV)
        cases.append((q, K, V, table, i64([0, news[0], sum(news)]), i64(lengths), max(news)))
    want = [F.fathom_paged_attn(*c) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        got = [F.fathom_paged_attn(*c, stream=streams[i % 2]) for i, c in enumerate(cases)]
        torch.cuda.synchronize()
        for w, g in zip(want, got):
            assert torch.equal(w, g)


def test_a_stream_of_another_device_is_refused():
    class Other:  # as a torch stream of the next device looks
        device_index, cuda_stream = torch.cuda.current_device() + 1, 0

    K, V = (torch.zeros((2, 1, 16, D), dtype=torch.float16, device=DEV) for _ in range(2))
    x = torch.ones((1, 1, D), dtype=torch.float16, device=DEV)
    with pytest.raises(ValueError, match="stream of the current device"):
        F.fathom_paged_write(x, x, i64([3]), K, V, stream=Other())
    F.fathom_paged_write(x, x, i64([3]), K, V, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert (K[0, 0, 3] == 1).all() and float(K.float().sum()) == D


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("n,new", [(64, 1), (64, 3), (160, 1), (600, 4), (5000, 1), (40000, 1), (130, 60), (3000, 60)])
def test_attn_infinities_in_seen_places(n, new, dt):
    """A value of V that is not finite reaches every token that sees its row, wherever the row lies in a block and however
    small its probability is: Inf as Inf, Inf of both signs and NaN as NaN.  Other channels, heads and tokens are as if it
    were not there."""
    t, G = TYPES[dt], 4
    for seed in range(3):
        rng = np.random.default_rng(40 + seed)
        table, K, V, Kr, Vr = pools(rng, [n], 2, 16, t)
        row = lambda pool, i: pool[int(table[0, i // 16]), 0, i % 16]  # noqa: E731
        q = torch.from_numpy(np.abs(rng.standard_normal((new, 2 * G, D))).astype(np.float32)).to(t)
        # key 7 scores about -900 and the last old one about +180: after it, earlier keys' probabilities are below 2^-149
        for i, x in ((7, -100.0), (n - new - 1, 20.0)):
            row(K, i).fill_(x)
            Kr[0][0, i] = x
        inf = float("inf")
        for i, c, x in ((5, 3, inf), (5, 77, -inf), (5, 9, inf), (41, 9, -inf), (33, 20, float("nan")), (7, 50, inf),
                        (n - new - 1, 100, -inf), (45, 60, inf)):
            row(V, i)[c] = x
            Vr[0][0, i, c] = 0.0
        first = np.where(np.arange(new) % 2 == 1, 12, 0)  # the odd tokens do not see keys 5 and 7
        out, st = torch.empty((new, 2 * G, D), dtype=t, device=DEV), F.new_status()
        F.fathom_paged_attn(q.to(DEV), K, V, table, i64([0, new]), i64([n]), new, first=i64(first.tolist()), out=out,
                            dev_status=st)
        assert status(st) == 0
        out = out.cpu().double()
        even, odd = out[0::2, :G], out[1::2, :G]
        assert (even[..., 3] == inf).all() and (even[..., 77] == -inf).all() and (even[..., 50] == inf).all()
        assert torch.isnan(even[..., 9]).all() and (odd[..., 9] == -inf).all()
        for part in (even, odd):
            assert torch.isnan(part[..., 20]).all() and (part[..., 100] == -inf).all() and (part[..., 60] == inf).all()
        eps = torch.finfo(t).eps
        for h in range(2):
            got = out[:, h * G:(h + 1) * G].numpy()
            ref, mag, top = O.paged_attn(q[:, h * G:(h + 1) * G].double().numpy(), Kr[0][h].double().numpy(),
                                         Vr[0][h].double().numpy(), n, G, 1 / np.sqrt(D), first=first)
            # the tolerance above; head 0's scores reach some hundreds, whose fp32 error its last term counts
            tol = eps / 2 * np.abs(ref) + mag * ((eps / 2 if new * G > 32 else eps * eps) + 64 * 2.0 ** -24 +
                                                 2 * (D + 8) * 2.0 ** -24 * top[..., None]) * (1 + eps) + 2.0 ** -25
            on = np.ones((new, G, D), bool)
            if h == 0:
                on[:, :, [9, 20, 60, 100]] = False
                on[0::2, :, [3, 50, 77]] = False
            err = np.abs(np.where(on, got, ref) - ref)
            assert (err <= tol).all(), (seed, h)


def test_sparse_and_dense_agree_on_infinities():
    """One token over all of its rows, dense and selected: infinities come out alike."""
    rng = np.random.default_rng(44)
    n = 96
    table, K, V, _, _ = pools(rng, [n], 1, 16, torch.float16)
    for i, c in ((0, 1), (40, 2), (95, 3)):
        V[int(table[0, i // 16]), 0, i % 16, c] = float("inf")
    q = torch.from_numpy(rng.standard_normal((1, 4, D)).astype(np.float32)).half().to(DEV)
    idx = torch.arange(n, dtype=torch.int32, device=DEV).expand(1, 4, n).contiguous()
    a = F.fathom_paged_attn(q, K, V, table, i64([0, 1]), i64([n]), 1).float()
    b = F.fathom_paged_sparse_attn(q, K, V, table, i64([n]), idx)
    assert torch.equal(torch.isinf(a), torch.isinf(b)) and torch.isinf(a[..., 1:4]).all()


def test_write_up_to_its_limit_of_rows():
    """2^28 rows and more (of one source row, stride 0): more threads than a grid's axis counts."""
    H, page, P = 1024, 16, 3
    K, V = (torch.zeros((P, H, page, D), dtype=torch.float16, device=DEV) for _ in range(2))
    x = torch.arange(D, dtype=torch.float32, device=DEV).half()
    for T in ((1 << 18), (1 << 18) + 5, 1 << 20):
        K.zero_(), V.zero_()
        slots = torch.full((T,), -1, dtype=torch.int64, device=DEV)
        at = {0: 3, T // 2: 17, T - 1: P * page - 1}
        for i, s in at.items():
            slots[i] = s
        F.fathom_paged_write(x.expand(T, H, D), (2 * x).expand(T, H, D), slots, K, V)
        for pool, want in ((K, x), (V, 2 * x)):
            rows = pool.transpose(1, 2).reshape(P * page, H, D)
            for s in range(P * page):
                assert (rows[s] == (want if s in at.values() else 0 * want)).all(), (T, s)


# ---------------------------------------------------------------- map, more
@pytest.mark.parametrize("S,page,L", [(3, 16, 5), (64, 32, 9), (300, 16, 40), (1500, 64, 20)])
@pytest.mark.parametrize("alias", ["n", "n and state", "n_old"])
def test_map_in_place_of_its_inputs(S, page, L, alias):
    """n_now may be n or n_old, state_out may be state: the same results, in one workgroup and in two launches."""
    rng = np.random.default_rng(S + 1)
    n_old, n, table, ring, state, T = random_map(rng, S, page, L, 3, 4)
    want = O.paged_map(n_old, n, page, table, ring, state, T, 2)
    t, r, st = torch.from_numpy(table).to(DEV), torch.from_numpy(ring).to(DEV), F.new_status()
    a, b, s0 = i64(n_old), i64(n), i64(state)
    kw = dict(n_now=a if alias == "n_old" else b)
    if "state" in alias:
        kw["state_out"] = s0
    got = F.fathom_paged_map(a, b, page, t, r, s0, T, 2, dev_status=st, **kw)
    for name, g, w in zip(("table", "ring", "slots", "start", "n_now", "n_unit", "state"), (t, r, *got), want):
        assert np.array_equal(g.cpu().numpy(), w), name
    assert status(st) == (F.FATHOM_DEV_PAGES_SHORT if want[7] else 0) | (F.FATHOM_DEV_BAD_N if want[8] else 0)


def test_a_step_with_too_few_pages():
    """The ring runs dry in the middle of a step: requests that are served come out right, the rows of one that is not are
    the last of its old tokens to the attention, or left where it has fewer, and what is cached stays as it was."""
    rng = np.random.default_rng(37)
    H, G, page, L = 2, 4, 16, 12
    old, new = [40, 30, 5, 64, 50], [12, 40, 30, 1, 20]  # two free pages: request 0 takes one, request 1 wants three
    n = [a + b for a, b in zip(old, new)]
    table, K, V, Kr, Vr = pools(rng, old, H, page, torch.float16, spare=2)
    table = torch.cat([table, torch.full((5, L - table.shape[1]), -1, dtype=torch.int32, device=DEV)], 1)
    P = K.shape[0]
    free = sorted(set(range(P)) - set(table[table >= 0].tolist()))
    ring = torch.tensor(free + [-1] * (P - len(free)), dtype=torch.int32, device=DEV)
    T, st = sum(new), F.new_status()
    rows = [torch.from_numpy(rng.standard_normal((T, m, D)).astype(np.float32)).half() for m in (H * G, H, H)]
    slots, start, now, _, state = F.fathom_paged_map(i64(old), i64(n), page, table, ring, i64([0, len(free)]), T, H,
                                                     dev_status=st)
    assert status(st) == F.FATHOM_DEV_PAGES_SHORT
    served = (now == i64(n)).tolist()  # how a caller tells them
    assert served == [True, False, False, False, False]
    assert start.tolist() == [0, *np.cumsum(new).tolist()] and now.tolist() == [52, 30, 5, 64, 50]
    before = K.clone(), V.clone()
    F.fathom_paged_write(rows[1].to(DEV), rows[2].to(DEV), slots, K, V, dev_status=st)
    out = torch.full((T, H * G, D), 5.0, dtype=torch.float16, device=DEV)
    F.fathom_paged_attn(rows[0].to(DEV), K, V, table, start, now, max(new), out=out, dev_status=st)
    assert status(st) == F.FATHOM_DEV_PAGES_SHORT | F.FATHOM_DEV_BAD_N  # requests 1 and 2 have more rows than tokens
    for s in range(5):
        a, b = sum(new[:s]), sum(new[:s + 1])
        if not served[s] and new[s] > old[s]:
            assert (out[a:b] == 5.0).all()
            continue
        for h in range(H):
            kv = [x[s][h] for x in (Kr, Vr)]
            if served[s]:
                kv = [torch.cat([x, y[a:b, h]]) for x, y in zip(kv, rows[1:])]
            heads = slice(h * G, (h + 1) * G)
            m = n[s] if served[s] else old[s]
            assert close(out[a:b, heads], rows[0][a:b, heads], *kv, m, G, new[s] * G > 32), (s, h)
    taken = sorted({int(x) // page for x in slots.tolist() if x >= 0})
    kept = [p for p in range(P) if p not in taken]
    for x, y in zip(before, (K, V)):
        assert torch.equal(x[kept].nan_to_num(9.0), y[kept].nan_to_num(9.0))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("slope", [2.0 ** 16, 2.0 ** 20, 1e6])
def test_attn_bias_that_leaves_one_key(slope, new, dt):
    """Scores of far keys of -10^9 and below: the probabilities taken against them stay finite, and a token is left with its
    own key."""
    rng = np.random.default_rng(33)
    n, t = 20000, TYPES[dt]
    table, K, V, _, Vr = pools(rng, [n], 1, 64, t)
    q = torch.from_numpy(rng.standard_normal((new, 2, D)).astype(np.float32)).to(t).to(DEV)
    out = F.fathom_paged_attn(q, K, V, table, i64([0, new]), i64([n]), new,
                              slopes=torch.full((2,), slope, dtype=torch.float32, device=DEV)).cpu()
    assert torch.equal(out, Vr[0][0, n - new:, None].expand(new, 2, D))


@pytest.mark.parametrize("new", [1, 40])
def test_attn_large_scores(new):
    """One key's score is 2^25, the others' some tens: it is all that counts."""
    rng = np.random.default_rng(34)
    n = 300
    table, K, V, Kr, Vr = pools(rng, [n], 1, 16, torch.float16, scale=0.01)
    K[int(table[0, 100 // 16]), 0, 100 % 16] = 1024.0
    q = torch.full((new, 2, D), 1024.0, dtype=torch.float16, device=DEV)
    out = F.fathom_paged_attn(q, K, V, table, i64([0, new]), i64([n]), new, sm_scale=0.25).cpu()
    assert torch.equal(out, Vr[0][0, 100].expand(new, 2, D))


@pytest.mark.parametrize("max_new", [64, 1 << 40, (1 << 63) - 1])
def test_pack_append_under_any_bound(max_new):
    """max_new is a bound on new tokens, however large: paged or not, the store grows by what there is."""
    rng = np.random.default_rng(38)
    lengths, H = [500, 129], 2
    table, K, _, Kr, _ = pools(rng, lengths, H, 16, torch.float16)
    flat = torch.zeros((4, 500, D))
    for s, n in enumerate(lengths):
        flat[2 * s:2 * s + 2, :n] = Kr[s].float()
    flat, n, st = flat.to(DEV), i64(lengths), F.new_status()
    nu = n.repeat_interleave(H)
    want = F.fathom_pack(flat, nu)
    for call in ("paged", "fp32", "fp16"):
        p, s = F.fathom_pack(flat, nu - 50)
        if call == "paged":
            F.fathom_paged_pack(K, table, n, p, s, n - 50, max_new, dev_status=st)
        else:
            F.fathom_pack_append(flat if call == "fp32" else flat.half(), nu - 50, nu, max_new, p, s, dev_status=st)
        assert torch.equal(p, want[0]) and torch.equal(s, want[1]) and status(st) == 0, call
