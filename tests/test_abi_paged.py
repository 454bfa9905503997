"""CPU checks of the paged calls: argument errors are found on the host before any launch, and the plain map of
oracle/paged.py does what the header says.  No call here reaches a kernel."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import paged as P


@pytest.fixture(scope="module")
def fl():
    import paper_2609_17652_amd as F
    if not os.path.exists(F.LIB_PATH):
        from paper_2609_17652_amd import build
        build.build()
    return F


FAKE, ODD = 0x10000, 0x10004  # never dereferenced
S0 = C.c_void_p(0)


def _pg(fl, **kw):
    d = dict(K=FAKE, V=FAKE, dt=1, H=2, page=64, P=10, ld_page=2 * 64 * 128, ld_head=64 * 128, ld_tok=128)
    d.update(kw)
    return fl._Pages(**d)


BAD_PAGES = [(dict(dt=0), "UNSUPPORTED"), (dict(dt=5), "UNSUPPORTED"), (dict(H=0), "UNSUPPORTED"),
             (dict(H=1025), "UNSUPPORTED"), (dict(page=8), "UNSUPPORTED"), (dict(page=48), "UNSUPPORTED"),
             (dict(page=2048), "UNSUPPORTED"), (dict(P=-1), "INVALID"), (dict(P=1 << 31), "UNSUPPORTED"),
             (dict(ld_tok=120), "INVALID"), (dict(ld_tok=132), "INVALID"), (dict(ld_tok=(1 << 20) + 8), "UNSUPPORTED"),
             (dict(ld_head=4), "INVALID"), (dict(ld_page=-8), "INVALID"), (dict(K=0), "INVALID"), (dict(K=ODD), "INVALID")]


def _attn(fl, pg, S=1, T=1, D=128, G=4, max_new=1, scale=1.0, cap=0.0, q=FAKE, ldq=128, out=FAKE, ws=FAKE, ws_bytes=None,
          ld_table=4, table=FAKE, start=FAKE, n=FAKE, first=None):
    need = fl.fathom_paged_attn_workspace_size(T, S, 2, G, max_new)
    return fl.lib().fathom_paged_attn(q, ldq, 128, C.byref(pg), table, ld_table, start, n, S, T, max_new, G, D,
                                      C.c_float(scale), C.c_float(cap), None, None, first, out, ws,
                                      need if ws_bytes is None else ws_bytes, None, S0)


@pytest.mark.parametrize("change,code", BAD_PAGES)
def test_pages_are_checked_by_every_call(fl, change, code):
    want = getattr(fl, "FATHOM_ERR_" + code)
    L, pg = fl.lib(), _pg(fl, **change)
    assert _attn(fl, pg) == want
    assert L.fathom_paged_write(FAKE, FAKE, 1, 256, 128, 256, 128, FAKE, 1, 128, C.byref(pg), None, S0) == want
    assert L.fathom_paged_pack(C.byref(pg), FAKE, 4, None, FAKE, 0, 1, 128, 4, FAKE, FAKE, None, S0) == want
    assert L.fathom_paged_sparse_attn(FAKE, 0, C.byref(pg), FAKE, 4, FAKE, 1, 4, 128, FAKE, 8, 4, 32, C.c_float(1.0), FAKE,
                                      FAKE, 1 << 20, None, S0) == want


def test_attn_refusals(fl):
    pg = _pg(fl)
    I, U, W = fl.FATHOM_ERR_INVALID, fl.FATHOM_ERR_UNSUPPORTED, fl.FATHOM_ERR_WORKSPACE
    assert _attn(fl, pg, D=64) == U
    assert _attn(fl, pg, G=0) == U and _attn(fl, pg, G=9) == U
    assert _attn(fl, pg, S=4097) == U and _attn(fl, pg, S=-1) == I
    assert _attn(fl, pg, T=-1) == I and _attn(fl, pg, max_new=-1) == I
    assert _attn(fl, pg, T=1 << 30) == U
    assert _attn(fl, pg, scale=float("nan")) == I and _attn(fl, pg, scale=float("inf")) == I
    assert _attn(fl, pg, cap=-1.0) == I and _attn(fl, pg, cap=float("nan")) == I and _attn(fl, pg, cap=float("inf")) == I
    assert _attn(fl, pg, ldq=4) == I and _attn(fl, pg, ldq=-128) == I
    assert _attn(fl, pg, q=ODD) == I and _attn(fl, pg, out=ODD) == I and _attn(fl, pg, first=ODD) == I
    assert _attn(fl, pg, q=None) == I and _attn(fl, pg, table=None) == I and _attn(fl, pg, start=None) == I
    assert _attn(fl, pg, ws=None) == I and _attn(fl, pg, ws=0x10010) == I and _attn(fl, pg, ws_bytes=100) == W
    assert _attn(fl, pg, ld_table=1 << 26) == U and _attn(fl, pg, ld_table=-1) == I
    assert _attn(fl, _pg(fl, P=0)) == I
    assert _attn(fl, pg, S=0) == 0 and _attn(fl, pg, T=0, ws_bytes=0) == 0  # nothing to do


@pytest.mark.parametrize("cap,code", [(1e-30, "U"), (2.0 ** -11, "U"), (1025.0, "U"), (1e30, "U"), (2.0 ** -10, "ok"),
                                      (1024.0, "ok"), (0.0, "ok")])
def test_attn_cap_range(fl, cap, code):
    """No rows: nothing is launched."""
    assert _attn(fl, _pg(fl), cap=cap, T=0) == (fl.FATHOM_ERR_UNSUPPORTED if code == "U" else 0)


def test_attn_table_positions_are_counted_in_32_bits(fl):
    """4096 requests of 2^23 positions are the most: S*ld_table*page <= 2^35."""
    pg = _pg(fl)
    most = (1 << 23) // pg.page
    assert _attn(fl, pg, S=4096, ld_table=most, T=0) == 0
    assert _attn(fl, pg, S=4096, ld_table=most + 1, T=0) == fl.FATHOM_ERR_UNSUPPORTED


def test_write_pack_sparse_refusals(fl):
    L, pg = fl.lib(), _pg(fl)
    I, U = fl.FATHOM_ERR_INVALID, fl.FATHOM_ERR_UNSUPPORTED

    def write(K=FAKE, sdt=1, ld=256, T=1, slots=FAKE, p=pg):
        return L.fathom_paged_write(K, FAKE, sdt, ld, 128, 256, 128, slots, T, 128, C.byref(p), None, S0)

    assert write(sdt=2) == U and write(sdt=7) == U and write(T=1 << 30) == U
    assert write(T=-1) == I and write(ld=-8) == I and write(ld=4) == I and write(sdt=0, ld=2) == I
    assert write(K=ODD) == I and write(slots=ODD) == I and write(slots=None) == I and write(K=None) == I
    assert write(T=0, K=None, slots=None) == 0
    assert write(p=_pg(fl, V=0)) == I

    def pack(S=1, nb=4, n=FAKE, old=None, new=0, planes=FAKE, H=2):
        return L.fathom_paged_pack(C.byref(_pg(fl, V=0, H=H)), FAKE, 4, old, n, new, S, 128, nb, planes, FAKE, None, S0)

    assert pack(S=-1) == I and pack(nb=-1) == I and pack(n=None) == I and pack(planes=None) == I and pack(planes=ODD) == I
    assert pack(old=FAKE, new=-1) == I and pack(old=ODD, new=1) == I
    assert pack(S=4096, H=16) == U  # 65536 units
    assert pack(S=0) == 0 and pack(nb=0) == 0

    def sparse(S=1, G=4, k=8, sink=4, local=32, qdt=0, q=FAKE, idx=FAKE, ws=FAKE, nbytes=1 << 20):
        return L.fathom_paged_sparse_attn(q, qdt, C.byref(pg), FAKE, 4, FAKE, S, G, 128, idx, k, sink, local,
                                          C.c_float(1.0), FAKE, ws, nbytes, None, S0)

    assert sparse(G=9) == U and sparse(k=9000) == U and sparse(sink=1000, local=100) == U and sparse(qdt=3) == U
    assert sparse(local=(1 << 31) - 1) == U and sparse(S=4096, G=8) == U
    assert sparse(k=-1) == I and sparse(q=None) == I and sparse(idx=None) == I and sparse(idx=0x10002) == I
    assert sparse(ws=0x10010) == I and sparse(nbytes=8) == fl.FATHOM_ERR_WORKSPACE
    assert sparse(S=0) == 0


def test_map_refusals(fl):
    def m(S=1, H=1, page=64, L=4, P=8, T=4, n_old=FAKE, n=FAKE, table=FAKE, ring=FAKE, state=FAKE, slots=FAKE, start=FAKE,
          now=FAKE, unit=None, out=FAKE):
        return fl.lib().fathom_paged_map(n_old, n, S, H, page, table, L, ring, P, state, slots, T, start, now, unit, out,
                                         None, S0)

    I, U = fl.FATHOM_ERR_INVALID, fl.FATHOM_ERR_UNSUPPORTED
    assert m(S=-1) == I and m(L=-1) == I and m(P=-1) == I and m(T=-1) == I
    assert m(S=4097) == U and m(H=0) == U and m(H=1025) == U
    assert m(page=8) == U and m(page=96) == U and m(page=2048) == U
    assert m(P=1 << 31) == U and m(T=1 << 31) == U and m(L=1 << 25) == U
    for k in ("n_old", "n", "state", "start", "now", "out", "slots"):
        assert m(**{k: None}) == I and m(**{k: 0x10004}) == I, k
    for k in ("table", "ring"):
        assert m(**{k: None}) == I and m(**{k: 0x10002}) == I, k
    assert m(unit=0x10004) == I


def test_binding_refuses_host_tensors(fl):
    z = torch.zeros
    with pytest.raises(ValueError):
        fl.fathom_paged_attn(z(1, 4, 128).half(), z(2, 1, 16, 128).half(), z(2, 1, 16, 128).half(), z(1, 2).int(),
                             z(2).long(), z(1).long(), 1)
    with pytest.raises(ValueError):
        fl.fathom_paged_map(z(1).long(), z(1).long(), 16, z(1, 2).int(), z(4).int(), z(2).long(), 4)


def test_constants_match_header(fl):
    src = open(os.path.join(os.path.dirname(fl.HERE), "include", "fathom.h")).read()
    for name in ("FATHOM_DEV_BAD_PAGE", "FATHOM_DEV_PAGES_SHORT", "FATHOM_MAX_SEQS"):
        val = src.split(f"#define {name} ")[1].split()[0].rstrip("u")
        assert int(val) == getattr(fl, name)
    assert "FATHOM_BF16 = 2" in src and fl.FATHOM_BF16 == 2


def test_plain_map_by_hand():
    """Two requests, pages of 16: the first grows over a page, the second ends."""
    table = np.array([[5, -1, -1], [3, 1, -1]], np.int32)
    ring = np.array([0, 7, 2, 4, 6, 9, 9, 9], np.int32)
    t, r, slots, start, now, unit, st, short, bad = P.paged_map([10, 20], [18, 0], 16, table, ring, [1, 4], 9, 2)
    assert t.tolist() == [[5, 7, -1], [3, 1, -1]]  # takes ring[1]; what ends keeps its entries
    assert r.tolist() == [0, 7, 2, 4, 6, 3, 1, 9]  # returned behind the four free ones
    assert slots.tolist() == [90, 91, 92, 93, 94, 95, 112, 113, -1]
    assert start.tolist() == [0, 8, 8] and now.tolist() == [18, 0] and unit.tolist() == [18, 18, 0, 0]
    assert st.tolist() == [2, 5] and not short and not bad


def test_map_ends_requests_behind_rows_that_do_not_fit():
    """A request without new rows is served wherever it stands: the pages it returns are no longer its own."""
    table = np.array([[-1, -1], [4, 2], [3, -1]], np.int32)
    args = [0, 30, 16], [20, 0, 5], 16, table, np.array([0, 1, 5, -1, -1, -1], np.int32), [0, 3], 10
    _, ring, slots, start, n_now, _, state, short, bad_n = P.paged_map(*args, 1)
    assert n_now.tolist() == [0, 0, 5] and ring.tolist() == [0, 1, 5, 4, 2, -1] and state.tolist() == [0, 5]
    assert (slots == -1).all() and start.tolist() == [0, 20, 20, 20] and bad_n and not short


def test_packed_pages_are_the_structure(fl):
    """The binding's bytes are fathom_pages as ctypes lays it out."""
    args = 0x1000, 0x2000, fl.FATHOM_BF16, 8, 64, 12345, 1 << 40, 1 << 20, 1 << 7
    assert fl._pack_pages(*args) == bytes(fl._Pages(*args))
    K = torch.zeros((3, 2, 16, 128), dtype=torch.float16)
    pg, H, D = fl._pages(K, None)
    want = fl._Pages(K.data_ptr(), None, fl.FATHOM_F16, 2, 16, 3, 4096, 2048, 128)
    assert pg == bytes(want) and (H, D) == (2, 128)


@pytest.mark.parametrize("page", [16, 64, 1024])
def test_positions_leave_room_in_32_bits(fl, page):
    """2^31 - 1024 positions a request are the most, for every call that takes a table; blocks behind the last are counted
    beyond."""
    most = ((1 << 31) - 1024) // page
    L, pg = fl.lib(), _pg(fl, page=page)
    for ld, want in ((most, 0), (most + 1, fl.FATHOM_ERR_UNSUPPORTED)):
        assert _attn(fl, pg, ld_table=ld, T=0) == want
        assert L.fathom_paged_pack(C.byref(pg), FAKE, ld, None, FAKE, 0, 0, 128, 4, FAKE, FAKE, None, S0) == want
        assert L.fathom_paged_sparse_attn(FAKE, 0, C.byref(pg), FAKE, ld, FAKE, 0, 4, 128, FAKE, 8, 4, 32, C.c_float(1.0),
                                          FAKE, FAKE, 1 << 20, None, S0) == want
        # (without its lengths: refused for them where the table is not)
        assert L.fathom_paged_map(None, FAKE, 1, 1, page, FAKE, ld, FAKE, 8, FAKE, FAKE, 4, FAKE, FAKE, None, FAKE, None,
                                  S0) == (want or fl.FATHOM_ERR_INVALID)
