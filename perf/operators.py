"""The paged KV cache's operators as a program that serves with them calls them, and the same in plain torch.

A request's keys and values lie in pages of a common pool; a block table per request lists its pages.  A serving step
maps its new tokens to slots (pages taken from and returned to a ring of free pages), writes their K and V rows there,
and attends: a chunk of a prompt or a decode step over all cached rows (`attn`), or over the rows that the bit-plane
scan selected (`sparse`), whose planes are packed from the pages (`pack`).

`own` chooses the side: False computes each operator from elementary torch operations in 32 bits or more, True calls
the package.  Keys have log-normal channel scales as in `paper_2609_17652_amd.synth`; everything is drawn from the seed.
"""
import math
import random

import torch

own = False

D = 128
DEV = "cuda"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # a decode step of 64 requests, one new token each: latency is all that counts
        _map("map_decode64", S=64, H=8, n_lo=1000, n_hi=65536, new_hi=1, page=64, mix=False),
        # a step in which requests begin (prompts of up to 8192 tokens), go on and end, small pages
        _map("map_mixed512", S=512, H=8, n_lo=1, n_hi=32768, new_hi=8192, page=16, mix=True),
        # the new rows of that decode step, taken from the fused projection's output
        _write("write_decode64", S=64, H=8, n_lo=1000, n_hi=16384, new_lo=1, new_hi=1, page=64, dt="f16", src="f16"),
        # the rows of long prompts, fp32 rows rounded into a bf16 cache
        _write("write_prompts_bf16", S=6, H=8, n_lo=0, n_hi=5000, new_lo=9001, new_hi=32001, page=64, dt="bf16",
               src="f32"),
        # the bit-plane store of 32 requests x 8 heads follows one token
        _pack("pack_append32", S=32, H=8, n_lo=500, n_hi=16384, page=64, append=1),
        # the bit-plane store of prefilled prompts, one layer
        _pack("pack_prompts", S=4, H=8, n_lo=30011, n_hi=131072, page=128, append=0),
        # the smallest attention: one request at 4096 tokens, one new token
        _attn("attn_decode_1x4k", S=1, H=8, G=4, n_lo=4095, n_hi=4095, new_lo=1, new_hi=1, page=64, dt="f16"),
        # a decode step of 32 requests of very different lengths
        _attn("attn_decode32_ragged", S=32, H=8, G=4, n_lo=1000, n_hi=65535, new_lo=1, new_hi=1, page=64, dt="f16"),
        # a chunk of a long prompt over what is cached: the largest
        _attn("attn_chunk2k_64k", S=1, H=8, G=4, n_lo=65536, n_hi=65536, new_lo=2048, new_hi=2048, page=64, dt="bf16"),
        # prompts of packed documents with a shared prefix, capped scores and a distance bias, odd lengths, token-major
        # pages
        _attn("attn_docs_cap_bias", S=6, H=2, G=8, n_lo=0, n_hi=3001, new_lo=301, new_hi=5003, page=16, dt="bf16",
              cap=30.0, bias=True, prefix=True, docs=True, major="token"),
        # sparse decode of one short request
        _sparse("sparse_1x4k", S=1, H=8, G=4, n_lo=4096, n_hi=4096, page=64, k=64, sink=4, local=32, q="f32"),
        # sparse decode of 16 long requests
        _sparse("sparse16_k2048", S=16, H=8, G=4, n_lo=20011, n_hi=65536, page=64, k=2012, sink=4, local=32, q="f16"),
    ]


def _map(name, S, H, n_lo, n_hi, new_hi, page, mix):
    """Slots for S requests of n_lo..n_hi cached tokens; mix: some begin, some end, the others get one token."""
    return dict(name=name, kind="map", S=S, H=H, n_lo=n_lo, n_hi=n_hi, new_hi=new_hi, page=page, mix=mix)


def _write(name, S, H, n_lo, n_hi, new_lo, new_hi, page, dt, src, major="head"):
    return dict(name=name, kind="write", S=S, H=H, n_lo=n_lo, n_hi=n_hi, new_lo=new_lo, new_hi=new_hi, page=page, dt=dt,
                src=src, major=major)


def _pack(name, S, H, n_lo, n_hi, page, append, dt="f16", major="head"):
    """append: tokens by which the store grows (0: packed whole)."""
    return dict(name=name, kind="pack", S=S, H=H, n_lo=n_lo, n_hi=n_hi, page=page, append=append, dt=dt, major=major)


def _attn(name, S, H, G, n_lo, n_hi, new_lo, new_hi, page, dt, cap=0.0, bias=False, prefix=False, docs=False,
          major="head"):
    """n_lo..n_hi tokens cached before the call's new_lo..new_hi."""
    return dict(name=name, kind="attn", S=S, H=H, G=G, n_lo=n_lo, n_hi=n_hi, new_lo=new_lo, new_hi=new_hi, page=page,
                dt=dt, cap=cap, bias=bias, prefix=prefix, docs=docs, major=major)


def _sparse(name, S, H, G, n_lo, n_hi, page, k, sink, local, q, dt="f16", major="head"):
    return dict(name=name, kind="sparse", S=S, H=H, G=G, n_lo=n_lo, n_hi=n_hi, page=page, k=k, sink=sink, local=local,
                q=q, dt=dt, major=major)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["map", "write", "pack", "attn", "attn", "attn", "sparse"])
    H, page = rng.choice([1, 2, 4, 8, 8]), rng.choice([16, 32, 64, 64, 128, 256])
    major = rng.choice(["head", "head", "token"])
    dt = rng.choice(["f16", "bf16"])
    if kind == "map":
        mix = rng.random() < 0.5
        c = _map("", S=log(1, 512), H=H, n_lo=1, n_hi=log(1000, 65536), new_hi=log(2, 8192) if mix else 1, page=page,
                 mix=mix)
    elif kind == "write":
        S = log(1, 128)
        new = log(1, max(1, 100000 // S))
        c = _write("", S=S, H=H, n_lo=0, n_hi=log(10, 8192), new_lo=new // 2 + 1, new_hi=new, page=page, dt=dt,
                   src=rng.choice([dt, "f32"]), major=major)
    elif kind == "pack":
        S = log(1, 32)
        n = log(200, max(400, min(131072, (1 << 22) // (S * H))))
        c = _pack("", S=S, H=H, n_lo=n // 3 + 1, n_hi=n, page=page, append=rng.choice([0, 0, 1, 1, log(2, 150)]), dt=dt,
                  major=major)
    elif kind == "sparse":
        S = log(1, 16)
        n = log(2000, 65536)
        c = _sparse("", S=S, H=H, G=rng.choice([1, 2, 4, 8]), n_lo=n // 2 + 1, n_hi=n, page=page,
                    k=min(log(16, 1024), n // 4), sink=rng.choice([0, 4]), local=rng.choice([0, 32]),
                    q=rng.choice(["f16", "f32"]), dt=dt, major=major)
    else:
        G = rng.choice([1, 2, 3, 4, 4, 5, 8])
        opt = dict(cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.3, prefix=rng.random() < 0.3,
                   docs=rng.random() < 0.3)
        if rng.random() < 0.5:  # decode steps, some of a few tokens per request
            S = log(1, 64)
            n = log(50, min(65536, (1 << 20) // S))
            new = rng.choice([1, 1, 1, 2, 5, 8])
        else:  # chunks of prompts
            S = log(1, 8)
            new = log(20, 4096 // S)
            n = log(30, 16384)
        c = _attn("", S=S, H=H, G=G, n_lo=n // 4, n_hi=n, new_lo=(new + 1) // 2, new_hi=new, page=page, dt=dt,
                  major=major, **opt)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * seed + 29)


def _between(lo, hi, k, gen):
    return torch.randint(lo, hi + 1, (k,), generator=gen, device=DEV)


def _requests(c, gen):
    """Cached and new tokens of the case's requests: the case fixes the pairs (and so every shape), the seed their
    order."""
    fixed, S = random.Random("%d %d %d" % (c["S"], c["n_lo"], c["n_hi"])), c["S"]
    pairs = []
    for i in range(S):
        old = fixed.randint(c["n_lo"], c["n_hi"])
        if c["kind"] == "map":
            new = 1
            if c["mix"] and i % 10 == 0:  # one request in ten ends
                new = -old
            elif c["mix"] and i % 10 > 7:  # two in ten begin
                old, new = 0, fixed.randint(1, c["new_hi"])
        elif c["kind"] == "pack":
            new = c["append"]
        elif c["kind"] == "sparse":
            new = 0
        else:
            new = fixed.randint(c["new_lo"], c["new_hi"])
        pairs.append((old, new))
    x = torch.tensor(pairs, device=DEV)[torch.randperm(S, generator=gen, device=DEV)]
    return x[:, 0].contiguous(), x[:, 1].contiguous()


def _pages(c, lengths, gen):
    """Block tables for the lengths (a shuffled pool), and empty pages [P][H][page][D] of the case's layout."""
    page, need = c["page"], [(m + c["page"] - 1) // c["page"] for m in lengths]
    P, L = sum(need) + 3, max(max(need), 1)
    pool = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(need), L), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = pool[at:at + m]
        at += m
    if c["major"] == "head":
        make = lambda: torch.zeros((P, c["H"], page, D), dtype=TYPES[c["dt"]], device=DEV)  # noqa: E731
    else:
        make = lambda: torch.zeros((P, page, c["H"], D), dtype=TYPES[c["dt"]], device=DEV).transpose(1, 2)  # noqa: E731
    return table, make(), make()


def _fill(pages, gen, scale):
    """Random rows in every page (a pool holds what earlier requests left there), a part of the pool at a time."""
    for p in range(0, pages.shape[0], 4096):
        x = torch.randn(pages[p:p + 4096].shape, generator=gen, device=DEV)
        pages[p:p + 4096] = x * scale if scale is not None else x


def _inputs(c, seed):
    gen = _rng(seed)
    S, d = c["S"], {}
    n_old, new = _requests(c, gen)
    n = n_old + new
    if c["kind"] == "map":
        page = c["page"]
        L = (max(c["n_hi"] + 1, c["new_hi"]) + page - 1) // page
        held, need = ((n_old + page - 1) // page).tolist(), ((n + page - 1) // page).tolist()
        P = sum(max(a, b) for a, b in zip(held, need)) + 7
        pool = torch.randperm(P, generator=gen, device=DEV).to(torch.int32)
        table = torch.full((S, L), -1, dtype=torch.int32, device=DEV)
        at = 0
        for s, m in enumerate(held):
            table[s, :m] = pool[at:at + m]
            at += m
        ring, head = torch.full((P,), -1, dtype=torch.int32, device=DEV), P // 3
        ring[(head + torch.arange(P - at, device=DEV)) % P] = pool[at:]
        d.update(n_old=n_old, n=n, table=table, ring=ring, T=int(new.clamp(min=0).sum()) + 5,
                 state=torch.tensor([head, P - at], device=DEV))
        return d
    d.update(n=n, n_host=n.tolist(), new_host=new.tolist())
    d["table"], d["K"], d["V"] = _pages(c, d["n_host"], gen)
    if c["kind"] != "write":
        _fill(d["K"], gen, torch.exp(0.5 * torch.randn((D,), generator=gen, device=DEV)))
        if c["kind"] != "pack":
            _fill(d["V"], gen, None)
    d["start"] = torch.cat([torch.zeros_like(n[:1]), new.cumsum(0)])
    T, H = sum(d["new_host"]), c["H"]
    if c["kind"] == "write":
        # the fused projection's output: a query head, then K and V heads, of every new token
        qkv = torch.randn((T, 3 * H, D), generator=gen, device=DEV).to(TYPES[c["src"]])
        d.update(Knew=qkv[:, H:2 * H], Vnew=qkv[:, 2 * H:])
        s = torch.repeat_interleave(torch.arange(S, device=DEV), new)
        pos = n[s] - new[s] + torch.arange(T, device=DEV) - d["start"][s]
        d["slots"] = d["table"][s, pos // c["page"]].long() * c["page"] + pos % c["page"]
    elif c["kind"] == "pack":
        d["n_old"] = n_old
    elif c["kind"] == "sparse":
        q = 2.0 * torch.randn((S * H, c["G"], D), generator=gen, device=DEV)
        d["q"] = q.to(TYPES[c["q"]])
        idx = torch.empty((S, H * c["G"], c["k"]), dtype=torch.int32, device=DEV)
        for s, m in enumerate(d["n_host"]):
            r = torch.rand((H * c["G"], m - c["sink"] - c["local"]), generator=gen, device=DEV)
            idx[s] = r.topk(c["k"], dim=1).indices.int() + c["sink"]
        d["idx"] = idx.view(S * H, c["G"], c["k"])
    else:
        HG = H * c["G"]
        qkv = torch.randn((T, HG + 2 * H, D), generator=gen, device=DEV)
        d["q"] = (2.0 * qkv).to(TYPES[c["dt"]])[:, :HG]
        if c["bias"]:
            d["slopes"] = 2.0 ** -(8.0 * (torch.arange(HG, device=DEV) + 1) / HG)
        if c["prefix"]:
            d["prefix"] = _between(1, 200, S, gen)
        if c["docs"]:  # documents of about 700 tokens, packed one after another in each request
            s = torch.repeat_interleave(torch.arange(S, device=DEV), new)
            pos = n[s] - new[s] + torch.arange(T, device=DEV) - d["start"][s]
            size = _between(300, 1100, S, gen)[s]
            d["first"] = pos // size * size
    return d


def _map_state(c, d):
    """Where the call puts what it computes; the ring and the table are the program's own, changed in place."""
    S, H = c["S"], c["H"]
    i64 = dict(dtype=torch.int64, device=DEV)
    d.update(slots=torch.empty((d["T"],), **i64), start=torch.empty((S + 1,), **i64), n_now=torch.empty((S,), **i64),
             n_unit=torch.empty((S * H,), **i64), state_out=torch.empty((2,), **i64))


def prepare(case, seed):
    c, d = case, _inputs(case, seed)
    d["case"] = c
    S, H = c["S"], c["H"]
    if c["kind"] == "map":
        _map_state(c, d)
    elif c["kind"] == "pack":
        nb = (max(d["n_host"]) + 63) // 64
        d.update(planes=torch.zeros((S * H, D, 4, nb), dtype=torch.int64, device=DEV),
                 scales=torch.zeros((S * H, D, nb), dtype=torch.int16, device=DEV))
        if c["append"]:  # the store before the call
            _plain_pack(c, d, d["n_old"].tolist())
    elif c["kind"] == "sparse":
        d["out"] = torch.empty((S * H, c["G"], D), dtype=torch.float32, device=DEV)
    elif c["kind"] == "attn":
        d["out"] = torch.empty((d["q"].shape[0], H * c["G"], D), dtype=TYPES[c["dt"]], device=DEV)
    if own:
        import paper_2609_17652_amd as F
        d["F"], d["st"] = F, F.new_status(DEV)
        u8 = dict(dtype=torch.uint8, device=DEV)
        if c["kind"] == "attn":
            d["max_new"] = max(d["new_host"])
            d["ws"] = torch.empty((F.fathom_paged_attn_workspace_size(d["q"].shape[0], S, H, c["G"], d["max_new"]),),
                                  **u8)
        elif c["kind"] == "sparse":
            d["ws"] = torch.empty((F.fathom_sparse_attn_workspace_size(S * H, c["G"], c["k"], c["sink"], c["local"]),),
                                  **u8)
    return d


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if not own:
        return _PLAIN[c["kind"]](c, s)
    F = s["F"]
    if c["kind"] == "map":
        F.fathom_paged_map(s["n_old"], s["n"], c["page"], s["table"], s["ring"], s["state"], s["T"], c["H"], s["slots"],
                           s["start"], s["n_now"], s["n_unit"], s["state_out"], s["st"])
        return {x: s[x] for x in ("table", "ring", "state_out", "slots", "start", "n_now", "n_unit")}
    if c["kind"] == "write":
        F.fathom_paged_write(s["Knew"], s["Vnew"], s["slots"], s["K"], s["V"], s["st"])
        return {"K": s["K"], "V": s["V"]}
    if c["kind"] == "pack":
        F.fathom_paged_pack(s["K"], s["table"], s["n"], s["planes"], s["scales"], s["n_old"] if c["append"] else None,
                            c["append"], s["st"])
        return {"planes": s["planes"], "scales": s["scales"]}
    if c["kind"] == "sparse":
        return F.fathom_paged_sparse_attn(s["q"], s["K"], s["V"], s["table"], s["n"], s["idx"], c["sink"], c["local"],
                                          None, s["out"], s["st"], ws=s["ws"])
    return F.fathom_paged_attn(s["q"], s["K"], s["V"], s["table"], s["start"], s["n"], s["max_new"], None, c["cap"],
                               s.get("slopes"), s.get("prefix"), s.get("first"), s["out"], s["ws"], s["st"])


def _plain_map(c, s):
    page, n_old, n, table, ring, T, H = c["page"], s["n_old"], s["n"], s["table"], s["ring"], s["T"], c["H"]
    S, L = table.shape
    P, head, count = ring.numel(), s["state"][0], s["state"][1]
    zero = torch.zeros_like(n)
    ok = (n_old >= 0) & (n_old <= L * page) & (n >= 0) & (n <= L * page)
    new = torch.where(ok, (n - n_old).clamp(min=0), zero)
    start = torch.cat([zero[:1], new.cumsum(0)])
    before, after = (n_old + page - 1) // page, (n + page - 1) // page
    take, back = torch.where(ok, (after - before).clamp(min=0), zero), torch.where(ok, (before - after).clamp(min=0), zero)
    taken, returned = take.cumsum(0), back.cumsum(0)
    served = ok & (start[1:] <= T) & ((take == 0) | (taken <= count))
    j = torch.arange(L, device=DEV)
    grow = served[:, None] & (j >= before[:, None]) & (j < after[:, None])
    at = (head + (taken - take - before)[:, None] + j) % P
    table = torch.where(grow, ring[at], table)
    popped, total = torch.where(served, take, zero).sum(), returned[-1]
    fits = count + total <= P
    give = ok[:, None] & fits & (j >= after[:, None]) & (j < before[:, None])
    to = torch.where(give, (head + count + (returned - back - after)[:, None] + j) % P, torch.full_like(at, P))
    ring = torch.cat([ring, ring[:1]]).scatter(0, to.flatten(), table.flatten())[:P]
    state_out = torch.stack([(head + popped) % P, count - popped + torch.where(fits, total, zero[0])])
    n_now = torch.where(served, n, torch.where((n_old >= 0) & (n_old <= L * page), n_old, zero))
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(start[1:].contiguous(), t, right=True).clamp(max=S - 1)
    pos = n_old[r] + t - start[r]
    on = (t < start[S]) & served[r]
    pid = table[r, torch.where(on, pos // page, torch.zeros_like(pos))].long()
    slots = torch.where(on & (pid >= 0) & (pid < P), pid * page + pos % page, torch.full_like(t, -1))
    return {"table": table, "ring": ring, "state_out": state_out, "slots": slots, "start": start, "n_now": n_now,
            "n_unit": n_now.repeat_interleave(H)}


def _plain_write(c, s):
    page, slots = c["page"], s["slots"]
    for pages, rows in ((s["K"], s["Knew"]), (s["V"], s["Vnew"])):
        pages[slots // page, :, slots % page] = rows.to(pages.dtype)
    return {"K": s["K"], "V": s["V"]}


def _rows(pages, ids, m):
    """The first m rows [H][m][D] of the pages `ids`."""
    x = pages[ids.long()]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, D)[:, :m]


def _plain_pack(c, s, upto=None):
    """Planes and scales of the blocks from the one that holds the first new token (or of all blocks)."""
    page, H, nb_cap = c["page"], c["H"], s["scales"].shape[-1]
    planes, scales = s["planes"].view(-1, H, D, 4, nb_cap), s["scales"].view(-1, H, D, nb_cap)
    lengths = s["n_host"] if upto is None else upto
    place = torch.arange(64, device=DEV)
    for i, m in enumerate(lengths):
        b0 = (m - c["append"]) // 64 if c["append"] and upto is None else 0
        nb = (m + 63) // 64
        if nb > b0:
            p0 = 64 * b0 // page
            off = 64 * b0 - p0 * page
            x = _rows(s["K"], s["table"][i, p0:(m + page - 1) // page], m - p0 * page)[:, off:].double()
            x = torch.nn.functional.pad(x, (0, 0, 0, (nb - b0) * 64 - x.shape[1])).view(H, nb - b0, 64, D)
            a = x.abs().amax(2).half()
            step = a.double().unsqueeze(2) / 8
            code = torch.floor(x / torch.where(step > 0, step, torch.ones_like(step))).clamp(-8, 7).long() + 8
            on = (64 * b0 + torch.arange((nb - b0) * 64, device=DEV) < m).view(1, nb - b0, 64, 1)
            for p in range(4):
                word = torch.where(on, (code >> (3 - p)) & 1, torch.zeros_like(code)) << place.view(1, 1, 64, 1)
                planes[i, :, :, p, b0:nb] = word.sum(2).transpose(1, 2)
            scales[i, :, :, b0:nb] = a.view(torch.int16).transpose(1, 2)
        if not c["append"]:
            planes[i, :, :, :, nb:] = 0
            scales[i, :, :, nb:] = 0
    return {"planes": s["planes"], "scales": s["scales"]}


def _bounds(s, i, new, m):
    """Positions of request i's new tokens and the first and one past the last position each sees."""
    a = sum(s["new_host"][:i])
    pos = torch.arange(m - new, m, device=DEV)
    hi = pos + 1
    if "prefix" in s:
        hi = torch.maximum(hi, s["prefix"][i].clamp(max=m))
    lo = s["first"][a:a + new] if "first" in s else torch.zeros_like(pos)
    return a, pos, lo, hi


def _plain_attn(c, s):
    H, G, q, out = c["H"], c["G"], s["q"], s["out"]
    scale = 1 / math.sqrt(D)
    for i, (m, new) in enumerate(zip(s["n_host"], s["new_host"])):
        a, pos, lo, hi = _bounds(s, i, new, m)
        j = torch.arange(m, device=DEV)
        seen = ((j >= lo[:, None]) & (j < hi[:, None])).repeat_interleave(G, 0)
        ids = s["table"][i, :(m + c["page"] - 1) // c["page"]]
        K, V = _rows(s["K"], ids, m), _rows(s["V"], ids, m)
        qh = q[a:a + new].reshape(new, H, G, D).permute(1, 0, 2, 3).reshape(H, new * G, D)
        few = max(1, (1 << 29) // (new * G * m))  # heads at a time: scores of 2 GB
        for h in range(0, H, few):
            z = torch.matmul(qh[h:h + few].float(), K[h:h + few].float().transpose(1, 2)) * scale
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if "slopes" in s:
                far = (pos[:, None] - j).abs().float()
                sl = s["slopes"].view(H, 1, G, 1)[h:h + few]
                z = z - (sl * far[None, :, None, :]).reshape(z.shape[0], new * G, m)
            z = torch.where(seen, z, torch.full_like(z[:1, :1, :1], -math.inf))
            top = z.amax(2, keepdim=True)
            z = torch.exp(z - torch.where(torch.isinf(top), torch.zeros_like(top), top))
            den = z.sum(2, keepdim=True)
            o = torch.matmul(z, V[h:h + few].float()) / torch.where(den > 0, den, torch.ones_like(den))
            o = o.view(-1, new, G, D).permute(1, 0, 2, 3)
            out[a:a + new].view(new, H, G, D)[:, h:h + few] = o.to(out.dtype)
    return out


def _plain_sparse(c, s):
    S, H, G, page = c["S"], c["H"], c["G"], c["page"]
    n, q, out = s["n"], s["q"].float().view(S, H, G, D), s["out"].view(S, H, G, D)
    fixed = torch.cat([torch.arange(c["sink"], device=DEV).expand(S, -1),
                       n[:, None] - c["local"] + torch.arange(c["local"], device=DEV)], 1)
    rows = torch.cat([fixed[:, None].expand(S, H * G, -1), s["idx"].long().view(S, H * G, -1)], 2)
    pid = torch.gather(s["table"].long(), 1, (rows // page).flatten(1)).view(rows.shape)
    head = torch.arange(H, device=DEV).repeat_interleave(G).view(1, H * G, 1)
    for i in range(S):  # a request at a time: fp32 copies of its rows
        at = (pid[i:i + 1], head, rows[i:i + 1] % page)
        K, V = s["K"][at][0].float(), s["V"][at][0].float()
        z = torch.matmul(K, q[i].reshape(H * G, D, 1))[:, :, 0] / math.sqrt(D)
        z = torch.exp(z - z.amax(1, keepdim=True))
        o = torch.matmul(z[:, None], V)[:, 0] / z.sum(1, keepdim=True)
        out[i] = o.view(H, G, D)
    return s["out"]


_PLAIN = {"map": _plain_map, "write": _plain_write, "pack": _plain_pack, "attn": _plain_attn, "sparse": _plain_sparse}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    S, H = c["S"], c["H"]
    if c["kind"] == "map":
        mean = (c["n_lo"] + c["n_hi"]) / 2
        rows = S * (0.7 + 0.2 * (1 + c["new_hi"]) / 2) if c["mix"] else S
        pages = rows / c["page"] + (S * 0.1 * mean / c["page"] if c["mix"] else 0)
        return {"bytes": 24 * S + 8 * rows + 8 * pages + 8 * (S + 1) + 8 * S * H + 32, "flops": 0}
    n = (c["n_lo"] + c["n_hi"]) / 2
    if c["kind"] == "write":
        rows = S * (c["new_lo"] + c["new_hi"]) / 2
        return {"bytes": rows * (2 * H * D * ((4 if c["src"] == "f32" else 2) + 2) + 8), "flops": 0}
    if c["kind"] == "pack":
        tok = S * H * (32.5 + c["append"] if c["append"] else n)
        return {"bytes": tok * (2 * D + 68) + 4 * S * (n / c["page"] if not c["append"] else 2), "flops": 8 * tok * D}
    G = c["G"]
    if c["kind"] == "sparse":
        rows = S * H * G * (c["k"] + c["sink"] + c["local"])
        return {"bytes": rows * 4 * D + S * H * G * (c["k"] * 4 + D * (4 if c["q"] == "f32" else 2) + 4 * D),
                "flops": 4 * rows * D}
    new = (c["new_lo"] + c["new_hi"]) / 2
    seen = n + (new + 1) / 2
    read = n + new
    if c["docs"]:  # about 700 tokens a document: half of one before a token, and what is cached of the first
        seen = min(seen, 350)
        read = min(read, new + 350)
    return {"bytes": S * (4 * D * H * read + 4 * D * H * G * new + 4 * read / c["page"]),
            "flops": 4 * D * H * G * S * new * seen}


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    c = case
    if c["kind"] in ("map", "pack"):  # whole numbers
        return None
    d = _inputs(case, seed)
    if c["kind"] == "write":
        o = {}
        for name, rows in (("K", d["Knew"]), ("V", d["Vnew"])):
            x = torch.zeros((d[name].shape[0] * c["page"], c["H"], D), dtype=torch.float64, device=DEV)
            x[d["slots"]] = rows.double()
            o[name] = x.view(-1, c["page"], c["H"], D).transpose(1, 2)
        return o
    H, G = c["H"], c["G"]
    if c["kind"] == "sparse":
        out = torch.empty((c["S"], H, G, D), dtype=torch.float64, device=DEV)
        q, idx = d["q"].view(c["S"], H, G, D), d["idx"].view(c["S"], H, G, -1)
        for i, m in enumerate(d["n_host"]):
            ids = d["table"][i, :(m + c["page"] - 1) // c["page"]].long()
            ends = torch.cat([torch.arange(c["sink"], device=DEV), torch.arange(m - c["local"], m, device=DEV)])
            for h in range(H):
                K, V = (d[x][ids, h].reshape(-1, D) for x in ("K", "V"))
                for g in range(G):
                    r = torch.cat([ends, idx[i, h, g].long()])
                    w = torch.softmax(K[r].double() @ q[i, h, g].double() / math.sqrt(D), 0)
                    out[i, h, g] = w @ V[r].double()
        return out.view(-1, G, D)
    out = torch.zeros(d["q"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for i, (m, new) in enumerate(zip(d["n_host"], d["new_host"])):
        ids = d["table"][i, :(m + c["page"] - 1) // c["page"]].long()
        j = torch.arange(m, device=DEV)
        for h in range(H):
            K, V = (d[x][ids, h].reshape(-1, D)[:m].double() for x in ("K", "V"))
            step = max(1, (1 << 27) // m)  # tokens at a time: scores of 1 GB
            for g in range(G):
                for t in range(0, new, step):
                    e = min(new, t + step)
                    p = (m - new + torch.arange(t, e, device=DEV)).view(-1, 1)
                    z = (d["q"][row + t:row + e, h * G + g].double() / math.sqrt(D)) @ K.T
                    if c["cap"] > 0:
                        z = torch.tanh(z / c["cap"]) * c["cap"]
                    if c["bias"]:
                        z -= d["slopes"][h * G + g].double() * (p - j).abs()
                    hide = j > p
                    if c["prefix"]:
                        hide &= j >= d["prefix"][i]
                    if c["docs"]:
                        hide |= j < d["first"][row + t:row + e].view(-1, 1)
                    z.masked_fill_(hide, -math.inf)
                    w = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
                    out[row + t:row + e, h * G + g] = w.masked_fill(hide, 0.0) @ V
        row += new
    return out
