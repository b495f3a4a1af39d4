"""Serving from a cache of pages: prompts in chunks, windows, and caches that are cut down, as cases that can be timed.

Kinds:
  rotate  new tokens enter one layer's cache: RMS norm of each head's query and key, rotary positions, and K and V to
          their places in the pages
  chunk   causal attention of each sequence's new tokens (one, or a chunk of a prompt) over its cache pages, with or
          without a sliding window behind a few first tokens that stay visible
  weigh   the same, and every cached token's accumulated attention weight grows by what the new queries gave it
  evict   sequences are cut down to the tokens of the largest accumulated weight, layer by layer and head by head, and
          grow again to their length

``own`` chooses what ``run`` calls: the plain form (elementary torch operations in 32 bits) or the framework.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
EPS = 1e-6


# ---- cases

def _rotate(name, tokens, seqs, heads, kv_heads, dim, rot, page, far=0, norm=True, interleaved=False, dtype="bf16"):
    return dict(name=name, kind="rotate", tokens=tokens, seqs=seqs, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot,
                page=page, far=far, norm=norm, interleaved=interleaved, dtype=dtype)


def _chunk(name, rows, heads, kv_heads, dim, new_lo, new_hi, len_lo, len_hi, page, window=0, sinks=0, dtype="bf16",
           kind="chunk"):
    return dict(name=name, kind=kind, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, new_lo=new_lo, new_hi=new_hi,
                len_lo=len_lo, len_hi=len_hi, page=page, window=window, sinks=sinks, dtype=dtype)


def _evict(name, layers, seqs, kv_heads, dim, page, len_lo, len_hi, keep, sinks, recent):
    return dict(name=name, kind="evict", layers=layers, seqs=seqs, kv_heads=kv_heads, dim=dim, page=page, len_lo=len_lo,
                len_hi=len_hi, keep=keep, sinks=sinks, recent=recent)


def listed():
    return [
        # one user's next token in one layer of the repository's shape (4 KV heads of 128): what a call costs by itself
        _rotate("rotate_one", 1, 1, 32, 4, 128, 128, 16),
        # prompts of four users prefilled together: bound by the memory
        _rotate("rotate_chunk", 8192, 4, 32, 4, 128, 128, 16),
        # small and odd: half of each narrow head turns, in neighbouring pairs, at positions past a million
        _rotate("rotate_odd", 77, 5, 6, 2, 64, 32, 24, far=1 << 20, interleaved=True, dtype="fp16"),
        # one user's next token behind the repository's prompt of 4,096 tokens and 300 of the user's own
        _chunk("chunk_one", 1, 32, 4, 128, 1, 1, 4396, 4396, 16),
        # the repository's decode batch, each row with a history of its own and no shared prefix
        _chunk("chunk_b64", 64, 32, 4, 128, 1, 1, 1, 8192, 16),
        # a chunk of a long prompt behind the part that is cached already: most of the work is products
        _chunk("chunk_prompt", 1, 32, 4, 128, 4096, 4096, 8192, 8192, 16),
        # chunks of long documents under a window of 1,024 tokens and four first ones
        _chunk("chunk_window", 4, 32, 4, 128, 1000, 2048, 16384, 32768, 16, window=1024, sinks=4),
        # a mixed batch, small and odd: single tokens, short chunks and rows without any
        _chunk("chunk_odd", 9, 6, 2, 64, 0, 130, 130, 1003, 24, dtype="fp16"),
        # the decode batch again, with the weights that eviction goes by
        _chunk("weigh_b64", 64, 32, 4, 128, 1, 1, 1, 4096, 16, kind="weigh"),
        # a prompt's second half, with the weights
        _chunk("weigh_prompt", 1, 32, 4, 128, 2048, 2048, 4096, 4096, 16, kind="weigh"),
        # a few short sequences of one layer: what the calls cost by themselves
        _evict("evict_small", 1, 4, 4, 128, 16, 520, 700, 512, 4, 32),
        # the repository's 48 layers, eight sequences cut to 1,024 tokens
        _evict("evict_48", 48, 8, 4, 128, 16, 1100, 2200, 1024, 4, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv_heads = rng.choice([1, 2, 4, 8])
    return kv_heads * rng.choice([1, 2, 3, 4, 7, 8, 16]), kv_heads


def draw(rng):
    r = rng.random()
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([1, 8, 16, 24, 64, 256])
    if r < 0.25:
        heads, kv_heads = _heads(rng)
        dim = rng.choice([64, 128, 128])
        # no more values than rotate_chunk's
        tokens = _log(rng, 1, 8192 * 40 * 128 // (dim * max(40, heads + 2 * kv_heads)))
        return _rotate(None, tokens, min(tokens, _log(rng, 1, 64)), heads, kv_heads, dim,
                       rng.choice([dim, dim, dim // 2, dim - 16]), page, rng.choice([0, 0, 1 << 20]),
                       rng.random() < 0.7, rng.random() < 0.4, dtype)
    if r < 0.75:
        kind = rng.choice(["chunk", "chunk", "weigh"])
        heads, kv_heads = _heads(rng)
        dim = rng.choice([64, 128, 128])
        window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 1, 4096), rng.choice([0, 1, 4, 30]))])
        if rng.random() < 0.5:   # single tokens: no more bytes than the listed batch's
            rows = _log(rng, 1, 64)
            top = (8192 if kind == "chunk" else 4096) * 64 * 4 // (rows * max(kv_heads, 4))
            len_hi = _log(rng, 1, min(131072, top))
            return _chunk(None, rows, heads, kv_heads, dim, 1, 1, rng.choice([1, len_hi]), len_hi, page, window, sinks,
                          dtype, kind)
        rows = _log(rng, 1, 12)
        new_hi = _log(rng, 2, max(2, (4096 if kind == "chunk" else 2048) * 32 // (rows * max(32, heads))))
        # no more products than the listed prompt's, counted by the tokens that its queries see
        top = (6000 if kind == "chunk" else 1500) * (4096 if kind == "chunk" else 2048) * 32 // (rows * new_hi * heads)
        len_hi = max(new_hi, min(_log(rng, new_hi, 16 * new_hi), top, 65536))
        return _chunk(None, rows, heads, kv_heads, dim, rng.choice([0, 1, new_hi]), new_hi,
                      rng.choice([new_hi, len_hi]), len_hi, page, window, sinks, dtype, kind)
    layers = _log(rng, 1, 24)
    kv_heads = rng.choice([1, 2, 4])
    page = rng.choice([8, 16, 24])
    len_hi = _log(rng, 40, 4000)
    keep = max(1, min(len_hi, int(len_hi * rng.uniform(0.2, 1.05))))
    sinks = rng.choice([0, 1, 4, 30])
    sinks = sinks if sinks <= keep // 2 else 0
    return _evict(None, layers, _log(rng, 1, 8), kv_heads, rng.choice([64, 128]), page,
                  rng.choice([len_hi // 2, len_hi]), len_hi, keep, sinks, rng.randint(0, keep - sinks) // 2)


# ---- inputs

def _randn(gen, shape, dtype, std):
    """Normal values of the seed, drawn on the GPU a slice at a time."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    step = 1 << 26
    for a in range(0, flat.numel(), step):
        b = min(a + step, flat.numel())
        flat[a:b] = torch.randn(b - a, generator=gen, device="cuda", dtype=torch.float32).mul_(std)
    return out


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _cache(rng, lens, pt, pages, longest):
    """Slots in some order, one for each length and one left empty: (slot ids, tables, refs, lengths by slot)."""
    n = len(lens)
    held = -(-lens // pt)
    perm = rng.permutation(pages)
    slot = rng.permutation(n + 1)[:n]
    tables = np.full((n + 1, -(-longest // pt) + 1), -1, dtype=np.int32)
    refs = np.zeros(pages, dtype=np.int32)
    by_slot = np.zeros(n + 1, dtype=np.int32)
    at = 0
    for i, s in enumerate(slot):
        ids = perm[at:at + held[i]]
        at += held[i]
        tables[s, :held[i]] = ids
        refs[ids] = 1
        by_slot[s] = lens[i]
    return slot.astype(np.int32), tables, refs, by_slot


def _freqs(case):
    """Angle for each position and pair, in 64 bits."""
    return 10000.0 ** (-np.arange(0, case["rot"], 2) / case["rot"])


def _rotate_inputs(case, seed):
    rng, gen = np.random.default_rng(seed), _gen(seed)
    T, S, D, Hk = case["tokens"], case["seqs"], case["dim"], case["kv_heads"]
    dt = DTYPES[case["dtype"]]
    new = np.diff(np.concatenate([[0], np.sort(rng.choice(np.arange(1, T), S - 1, replace=False)), [T]])) if S > 1 else np.array([T])
    before = rng.integers(0, 300, S)
    slot, tables, refs, lens = _cache(rng, before + new, case["page"], (T + 300 * S) // case["page"] + S, T + 300)
    slots = np.repeat(slot, new).astype(np.int32)
    pos = np.concatenate([b + np.arange(n) for b, n in zip(before, new)]).astype(np.int32)
    order = rng.permutation(T)   # tokens in no order of their own
    slots, pos = slots[order], pos[order]
    qkv = _randn(gen, (T, (case["heads"] + 2 * Hk) * D), dt, 1.0)
    w = [(1 + 0.2 * torch.randn(D, generator=gen, device="cuda")).to(dt) for _ in range(2)] if case["norm"] else [None] * 2
    pool = _randn(gen, (1, 2, refs.size, case["page"], Hk, D), dt, 1.0)
    return (pool, qkv, w, *map(_dev, (tables, refs, lens, slots, pos, pos + np.int32(case["far"]), _freqs(case))))


def _lengths(case, rng):
    # the batch's new tokens are as many whatever the seed; which row has how many is the seed's
    new = np.random.default_rng(case["rows"]).integers(case["new_lo"], case["new_hi"] + 1, case["rows"])
    new = rng.permutation(new)
    lens = rng.integers(case["len_lo"], case["len_hi"] + 1, case["rows"])
    return np.maximum(new, lens), new


def _chunk_inputs(case, seed):
    rng, gen = np.random.default_rng(seed), _gen(seed)
    lens, new = _lengths(case, rng)
    dt = DTYPES[case["dtype"]]
    slot, tables, refs, by_slot = _cache(rng, lens, case["page"], int((-(-lens // case["page"])).sum()) + 3,
                                         max(case["len_hi"], case["new_hi"]))
    starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    pool = _randn(gen, (1, 2, refs.size, case["page"], case["kv_heads"], case["dim"]), dt, 1.0)
    # queries wide enough that a row's probabilities are uneven
    q = _randn(gen, (max(1, int(starts[-1])), case["heads"], case["dim"]), dt, 2.0)
    weights = None
    if case["kind"] == "weigh":   # what earlier queries have left
        weights = torch.rand((by_slot.size, case["kv_heads"], tables.shape[1] * case["page"]), generator=gen, device="cuda")
    return (lens, new), pool, q, weights, *map(_dev, (tables, refs, by_slot, slot, starts))


def _evict_inputs(case, seed):
    rng, gen = np.random.default_rng(seed), _gen(seed)
    lens = rng.integers(max(1, case["len_lo"]), case["len_hi"] + 1, case["seqs"])
    lens[0] = case["len_hi"]
    keep = np.minimum(lens, case["keep"]).astype(np.int32)
    slot, tables, refs, by_slot = _cache(rng, lens, case["page"], case["seqs"] * -(-case["len_hi"] // case["page"]) + 3,
                                         case["len_hi"])
    pool = _randn(gen, (case["layers"], 2, refs.size, case["page"], case["kv_heads"], case["dim"]), torch.bfloat16, 1.0)
    # a few tokens have most of the weight; some have had none yet
    w = torch.randn((case["layers"], by_slot.size, case["kv_heads"], tables.shape[1] * case["page"]), generator=gen,
                    device="cuda").mul_(2.0).exp_()
    w[torch.rand(w.shape, generator=gen, device="cuda") < 0.1] = 0.0
    return (lens, keep), pool, w, *map(_dev, (tables, refs, by_slot, slot, keep, (lens - keep).astype(np.int32)))


def prepare(case, seed):
    st = dict(case=case)
    kind = case["kind"]
    if kind == "rotate":
        (st["pool"], st["qkv"], st["w"], st["tables"], st["refs"], st["lens"], st["slots"], st["pos"], st["positions"],
         st["freqs"]) = _rotate_inputs(case, seed)
        H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
        heads = st["qkv"].view(case["tokens"], H + 2 * Hk, D)
        st["q"], st["k"], st["v"] = heads[:, :H], heads[:, H:H + Hk], heads[:, H + Hk:]
        st["q_out"] = torch.empty((case["tokens"], H, D), dtype=st["qkv"].dtype, device="cuda")
    elif kind in ("chunk", "weigh"):
        (st["host"], st["pool"], st["q"], st["weights"], st["tables"], st["refs"], st["lens"], st["slots"],
         st["starts"]) = _chunk_inputs(case, seed)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(st["q"].shape[:2], dtype=torch.float32, device="cuda")
    else:
        (st["host"], st["pool"], st["weights"], st["tables"], st["refs"], st["lens"], st["slots"], st["keep"],
         st["back"]) = _evict_inputs(case, seed)
        st["kept"] = torch.full((case["layers"], case["seqs"], case["kv_heads"], int(st["host"][1].max())), -1,
                                dtype=torch.int32, device="cuda")
        st["weights_out"] = torch.zeros_like(st["weights"])
    if own:
        from paper_2609_09800_amd import hbf
        st["op"] = hbf.KvPages(st["pool"], refs=st["refs"], tables=st["tables"], lens=st["lens"])
    return st


# ---- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"rotate": _rotate_own, "chunk": _chunk_own, "weigh": _chunk_own, "evict": _evict_own}[kind](state)
    return {"rotate": _rotate_plain, "chunk": _chunk_plain, "weigh": _chunk_plain, "evict": _evict_plain}[kind](state)


def _bits(pool):
    return pool.view(torch.int16)


def _rotate_own(s):
    c = s["case"]
    s["op"].write_rotated(0, s["q"], s["k"], s["v"], s["slots"], s["pos"], s["freqs"], q_out=s["q_out"],
                          q_weight=s["w"][0], k_weight=s["w"][1], eps=EPS, positions=s["positions"],
                          interleaved=c["interleaved"])
    return s["q_out"], s["pool"]


def _chunk_own(s):
    c = s["case"]
    s["op"].attention(0, s["q"], s["out"], s["slots"], s["starts"], lse=s["lse"], weights=s["weights"],
                      window=c["window"], sinks=c["sinks"])
    return (s["out"], s["lse"]) if s["weights"] is None else (s["out"], s["lse"], s["weights"])


def _evict_own(s):
    c = s["case"]
    s["op"].evict(s["slots"], s["keep"], s["weights"], s["kept"], sinks=c["sinks"], recent=c["recent"],
                  weights_out=s["weights_out"])
    kept_lens = s["lens"].clone()
    s["op"].extend(s["slots"], s["back"])
    return _bits(s["pool"]), s["tables"], s["refs"], s["lens"], kept_lens, s["kept"], s["weights_out"]


def _rotate_plain(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2

    def norm(x, w):
        x = x.float()
        if w is None:
            return x
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()

    angle = s["positions"].double()[:, None] * s["freqs"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turn(x):
        if c["interleaved"]:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            both = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:rot]
            both = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        return torch.cat([both, x[..., rot:]], -1)

    dt = s["pool"].dtype
    s["q_out"].copy_(turn(norm(s["q"], s["w"][0])).to(dt))
    pos = s["pos"].long()
    page = s["tables"][s["slots"].long(), pos // c["page"]].long()
    s["pool"][0, 0, page, pos % c["page"]] = turn(norm(s["k"], s["w"][1])).to(dt)
    s["pool"][0, 1, page, pos % c["page"]] = s["v"]
    return s["q_out"], s["pool"]


def _chunk_plain(s):
    c = s["case"]
    Hk, D, pt = c["kv_heads"], c["dim"], c["page"]
    G = c["heads"] // Hk
    kp, vp = s["pool"][0]
    at = 0
    for i, (L, n) in enumerate(zip(s["host"][0].tolist(), s["host"][1].tolist())):
        if n == 0:
            continue
        pages = s["tables"][s["slots"][i].long(), :-(-L // pt)].long()
        k = kp[pages].float().view(-1, Hk, D)[:L].permute(1, 2, 0).contiguous()
        v = vp[pages].float().view(-1, Hk, D)[:L].transpose(0, 1).contiguous()
        q = (s["q"][at:at + n].float() / math.sqrt(D)).view(n, Hk, G, D).transpose(0, 1).reshape(Hk, n * G, D)
        j, p = torch.arange(L, device="cuda")[None, :], torch.arange(L - n, L, device="cuda")[:, None]
        seen = j <= p
        if c["window"]:
            seen = seen & ((j > p - c["window"]) | (j < c["sinks"]))
        sc = torch.matmul(q, k).view(Hk, n, G, L).masked_fill_(~seen[None, :, None, :], -math.inf)
        m = sc.amax(-1, keepdim=True)
        e = torch.exp(sc.sub_(m))
        l = e.sum(-1, keepdim=True)
        o = torch.matmul(e.view(Hk, n * G, L), v).view(Hk, n, G, D) / l
        s["out"][at:at + n] = o.transpose(0, 1).reshape(n, Hk * G, D).to(s["q"].dtype)
        s["lse"][at:at + n] = (m + torch.log(l))[..., 0].transpose(0, 1).reshape(n, Hk * G)
        if s["weights"] is not None:
            s["weights"][s["slots"][i].long(), :, :L] += (e / l).view(Hk, n * G, L).sum(1)
        at += n
    return (s["out"], s["lse"]) if s["weights"] is None else (s["out"], s["lse"], s["weights"])


def _evict_plain(s):
    c = s["case"]
    pt, s0, rec = c["page"], c["sinks"], c["recent"]
    pool, tables, refs, lens = s["pool"], s["tables"], s["refs"], s["lens"]
    N, Hk, D = c["layers"], c["kv_heads"], c["dim"]
    slots = s["slots"].long()
    for i, (L, keep) in enumerate(zip(s["host"][0].tolist(), s["host"][1].tolist())):
        slot = slots[i]
        w = s["weights"].index_select(1, slot[None])[:, 0, :, :L]
        m = keep - rec if keep < L else keep   # the middle ends here afterwards
        src = torch.arange(keep, device="cuda").expand(N, Hk, keep).clone()
        if keep < L:
            mid = w[:, :, s0:L - rec]
            best = torch.sort(mid, dim=-1, descending=True, stable=True)[1][..., :m - s0]
            chosen = torch.zeros_like(mid, dtype=torch.bool).scatter_(-1, best, True)
            stay, move = chosen[..., :m - s0], chosen[..., m - s0:]
            if m > s0:
                # those behind the middle's new end, in order, to the places that are free before it, in order
                movers = m + torch.argsort((~move).to(torch.int8), dim=-1, stable=True)
                rank = (torch.cumsum((~stay).long(), -1) - 1).clamp(0, move.shape[-1] - 1)
                src[..., s0:m] = torch.where(stay, src[..., s0:m], movers.gather(-1, rank))
            src[..., m:] += L - keep
            tok = pool[:, :, tables[slot, :-(-L // pt)].long()].view(N, 2, -1, Hk, D)
            new = tok.gather(2, src.transpose(1, 2)[:, None, :, :, None].expand(N, 2, keep, Hk, D))
            tok[:, :, :keep] = new
            first = tables[slot, :-(-keep // pt)].long()
            pool[:, :, first] = tok[:, :, :first.numel() * pt].view(N, 2, -1, pt, Hk, D)
            gone = tables[slot, -(-keep // pt):-(-L // pt)].long()
            refs[gone] -= 1
            tables[slot, -(-keep // pt):-(-L // pt)] = -1
            lens[slot] = keep
        s["kept"][:, i, :, :keep] = src.to(torch.int32)
        s["kept"][:, i, :, keep:] = -1
        s["weights_out"][:, slot, :, :keep] = w.gather(-1, src)
        s["weights_out"][:, slot, :, keep:L] = 0.0
    kept_lens = lens.clone()
    # extend: every sequence grows back, with the lowest free pages, in order
    before = torch.div(lens[slots] + pt - 1, pt, rounding_mode="floor")
    lens[slots] += s["back"]
    need = torch.div(lens[slots] + pt - 1, pt, rounding_mode="floor") - before
    free = torch.argsort((refs != 0).to(torch.int8), stable=True).to(torch.int32)
    off = torch.cumsum(need, 0) - need
    col = torch.arange(tables.shape[1], device="cuda")[None, :] - before[:, None]
    take = (col >= 0) & (col < need[:, None])
    rank = (off[:, None] + col).clamp(0, refs.numel() - 1)
    tables[slots] = torch.where(take, free[rank], tables[slots])
    refs[free[rank[take]].long()] = 1
    return _bits(pool), tables, refs, lens, kept_lens, s["kept"], s["weights_out"]


# ---- what a pass cannot do without

def _seen(case, lens, new):
    """(query, token) pairs of one head, and tokens that some query of a row sees."""
    pairs = tokens = 0
    for L, n in zip(lens.tolist(), new.tolist()):
        if n == 0:
            continue
        p = np.arange(L - n, L) + 1
        if case["window"]:
            sinks = np.minimum(case["sinks"], p)
            pairs += int(np.maximum(np.minimum(p, case["window"]), np.minimum(p, case["window"] + sinks)).sum())
            tokens += min(L, n - 1 + case["window"] + case["sinks"])
        else:
            pairs += int(p.sum())
            tokens += L
    return pairs, tokens


def work(case):
    kind, Hk, D = case["kind"], case["kv_heads"], case["dim"]
    if kind == "rotate":
        values = case["tokens"] * (case["heads"] + 2 * Hk) * D
        return {"bytes": int(4 * values + 12 * case["tokens"]), "flops": int(7 * values)}
    rng = np.random.default_rng(1)
    if kind in ("chunk", "weigh"):
        pairs = tokens = new_all = 0
        for _ in range(8):
            lens, new = _lengths(case, rng)
            a, b = _seen(case, lens, new)
            pairs, tokens, new_all = pairs + a / 8, tokens + b / 8, new_all + new.sum() / 8
        qo = new_all * case["heads"] * (4 * D + 4)
        w = tokens * Hk * 8 if kind == "weigh" else 0
        return {"bytes": int(qo + tokens * (Hk * D * 4 + 4 / case["page"]) + w), "flops": int(4 * case["heads"] * D * pairs)}
    L = (max(1, case["len_lo"]) + case["len_hi"]) / 2
    keep = min(L, case["keep"])
    mid_old, mid_new = L - case["sinks"] - case["recent"], keep - case["sinks"] - case["recent"]
    moved = mid_new * (mid_old - mid_new) / max(mid_old, 1) + (case["recent"] if keep < L else 0)
    heads = case["layers"] * case["seqs"] * Hk
    # weights read, written as kept; kept lists; the tokens that move, read and written, K and V
    return {"bytes": int(heads * (4 * L + 4 * L + 4 * keep + moved * D * 2 * 2 * 2)), "flops": 0}


# ---- the definition, in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind == "rotate":
        return _rotate_exact(case, seed)
    if kind in ("chunk", "weigh"):
        return _chunk_exact(case, seed)
    return None   # copies and whole numbers


def _rotate_exact(case, seed):
    pool, qkv, w, tables, _, _, slots, pos, positions, freqs = _rotate_inputs(case, seed)
    H, Hk, D, pairs = case["heads"], case["kv_heads"], case["dim"], case["rot"] // 2
    x = qkv.view(case["tokens"], H + 2 * Hk, D).double()
    turn = torch.polar(torch.ones((case["tokens"], pairs), dtype=torch.float64, device="cuda"),
                       positions.double()[:, None] * freqs[None, :])
    done = []
    for lo, hi, weight in ((0, H, w[0]), (H, H + Hk, w[1])):
        y = x[:, lo:hi]
        if weight is not None:
            y = y / (y.square().sum(-1, keepdim=True) / D + EPS).sqrt() * weight.double()
        y = y.clone()
        pick = (slice(0, case["rot"], 2), slice(1, case["rot"], 2)) if case["interleaved"] else (slice(0, pairs), slice(pairs, 2 * pairs))
        z = torch.complex(y[..., pick[0]].contiguous(), y[..., pick[1]].contiguous()) * turn[:, None, :]
        y[..., pick[0]], y[..., pick[1]] = z.real, z.imag
        done.append(y)
    out = pool.double()
    flat = (tables[slots.long(), (pos // case["page"]).long()].long() * case["page"] + pos % case["page"])
    out[0, 0].view(-1, Hk, D).index_copy_(0, flat, done[1])
    out[0, 1].view(-1, Hk, D).index_copy_(0, flat, x[:, H + Hk:].contiguous())
    return done[0], out


def _chunk_exact(case, seed):
    (lens, new), pool, q, weights, tables, _, _, slots, _ = _chunk_inputs(case, seed)
    Hq, Hk, D, pt = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device="cuda")
    total = None if weights is None else weights.double()
    at = 0
    for i in range(case["rows"]):
        L, n = int(lens[i]), int(new[i])
        slot = int(slots[i])
        pages = tables[slot, :-(-L // pt)].long()
        pos = torch.arange(L - n, L, device="cuda")
        dist = pos[:, None] - torch.arange(L, device="cuda")[None, :]
        hidden = dist < 0
        if case["window"]:
            hidden |= (dist >= case["window"]) & (torch.arange(L, device="cuda") >= case["sinks"])[None, :]
        for h in range(Hq if n else 0):
            kk, vv = (pool[0, x, pages, :, h // (Hq // Hk)].double().reshape(-1, D)[:L] for x in range(2))
            sc = torch.nn.functional.linear(q[at:at + n, h].double(), kk) * D ** -0.5
            sc.masked_fill_(hidden, -math.inf)
            p = torch.softmax(sc, dim=-1)
            out[at:at + n, h] = p @ vv
            lse[at:at + n, h] = torch.logsumexp(sc, dim=-1)
            if total is not None:
                total[slot, h // (Hq // Hk), :L] += p.sum(0)
        at += n
    return (out, lse) if total is None else (out, lse, total)
