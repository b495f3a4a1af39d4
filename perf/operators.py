"""One decode layer's operators over weights and KV pages, as cases that can be timed.

Kinds:
  moe      a whole mixture-of-experts layer for a few tokens: router, top-k, SwiGLU experts, weighted sum
  attn     decode attention of a batch whose rows share one long prefix and each have own tokens, over cache pages
  kv_step  the cache pages between two decode steps: sequences end, new ones fork from their parents, grow by a
           token and get its K and V (every layer's)
  kv_pack  the cache's compaction: live pages move to the front of the pool, tables and counts follow

``own`` chooses what ``run`` calls: the plain form (elementary torch operations in 32 bits) or the framework.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ---- cases

def _moe(name, tokens, experts, topk, hidden, ffn, dtype="bf16", zipf=1.1):
    return dict(name=name, kind="moe", tokens=tokens, experts=experts, topk=topk, hidden=hidden, ffn=ffn, dtype=dtype,
                zipf=zipf)


def _attn(name, rows, heads, kv_heads, dim, prefix, own_lo, own_hi, page, dtype="bf16"):
    return dict(name=name, kind="attn", rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, prefix=prefix,
                own_lo=own_lo, own_hi=own_hi, page=page, dtype=dtype)


def _step(name, layers, kv_heads, dim, page, parents, each, len_lo, len_hi):
    return dict(name=name, kind="kv_step", layers=layers, kv_heads=kv_heads, dim=dim, page=page, parents=parents,
                each=each, len_lo=len_lo, len_hi=len_hi)


def _pack(name, layers, kv_heads, dim, page, pages, live, len_hi):
    return dict(name=name, kind="kv_pack", layers=layers, kv_heads=kv_heads, dim=dim, page=page, pages=pages,
                live=live, len_hi=len_hi)


def listed():
    return [
        # one token of one user through the repository's MoE layer (128 experts, top 8): eight experts' weights
        _moe("moe_one", 1, 128, 8, 2048, 768),
        # a small serving batch
        _moe("moe_b16", 16, 128, 8, 2048, 768),
        # the 64-token decode batch of the repository's traces: most experts of the layer are read
        _moe("moe_b64", 64, 128, 8, 2048, 768),
        # a small layer of odd sizes in the other type: what a call costs by itself
        _moe("moe_odd", 5, 20, 3, 328, 104, "fp16", 0.0),
        # one user behind the repository's shared system prompt (4,096 tokens, 4 KV heads of 128)
        _attn("attn_one", 1, 32, 4, 128, 4096, 300, 300, 16),
        # a batch behind the same prompt with histories of its own: most of the bytes are the rows' own
        _attn("attn_b64", 64, 32, 4, 128, 4096, 1, 1024, 16),
        # a batch behind a long shared document: most of the work is the prefix, read once for 64 rows
        _attn("attn_doc", 64, 32, 4, 128, 32771, 1, 256, 16),
        # small, odd: narrow heads, pages of 24 tokens, rows that have no token of their own yet
        _attn("attn_odd", 7, 6, 2, 64, 1003, 0, 130, 24, "fp16"),
        # parallel samples of two prompts, one layer's cache: what the calls cost by themselves
        _step("kv_step_small", 1, 4, 128, 16, 2, 4, 100, 700),
        # the repository's 48 layers, 8 samples of each of 8 prompts begin (a KV page of a layer is 16 KiB)
        _step("kv_step_48", 48, 4, 128, 16, 8, 8, 100, 1100),
        # a small pool with a few holes
        _pack("kv_pack_small", 1, 4, 128, 16, 512, 0.6, 300),
        # a large pool, two fifths of it freed by sequences that ended
        _pack("kv_pack_8", 8, 4, 128, 16, 4096, 0.6, 2000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    r = rng.random()
    if r < 0.4:
        hidden, ffn = rng.choice([(2048, 768), (2048, 768), (8 * rng.randint(16, 256), 8 * rng.randint(8, 96))])
        experts = rng.choice([8, 20, 32, 64, 100, 128])
        return _moe(None, _log(rng, 1, 64), experts, rng.randint(1, min(8, experts)), hidden, ffn,
                    rng.choice(["bf16", "bf16", "fp16"]), rng.choice([0.0, 1.1]))
    if r < 0.8:
        kv_heads = rng.choice([1, 2, 4, 8])
        group = rng.choice([1, 2, 3, 4, 7, 8, 16])
        rows = _log(rng, 1, 64)
        # prefix work stays below attn_doc's (64 * 32 query heads over 32,771 tokens), own pages below attn_b64's
        top = min(131072, 64 * 32 * 32771 // (rows * kv_heads * group), 32771 * 4 // kv_heads)
        own_hi = _log(rng, 1, 1024 if kv_heads <= 4 else 512)
        return _attn(None, rows, kv_heads * group, kv_heads, rng.choice([64, 128, 128]), _log(rng, 64, max(64, top)),
                     rng.choice([0, 1, own_hi]), own_hi, rng.choice([1, 8, 16, 24, 64, 256]),
                     rng.choice(["bf16", "bf16", "fp16"]))
    if r < 0.9:
        hi = _log(rng, 20, 2000)
        return _step(None, _log(rng, 1, 30), rng.choice([1, 2, 4]), rng.choice([64, 128]), rng.choice([1, 8, 16, 24]),
                     _log(rng, 1, 8), _log(rng, 1, 8), _log(rng, 1, hi), hi)
    layers, page = _log(rng, 1, 8), rng.choice([8, 16, 24])
    return _pack(None, layers, rng.choice([1, 2, 4]), rng.choice([64, 128]), page,
                 _log(rng, 100, min(20000, 4096 * 16 * 8 // (page * layers))), rng.uniform(0.1, 0.95), _log(rng, 20, 1500))


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


def _logw(case, rng):
    """Log popularity of each expert (Zipf over a random order, as in the repository's traces)."""
    rank = rng.permutation(case["experts"]).astype(np.float64) + 1.0
    return -case["zipf"] * np.log(rank)


def _moe_inputs(case, seed):
    T, E, H, F = case["tokens"], case["experts"], case["hidden"], case["ffn"]
    dt = DTYPES[case["dtype"]]
    gen = _gen(seed)
    # the tokens share a direction along which the router's rows carry the experts' popularity
    c = torch.randn(H, generator=gen, device="cuda")
    logw = torch.from_numpy(_logw(case, np.random.default_rng(seed))).cuda().float()
    x = (torch.randn((T, H), generator=gen, device="cuda") + c).to(dt)
    router = (torch.randn((E, H), generator=gen, device="cuda") / math.sqrt(H) + logw[:, None] * c / c.square().sum()).to(dt)
    gate_up = _randn(gen, (E, 2 * F, H), dt, 1 / math.sqrt(H))
    down = _randn(gen, (E, H, F), dt, 1 / math.sqrt(F))
    return x, router, gate_up, down


def _attn_inputs(case, seed):
    R, L, pt = case["rows"], case["prefix"], case["page"]
    dt = DTYPES[case["dtype"]]
    gen = _gen(seed)
    rng = np.random.default_rng(seed)
    own_lens = rng.integers(case["own_lo"], case["own_hi"] + 1, R)
    np_pre = -(-L // pt)
    cols = max(1, -(-case["own_hi"] // pt))
    held = -(-own_lens // pt)
    pages = np_pre + int(held.sum()) + 5
    perm = rng.permutation(pages)
    tables = np.full((R, cols), -1, dtype=np.int32)
    at = np_pre
    for r in range(R):
        tables[r, :held[r]] = perm[at:at + held[r]]
        at += held[r]
    pool = _randn(gen, (1, 2, pages, pt, case["kv_heads"], case["dim"]), dt, 1.0)
    # queries wide enough that a row's probabilities are uneven
    q = _randn(gen, (R, case["heads"], case["dim"]), dt, 2.0)
    return (pool, q, torch.from_numpy(perm[:np_pre].astype(np.int32)).cuda(), torch.from_numpy(tables).cuda(),
            torch.from_numpy(own_lens.astype(np.int32)).cuda())


def _step_inputs(case, seed):
    pt, npar, each = case["page"], case["parents"], case["each"]
    n = npar * each
    rng = np.random.default_rng(seed)
    lens = rng.integers(case["len_lo"], case["len_hi"] + 1, npar)
    held = -(-lens // pt)
    cols = -(-(case["len_hi"] + 1) // pt) + 1
    pages = npar * -(-case["len_hi"] // pt) + 2 * n + 8
    perm = rng.permutation(pages)
    slots = npar + n + 1
    tables = np.full((slots, cols), -1, dtype=np.int32)
    refs = np.zeros(pages, dtype=np.int32)
    all_lens = np.zeros(slots, dtype=np.int32)
    order = rng.permutation(slots)
    par, kid = order[:npar], order[npar:npar + n]
    at = 0
    for i, s in enumerate(par):
        ids = perm[at:at + held[i]]
        at += held[i]
        tables[s, :held[i]] = ids
        refs[ids] = 1
        all_lens[s] = lens[i]
    gen = _gen(seed)
    pool = _randn(gen, (case["layers"], 2, pages, pt, case["kv_heads"], case["dim"]), torch.bfloat16, 1.0)
    new = _randn(gen, (2, case["layers"], n, case["kv_heads"], case["dim"]), torch.bfloat16, 1.0)
    parents = np.repeat(par, each).astype(np.int32)
    pos = np.repeat(lens, each).astype(np.int32)   # where the children's new token goes
    dev = [torch.from_numpy(a).cuda() for a in (tables, refs, all_lens, parents, kid.astype(np.int32), pos)]
    return (pool, new[0], new[1], *dev)


def _pack_inputs(case, seed):
    pt, pages = case["page"], case["pages"]
    rng = np.random.default_rng(seed)
    cols = -(-case["len_hi"] // pt)
    free = list(rng.permutation(pages)[:max(1, int(case["live"] * pages))])
    slots = 2 + len(free) * pt * 5 // (2 * case["len_hi"])   # enough for the pages, the rest stay empty
    rows, lens = [], []
    refs = np.zeros(pages, dtype=np.int32)
    while free and len(rows) < slots:
        ln = int(rng.integers(1, case["len_hi"] + 1))
        held = min(-(-ln // pt), len(free))
        ln = min(ln, held * pt)
        row = np.full(cols, -1, dtype=np.int32)
        row[:held] = free[:held]
        if rows and lens[-1] >= pt and rng.random() < 0.3:   # the first pages of the sequence before, shared
            k = min(held, lens[-1] // pt)
            row[:k] = rows[-1][:k]
        refs[row[:held]] += 1
        free = free[held:]
        rows.append(row)
        lens.append(ln)
    while len(rows) < slots:
        rows.append(np.full(cols, -1, dtype=np.int32))
        lens.append(0)
    pool = _randn(_gen(seed), (case["layers"], 2, pages, pt, case["kv_heads"], case["dim"]), torch.bfloat16, 1.0)
    return (pool, torch.from_numpy(np.stack(rows)).cuda(), torch.from_numpy(refs).cuda(),
            torch.from_numpy(np.array(lens, dtype=np.int32)).cuda())


def prepare(case, seed):
    st = dict(case=case)
    kind = case["kind"]
    if kind == "moe":
        st["x"], st["router"], st["gate_up"], st["down"] = _moe_inputs(case, seed)
        if own:
            from paper_2609_09800_amd import hbf
            st["op"] = hbf.MoeLayer(st["gate_up"], st["down"], case["topk"], router=st["router"], max_tokens=case["tokens"])
            st["y"] = torch.empty_like(st["x"])
            st["ids"] = torch.empty((case["tokens"], case["topk"]), dtype=torch.int32, device="cuda")
            st["w"] = torch.empty((case["tokens"], case["topk"]), dtype=torch.float32, device="cuda")
    elif kind == "attn":
        st["pool"], st["q"], st["prefix"], st["tables"], st["own_lens"] = _attn_inputs(case, seed)
        if own:
            from paper_2609_09800_amd import hbf
            st["op"] = hbf.KvPages(st["pool"])
            st["out"] = torch.empty_like(st["q"])
            st["lse"] = torch.empty((case["rows"], case["heads"]), dtype=torch.float32, device="cuda")
    elif kind == "kv_step":
        (st["pool"], st["k"], st["v"], st["tables"], st["refs"], st["lens"], st["parents"], st["kids"],
         st["pos"]) = _step_inputs(case, seed)
        st["one"] = torch.ones_like(st["kids"])
        if own:
            from paper_2609_09800_amd import hbf
            st["op"] = hbf.KvPages(st["pool"], refs=st["refs"], tables=st["tables"], lens=st["lens"])
    else:
        st["pool"], st["tables"], st["refs"], st["lens"] = _pack_inputs(case, seed)
        if own:
            from paper_2609_09800_amd import hbf
            st["op"] = hbf.KvPages(st["pool"], refs=st["refs"], tables=st["tables"], lens=st["lens"])
            st["remap"] = torch.empty_like(st["refs"])
            st["refs_out"] = torch.empty_like(st["refs"])
            st["tables_out"] = torch.empty_like(st["tables"])
    return st


# ---- one pass

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"moe": _moe_own, "attn": _attn_own, "kv_step": _step_own, "kv_pack": _pack_own}[kind](state)
    return {"moe": _moe_plain, "attn": _attn_plain, "kv_step": _step_plain, "kv_pack": _pack_plain}[kind](state)


def _bits(pool):
    return pool.view(torch.int16)


def _moe_own(s):
    s["op"].forward(s["x"], s["y"], s["ids"], s["w"])
    return s["y"], s["ids"], s["w"]


def _attn_own(s):
    s["op"].prefix_attention(0, s["q"], s["out"], s["prefix"], s["case"]["prefix"], s["tables"], s["own_lens"], lse=s["lse"])
    return s["out"], s["lse"]


def _step_own(s):
    op = s["op"]
    op.free(s["kids"])
    op.fork(s["parents"], s["kids"])
    op.extend(s["kids"], s["one"])
    op.write(s["k"], s["v"], s["kids"], s["pos"])
    return _bits(s["pool"]), s["tables"], s["refs"], s["lens"]


def _pack_own(s):
    s["op"].compact(s["remap"], tables_out=s["tables_out"], refs_out=s["refs_out"])
    return _bits(s["pool"]), s["tables_out"], s["refs_out"], s["remap"]


def _moe_plain(s):
    c = s["case"]
    T, k, F = c["tokens"], c["topk"], c["ffn"]
    x = s["x"].float()
    logits = x @ s["router"].float().t()
    top, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k]
    # the softmax over all experts, renormalised over the chosen ones
    w = torch.exp(top - top[:, :1])
    w = w / w.sum(dim=1, keepdim=True)
    pairs = ids.reshape(-1)
    parts = []
    for a in range(0, T * k, 32):
        e = pairs[a:a + 32]
        xt = x[torch.arange(a, a + e.numel(), device="cuda") // k]
        gu = torch.matmul(s["gate_up"][e].float(), xt[:, :, None])[:, :, 0]
        g, u = gu[:, :F], gu[:, F:]
        h = g / (1 + torch.exp(-g)) * u
        parts.append(torch.matmul(s["down"][e].float(), h[:, :, None])[:, :, 0])
    y = (torch.cat(parts).view(T, k, -1) * w[:, :, None]).sum(dim=1)
    return y.to(s["x"].dtype), ids.to(torch.int32), w


def _attn_plain(s):
    c = s["case"]
    R, Hq, Hk, D, pt, L = c["rows"], c["heads"], c["kv_heads"], c["dim"], c["page"], c["prefix"]
    G = Hq // Hk
    kp, vp = s["pool"][0]
    q = s["q"].float().view(R, Hk, G, D) / math.sqrt(D)
    # the prefix, all rows at once, a head at a time
    k0 = kp[s["prefix"].long()].float().view(-1, Hk, D)[:L]
    v0 = vp[s["prefix"].long()].float().view(-1, Hk, D)[:L]
    sc0 = torch.stack([(q[:, h].reshape(R * G, D) @ k0[:, h].t()).view(R, G, L) for h in range(Hk)], 1)
    # each row's own pages, padded to the longest
    t = s["tables"].long().clamp(min=0)
    k1 = kp[t].float().view(R, -1, Hk, D).transpose(1, 2).contiguous()
    v1 = vp[t].float().view(R, -1, Hk, D).transpose(1, 2).contiguous()
    seen = torch.arange(k1.shape[2], device="cuda")[None, :] < s["own_lens"][:, None]
    sc1 = torch.matmul(q, k1.transpose(2, 3).contiguous())
    sc1 = sc1.masked_fill(~seen[:, None, None, :], -math.inf)
    m = torch.maximum(sc0.amax(-1), sc1.amax(-1))
    p0, p1 = torch.exp(sc0 - m[..., None]), torch.exp(sc1 - m[..., None])
    l = p0.sum(-1) + p1.sum(-1)
    o0 = torch.stack([(p0[:, h].reshape(R * G, L) @ v0[:, h]).view(R, G, D) for h in range(Hk)], 1)
    o = (o0 + torch.matmul(p1, v1)) / l[..., None]
    return o.reshape(R, Hq, D).to(s["q"].dtype), (m + torch.log(l)).reshape(R, Hq)


def _step_plain(s):
    pool, tables, refs, lens = s["pool"], s["tables"], s["refs"], s["lens"]
    pt = s["case"]["page"]
    kids, par = s["kids"].long(), s["parents"].long()
    cols = torch.arange(tables.shape[1], device="cuda")
    n = kids.numel()
    # free: the children of the step before give their pages back
    rows, held = tables[kids], (lens[kids] + pt - 1) // pt
    live = cols[None, :] < held[:, None]
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), -live.view(-1).to(torch.int32))
    tables[kids] = torch.where(live, -1, rows)
    lens[kids] = 0
    # fork: full pages are shared, a last page that is part full is copied to the lowest free one
    rows, pl = tables[par], lens[par]
    full, part = pl // pt, pl % pt
    shared = cols[None, :] < full[:, None]
    refs.index_add_(0, rows.clamp(min=0).view(-1).long(), shared.view(-1).to(torch.int32))
    free = torch.argsort((refs != 0).to(torch.int32), stable=True)
    rank = torch.empty_like(kids)
    rank[torch.argsort((part == 0).to(torch.int32), stable=True)] = torch.arange(n, device="cuda")
    new = free[rank]
    has = (part > 0).to(torch.int32)
    refs.index_add_(0, new, has)
    at_part = (cols[None, :] == full[:, None]) & (part > 0)[:, None]
    tables[kids] = torch.where(shared, rows, torch.where(at_part, new[:, None].to(torch.int32), tables[kids]))
    lens[kids] = pl
    src = tables[par, full.long().clamp(max=tables.shape[1] - 1)].clamp(min=0).long()
    keep = (torch.arange(pt, device="cuda")[None, :] < part[:, None])[None, None, :, :, None, None]
    pool[:, :, new] = torch.where(keep, pool[:, :, src], pool[:, :, new])
    # extend: one more token each; those at a page's end get the lowest free pages, in order
    ln = lens[kids]
    need = (ln % pt == 0).to(torch.int32)
    free = torch.argsort((refs != 0).to(torch.int32), stable=True)
    new = free[(torch.cumsum(need, 0) - need).long()]
    refs.index_add_(0, new, need)
    at = (ln // pt).long()
    tables[kids, at] = torch.where(need > 0, new.to(torch.int32), tables[kids, at])
    lens[kids] = ln + 1
    # write: the new token's K and V
    pos = s["pos"].long()
    pg = tables[kids, pos // pt].long()
    pool[:, 0, pg, pos % pt] = s["k"]
    pool[:, 1, pg, pos % pt] = s["v"]
    return _bits(pool), tables, refs, lens


def _pack_plain(s):
    pool, tables, refs, lens = s["pool"], s["tables"], s["refs"], s["lens"]
    pt = s["case"]["page"]
    page = torch.arange(refs.numel(), device="cuda")
    live = refs > 0
    n_live = live.sum()
    src = torch.nonzero(live & (page >= n_live))[:, 0]
    dst = torch.nonzero(~live & (page < n_live))[:, 0]
    remap = torch.where(live, page, -1)
    remap[src] = dst
    refs_out = refs.clone()
    refs_out[dst] = refs[src]
    refs_out[src] = 0
    held = (lens + pt - 1) // pt
    used = torch.arange(tables.shape[1], device="cuda")[None, :] < held[:, None]
    tables_out = torch.where(used, remap[tables.clamp(min=0).long()].to(torch.int32), tables)
    pool[:, :, dst] = pool[:, :, src]
    return _bits(pool), tables_out, refs_out, remap.to(torch.int32)


# ---- what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind == "moe":
        T, E, k, H, F = case["tokens"], case["experts"], case["topk"], case["hidden"], case["ffn"]
        # distinct experts that the tokens choose, by drawing the router's choices as the inputs do
        rng = np.random.default_rng(1)
        act = 0
        for _ in range(8):
            z = rng.standard_normal((T, E)) * math.sqrt(2) + _logw(case, rng)[None, :]
            act += np.unique(np.argsort(-z, axis=1)[:, :k]).size
        act /= 8
        return {"bytes": int(2 * (act * 3 * F * H + E * H + 2 * T * H) + 8 * T * k),
                "flops": int(2 * T * (k * 3 * F * H + E * H))}
    if kind == "attn":
        own_tok = case["rows"] * (case["own_lo"] + case["own_hi"]) / 2
        qo = case["rows"] * case["heads"] * (case["dim"] * 4 + 4)
        kv = (case["prefix"] + own_tok) * case["kv_heads"] * case["dim"] * 4
        ids = 4 * (case["prefix"] + own_tok) / case["page"]
        return {"bytes": int(qo + kv + ids),
                "flops": int(4 * case["heads"] * case["dim"] * (case["rows"] * case["prefix"] + own_tok))}
    tok = case["layers"] * 2 * case["kv_heads"] * case["dim"] * 2
    if kind == "kv_step":
        n = case["parents"] * case["each"]
        rows = (case["len_lo"] + case["len_hi"]) / 2 / case["page"]
        # part pages read and written, new tokens read and written, table rows cleared, read and written, counts twice
        return {"bytes": int(n * (tok * (case["page"] - 1) + 2 * tok + 4 * rows * 7)), "flops": 0}
    moved = case["pages"] * case["live"] * (1 - case["live"])
    return {"bytes": int(moved * tok * case["page"] * 2 + case["pages"] * 12 + case["pages"] * case["live"] * 8),
            "flops": 0}


# ---- the definition, in 64 bits

def exact(case, seed):
    kind = case["kind"]
    if kind == "moe":
        return _moe_exact(case, seed)
    if kind == "attn":
        return _attn_exact(case, seed)
    return None   # copies and whole numbers


def _moe_exact(case, seed):
    x, router, gate_up, down = _moe_inputs(case, seed)
    T, E, k, F = case["tokens"], case["experts"], case["topk"], case["ffn"]
    xd = x.double()
    prob = torch.softmax(torch.nn.functional.linear(xd, router.double()), dim=1).cpu().numpy()
    ids = np.zeros((T, k), dtype=np.int64)
    w = np.zeros((T, k))
    for t in range(T):
        best = sorted(range(E), key=lambda e: (-prob[t, e], e))[:k]
        ids[t] = best
        w[t] = prob[t, best] / prob[t, best].sum()
    y = torch.zeros((T, case["hidden"]), dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if t.size == 0:
            continue
        td = torch.from_numpy(t).cuda()
        both = gate_up[e].double() @ xd[td].t().contiguous()
        h = torch.nn.functional.silu(both[:F]) * both[F:]
        y.index_add_(0, td, (down[e].double() @ h).t().contiguous() * torch.from_numpy(w[t, j]).cuda()[:, None])
    return y, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(w).cuda()


def _attn_exact(case, seed):
    pool, q, prefix, tables, own_lens = _attn_inputs(case, seed)
    R, Hq, Hk, D, pt = case["rows"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros((R, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((R, Hq), dtype=torch.float64, device="cuda")
    lens = own_lens.tolist()
    for h in range(Hk):
        head = slice(h * (Hq // Hk), (h + 1) * (Hq // Hk))
        k0 = pool[0, 0, prefix.long(), :, h].double().reshape(-1, D)[:case["prefix"]]
        v0 = pool[0, 1, prefix.long(), :, h].double().reshape(-1, D)[:case["prefix"]]
        for r in range(R):
            own_pages = tables[r, :-(-lens[r] // pt)].long()
            kk = torch.cat([k0, pool[0, 0, own_pages, :, h].double().reshape(-1, D)[:lens[r]]])
            vv = torch.cat([v0, pool[0, 1, own_pages, :, h].double().reshape(-1, D)[:lens[r]]])
            sc = torch.nn.functional.linear(q[r, head].double(), kk) * D ** -0.5
            out[r, head] = torch.softmax(sc, dim=-1) @ vv
            lse[r, head] = torch.logsumexp(sc, dim=-1)
    return out, lse
