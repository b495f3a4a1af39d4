"""A KV cache's pages (extend, fork, free, copy, compact, write) against a
sequential model of the same rules in plain Python: every table, count,
length and byte of the pool must be equal."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL, ENOMEM, ENOWORKSPACE = 0, -1, -8, -4


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


class Plain:
    """The rules of include/hbf.h, one entry after another, on numpy arrays."""

    def __init__(self, pool, refs, tables, lens):
        self.pool, self.refs, self.tables, self.lens = pool, refs, tables, lens
        self.pt = pool.shape[3]

    def held(self, length):
        return -(-int(length) // self.pt)

    def take(self):
        p = int(np.flatnonzero(self.refs == 0)[0])
        self.refs[p] = 1
        return p

    def extend(self, slots, add):
        for s, a in zip(slots, add):
            for c in range(self.held(self.lens[s]), self.held(self.lens[s] + a)):
                self.tables[s, c] = self.take()
            self.lens[s] += a

    def fork(self, parents, children):
        for p, c in zip(parents, children):
            n = int(self.lens[p])
            for i in range(n // self.pt):
                self.tables[c, i] = self.tables[p, i]
                self.refs[self.tables[p, i]] += 1
            part = n % self.pt
            if part:
                new = self.take()
                self.tables[c, n // self.pt] = new
                self.pool[:, :, new, :part] = self.pool[:, :, self.tables[p, n // self.pt], :part]
            self.lens[c] = n

    def free(self, slots):
        for s in slots:
            for i in range(self.held(self.lens[s])):
                self.refs[self.tables[s, i]] -= 1
                self.tables[s, i] = -1
            self.lens[s] = 0

    def copy(self, src, dst):
        self.pool[:, :, dst] = self.pool[:, :, src].copy()

    def compact(self):
        live = np.flatnonzero(self.refs > 0)
        m = live.size
        src, dst = live[live >= m], np.flatnonzero(self.refs[:m] == 0)
        remap = np.full(self.refs.size, -1, dtype=np.int32)
        remap[live] = live
        remap[src] = dst
        self.pool[:, :, dst] = self.pool[:, :, src].copy()
        self.refs[dst] = self.refs[src]
        self.refs[src] = 0
        for s in range(self.lens.size):
            h = self.held(self.lens[s])
            self.tables[s, :h] = remap[self.tables[s, :h]]
        return remap

    def write(self, k, v, slots, pos, layer):
        for i, (s, p) in enumerate(zip(slots, pos)):
            page = self.tables[s, p // self.pt]
            for l in range(k.shape[0]):
                self.pool[layer + l, 0, page, p % self.pt] = k[l, i]
                self.pool[layer + l, 1, page, p % self.pt] = v[l, i]


class Both:
    """The cache on the GPU and its model, put through the same calls."""

    def __init__(self, torch, layers, pages, pt, heads, dim, slots, cols, seed=0, extra_cols=0, max_list=256):
        from paper_2609_09800_amd import hbf
        self.torch = torch
        rng = np.random.default_rng(seed)
        pool = rng.integers(-30000, 30000, (layers, 2, pages, pt, heads, dim)).astype(np.int16)
        tables = np.full((slots, cols + extra_cols), -1, dtype=np.int32)
        self.plain = Plain(pool, np.zeros(pages, np.int32), tables[:, :cols], np.zeros(slots, np.int32))
        dev = torch.from_numpy(tables).cuda()
        self.t = dict(pool=torch.from_numpy(pool).cuda().view(torch.bfloat16), refs=self.dev(self.plain.refs),
                      tables=dev[:, :cols], lens=self.dev(self.plain.lens))
        self.kv = hbf.KvPages(self.t["pool"], refs=self.t["refs"], tables=self.t["tables"], lens=self.t["lens"],
                              max_list=max_list)

    def dev(self, a):
        return self.torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def hold(self, page):
        """The caller holds a page itself."""
        self.plain.refs[page] += 1
        self.t["refs"][page] += 1

    def call(self, name, *lists):
        getattr(self.plain, name)(*lists)
        assert getattr(self.kv, name)(*[self.dev(x) for x in lists]) == OK

    def write(self, rng, slots, pos, layer, layers):
        heads, dim = self.plain.pool.shape[4:]
        k, v = (rng.integers(-30000, 30000, (layers, len(slots), heads, dim)).astype(np.int16) for _ in range(2))
        self.plain.write(k, v, slots, pos, layer)
        half = [self.torch.from_numpy(x).cuda().view(self.torch.bfloat16) for x in (k, v)]
        assert self.kv.write(*half, self.dev(slots), self.dev(pos), first_layer=layer) == OK

    def compact(self):
        want = self.plain.compact()
        remap = self.torch.full((want.size,), -7, dtype=self.torch.int32, device="cuda")
        assert self.kv.compact(remap) == OK
        assert np.array_equal(remap.cpu().numpy(), want)

    def same(self):
        assert self.kv.get_status() == OK
        for name in ("refs", "tables", "lens"):
            got = self.t[name].cpu().numpy()
            assert np.array_equal(got, getattr(self.plain, name)), name
        got = self.t["pool"].view(self.torch.int16).cpu().numpy()
        assert np.array_equal(got, self.plain.pool), "pool"


@pytest.mark.parametrize("layers,pages,pt,heads,dim,slots,cols", [
    (1, 40, 16, 1, 8, 6, 12), (3, 700, 8, 2, 64, 40, 30), (2, 9000, 1, 1, 8, 30, 700), (1, 4097, 24, 1, 16, 64, 50),
    (5, 300, 5, 4, 24, 20, 21), (1, 20000, 2, 1, 8, 40, 900), (2, 16390, 3, 1, 8, 90, 1200)])
def test_random_life_of_a_cache(torch, layers, pages, pt, heads, dim, slots, cols):
    say(f"kv life {layers} {pages} {pt} {heads} {dim} {slots} {cols}")
    rng = np.random.default_rng(pages)
    b = Both(torch, layers, pages, pt, heads, dim, slots, cols, seed=pages, extra_cols=3)
    p = b.plain
    b.hold(pages - 1)
    for step in range(40):
        empty = np.flatnonzero(p.lens == 0)
        some = rng.permutation(slots)
        what = rng.integers(0, 6)
        free_pages = int((p.refs == 0).sum())
        if what <= 1:
            s, add, need = [], [], 0
            for x in some[:rng.integers(1, slots)]:
                a = int(rng.integers(0, pt * 4))
                n = p.held(p.lens[x] + a) - p.held(p.lens[x])
                if p.held(p.lens[x] + a) <= cols and need + n <= free_pages:
                    s.append(x), add.append(a)
                    need += n
            b.call("extend", s, add)
            b.write(rng, [x for x in s if p.lens[x]], [int(rng.integers(0, p.lens[x])) for x in s if p.lens[x]],
                    0, layers)
        elif what == 2 and empty.size and (p.lens > 0).any():
            kids = rng.permutation(empty)[:min(empty.size, free_pages)]
            b.call("fork", rng.choice(np.flatnonzero(p.lens > 0), kids.size), kids)
        elif what == 3:
            b.call("free", some[:rng.integers(0, max(1, slots // 3))])
        elif what == 4:
            b.compact()
        else:
            x = rng.permutation(pages)
            k = int(rng.integers(1, pages // 2))
            b.call("copy", x[:k], x[pages // 2:pages // 2 + k])
        if step % 8 == 7:
            b.same()
    b.same()


def test_fork_lengths_around_a_page(torch):
    """Lengths 0, 1, a page less one, a page, a page and one; many children of one parent; the new tokens of each
    child are its own."""
    pt = 16
    b = Both(torch, 2, 64, pt, 2, 8, 30, 4)
    b.call("extend", [0, 1, 2, 3], [1, pt - 1, pt, pt + 1])
    b.call("fork", [0, 1, 2, 3, 4, 1, 3, 3], [10, 11, 12, 13, 14, 15, 16, 17])   # 4 is empty
    b.same()
    b.call("extend", [10, 11, 12, 13, 14, 15, 16, 17], [1] * 8)
    b.write(np.random.default_rng(1), [10, 11, 12, 13, 14, 15, 16, 17], [1, 15, 16, 17, 0, 15, 17, 17], 1, 1)
    b.same()
    b.call("free", [3, 0, 12])
    b.compact()
    b.same()


def test_empty_lists_and_full_pool(torch):
    b = Both(torch, 1, 8, 4, 1, 8, 4, 8)
    for name in ("extend", "fork", "copy"):
        b.call(name, [], [])
    b.call("free", [])
    b.compact()                                  # nothing in use
    b.call("extend", [2], [32])                  # every page
    b.compact()
    b.same()
    b.call("free", [2, 2, 2])                    # freed once
    b.same()


def test_large_pool_many_tiles(torch):
    """More than a tile of pages per workgroup of the plan, and a prompt's worth of pages at once."""
    b = Both(torch, 1, 30000, 1, 1, 8, 5, 12000)
    b.call("extend", [0, 1], [11000, 9000])
    b.call("free", [0])
    b.call("extend", [3, 0], [1, 10998])
    b.compact()
    b.same()


@pytest.mark.parametrize("pages", [50, 17000])
def test_compact_to_other_arrays(torch, pages):
    b = Both(torch, 2, pages, 4, 1, 8, 6, 8, extra_cols=2)
    b.call("extend", [0, 1, 2], [30, 17, 25])
    b.call("fork", [1], [4])
    b.call("free", [0])
    before = {k: v.cpu().clone() for k, v in b.t.items()}
    remap, refs = (torch.full((pages,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    tables = torch.full((6, 10), -9, dtype=torch.int32, device="cuda")[:, :8]
    for _ in range(2):   # the same again: pages that moved keep their bytes
        assert b.kv.compact(remap, tables_out=tables, refs_out=refs) == OK
    assert b.kv.get_status() == OK
    for k in ("refs", "tables", "lens"):
        assert torch.equal(b.t[k].cpu(), before[k])
    want = b.plain.compact()
    assert np.array_equal(remap.cpu().numpy(), want)
    assert np.array_equal(refs.cpu().numpy(), b.plain.refs)
    assert np.array_equal(tables.cpu().numpy(), b.plain.tables)
    assert np.array_equal(b.t["pool"].view(torch.int16).cpu().numpy(), b.plain.pool)


def test_page_bytes_past_32_bits(torch):
    """Offsets past 2^32 bytes: pages of a pool of 5 GiB."""
    from paper_2609_09800_amd import hbf
    pages, pt = 20, 1 << 16
    pool = torch.zeros((2, 2, pages, pt, 4, 128), dtype=torch.bfloat16, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    tables = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(3, dtype=torch.int32, device="cuda")
    kv = hbf.KvPages(pool, refs=refs, tables=tables, lens=lens)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    refs[:17] = 1
    assert kv.extend(i(1), i(pt + 9)) == OK
    k = torch.randn((2, 1, 4, 128), device="cuda").bfloat16()
    assert kv.write(k, -k, i(1), i(pt + 8)) == OK
    assert kv.fork(i(1), i(2)) == OK
    assert kv.get_status() == OK
    assert tables[1].tolist()[:2] == [17, 18] and tables[2].tolist()[:2] == [17, 19]
    assert torch.equal(pool[:, 0, 19, 8], k[:, 0]) and torch.equal(pool[:, 1, 19, 8], -k[:, 0])
    assert kv.copy(i(19), i(0)) == OK
    assert torch.equal(pool[:, 1, 0, 8], -k[:, 0])
    assert not pool[:, :, 0, :8].any() and not pool[:, :, 0, 9:].any()


BAD = [
    ("extend", [0, 0], [1, 1], EINVAL), ("extend", [9], [1], EINVAL), ("extend", [-1], [1], EINVAL),
    ("extend", [0], [-1], EINVAL), ("extend", [0], [33], EINVAL), ("extend", [1], [1], EINVAL),
    ("extend", [0, 2], [25, 25], ENOMEM), ("extend", [0], [2**31 - 1], EINVAL),
    ("fork", [1], [1], EINVAL), ("fork", [1, 1], [3, 3], EINVAL), ("fork", [1], [7], EINVAL),
    ("fork", [-2], [3], EINVAL), ("fork", [1, 3], [3, 4], EINVAL), ("fork", [0], [1], EINVAL),
    ("copy", [0, 1], [2, 2], EINVAL), ("copy", [0, 2], [2, 3], EINVAL), ("copy", [0], [12], EINVAL),
    ("copy", [-1], [1], EINVAL), ("copy", [3], [3], EINVAL),
]


@pytest.mark.parametrize("pages", [12, 17000])
@pytest.mark.parametrize("name,first,second,want", BAD)
def test_refused_calls_change_nothing(torch, name, first, second, want, pages):
    b = Both(torch, 1, pages, 4, 1, 8, 6, 8)
    b.call("extend", [0, 1], [7, 6])
    b.hold(b.plain.tables[1, 1])     # slot 1's part-full page is held twice
    if pages > 12:
        if name == "copy" and max(first + second) == 12:
            second = [pages]
        for page in range(12, pages):    # as full as the small pool
            b.plain.refs[page] += 1
        b.t["refs"][12:] += 1
    assert getattr(b.kv, name)(b.dev(first), b.dev(second)) == OK
    assert b.kv.get_status() == want
    assert b.kv.get_status() == OK   # cleared
    b.same()
    b.call("extend", [0], [5])       # and the next call is served
    b.same()


def test_damaged_tables_are_refused(torch):
    b = Both(torch, 1, 12, 4, 1, 8, 6, 8)
    b.call("extend", [0, 1], [7, 6])
    remap = torch.zeros(12, dtype=torch.int32, device="cuda")
    for table, refs, length in (((0, 0, 99), None, None), ((0, 0, -5), None, None), (None, (0, 0), None),
                                (None, None, (2, -3)), (None, None, (2, 33)), (None, (11, -1), None)):
        saved = {k: v.clone() for k, v in b.t.items()}
        if table:
            b.t["tables"][table[0], table[1]] = table[2]
        if refs:
            b.t["refs"][refs[0]] = refs[1]
        if length:
            b.t["lens"][length[0]] = length[1]
        damaged = {k: v.clone() for k, v in b.t.items()}
        assert b.kv.compact(remap) == OK and b.kv.get_status() == EINVAL
        if refs != (11, -1):
            slot = length[0] if length else 0
            assert b.kv.fork(b.dev([slot]), b.dev([4])) == OK and b.kv.get_status() == EINVAL
        for k, v in b.t.items():
            assert torch.equal(v.view(torch.int16) if k == "pool" else v,
                               damaged[k].view(torch.int16) if k == "pool" else damaged[k])
            v.copy_(saved[k])
    b.same()


def test_free_and_write_leave_bad_entries_out(torch):
    b = Both(torch, 1, 12, 4, 1, 8, 6, 8)
    b.call("extend", [0, 1], [7, 6])
    assert b.kv.free(b.dev([-1, 1, 6])) == OK
    assert b.kv.get_status() == EINVAL
    b.plain.free([1])
    b.same()
    k = torch.ones((1, 4, 1, 8), dtype=torch.bfloat16, device="cuda")
    assert b.kv.write(k, k, b.dev([0, 0, 9, 1]), b.dev([7, -1, 0, 0])) == OK   # behind the end; slot out of range; empty
    assert b.kv.get_status() == EINVAL
    b.same()


def test_arguments(torch):
    from paper_2609_09800_amd import hbf
    b = Both(torch, 2, 12, 4, 1, 8, 6, 8, max_list=2)
    assert b.kv.extend(b.dev([0, 1, 2]), b.dev([1, 1, 1])) == ENOWORKSPACE
    assert b.kv.fork(b.dev([0, 1, 2]), b.dev([3, 4, 5])) == ENOWORKSPACE
    k = torch.ones((1, 1, 1, 8), dtype=torch.bfloat16, device="cuda")
    for args in ((k.float(), k, b.dev([0]), b.dev([0])), (k, k[:, :0], b.dev([0]), b.dev([0])),
                 (k, k, b.dev([0]).long(), b.dev([0])), (k, k, b.dev([0]), b.dev([0, 1])), (k.cpu(), k, b.dev([0]), b.dev([0]))):
        with pytest.raises(hbf.HbfError):
            b.kv.write(*args)
    assert b.kv.write(k, k, b.dev([0]), b.dev([0]), first_layer=2) == EINVAL
    with pytest.raises(hbf.HbfError):
        b.kv.extend(b.dev([0]), b.dev([1, 2]))
    with pytest.raises(hbf.HbfError):
        b.kv.compact(torch.zeros(11, dtype=torch.int32, device="cuda"))
    with pytest.raises(hbf.HbfError):
        b.kv.compact(torch.zeros(12, dtype=torch.int32, device="cuda"), tables_out=torch.zeros((6, 7), dtype=torch.int32, device="cuda"))
    with pytest.raises(hbf.HbfError):
        hbf.KvPages(b.t["pool"]).free(b.dev([0]))
    with pytest.raises(hbf.HbfError):
        hbf.KvPages(b.t["pool"].float())
    with pytest.raises(hbf.HbfError):
        hbf.KvPages(b.t["pool"], refs=b.t["refs"][:-1], tables=b.t["tables"], lens=b.t["lens"])
    with pytest.raises(hbf.HbfError):   # tokens of 8 bytes
        hbf.KvPages(torch.zeros((1, 2, 4, 4, 1, 4), dtype=torch.bfloat16, device="cuda"), refs=b.dev([0] * 4),
                    tables=b.dev([[0]]), lens=b.dev([0]))
    b.same()


def test_another_stream(torch):
    b = Both(torch, 1, 40, 4, 1, 8, 6, 8)
    s = torch.cuda.Stream()
    slots, add = b.dev([0, 1]), b.dev([9, 10])
    s.wait_stream(torch.cuda.current_stream())
    assert b.kv.extend(slots, add, stream=s) == OK
    assert b.kv.get_status(stream=s) == OK
    b.plain.extend([0, 1], [9, 10])
    b.same()


def test_replayed_graph(torch):
    """A captured step (free, fork, extend, write) replayed, with eager work between the replays."""
    b = Both(torch, 2, 60, 4, 1, 8, 10, 8)
    b.call("extend", [0, 1], [7, 12])
    par, kid, one, pos = b.dev([0, 0, 1]), b.dev([4, 5, 6]), b.dev([1, 1, 1]), b.dev([7, 7, 12])
    k = torch.zeros((2, 3, 1, 8), dtype=torch.bfloat16, device="cuda")

    def step():
        b.kv.free(kid)
        b.kv.fork(par, kid)
        b.kv.extend(kid, one)
        b.kv.write(k, k, kid, pos)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for r in range(4):
        k.fill_(r + 1.0)
        bits = np.full((2, 3, 1, 8), k.view(torch.int16).flatten()[0].item(), dtype=np.int16)
        g.replay()
        torch.cuda.synchronize()
        for _ in range(2 if r == 0 else 1):
            b.plain.free([4, 5, 6])
            b.plain.fork([0, 0, 1], [4, 5, 6])
            b.plain.extend([4, 5, 6], [1, 1, 1])
        b.plain.write(bits, bits, [4, 5, 6], [7, 7, 12], 0)
        b.same()
