"""The decode-layer operators on a stream that is not the current one: what the
call reads and overwrites is there before it, the stream is busy while the host
goes on, and the objects go before their work is done."""
import pytest

import test_gpu_kv_attention as attention
import test_gpu_moe as moe

pytestmark = pytest.mark.gpu
OK = 0


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


def busy(torch):
    """A stream with tens of milliseconds of work, behind all that the current one has."""
    a = torch.zeros((8192, 8192), dtype=torch.bfloat16, device="cuda")
    a @ a
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(60):
            a @ a
    a.record_stream(s)
    return s


def dropped(torch, s, blocks):
    """New blocks of those sizes are others while the stream is busy."""
    was = [(b.untyped_storage().data_ptr(), b.untyped_storage().nbytes()) for b in blocks]
    assert not s.query()
    return was


def others(torch, s, was):
    new = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _, n in was]
    assert not s.query()
    assert not {a for a, _ in was} & {t.data_ptr() for t in new}
    return new


@pytest.mark.parametrize("rows,lens", [(1, [20]), (40, [0, 130] * 20)])
def test_attention(torch, rows, lens):
    from paper_2609_09800_amd import hbf
    attention.say(f"attention on a busy stream {rows}")
    pool, q, prefix, tables, ln = attention.make(torch, rows, 8, 2, 64, 900, lens, 16, seed=41)
    want, want_lse = attention.run(torch, pool, q, prefix, 900, tables, ln)[1:]
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    kv = hbf.KvPages(pool)
    s = busy(torch)
    assert kv.prefix_attention(0, q, out, prefix, 900, tables, ln, lse=lse, stream=s) == OK
    was = dropped(torch, s, [kv._attn_ws._t, kv._attn_status])
    del kv
    new = others(torch, s, was)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert not any(bool(t.any()) for t in new)


@pytest.mark.parametrize("tokens", [1, 20])
def test_moe_layer(torch, tokens):
    from paper_2609_09800_amd import hbf
    moe.say(f"moe on a busy stream {tokens}")
    x, router, gate_up, down = moe.make(torch, tokens, 16, 256, 64, "bfloat16", seed=42)
    _, want, want_ids, want_w = moe.run(torch, x, gate_up, down, 4, router=router)
    y = torch.full_like(x, 7.0)
    ids = torch.full((tokens, 4), -7, dtype=torch.int32, device="cuda")
    w = torch.full((tokens, 4), 7.0, device="cuda")
    layer = hbf.MoeLayer(gate_up, down, 4, router=router)
    s = busy(torch)
    assert layer.forward(x, y, ids, w, stream=s) == OK
    was = dropped(torch, s, [layer._ws, layer._status])
    del layer
    new = others(torch, s, was)
    s.synchronize()
    assert torch.equal(y, want) and torch.equal(ids, want_ids) and torch.equal(w, want_w)
    assert not any(bool(t.any()) for t in new)


def test_cache_pages(torch):
    from paper_2609_09800_amd import hbf
    attention.say("cache pages on a busy stream")
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((2, 2, 40, 4, 1, 8), dtype=torch.bfloat16, device="cuda")
    refs, tables, lens = torch.zeros(40, **i32), torch.full((6, 8), -1, **i32), torch.zeros(6, **i32)
    kv = hbf.KvPages(pool, refs=refs, tables=tables, lens=lens)
    slots, add, pos, child = (torch.tensor(v, **i32) for v in ([0, 1], [9, 10], [8, 9], [4, 5]))
    k = torch.ones((2, 2, 1, 8), dtype=torch.bfloat16, device="cuda")
    s = busy(torch)
    assert kv.extend(slots, add, stream=s) == OK
    assert kv.write(k, k, slots, pos, stream=s) == OK
    assert kv.fork(slots, child, stream=s) == OK
    assert kv.free(slots, stream=s) == OK
    was = dropped(torch, s, [kv._ws])
    del kv
    new = others(torch, s, was)
    s.synchronize()
    assert lens.tolist() == [0, 0, 0, 0, 9, 10]
    assert tables[4].tolist() == [0, 1, 6] + [-1] * 5 and tables[5].tolist() == [3, 4, 7] + [-1] * 5
    assert refs.tolist() == [1, 1, 0, 1, 1, 0, 1, 1] + [0] * 32
    assert bool((pool[:, :, 6, 0] == 1).all()) and bool((pool[:, :, 7, 1] == 1).all())
    assert not any(bool(t.any()) for t in new)


def test_a_graph_s_scratch_outlasts_larger_calls(torch):
    """A captured call's scratch is nobody else's, however much scratch later calls of the object need."""
    from paper_2609_09800_amd import hbf
    attention.say("attention captured, then larger")
    pool, q, prefix, tables, ln = attention.make(torch, 40, 8, 2, 64, 900, [0, 130] * 20, 16, seed=43)
    small, one = q[:9].contiguous(), torch.empty_like(q[:9])
    kv = hbf.KvPages(pool)
    kv.prefix_attention(0, small, one, prefix, 300, tables[:9], ln[:9].contiguous())
    own9 = ln[:9].contiguous()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert kv.prefix_attention(0, small, one, prefix, 300, tables[:9], own9) == OK
    first = kv._attn_ws._t
    size = first.numel()
    del first
    out = torch.empty_like(q)
    assert kv.prefix_attention(0, q, out, prefix, 900, tables, ln) == OK
    assert kv._attn_ws._t.numel() >= 2 * size
    new = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for i in range(4):
        small.copy_(q[:9] * (i + 1) / 2)
        one.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(one, attention.run(torch, pool, small, prefix, 300, tables[:9], own9)[1])
        assert all(bool((t == 85).all()) for t in new)
    assert kv.get_status() == OK


def test_an_error_after_the_status_was_taken_is_kept(torch):
    from paper_2609_09800_amd import hbf
    attention.say("status on another stream")
    pool, q, prefix, tables, ln = attention.make(torch, 4, 8, 2, 64, 90, [20, 30, 16, 5], 16, seed=44)
    kv = attention.run(torch, pool, q, prefix, 90, tables, ln)[0]
    out, bad = torch.empty_like(q), ln.clone()
    bad[1] = -1
    x, router, gate_up, down = moe.make(torch, 3, 6, 64, 16, "bfloat16", seed=45)
    layer = hbf.MoeLayer(gate_up, down, 2)
    y, w = torch.empty_like(x), torch.ones((3, 2), device="cuda")
    ids = torch.full((3, 2), 6, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        assert kv.prefix_attention(0, q, out, prefix, 90, tables, bad, stream=s) == OK
        assert layer.forward(x, y, ids, w, stream=s) == OK
        assert kv.get_status(stream=s) == -1 and layer.get_status(stream=s) == -1
    assert kv.get_status(stream=s) == OK and layer.get_status(stream=s) == OK
    s.synchronize()
