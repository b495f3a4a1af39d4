"""Device blocks that the decode-layer objects keep, and the streams of the calls
that use them, with an allocator and a library that only take notes: a block has
to be made on the call's stream, or the allocator has to be told of that stream,
before the library gets its address.  (What goes wrong otherwise, memory in use
given to somebody else, depends on timing.)"""
import contextlib
import gc
import types
import weakref

import pytest

from paper_2609_09800_amd import hbf


class Stream:
    def __init__(self, number):
        self.cuda_stream = number

    def synchronize(self):
        pass


class Block:
    """As a tensor: `streams` has the one it was made on and those recorded."""
    is_cuda = True

    def __init__(self, notes, shape, dtype="int32"):
        self.notes, self.shape, self.dtype, self.device = notes, tuple(shape), dtype, None
        self.streams = [notes.current.cuda_stream]
        notes.made += 1
        self.address = 4096 * notes.made

    def numel(self):
        n = 1
        for x in self.shape:
            n *= x
        return n

    def dim(self):
        return len(self.shape)

    def stride(self, d=None):
        strides = [1]
        for x in self.shape[:0:-1]:
            strides.insert(0, strides[0] * x)
        return strides if d is None else strides[d]

    def data_ptr(self):
        return self.address

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)

    def item(self):   # (waits for the current stream)
        self.notes.status.append(("read", self.notes.current.cuda_stream))
        return hbf.HBF_EINVAL

    def zero_(self):
        self.notes.status.append(("cleared", self.notes.current.cuda_stream))

    def view(self, dtype):
        return self

    def __getitem__(self, part):
        return self


@pytest.fixture
def notes(monkeypatch):
    d = types.SimpleNamespace(made=0, current=Stream(1), calls=[], need=300, status=[])

    @contextlib.contextmanager
    def on(stream):
        before = d.current
        d.current = before if stream is None else stream
        yield
        d.current = before

    def entry(name):
        def call(*args):
            if name.endswith("_bytes"):
                args[-1]._obj.value = d.need
            else:
                d.calls.append(args[-1])
            return hbf.HBF_OK
        return call

    lib = types.SimpleNamespace(**{n: entry(n) for n in hbf.EXPORTED})
    fake = types.SimpleNamespace(
        cuda=types.SimpleNamespace(stream=on, current_stream=lambda device=None: d.current), Tensor=Block,
        int32="int32", float32="float32", bfloat16="bf16", float16="fp16", uint8="uint8",
        empty=lambda n, dtype, device: Block(d, (n,)))
    for name, value in (("torch", fake), ("_Tensor", Block), ("_int32", "int32"), ("_device", lambda: 0),
                        ("_raw_stream", lambda device: d.current.cuda_stream), ("_import_torch", lambda: lib),
                        ("_dev", lambda t, *a, **k: t), ("_strided", lambda t, *a, **k: t),
                        ("_dtype_code", lambda t: hbf.HBF_BF16),
                        ("_zeroed", lambda nbytes, device, zero=256: Block(d, (nbytes,)))):
        monkeypatch.setattr(hbf, name, value, raising=False)
    return d


def known(notes, first, call):
    """Calls on the current stream 1, on a stream given, and on another one that is current: every block from
    `first` on that an object keeps must be known there before the library is called."""
    for stream in (None, Stream(3), Stream(3), None):
        notes.calls.clear()
        assert call(stream) == hbf.HBF_OK
        raw = stream.cuda_stream if stream else 1
        assert notes.calls == [raw]
        for block in first():
            assert raw in block.streams
    notes.current = Stream(4)
    assert call(None) == hbf.HBF_OK
    for block in first():
        assert set(block.streams) == {1, 3, 4} and len(block.streams) == 3   # told once each


@pytest.mark.parametrize("name,lists", [("extend", 2), ("fork", 2), ("free", 1), ("copy", 2), ("compact", 1), ("write", 2)])
def test_a_cache_s_workspace_is_known_on_every_stream(notes, name, lists):
    pool = Block(notes, (2, 2, 64, 16, 1, 64), "bf16")
    kv = hbf.KvPages(pool, refs=Block(notes, (64,)), tables=Block(notes, (8, 4)), lens=Block(notes, (8,)))
    args = [Block(notes, (64,)) for _ in range(lists)]
    if name == "write":
        args = [Block(notes, (2, 64, 1, 64), "bf16") for _ in range(2)] + args
    known(notes, lambda: [kv._ws], lambda stream: getattr(kv, name)(*args, stream=stream))


def attention(notes):
    kv = hbf.KvPages(Block(notes, (1, 2, 64, 16, 1, 64), "bf16"))
    q, out, prefix = Block(notes, (3, 4, 64), "bf16"), Block(notes, (3, 4, 64), "bf16"), Block(notes, (4,))
    return kv, lambda stream, length=64: kv.prefix_attention(0, q, out, prefix, length, stream=stream)


def test_attention_s_words_and_scratch_are_known_on_every_stream(notes):
    kv, call = attention(notes)
    known(notes, lambda: [kv._attn_status, kv._attn_ws._t], call)


def test_attention_s_scratch_is_made_on_the_stream_of_its_call(notes):
    kv, call = attention(notes)
    assert call(Stream(2)) == hbf.HBF_OK
    assert kv._attn_ws._t.streams == [2] and notes.current.cuda_stream == 1
    notes.need = 10000
    assert call(Stream(5), 63) == hbf.HBF_OK   # grows
    assert kv._attn_ws._t.streams == [5] and kv._attn_ws._t.numel() >= 10000


def test_a_moe_layer_s_blocks_are_known_on_every_stream(notes):
    layer = hbf.MoeLayer(Block(notes, (4, 32, 64), "bf16"), Block(notes, (4, 64, 16), "bf16"), 2)
    x, y = Block(notes, (3, 64), "bf16"), Block(notes, (3, 64), "bf16")
    ids, weights = Block(notes, (3, 2)), Block(notes, (3, 2), "float32")
    known(notes, lambda: [layer._ws, layer._status], lambda stream: layer.forward(x, y, ids, weights, stream=stream))


def test_scratch_that_a_graph_may_have_captured_is_kept(notes):
    kv, call = attention(notes)
    blocks, sizes = [], []
    for length in range(64, 54, -1):   # a little more each time
        notes.need = notes.need + 100
        assert call(None, length) == hbf.HBF_OK
        if not blocks or blocks[-1]() is not kv._attn_ws._t:
            blocks.append(weakref.ref(kv._attn_ws._t))
            sizes.append(kv._attn_ws._t.numel())
    gc.collect()
    assert len(blocks) > 1 and all(b() is not None for b in blocks)
    assert sum(sizes[:-1]) < sizes[-1]
    del kv, call
    gc.collect()
    assert all(b() is None for b in blocks)


@pytest.mark.parametrize("given", [None, 6])
def test_a_status_is_read_and_cleared_in_its_stream_s_order(notes, given):
    """Cleared on another stream, the word could be cleared after the next call has set it."""
    kv, _ = attention(notes)
    layer = hbf.MoeLayer(Block(notes, (4, 32, 64), "bf16"), Block(notes, (4, 64, 16), "bf16"), 2)
    for thing in (kv, layer):
        notes.status.clear()
        assert thing.get_status(stream=Stream(given) if given else None) == hbf.HBF_EINVAL
        assert notes.status == [("read", given or 1), ("cleared", given or 1)]
