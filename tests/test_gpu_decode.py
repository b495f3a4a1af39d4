"""The decode-layer operators together (paper_2609_09800_amd.decode) against the
same steps in plain 64-bit operations, and the page traffic they hand to the
service model against the reference model.

Tolerance: the steps round to bfloat16 (unit roundoff 2^-8) where the plain ones
do not, about ten times per layer and value (norm, q, k, v, probabilities,
attention, its projection, two residuals, norm, the layer's result), each a
relative 2^-8 at most of a value no larger than the layer's: after n layers the
relative L2 difference stays below 10 n 2^-8, a tenth of that where the
roundings are independent.  The routes taken are compared layer by layer from the
steps' own inputs, so that no token is sent to other experts by a rounding.
"""
import numpy as np
import pytest

from paper_2609_09800_amd import workloads as wl

pytestmark = pytest.mark.gpu


def plain_step(torch, d, x, history):
    """Decoder.step in float64 from the plain history of K and V; the experts as the step chose them."""
    norm = lambda t: t * t.square().mean(1, keepdim=True).add(1e-6).rsqrt()
    kvh, dim, heads = wl.KV_HEADS, wl.KV_DIM, d.heads
    x = x.double()
    for l in range(d.layers):
        wq, wkv, wo = (w.double() for w in d.proj[l])
        h = norm(x)
        k, v = (h @ wkv.t()).view(d.rows, 2, kvh, dim).unbind(1)
        history[l][0].append(k)
        history[l][1].append(v)
        q = (h @ wq.t()).view(d.rows, heads, dim)
        out = torch.zeros_like(q)
        for r in range(d.rows):
            kk = torch.cat([history[l][0][0], *(t[r:r + 1] for t in history[l][0][1:])])
            vv = torch.cat([history[l][1][0], *(t[r:r + 1] for t in history[l][1][1:])])
            for j in range(heads):
                g = j // (heads // kvh)
                out[r, j] = torch.softmax(kk[:, g] @ q[r, j] * dim ** -0.5, 0) @ vv[:, g]
        x = x + out.view(d.rows, -1) @ wo.t()
        h = norm(x)
        gate_up, down, router = (t.double() for t in d.moe[l]._keep)
        p = torch.softmax(h @ router.t(), 1)
        y = torch.zeros_like(h)
        for t in range(d.rows):
            w = p[t, d.ids[l, t].long()]
            for e, we in zip(d.ids[l, t].tolist(), (w / w.sum()).tolist()):
                a = gate_up[e] @ h[t]
                f = a.numel() // 2
                y[t] += we * (down[e] @ (torch.nn.functional.silu(a[:f]) * a[f:]))
        x = x + y
    return x


@pytest.mark.parametrize("prefix", [32, 37])
def test_steps_against_plain(prefix):
    import torch
    from paper_2609_09800_amd import decode
    d = decode.Decoder(layers=2, rows=3, prefix=prefix, experts=8, topk=2, hidden=256, ffn=64, heads=8, own=30)
    print(f"[gpu-case] decode prefix {prefix}", flush=True)
    table = d.tables[0, :d.shared].long()
    history = [[[d.kv.pool[l, i, table].reshape(-1, wl.KV_HEADS, wl.KV_DIM)[:prefix].double()] for i in range(2)]
               for l in range(d.layers)]
    x = torch.randn((3, 256), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    for _ in range(18):   # past a page's end
        got = d.step(x)
        want = plain_step(torch, d, x, history)
        assert float((got.double() - want).norm() / want.norm()) < 10 * d.layers * 2.0 ** -8
        x = got
    assert d.kv.get_status() == 0
    assert d.lens.tolist() == [prefix] + [prefix + 18] * 3
    # the rows share the prompt's full pages, and nothing else
    full = prefix // d.kv.page_tokens
    assert torch.equal(d.tables[1:, :full], d.tables[:1, :full].expand(3, -1))
    own = d.tables[1:, full:-(-(prefix + 18) // d.kv.page_tokens)]
    assert own.unique().numel() == own.numel()


def test_pages_read_are_timed(oracle_mod):
    from paper_2609_09800_amd import decode
    import torch
    d = decode.Decoder(layers=3, rows=4, prefix=70, experts=8, topk=2, hidden=256, ffn=64, heads=8, own=20)
    d.step(torch.randn((4, 256), device="cuda").bfloat16())
    done, start = d.modeled_ns(compute_ns=1500)
    addr, start2 = d.read_pages()
    assert np.array_equal(start, start2) and addr.size == start[-1]
    chosen = d.ids.cpu().numpy()
    for l in range(3):
        n = 2 * (70 // 16) + np.unique(chosen[l]).size * d.pages_per_expert
        assert start[l + 1] - start[l] == n
    o = oracle_mod.OracleModel(**wl.geometry(16, 8, 4))
    for base, n in (d.weights, d.pool_range):
        o.register_range(base, n)
    t = 0
    for l in range(3):
        a = addr[start[l]:start[l + 1]].astype(np.uint64)
        rc, c = o.time_requests(a, np.full(a.size, t, dtype=np.int64))
        assert rc == 0
        t = int(c.max())
        assert done[l] == t
        t += 1500


def test_example_runs(capsys):
    from paper_2609_09800_amd import decode
    x = decode.main(["--layers", "2", "--rows", "3", "--prefix", "50", "--steps", "2"])
    assert bool(x.isfinite().all())
    assert capsys.readouterr().out.count("modeled") == 2
