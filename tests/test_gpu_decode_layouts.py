"""The decode-layer operators where a batch or a cache is laid out otherwise than
in their own tests: rows in another order and alone, tables wider than their
lengths, the prefix's pages in another order, weights behind 2^32 bytes, and the
routes of decode steps against their inputs."""
import math

import numpy as np
import pytest

from test_gpu_kv_attention import OK, U, check, make, reference, run, say
import test_gpu_moe as moe

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


@pytest.mark.parametrize("R,Hq,Hk,L", [(40, 8, 2, 700), (7, 6, 2, 500), (64, 4, 4, 3000)])
def test_a_row_s_place_does_not_matter(torch, R, Hq, Hk, L):
    """Rows in another order, and some of them alone, have the results of the batch but for rounding."""
    say(f"attention rows moved {R} {Hq} {Hk} {L}")
    lens = [int(x) for x in np.arange(R) * 7 % 90]
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, 128, L, lens, 16, seed=51)
    ref = reference(torch, pool[0], q, prefix, L, tables, ln, 128 ** -0.5)
    order = torch.from_numpy(np.random.default_rng(52).permutation(R)).cuda()
    for rows in (order, order[:1], order[-1:], order[: R // 2]):
        moved = [t[rows].contiguous() for t in (q, tables, ln)]
        _, out, lse = run(torch, pool, moved[0], prefix, L, moved[1], moved[2])
        check(torch, out, lse, [t[rows.cpu()] for t in ref], U["bfloat16"], L + 90, 128)


@pytest.mark.parametrize("R,Hq,Hk,L,cols", [(1, 8, 1, 300, 8192), (16, 32, 4, 2000, 2048), (64, 8, 2, 300, 500), (3, 4, 2, 0, 70000)])
def test_a_table_wider_than_its_lengths(torch, R, Hq, Hk, L, cols):
    """As the rows of a cache whose sequences may grow long; what lies behind a row's pages is not looked at."""
    say(f"attention wide table {R} {Hq} {Hk} {L} {cols}")
    lens = [int(x) for x in np.arange(R) * 37 % 200]
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, 64, L, lens, 16, seed=53)
    wide = torch.full((R, cols), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :tables.shape[1]] = torch.where(tables < 0, 1 << 30, tables)
    kv, out, lse = run(torch, pool, q, prefix, L, wide, ln)
    assert kv.get_status() == OK
    check(torch, out, lse, reference(torch, pool[0], q, prefix, L, tables, ln, 0.125), U["bfloat16"], L + 200, 64)


def test_rising_scores_in_any_page_order(torch):
    """Steps up and down of the running maximum, by the order of the pages."""
    pool, q, prefix, tables, ln = make(torch, 3, 8, 1, 64, 1504, [700, 0, 90], 16, seed=54)
    k = pool[0, 0, prefix.long()].view(-1, 64)
    k[:, 0] = torch.linspace(-30, 30, 1504, device="cuda").bfloat16()
    pool[0, 0, prefix.long()] = k.view(-1, 16, 1, 64)
    q[:, :, 0] = 40.0
    n = prefix.numel()
    shuffled = torch.from_numpy(np.random.default_rng(55).permutation(n)).cuda()
    for order in (torch.arange(n, device="cuda"), torch.arange(n - 1, -1, -1, device="cuda"), shuffled):
        pages = prefix[order].contiguous()
        say(f"attention page order from {int(order[0])}")
        kv, out, lse = run(torch, pool, q, pages, 1504, tables, ln)
        check(torch, out, lse, reference(torch, pool[0], q, pages, 1504, tables, ln, 0.125), U["bfloat16"], 2300, 64)


@pytest.mark.parametrize("tokens", [1, 9, 70])
def test_weights_behind_32_bits(torch, tokens):
    """Experts 2 GiB apart: the last ones' weights lie behind 2^32 bytes."""
    from paper_2609_09800_amd import hbf
    say(f"moe weights past 32 bits {tokens}")
    E, k, H, F = 4, 2, 128, 48
    x, router, gate_up, down = moe.make(torch, tokens, E, H, F, "bfloat16", seed=56)
    want = moe.run(torch, x, gate_up, down, k, router=router)
    stride = 1 << 30
    buf = torch.empty((E - 1) * stride + 3 * F * H, dtype=torch.bfloat16, device="cuda")
    gu = buf.as_strided((E, 2 * F, H), (stride, H, 1))
    dn = buf.as_strided((E, H, F), (stride, F, 1), 2 * F * H)
    gu.copy_(gate_up)
    dn.copy_(down)
    got = moe.run(torch, x, gu, dn, k, router=router)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2]) and torch.equal(got[3], want[3])
    assert bool((got[2] >= 2).any())


@pytest.mark.parametrize("rows", [2, 12])
def test_decode_steps_take_the_routes_of_their_inputs(torch, rows):
    """Each token's experts are the largest of its logits, or as large but for the fp32 products' rounding."""
    from paper_2609_09800_amd import decode
    say(f"decode routes {rows}")
    d = decode.Decoder(layers=2, rows=rows, prefix=37, experts=40, topk=4, hidden=256, ffn=64, heads=8, own=30)
    seen = []
    for layer in d.moe:
        def forward(x, y, ids, weights, layer=layer, call=layer.forward):
            rc = call(x, y, ids, weights)
            seen.append((layer, x.clone(), ids.clone(), weights.clone()))
            return rc
        layer.forward = forward
    x = torch.randn((rows, 256), generator=torch.Generator(device="cuda").manual_seed(57), device="cuda").bfloat16()
    for _ in range(3):
        x = d.step(x)
    assert len(seen) == 6 and any(len(set(i.flatten().tolist())) > 4 for _, _, i, _ in seen)
    for layer, h, ids, weights in seen:
        router = layer._keep[2].double()
        logits = h.double() @ router.t().contiguous()
        bound = 2 * (256 + 8) * 2.0 ** -23 * (h.double().abs() @ router.abs().t().contiguous()).amax(1, keepdim=True)
        chosen = logits.gather(1, ids.long())
        best = logits.sort(1, descending=True)[0][:, :4]
        assert bool(((chosen - best).abs() <= bound).all())
        assert all(len(set(r)) == 4 for r in ids.tolist())
        w = torch.softmax(chosen, 1)
        assert bool(((weights.double() - w).abs() <= (2 * bound + 60 * 2.0 ** -23) * w).all())
