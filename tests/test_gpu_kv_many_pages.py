"""Pools of very many pages: the copy's check holds a bit per page in LDS, past 64
KiB of it from 524,257 pages on (a word beside the bits)."""
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL = 0, -1


@pytest.mark.parametrize("pages", [524256, 524257, 524288, 524289, 1 << 20])
def test_copy_in_a_pool_of_very_many_pages(pages):
    import torch
    from paper_2609_09800_amd import hbf
    print(f"[gpu-case] copy of {pages} pages", flush=True)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros((1, 2, pages, 1, 1, 8), dtype=torch.bfloat16, device="cuda")
    pool.view(torch.int16)[0, :, :, 0, 0, 0] = torch.arange(pages, device="cuda").to(torch.int16)
    kv = hbf.KvPages(pool, refs=torch.zeros(pages, **i32), tables=torch.full((1, 1), -1, **i32), lens=torch.zeros(1, **i32))
    want = pool.clone()
    src, dst = torch.tensor([0, pages - 1, 77], **i32), torch.tensor([pages - 2, 5, pages // 2], **i32)
    want[:, :, dst.long()] = pool[:, :, src.long()]
    assert kv.copy(src, dst) == OK
    assert kv.get_status() == OK
    assert torch.equal(pool.view(torch.int16), want.view(torch.int16))
    assert kv.copy(src, dst.flip(0).clamp(min=pages - 2)) == OK   # a destination twice
    assert kv.get_status() == EINVAL
    assert torch.equal(pool.view(torch.int16), want.view(torch.int16))
