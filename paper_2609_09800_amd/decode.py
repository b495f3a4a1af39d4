"""Decode steps of a small layered model whose expert weights and shared KV
prefix lie in HBF: the decode-layer operators run together, and the service
model gives the time that the pages they read would take.

    python -m paper_2609_09800_amd.decode [--layers 4] [--rows 16] [--prefix 1024] [--steps 3]

Every row is a sample of one prompt: the rows' slots are forked from the
prompt's, so that their table rows begin with the same pages.  A step of a layer
writes the new tokens' K and V, attends over the shared prefix and each row's
own pages, and runs the mixture-of-experts layer.  What it read from HBF, the
prefix's pages of that layer and the pages of the experts that some token chose,
goes to ``Model.time_layers``: layer after layer, each issued when the one before
is there.  Projections and norms are plain torch operations, and the
weights are random: the example stands for the traffic, not for a trained model.
"""
import argparse

import numpy as np
import torch

from paper_2609_09800_amd import hbf
from paper_2609_09800_amd import workloads as wl


class Decoder:
    """`layers` decode layers of wl's MoE shape (smaller where asked), `rows`
    samples behind a prompt of `prefix` tokens."""

    def __init__(self, layers=4, rows=16, prefix=1024, experts=32, topk=wl.MOE_TOPK, hidden=wl.MOE_HIDDEN,
                 ffn=wl.MOE_FFN, heads=32, own=64, seed=0):
        self.layers, self.rows, self.prefix, self.hidden, self.heads = layers, rows, prefix, hidden, heads
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").mul_(shape[-1] ** -0.5).bfloat16()
        # experts: one block each of gate, up and down, whole HBF pages (wl.PAGES_PER_EXPERT of the paper's shape)
        block = 3 * ffn * hidden
        self.pages_per_expert = -(-block * 2 // wl.PAGE)
        size = self.pages_per_expert * wl.PAGE // 2
        self.weights, view = self._hbf_range(layers * experts * size)
        experts_of = view.view(layers, experts, size)
        experts_of.normal_(generator=gen).mul_(hidden ** -0.5)
        self.expert_base = view.data_ptr()
        self.experts = experts
        self.moe = [hbf.MoeLayer(experts_of[l, :, :2 * ffn * hidden].unflatten(1, (2 * ffn, hidden)),
                                 experts_of[l, :, 2 * ffn * hidden:block].unflatten(1, (hidden, ffn)), topk,
                                 router=rand(experts, hidden), max_tokens=rows) for l in range(layers)]
        kv, dim = wl.KV_HEADS, wl.KV_DIM
        self.proj = [(rand(heads * dim, hidden), rand(2 * kv * dim, hidden), rand(hidden, heads * dim))
                     for _ in range(layers)]
        # the cache: 16 tokens of a layer's K or V are one HBF page
        pt = wl.PAGE // (kv * dim * 2)
        self.shared = -(-prefix // pt)
        pages = self.shared + rows * (-(-own // pt) + 2)
        self.pool_range, pool = self._hbf_range(layers * 2 * pages * pt * kv * dim)
        pool = pool.view(layers, 2, pages, pt, kv, dim)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables = torch.full((rows + 1, self.shared + -(-own // pt) + 1), -1, **i32)
        self.lens = torch.zeros(rows + 1, **i32)
        self.kv = hbf.KvPages(pool, refs=torch.zeros(pages, **i32), tables=self.tables, lens=self.lens)
        self.slots = torch.arange(1, rows + 1, **i32)
        prompt = torch.zeros(1, **i32)
        self._ok(self.kv.extend(prompt, torch.full((1,), prefix, **i32)))
        k, v = (torch.randn((layers, prefix, kv, dim), generator=gen, device="cuda").bfloat16() for _ in range(2))
        self._ok(self.kv.write(k, v, prompt.expand(prefix).contiguous(), torch.arange(prefix, **i32)))
        # full pages are shared by all rows; the rest of the prompt is copied to each row's own page
        self._ok(self.kv.fork(prompt.expand(rows).contiguous(), self.slots))
        self.full = prefix // pt * pt
        self.one = torch.ones(rows, **i32)
        self.ids = torch.zeros((layers, rows, topk), **i32)
        self.model = hbf.Model(**wl.geometry(16, 8, 4))
        for t in (self.weights, self.pool_range):
            self._ok(self.model.register_range(*t)[0])

    @staticmethod
    def _ok(rc):
        if rc != hbf.HBF_OK:
            raise hbf.HbfError(rc, "decode")

    def _hbf_range(self, values):
        """A page-aligned bfloat16 buffer: ((base, bytes) to register, the values)."""
        nbytes = -(-values * 2 // wl.PAGE) * wl.PAGE
        buf = torch.empty(nbytes + wl.PAGE, dtype=torch.uint8, device="cuda")
        off = -buf.data_ptr() % wl.PAGE
        return (buf.data_ptr() + off, nbytes), buf[off:off + nbytes].view(torch.bfloat16)[:values]

    def step(self, x):
        """One token per row through every layer; x: bfloat16 [rows, hidden]."""
        kv_heads, dim, pt = wl.KV_HEADS, wl.KV_DIM, self.kv.page_tokens
        self._ok(self.kv.extend(self.slots, self.one))
        pos = self.lens[1:] - 1
        own = self.lens[1:] - self.full
        prefix_pages = self.tables[1, :self.full // pt].contiguous()
        norm = lambda t: (t.float() * t.float().square().mean(1, keepdim=True).add(1e-6).rsqrt()).bfloat16()
        for l in range(self.layers):
            wq, wkv, wo = self.proj[l]
            h = norm(x)
            k, v = (h @ wkv.t()).view(self.rows, 2, kv_heads, dim).unbind(1)
            self._ok(self.kv.write(k.contiguous(), v.contiguous(), self.slots, pos, first_layer=l))
            q = (h @ wq.t()).view(self.rows, self.heads, dim)
            out = torch.empty_like(q)
            self._ok(self.kv.prefix_attention(l, q, out, prefix_pages, self.full, self.tables[1:, self.full // pt:], own))
            x = x + out.view(self.rows, -1) @ wo.t()
            h = norm(x)
            y = torch.empty_like(h)
            weights = torch.empty(self.ids[l].shape, dtype=torch.float32, device="cuda")
            self._ok(self.moe[l].forward(h, y, self.ids[l], weights))
            x = x + y
        return x

    def read_pages(self):
        """(addresses of the HBF pages that the last step read, layer by layer; layer_start)."""
        chosen = self.ids.cpu().numpy()
        shared = self.tables[1, :self.full // self.kv.page_tokens].cpu().numpy().astype(np.int64)
        addr, start = [], [0]
        for l in range(self.layers):
            planes = (np.array([2 * l, 2 * l + 1])[:, None] * self.kv.pages + shared[None, :]).ravel()
            act = np.unique(chosen[l]).astype(np.int64)
            ex = ((l * self.experts + act)[:, None] * self.pages_per_expert
                  + np.arange(self.pages_per_expert)[None, :]).ravel()
            addr.append(np.concatenate([self.pool_range[0] + planes * wl.PAGE, self.expert_base + ex * wl.PAGE]))
            start.append(start[-1] + addr[-1].size)
        return np.concatenate(addr), np.array(start, dtype=np.int64)

    def modeled_ns(self, compute_ns=2000):
        """When each layer's pages of the last step would be there, from an idle device, in ns."""
        addr, start = self.read_pages()
        a = torch.from_numpy(addr).cuda()
        issue, complete = torch.empty_like(a), torch.empty_like(a)
        done = torch.empty(self.layers, dtype=torch.int64, device="cuda")
        self.model.reset()
        self._ok(self.model.time_layers(a, start, 0, compute_ns, issue, complete, done))
        self._ok(self.model.get_status())
        return done.cpu().numpy(), start


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("layers", 4), ("rows", 16), ("prefix", 1024), ("steps", 3)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    d = Decoder(layers=a.layers, rows=a.rows, prefix=a.prefix, own=a.prefix % 16 + a.steps)
    x = torch.randn((a.rows, d.hidden), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    for s in range(a.steps):
        t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        t0.record()
        x = d.step(x)
        t1.record()
        done, start = d.modeled_ns()
        print(f"step {s}: {t0.elapsed_time(t1) * 1e3:.0f} us on the GPU; {start[-1]} HBF pages, "
              f"{done[-1] / 1e3:.0f} us modeled ({', '.join(f'{t / 1e3:.0f}' for t in done)} by layer)")
    for what in (d.kv, *d.moe):
        Decoder._ok(what.get_status())
    return x


if __name__ == "__main__":
    main()
