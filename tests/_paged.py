"""A paged batch for the tests: pools whose unused places hold NaN, tables, lengths, on the CPU and as float64 numpy."""
import numpy as np
import torch

import oracle
from paper_2509_15763_amd import synth


class Paged:
    """lens: rows in use per sequence; news: new rows of each.  missing: (sequence, page) pairs whose table entry names no page."""

    def __init__(self, lens, news, page, Hq, Hkv, D, e4m3=False, seed=0, missing=(), extra_pages=2, behind=0, cols=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.news, self.page, self.Hq, self.Hkv, self.D, self.e4m3 = list(lens), list(news), page, Hq, Hkv, D, e4m3
        B = len(lens)
        per = [-(-n // page) for n in lens]
        n_pages = sum(per) + extra_pages
        cols = cols or max(max(per), 1)
        ids = torch.randperm(n_pages, generator=g)
        self.table = torch.full((B, cols), -1, dtype=torch.int32)
        at = 0
        for b in range(B):
            self.table[b, :per[b]] = ids[at:at + per[b]].int()
            at += per[b]
        self.kv_len = torch.tensor(lens, dtype=torch.int32)
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        self.cu, self.T = torch.tensor(cu, dtype=torch.int32), cu[-1] + behind
        self.ks, self.vs = synth.e4m3_scales(Hkv, seed) if e4m3 else (None, None)
        used = torch.zeros(n_pages, page, dtype=torch.bool)
        for b in range(B):
            for j in range(lens[b]):
                used[self.table[b, j // page], j % page] = True

        def pool(scale):
            x = torch.randn(n_pages, Hkv, page, D, generator=g).to(torch.bfloat16)
            if e4m3:
                x = torch.from_numpy(oracle.quantize_e4m3(x.float().numpy(), scale.numpy()))
            x.permute(0, 2, 1, 3)[~used] = 0x7F if e4m3 else float("nan")
            return x

        self.k, self.v = pool(self.ks), pool(self.vs)
        for t, (b, pg) in enumerate(missing):
            self.table[b, pg] = (-1, n_pages, -2 ** 31, 2 ** 31 - 1)[t % 4]
        self.q = torch.randn(self.T, Hq, D, generator=g).to(torch.bfloat16)
        self.weight = torch.rand(n_pages, Hkv, page, generator=g)

    @property
    def max_new(self):
        return max(max(self.news), 1)

    @property
    def max_kv(self):
        return max(max(self.lens), 1)

    def values(self):
        """The pools in float64."""
        if not self.e4m3:
            return self.k.double().numpy(), self.v.double().numpy()
        return tuple(oracle.dequantize_e4m3(x.numpy(), s.numpy()) for x, s in ((self.k, self.ks), (self.v, self.vs)))

    def want(self, r, W, weigh=0, **mask):
        k, v = self.values()
        return oracle.paged_attn(self.q.transpose(0, 1).double().numpy(), k, v, self.table.tolist(), self.lens, self.cu.tolist(), r, W,
                                 weigh=weigh, **mask)

    def want_weight(self, added, decay):
        """The whole pool of weights afterwards."""
        w = self.weight.double().numpy().copy()
        for b, add in enumerate(added):
            if self.news[b] == 0:
                continue
            for j in range(add.shape[1]):
                pg = int(self.table[b, j // self.page])
                if 0 <= pg < w.shape[0]:
                    w[pg, :, j % self.page] = add[:, j] + (decay * w[pg, :, j % self.page] if decay else 0.0)
        return w

    def cuda(self):
        c = object.__new__(Paged)
        c.__dict__ = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in self.__dict__.items()}
        return c

    @property
    def scales(self):
        return dict(k_scale=self.ks, v_scale=self.vs)
