"""Pools of 8-bit pages for the GPU tests: code values and scales, and the same on the GPU."""
import numpy as np
import torch

from oracle import qcf_oracle as orc
from paper_2604_08585_amd import binding as qb
from paper_2604_08585_amd import inputs
from gpu_util import DEV, i32

E4M3 = torch.float8_e4m3fn
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def say(*a):
    print(*a, flush=True)


def shape(H, Hkv, D, dtype, style=0, base=500000.0):
    return inputs.LayerShape(H * D, H, Hkv, D, base, dtype, style)


def normal(rng, size, dtype, std=1.0):
    return inputs.round_to_dtype((rng.standard_normal(size) * std).astype(np.float32), dtype)


class Paged8:
    """Random codes in shuffled pages, scales of 2^-9 to 2^-6; `order` puts heads or tokens next to each other."""

    def __init__(self, rng, sh, page, lens, order="token", spare=3, width=None, bounds=True):
        self.sh, self.page, self.order = sh, page, order
        Hkv, D, self.dt = sh.n_kv_heads, sh.head_dim, inputs.torch_dtype(sh.dtype)
        counts = [-(-n // page) for n in lens]
        n_pages = sum(counts) + spare
        perm = rng.permutation(n_pages)
        self.table = np.full((len(lens), max(counts + [1]) if width is None else width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(counts):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.codes = [orc.e4m3(np.clip(rng.standard_normal((n_pages, page, Hkv, D)) * 120, -448, 448)) for _ in range(2)]
        self.scales = np.exp2(rng.integers(-9, -5, (n_pages, Hkv, 2, page // 16)).astype(np.float64))
        k = self.values()[0]
        self.bounds = np.stack([k.min(1), k.max(1)], axis=2)
        self.upload(bounds)

    def values(self):
        return orc.page8_values(self.codes, self.scales)

    def upload(self, bounds=True):
        def pool(a):
            t = torch.from_numpy(a.astype(np.float32)).to(E4M3).view(torch.uint8).to(DEV)
            t = t.transpose(1, 2).contiguous().transpose(1, 2) if self.order == "head" else t
            return t.view(E4M3)
        self.kd, self.vd = pool(self.codes[0]), pool(self.codes[1])
        self.sd = torch.from_numpy(self.scales.astype(np.float32)).to(DEV)
        self.bd = torch.from_numpy(self.bounds).to(device=DEV, dtype=self.dt) if bounds else None
        self.td = i32(self.table)
        self.cache = qb.page8_cache(self.kd, self.vd, self.sd, self.bd, self.td, self.dt)
        self.desc = qb.make_desc(self.sh)

    def got(self):
        """Code values of keys and values, and scales, from the GPU."""
        num = lambda t: t.view(torch.uint8).cpu().view(E4M3).double().numpy()
        return num(self.kd), num(self.vd), self.sd.double().cpu().numpy()
