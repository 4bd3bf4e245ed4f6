"""Shared helpers of the serving-step tests: a block-format cache as logical numpy
arrays (oracle/step.py) and as device buffers in each layout."""
import numpy as np
import torch

import oracle
from synth.configs import ModelShape

LAYOUTS = ("slot", "paged", "head")


def shape(hq, hkv, dh, theta=1e4, scaling=None):
    return ModelShape(1, 64 * hq, hq, hkv, dh, 256, 1000, theta, 1e-5, rope_scaling=scaling)


def quantised(rng, b, cap, hkv, dh, block, stds=(0.5, 2.0)):
    """Codes and exponents of values N(0, std^2), std of each (sequence, block,
    head) its own."""
    n = cap // block
    std = rng.uniform(*stds, (b, n, hkv))
    x = rng.standard_normal((b, n, block, hkv, dh)) * std[:, :, None, :, None]
    top = np.abs(x).max((2, 4))
    exps = np.vectorize(oracle.block_exponent)(top).astype(np.uint8)
    codes = oracle.e4m3_encode(x * 2.0 ** (127.0 - exps.astype(int))[:, :, None, :, None])
    return codes.reshape(b, cap, hkv, dh), exps


def values(codes, exps):
    block = codes.shape[1] // exps.shape[1]
    scale = 2.0 ** (np.repeat(exps.astype(int), block, 1) - 127.0)
    return oracle.e4m3_decode(codes) * scale[..., None]


class DeviceCache:
    """One layer's cache in `layout`, from logical arrays (numpy, codes of any
    one dtype; exps None for a cache without blocks)."""

    def __init__(self, pkg, codes, exps, seq_len, layout, page=128, seed=0, pos=None, scale=None):
        self.layout, self.page = layout, page
        b, cap = codes["k"].shape[:2]
        self.b, self.cap = b, cap
        d = {"tokens": torch.zeros(b, cap, dtype=torch.int32, device="cuda"),
             "pos": torch.zeros(b, cap, dtype=torch.int32, device="cuda") if pos is None
             else torch.from_numpy(np.ascontiguousarray(pos, np.int32)).cuda(),
             "seq_len": torch.tensor(list(seq_len), dtype=torch.int32, device="cuda")}
        if layout == "paged":
            # a few pages of the pool belong to nobody
            extra = 3
            perm = np.random.default_rng(seed).permutation(b * (cap // page) + extra)
            self.perm = perm[:b * (cap // page)].reshape(b, -1)
            self.n_pages = len(perm)
            d["block_table"] = torch.from_numpy(self.perm.astype(np.int32)).cuda()
            d["page_size"] = page
        if layout == "head":
            d["kv_layout"] = 1
        for n in "kv":
            d[n] = [self.put(codes[n], page)]
        if exps is not None:
            self.block = cap // exps["k"].shape[1]
            d["kv_block"] = self.block
            for n in "kv":
                d[n + "_exp"] = [self.put(exps[n], page // self.block)]
        if scale is not None:
            d["kv_scale"] = scale
        self.d, self.cache = d, pkg.Cache(d)

    def put(self, x, per_page):
        """Logical [B][n][...] in the layout, on the device; what nobody owns holds any bits."""
        t = torch.from_numpy(np.ascontiguousarray(x)) if isinstance(x, np.ndarray) else x
        if self.layout == "head":
            t = t.transpose(1, 2)
        elif self.layout == "paged":
            pool = torch.full((self.n_pages, per_page) + tuple(t.shape[2:]), 0x7F, dtype=torch.uint8) \
                if t.dtype == torch.uint8 else torch.full((self.n_pages, per_page) + tuple(t.shape[2:]),
                                                          float("nan"), dtype=t.dtype)
            pool[torch.from_numpy(self.perm.reshape(-1))] = t.reshape((-1, per_page) + tuple(t.shape[2:]))
            t = pool
        return t.contiguous().cuda()

    def get(self, name):
        """Logical numpy array [B][n][...] of d[name][0]."""
        t = self.d[name][0].cpu()
        if self.layout == "head":
            t = t.transpose(1, 2)
        elif self.layout == "paged":
            t = t[torch.from_numpy(self.perm.reshape(-1))].reshape((self.b, -1) + tuple(t.shape[2:]))
        return (t.float() if t.is_floating_point() else t).numpy()


def starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)


def device_rows(pkg, counts, pos=None):
    n = int(sum(counts))
    return pkg.Rows(n, torch.from_numpy(starts(counts)).cuda(),
                    None if pos is None else torch.from_numpy(np.ascontiguousarray(pos, np.int32)).cuda(),
                    max(counts))


def columns(parts, dtype, pad=0):
    """[n][heads][dh] arrays as strided columns of one device matrix of `dtype`, as a
    fused projection leaves them (pad: unused NaN columns after each)."""
    n = parts[0].shape[0]
    wide = sum(p[0].size + pad for p in parts)
    buf = torch.full((n, wide), float("nan"), dtype=dtype, device="cuda")
    out, at = [], 0
    for p in parts:
        w = p[0].size
        buf[:, at:at + w] = torch.from_numpy(p.reshape(n, w)).to(dtype).cuda()
        out.append(buf[:, at:at + w].view(n, *p.shape[1:]))
        at += w + pad
    return out
