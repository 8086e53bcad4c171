"""Inputs of the attention-side GPU tests: packed tensors, paged caches full of stale bits, page tables."""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention_oracle as ao

NAN_CODE = 0x7F


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def bf16(x):
    """fp32 numpy -> (device bf16 tensor, its values as fp64 numpy)."""
    t = torch.from_numpy(np.asarray(x, np.float32)).bfloat16()
    return t.cuda(), t.double().numpy()


class Cache:
    """A paged cache on the device whose unused slots hold NaN codes and NaN and infinite scales."""

    def __init__(self, moe, rng, lens, heads, dim, page, spare=2):
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(lens), max(need + [1])), -1, np.int32)
        at = 0
        for i, n in enumerate(need):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.lens, self.page, self.heads, self.dim = list(lens), page, heads, dim
        self.codes = {n: np.full((n_pages, heads, page, dim), NAN_CODE, np.uint8) for n in "kv"}
        self.scales = {n: rng.choice([np.nan, np.inf, -np.inf], (n_pages, heads, page)).astype(np.float32) for n in "kv"}
        self.values = {n: [] for n in "kv"}
        for i, n in enumerate(lens):
            for name in "kv":
                if n == 0:
                    self.values[name].append(np.zeros((heads, 0, dim), np.float32))
                    continue
                x = rng.standard_normal((heads, n, dim)).astype(np.float32) * np.exp(rng.standard_normal((heads, n, 1)))
                c, s = ao.quantize_head_rows(x.astype(np.float32))
                for t in range(n):
                    p, o = self.table[i, t // page], t % page
                    self.codes[name][p, :, o] = c[:, t]
                    self.scales[name][p, :, o] = s[:, t]
                self.values[name].append(ao.cached_rows(c, s))
        self.dev = moe.KVCache(*(torch.from_numpy(a).cuda() for a in (self.codes["k"], self.codes["v"], self.scales["k"],
                                                                      self.scales["v"])))
