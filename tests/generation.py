"""Shared by the tests of generation over a retained cache: seeded inputs, drafted trees, error bounds."""

from __future__ import annotations

import numpy as np
import torch

import paper_2406_12018_amd as api
from oracle import citrus_oracle as orc

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step of rounding to the type, relative


def config(B, L, Hq, Hkv, d, cap, dtype="bf16", **kw):
    kw = {**dict(chunk_len=8, budget=1, instr_len=1), **kw}
    return api.Config(batch=B, layers=L, q_heads=Hq, kv_heads=Hkv, head_dim=d, dtype=api.F32 if dtype == "f32" else api.BF16,
                      cache_capacity=cap, **kw)


class Rand:
    def __init__(self, seed, dtype):
        self.g, self.dtype = torch.Generator().manual_seed(seed), TORCH[dtype]

    def __call__(self, *shape, scale=1.0):
        return (torch.randn(shape, generator=self.g) * scale).to(self.dtype).to(DEV)


def tree_words(seed, nodes):
    """A random tree: every node's ancestors and itself as the bits of a word."""
    rng, words = np.random.default_rng(seed), [1]
    for t in range(1, nodes):
        words.append(words[int(rng.integers(max(0, t - 6), t))] | 1 << t)
    return words


def as_tensor(words):
    signed = np.array(words, dtype=np.uint64).astype(np.int64)
    return torch.from_numpy(signed).to(DEV)


def f64(t):
    return t.detach().to("cpu").to(torch.float64).numpy()


def weight_error(q, k, n, scale):
    """Bound on the relative error of a softmax weight of n states computed in 32 bits.  A logit is off by at most (d + 8) roundings
    (d products added up, the scale, base 2) of sum_i |q_i k_i| scale, the sum of n weights by n roundings of itself; weight =
    exp(logit) / sum of exp(logits): twice the logits' error, the sum's, and a few roundings of the exponential."""
    d = q.shape[-1]
    most = float(np.abs(q).reshape(-1, d).max(0) @ np.abs(k).reshape(-1, d).max(0)) * scale
    return 2.0 ** -24 * (2 * (d + 8) * most + n + 16)


def check_rows(got, ref, mag, error, dtype, what=""):
    """Rows sum_j p_j v_j: p off by `error` relative, and in bf16 rounded before its product, the result rounded to the type.
    mag = sum_j p_j |v_j| is what the former scale with."""
    bound = STEP[dtype] * np.abs(ref) + (error + (STEP["bf16"] if dtype == "bf16" else 2.0 ** -23)) * mag * (1 + STEP[dtype]) + 1e-30
    off = np.abs(got - ref)
    assert np.isfinite(got).all() and (off <= bound).all(), f"{what}: {(off > bound).sum()} of {off.size} outside, worst {np.max(off / bound):.3g} of its bound"


def same_bits(a, b, what=""):
    view = lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32) if t.is_floating_point() else t
    assert torch.equal(view(a), view(b)), what
