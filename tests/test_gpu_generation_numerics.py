"""Generation over a retained cache where errors have small bounds: logits that are exact, so that what is left of an error is the weights'
words, the sums and the rounding of the result.  Needs an MI355X."""

import numpy as np
import pytest
import torch

import paper_2406_12018_amd as api
from generation import DEV, STEP, as_tensor, f64
from oracle import citrus_oracle as orc
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu


def signs(seed, like):
    """-1, 0 and 1 at random: their products and sums are whole numbers, exact in 32 bits."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-1, 2, like.shape, generator=g).to(like.dtype).to(DEV)


def bound(ref, mag, n, dtype):
    """|result - ref| for exact dot products s.  A weight is exp2(s c - m) with s c - m off by four roundings of numbers below 8 (c itself, the
    product, the difference), 2^-24 * 32 in all, and an exponential of 2^-23: 2^-24 * 25 relative after the logarithm's factor.  In bf16 it is
    two words, off by 2^-8 * 2^-8.  At most n + n products of the two words' are added in 32 bits, and n weights in the divisor; joining,
    division and product are a few more.  mag = sum_j p_j |v_j| is what these scale with; the result is rounded to its type."""
    return STEP[dtype] * np.abs(ref) + mag * ((2.0 ** -16 if dtype == "bf16" else 0.0) + 2.0 ** -24 * (3 * n + 64)) * (1 + STEP[dtype])


FORMS = [  # B, L, Hq, Hkv, d, T, n: rows of a KV head up to 32, 64, 128, 256 and beyond; few units and many
    (1, 1, 4, 1, 128, 4, 90), (1, 1, 4, 1, 128, 16, 90), (1, 1, 4, 1, 128, 32, 90), (1, 1, 4, 1, 128, 40, 90), (1, 1, 4, 1, 128, 33, 70),
    (1, 1, 8, 1, 128, 64, 90), (1, 3, 9, 1, 128, 60, 500), (1, 130, 8, 2, 128, 24, 60), (1, 130, 8, 2, 128, 56, 60), (1, 130, 8, 2, 128, 40, 60),
    (1, 1, 4, 1, 64, 8, 90), (1, 1, 4, 1, 64, 32, 90), (1, 1, 8, 1, 64, 64, 90), (1, 130, 8, 2, 64, 40, 60),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", FORMS, ids=lambda s: "x".join(map(str, s)))
def test_rows_are_as_exact_whatever_form_serves_them(shape, dtype):
    case = Case(41, *shape, dtype=dtype)
    case.q, case.kd, case.kc = signs(1, case.q), signs(2, case.kd), signs(3, case.kc)
    out, _ = case.run()
    layers = sorted({0, case.cfg.layers // 2, case.cfg.layers - 1})
    for l in layers:
        q, kd, vd, kc, vc, got = (f64(t[0, l]) for t in (case.q, case.kd, case.vd, case.kc, case.vc, out))
        ref, _, mag = orc.tree_attn(q, kd, vd, case.words[0], kc, vc)
        off, most = np.abs(got - ref), bound(ref, mag, case.n + case.T, dtype)
        assert (off <= most).all(), f"layer {l}: {(off > most).sum()} of {off.size} outside, worst {np.max(off / most):.3g} of its bound"


SEVERAL_TILES = [  # ... to a wave, in every form: the reference that a row's weights are formed against may lag behind its maximum
    (1, 140, 8, 2, 128, 6, 200), (1, 128, 4, 2, 128, 6, 700), (1, 1, 8, 1, 128, 8, 700), (1, 1, 8, 1, 128, 14, 700), (1, 1, 8, 1, 128, 25, 700),
    (1, 1, 8, 1, 128, 64, 700), (1, 130, 8, 2, 128, 24, 150), (1, 130, 8, 2, 128, 56, 150), (1, 140, 8, 2, 64, 6, 200), (1, 128, 4, 2, 64, 6, 700),
    (1, 1, 8, 1, 64, 14, 700), (1, 1, 8, 1, 64, 25, 700), (1, 1, 8, 1, 64, 64, 700), (1, 130, 8, 2, 64, 24, 150),
]


def _same_rows(a, b, rows, what):
    for x, y in zip(a, b):
        x, y = x[:, :, :, rows].contiguous(), y[:, :, :, rows].contiguous()
        kind = torch.int16 if x.dtype == torch.bfloat16 else torch.int32
        differ = int((x.view(kind) != y.view(kind)).sum())
        assert differ == 0, f"{what}: {differ} of {x.numel()} values differ"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SEVERAL_TILES, ids=lambda s: "x".join(map(str, s)))
def test_a_row_depends_on_nothing_but_what_it_sees(shape, dtype):
    """Large and infinite keys that a node does not see, large queries of other nodes and of padding: its row keeps its bits."""
    case = Case(42, *shape, dtype=dtype)
    T = case.T
    left, right = list(range(0, T, 2)), list(range(1, T, 2))
    branches = [sum(1 << u for u in range(t + 1) if u % 2 == t % 2) for t in range(T)]
    case.words = [branches]
    clean, keys, queries = case.run(), case.kd.clone(), case.q.clone()
    case.kd[:, :, :, right] *= 50
    _same_rows(case.run(), clean, left, "large unseen keys")
    case.kd[:, :, :, right, 3] = float("inf")
    _same_rows(case.run(), clean, left, "unseen keys with an infinite element")
    case.kd.copy_(keys)
    case.q[:, :, :, right] *= 40
    _same_rows(case.run(), clean, left, "large queries of other nodes")
    case.words = [[w if t % 2 == 0 else 0 for t, w in enumerate(branches)]]
    for factor in (1.0, 100.0, float("inf")):
        case.q[:, :, :, right] = (queries[:, :, :, right] * factor).nan_to_num(1.0, float("inf"), float("-inf"))
        _same_rows(case.run(), clean, left, f"padding, queries times {factor}")
