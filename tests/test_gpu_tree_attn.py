"""Attention of drafted trees over the cache and the commit of their accepted paths, against the 64-bit oracle: every
count of rows and states around the tiles' edges, ragged and empty documents, padding, infinities in what a node does not see,
strides, streams and graphs.  Needs an MI355X."""

import numpy as np
import pytest
import torch

import paper_2406_12018_amd as api
from generation import DEV, Rand, as_tensor, check_rows, config, f64, same_bits, tree_words, weight_error
from oracle import citrus_oracle as orc

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, seed, B, L, Hq, Hkv, d, T, n, dtype="bf16", lens=None, trees=None, cap=None, **kw):
        self.cfg = config(B, L, Hq, Hkv, d, cap or max(n, 1), dtype, **kw)
        self.T, self.n, self.dtype = T, n, dtype
        make = Rand(seed, dtype)
        rows = self.cfg.cache_capacity
        self.q, self.kd, self.vd = make(B, L, Hq, T, d), make(B, L, Hkv, T, d, scale=0.6), make(B, L, Hkv, T, d)
        self.kc, self.vc = make(B, L, Hkv, rows, d, scale=0.6), make(B, L, Hkv, rows, d)
        self.given = lens
        self.lens = [n] * B if lens is None else [min(max(x, 0), n) for x in lens]
        trees = trees or [T] * B
        self.words = [tree_words(seed + b, t) + [0] * (T - t) for b, t in enumerate(trees)]

    def run(self, **kw):
        lse = torch.full(self.q.shape[:4], 7.0, dtype=torch.float32, device=DEV)
        ws = torch.full((api.generation_workspace_bytes(self.cfg, self.T) + 16,), 0xA5, dtype=torch.uint8, device=DEV)[:-16]
        lens = None if self.given is None else torch.tensor(self.given, dtype=torch.int32, device=DEV)
        out = api.citrus_tree_attn(self.cfg, self.q, self.kd, self.vd, as_tensor(self.words), self.kc, self.vc, self.n,
                                   **{**dict(cache_lens=lens, lse=lse, workspace=ws), **kw})
        torch.cuda.synchronize()
        return out, lse

    def check(self, out, lse):
        cfg = self.cfg
        scale = cfg.softmax_scale or cfg.head_dim ** -0.5
        q, kd, vd, kc, vc, out, lse = (f64(t) for t in (self.q, self.kd, self.vd, self.kc, self.vc, out, lse))
        for b in range(cfg.batch):
            n = self.lens[b]
            for l in range(cfg.layers):
                ref, ref_lse, mag = orc.tree_attn(q[b, l], kd[b, l], vd[b, l], self.words[b], kc[b, l, :, :n], vc[b, l, :, :n], scale)
                real = np.isfinite(ref_lse)
                assert (lse[b, l][~real] == -np.inf).all() and (out[b, l][~real] == 0).all(), "padding"
                error = weight_error(q[b, l], np.concatenate([kc[b, l, :, :n], kd[b, l]], axis=1), n + self.T, scale)
                check_rows(out[b, l], ref, mag, error, self.dtype, f"document {b} layer {l}")
                assert np.abs(lse[b, l][real] - ref_lse[real]).max(initial=0) <= error + 2.0 ** -22 * np.abs(ref_lse[real]).max(initial=1)


SHAPES = [  # B, L, Hq, Hkv, d, T, n
    (1, 1, 1, 1, 128, 1, 0), (1, 1, 4, 1, 64, 1, 1), (2, 1, 4, 2, 128, 1, 31), (1, 2, 8, 2, 128, 2, 32), (1, 1, 8, 8, 64, 3, 33),
    (2, 2, 6, 2, 128, 5, 63), (1, 1, 7, 1, 64, 9, 64), (1, 1, 16, 2, 128, 8, 65), (1, 1, 4, 4, 128, 31, 127), (1, 1, 4, 4, 64, 32, 128),
    (1, 1, 2, 2, 128, 33, 129), (1, 1, 8, 2, 128, 16, 255), (1, 1, 8, 2, 64, 17, 500), (1, 1, 8, 1, 128, 33, 300), (1, 1, 16, 2, 128, 64, 97),
    (1, 1, 40, 1, 128, 3, 200), (1, 1, 40, 1, 64, 64, 70), (3, 1, 2, 1, 64, 63, 0), (1, 3, 3, 3, 128, 64, 1), (1, 1, 8, 8, 128, 7, 1300),
    (1, 1, 4, 1, 128, 1, 4500), (1, 1, 8, 2, 64, 13, 5000), (1, 1, 8, 1, 128, 40, 2500), (2, 70, 4, 2, 64, 4, 40),
    (2, 5, 16, 1, 128, 64, 90), (1, 11, 9, 1, 64, 60, 33), (1, 1, 4, 1, 128, 64, 3000), (3, 3, 4, 1, 128, 40, 260),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_trees_against_64_bits(shape, dtype):
    case = Case(11, *shape, dtype=dtype)
    out, lse = case.run()
    case.check(out, lse)
    again, lse2 = case.run()
    same_bits(out, again)
    same_bits(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 6, 30, 64])
def test_ragged_documents_and_padding(T, d, dtype):
    """Lengths of zero, inside and at the ends of tiles, the longest, and ones outside 0 .. cache_len; trees of other sizes; what
    lies behind a document's length and in the padding is NaN."""
    lens = [0, 1, 32, 33, 300, -5, 1000, 64, 299]
    trees = [max(1, T - b) if b % 2 else T for b in range(len(lens))]
    case = Case(5, len(lens), 2, 6, 2, d, T, 300, dtype, lens=lens, trees=trees, cap=310, softmax_scale=0.11)
    clean = case.run()
    case.check(*clean)
    for b, n in enumerate(case.lens):
        case.kc[b, :, :, n:] = float("nan")
        case.vc[b, :, :, n:] = float("nan")
        for t in (case.q, case.kd, case.vd):
            t[b, :, :, trees[b]:] = float("nan")
    for a, b in zip(case.run(), clean):
        same_bits(a, b)


MANY_SHORT = [  # units that fill the chip more than once, with few keys each
    (2, 65, 4, 2, 128, 1, 0), (2, 70, 8, 2, 128, 5, 37), (3, 50, 4, 2, 128, 16, 300), (1, 1400, 1, 1, 128, 3, 20), (1, 90, 6, 6, 64, 2, 130),
    (2, 140, 8, 2, 64, 8, 31), (1, 2700, 1, 1, 64, 1, 33), (1, 32, 32, 32, 128, 1, 63),
]


@pytest.mark.parametrize("shape", MANY_SHORT, ids=lambda s: "x".join(map(str, s)))
def test_many_units_of_few_keys(shape):
    case = Case(12, *shape)
    out, lse = case.run()
    case.check(out, lse)
    again, lse2 = case.run()
    same_bits(out, again)
    same_bits(lse, lse2)


MANY_WIDE = [  # ... with more than 64 rows a unit: three, four, seven and eight blocks of 32, few keys and more
    (1, 130, 8, 2, 128, 24, 70), (2, 65, 16, 2, 128, 16, 0), (1, 130, 8, 2, 128, 56, 200), (2, 65, 16, 2, 128, 31, 130), (1, 130, 8, 2, 128, 60, 600),
    (1, 130, 8, 2, 64, 24, 70), (1, 130, 8, 2, 64, 64, 33), (1, 130, 8, 2, 64, 40, 300),
]


@pytest.mark.parametrize("shape", MANY_WIDE, ids=lambda s: "x".join(map(str, s)))
def test_many_units_of_more_rows(shape):
    case = Case(13, *shape)
    clean = case.run()
    case.check(*clean)
    T = case.T
    case.words = [[sum(1 << u for u in range(t + 1) if u % 2 == t % 2) for t in range(T)]] * case.cfg.batch
    clean = case.run()
    kd, vd = case.kd.clone(), case.vd.clone()
    kd[:, :, :, 1::2], vd[:, :, :, 1::2] = float("nan"), float("inf")
    for a, b in zip(_with(case, kd, vd), clean):
        same_bits(a[:, :, :, 0::2], b[:, :, :, 0::2])


@pytest.mark.parametrize("d", [64, 128])
def test_many_units_of_few_keys_ragged(d):
    """Documents of other lengths, padding, and a branch whose states are NaN or infinite beside one that does not see them."""
    lens, T = [0, 70, 31, 1, 64, 300], 6
    case = Case(6, len(lens), 50, 6, 2, d, T, 70, lens=lens, trees=[6, 1, 2, 6, 3, 5], cap=75)
    clean = case.run()
    case.check(*clean)
    for b, n in enumerate(case.lens):
        case.kc[b, :, :, n:] = float("nan")
        case.vc[b, :, :, n:] = float("-inf")
    for a, b in zip(case.run(), clean):
        same_bits(a, b)
    case.words = [[sum(1 << u for u in range(t + 1) if u % 2 == t % 2) for t in range(T)]] * len(lens)
    left, clean = [0, 2, 4], case.run()
    case.check(*clean)
    for bad_k, bad_v in ((float("nan"), 1.0), (1.0, float("inf"))):
        kd, vd = case.kd.clone(), case.vd.clone()
        kd[:, :, :, 1::2], vd[:, :, :, 1::2] = bad_k, bad_v
        out, lse = _with(case, kd, vd)
        same_bits(out[:, :, :, left], clean[0][:, :, :, left])
        same_bits(lse[:, :, :, left], clean[1][:, :, :, left])
        assert not torch.isfinite(out[:, :, :, 1::2].float()).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 45, 300])
def test_a_draft_in_the_memory_of_the_cache(n, dtype):
    """Behind the cache's rows, or at its beginning where there are none."""
    case = Case(9, 2, 2, 6, 2, 128, 7, n, dtype, cap=n + 9)
    apart = case.run()
    case.check(*apart)
    case.kc[:, :, :, n:n + 7], case.vc[:, :, :, n:n + 7] = case.kd, case.vd
    case.kd, case.vd = case.kc[:, :, :, n:n + 7], case.vc[:, :, :, n:n + 7]
    for a, b in zip(case.run(), apart):
        same_bits(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,n", [(2, 0), (2, 45), (10, 200), (10, 3000)])
def test_what_a_node_does_not_see_does_not_touch_it(Hq, n, d, dtype):
    """Two branches; the states of one are NaN or infinite: the rows of the other stay as they were, and its own say so."""
    T = 12
    case = Case(3, 1, 1, Hq, 2, d, T, n, dtype)
    left = [t for t in range(T) if t % 2 == 0]
    words = [sum(1 << u for u in range(t + 1) if u % 2 == t % 2) for t in range(T)]
    case.words = [words]
    clean = case.run()
    case.check(*clean)
    for bad_k, bad_v in ((float("nan"), float("nan")), (1.0, float("inf")), (float("-inf"), 1.0), (float("inf"), float("-inf"))):
        kd, vd = case.kd.clone(), case.vd.clone()
        kd[:, :, :, 1::2], vd[:, :, :, 1::2] = bad_k, bad_v
        out, lse = _with(case, kd, vd)
        same_bits(out[:, :, :, left], clean[0][:, :, :, left])
        same_bits(lse[:, :, :, left], clean[1][:, :, :, left])
        if bad_v != 1.0:
            assert not torch.isfinite(out[:, :, :, 1::2].float()).any()


def _with(case, kd, vd):
    kept, case.kd, case.vd = (case.kd, case.vd), kd, vd
    try:
        return case.run()
    finally:
        case.kd, case.vd = kept


def test_bits_behind_the_draft_are_ignored():
    case = Case(4, 1, 1, 8, 2, 128, 9, 50)
    want = case.run()
    case.words = [[w | 0xABCD << 40 | 1 << 63 | 1 << 9 for w in doc] for doc in case.words]
    for a, b in zip(case.run(), want):
        same_bits(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_in_the_cache_reach_every_row(dtype):
    """An infinite value in a state of the last, partly filled tile: the element is infinite in every row, the others stay finite."""
    case = Case(8, 1, 1, 4, 2, 128, 3, 77, dtype)
    case.vc[:, :, :, 76, 5] = float("inf")
    out, _ = case.run()
    assert (out[..., 5] == float("inf")).all() and torch.isfinite(torch.cat([out[..., :5], out[..., 6:]], -1).float()).all()


@pytest.mark.parametrize("dtype,d,T,n", [("bf16", 128, 1, 700), ("bf16", 64, 20, 90), ("f32", 128, 5, 130), ("bf16", 128, 64, 2100)])
def test_strides_and_shared_trees_give_the_same_bits(dtype, d, T, n):
    case = Case(21, 2, 3, 8, 2, d, T, n, dtype, lens=[n, n // 2])
    case.words[1] = case.words[0]
    out, lse = case.run()

    def token_major(t, spare):  # [B, S, L, H, d + spare], rows apart from each other
        b, l, h, s, dd = t.shape
        wide = torch.full((b, s, l, h, dd + spare), float("nan"), dtype=t.dtype, device=DEV)
        view = wide[..., :dd].permute(0, 2, 3, 1, 4)
        view.copy_(t)
        return view

    kept = {x: getattr(case, x) for x in ("q", "kd", "vd", "kc", "vc")}
    for i, (name, t) in enumerate(kept.items()):
        setattr(case, name, token_major(t, 8 * i))
    strided = token_major(torch.zeros_like(kept["q"]), 16)
    out2, lse2 = case.run(out=strided)
    same_bits(out, out2)
    same_bits(lse, lse2)
    words = as_tensor(case.words[0])
    lens = torch.tensor(case.lens, dtype=torch.int32, device=DEV)
    ws = api.alloc_generation_workspace(case.cfg, T)
    shared = api.citrus_tree_attn(case.cfg, case.q, case.kd, case.vd, words, case.kc, case.vc, n, cache_lens=lens, workspace=ws)
    same_bits(out, shared)


def test_rows_of_a_unit_that_nearly_span_the_limit():
    """Element offsets past 31 bits between units and byte offsets near 2^31 inside one."""
    d, n, stride = 128, 33, (2 ** 30 - 4096) // 33 // 8 * 8
    case = Case(2, 1, 1, 2, 2, d, 4, n)
    big = torch.empty(2 * 34 * stride + d, dtype=torch.bfloat16, device=DEV)
    kc = torch.as_strided(big, (1, 1, 2, n, d), (stride * 68, stride * 68, stride * 34, stride, 1))
    kc.copy_(case.kc[:, :, :, :n])
    want = case.run()
    case.kc = kc
    for a, b in zip(case.run(), want):
        same_bits(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_one_node_is_a_decoding_step_and_a_chain_a_chunk(d, dtype):
    """The framework's own operators on the same inputs; both sides round weights and results once each."""
    n, T = 450, 24
    case = Case(31, 1, 2, 8, 2, d, T, n, dtype, cap=n + 1, chunk_len=T)
    case.words = [[(1 << t + 1) - 1 for t in range(T)]]
    out, lse = case.run()
    lse2 = torch.empty_like(lse)
    chunk = api.citrus_chunk_attn(case.cfg, case.q, case.kc, case.vc, n, case.kd, case.vd, lse=lse2)
    tol = (2e-2, 1e-2) if dtype == "bf16" else (1e-5, 1e-5)
    torch.testing.assert_close(out.float(), chunk.float(), atol=tol[0], rtol=tol[1])
    torch.testing.assert_close(lse, lse2, atol=tol[0], rtol=tol[1])
    one = Case(32, 1, 2, 8, 2, d, 1, n, dtype, cap=n + 1)
    got, _ = one.run()
    step = api.citrus_decode_step(one.cfg, one.q, one.kd, one.vd, one.kc, one.vc, n, workspace=api.alloc_workspace(one.cfg))
    torch.testing.assert_close(got.float(), step.float(), atol=tol[0], rtol=tol[1])


@pytest.mark.parametrize("shape", [(1, 1, 8, 2, 128, 8, 900), (2, 40, 8, 4, 64, 40, 200), (1, 2, 8, 1, 128, 64, 4096)])
def test_replays_of_a_graph_and_other_streams(shape):
    case = Case(17, *shape)
    want = case.run()
    ws, out = api.alloc_generation_workspace(case.cfg, case.T), torch.zeros_like(case.q)
    words, stream = as_tensor(case.words), torch.cuda.Stream()
    call = lambda: api.citrus_tree_attn(case.cfg, case.q, case.kd, case.vd, words, case.kc, case.vc, case.n, out=out, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    same_bits(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for _ in range(3):
        out.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same_bits(out, want[0])


@pytest.mark.parametrize("Hq,Hkv,L,cap", [(8, 2, 1, 5000), (8, 8, 40, 300), (64, 1, 1, 700), (1, 1, 1, 40000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nothing_is_written_outside_the_workspace(Hq, Hkv, L, cap, dtype):
    """A workspace for 64 nodes serves every smaller tree and every length up to the capacity."""
    guard = 1 << 16
    for T in (1, 7, 33, 64):
        for n in sorted({0, 1, 33, cap // 3, cap}):
            case = Case(4, 1, L, Hq, Hkv, 64, T, n, dtype, cap=cap)
            size = api.generation_workspace_bytes(case.cfg, 64)
            buf = torch.full((size + 2 * guard,), 0xA5, dtype=torch.uint8, device=DEV)
            case.run(workspace=buf[guard:guard + size])
            assert bool((buf[:guard] == 0xA5).all()) and bool((buf[guard + size:] == 0xA5).all()), (T, n)


# ---- commit ----
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,T,P,L,Hkv", [(64, 1, 1, 1, 1), (128, 8, 4, 2, 8), (64, 64, 64, 3, 5), (128, 40, 7, 1, 32)])
def test_commit_moves_bits_and_nothing_else(d, T, P, L, Hkv, dtype):
    lens, accepted = [0, 5, 33, 90, 96, -3, 200, 17], [P, 0, min(P, 3), P, P, 1, -4, P + 9]
    B, n, cap = len(lens), 96, 98
    cfg, make = config(B, L, Hkv, Hkv, d, cap, dtype), Rand(6, dtype)
    kd, vd, kc, vc = make(B, L, Hkv, T, d), make(B, L, Hkv, T, d), make(B, L, Hkv, cap, d), make(B, L, Hkv, cap, d)
    rng = np.random.default_rng(T)
    path = rng.integers(0, T, (B, P)).astype(np.int32)  # the same node twice, too
    path[2, 0] = T        # no such node: its cache row stays
    path[3, -1] = -1
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    want_k, want_v, want_lens = kc.clone(), vc.clone(), []
    for b in range(B):
        at, m = min(max(lens[b], 0), n), min(max(accepted[b], 0), P)
        m = min(m, cap - at)
        for i in range(m):
            if 0 <= path[b, i] < T:
                want_k[b, :, :, at + i], want_v[b, :, :, at + i] = kd[b, :, :, path[b, i]], vd[b, :, :, path[b, i]]
        want_lens.append(at + m)
    new = api.citrus_tree_commit(cfg, kd, vd, dev(path), dev(accepted), kc, vc, n, cache_lens=dev(lens))
    same_bits(kc, want_k)
    same_bits(vc, want_v)
    assert new.tolist() == want_lens


def test_commit_with_one_length_and_strided_caches():
    B, L, H, T, d, cap = 2, 2, 4, 6, 64, 50
    cfg, make = config(B, L, H, H, d, cap), Rand(9, "bf16")
    kd, vd = make(B, L, H, T, d), make(B, L, H, T, d)
    wide = make(B, cap, L, H, 3 * d)
    before = wide.clone()
    kc, vc = wide[..., :d].permute(0, 2, 3, 1, 4), wide[..., 2 * d:].permute(0, 2, 3, 1, 4)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    new = api.citrus_tree_commit(cfg, kd, vd, dev([[4, 5], [0, 3]]), dev([1, 2]), kc, vc, 20)
    assert new.tolist() == [21, 22]
    for b, nodes in enumerate(([4], [0, 3])):
        for i, t in enumerate(nodes):
            before[b, 20 + i, :, :, :d], before[b, 20 + i, :, :, 2 * d:] = kd[b, :, :, t], vd[b, :, :, t]
    same_bits(wide, before)
