"""Generation over a retained cache without a GPU: what the library and the binding refuse before anything is launched, the
workspace's size, the oracle's pins."""

import ctypes as C

import numpy as np
import pytest
import torch

import paper_2406_12018_amd as api
from generation import Counts, check_counts, check_rows, heavy_places, rows_in_64, weight_error
from oracle import citrus_oracle as orc
from paper_2406_12018_amd import binding as B


def cfg(**kw):
    base = dict(batch=2, layers=1, q_heads=4, kv_heads=2, head_dim=64, chunk_len=32, budget=64, instr_len=8, dtype=B.F32)
    base.update(kw)
    return B.Config(**base)


def at(ptr=0x1000, s=64):
    return B.CTensor(ptr, s * 1024, s * 512, s * 128, s)


NULL = B.CTensor(None, 0, 0, 0, 0)
BIG = 1 << 40


def tree(c=None, q=at(), kd=at(0x2000), vd=at(0x3000), nodes=8, words=0x8000, stride=8, kc=at(0x5000), vc=at(0x6000), n=16, lens=None,
         out=at(0x9000), lse=None, ws=0x10000, size=BIG):
    return B._lib().citrus_tree_attn(C.byref(c or cfg().c()), q, kd, vd, nodes, words, stride, kc, vc, n, lens, out, lse, ws, size, None)


def commit(c=None, kd=at(0x2000), vd=at(0x3000), nodes=8, path=0x8000, path_len=4, accepted=0x8100, kc=at(0x5000), vc=at(0x6000), n=16,
           lens=None, new=0x8200):
    return B._lib().citrus_tree_commit(C.byref(c or cfg().c()), kd, vd, nodes, path, path_len, accepted, kc, vc, n, lens, new, None)


def evict(c=None, q=at(), kn=at(0x2000), vn=at(0x3000), kc=at(0x5000), vc=at(0x6000), acc=0x8000, tokens=70, recent=8, out=at(0x9000),
          gone=None, ws=0x10000, size=BIG):
    return B._lib().citrus_decode_evict_step(C.byref(c or cfg().c()), q, kn, vn, kc, vc, acc, tokens, recent, out, gone, ws, size, None)


@pytest.mark.parametrize("status,kw", [
    (B.ERR_SHAPE, dict(nodes=0)), (B.ERR_SHAPE, dict(nodes=65)), (B.ERR_SHAPE, dict(n=-1)), (B.ERR_SHAPE, dict(n=65)),
    (B.ERR_NULL, dict(words=None)), (B.ERR_SHAPE, dict(words=0x8004)), (B.ERR_SHAPE, dict(stride=7)), (B.ERR_SHAPE, dict(stride=-8)),
    (B.ERR_SHAPE, dict(lens=0x7002)), (B.ERR_NULL, dict(q=NULL)), (B.ERR_NULL, dict(kd=NULL)), (B.ERR_NULL, dict(vd=NULL)),
    (B.ERR_NULL, dict(kc=NULL)), (B.ERR_NULL, dict(vc=NULL)), (B.ERR_NULL, dict(out=NULL)), (B.ERR_SHAPE, dict(q=at(0x1008))),
    (B.ERR_SHAPE, dict(out=at(s=66))), (B.ERR_SHAPE, dict(kd=at(0x5000))), (B.ERR_SHAPE, dict(vd=at(0x6000))), (B.ERR_SHAPE, dict(out=at())),
    (B.ERR_WORKSPACE, dict(ws=None)), (B.ERR_WORKSPACE, dict(size=16)), (B.ERR_WORKSPACE, dict(ws=0x10008)),
    (B.ERR_SHAPE, dict(lse=0x7002)),
])
def test_tree_attention_refuses(status, kw):
    assert tree(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (B.ERR_SHAPE, dict(nodes=0)), (B.ERR_SHAPE, dict(nodes=65)), (B.ERR_SHAPE, dict(n=65)), (B.ERR_SHAPE, dict(path_len=0)),
    (B.ERR_SHAPE, dict(path_len=65)), (B.ERR_NULL, dict(path=None)), (B.ERR_NULL, dict(accepted=None)), (B.ERR_SHAPE, dict(path=0x8002)),
    (B.ERR_SHAPE, dict(accepted=0x8102)), (B.ERR_SHAPE, dict(new=0x8201)), (B.ERR_NULL, dict(kc=NULL)), (B.ERR_NULL, dict(vd=NULL)),
    (B.ERR_SHAPE, dict(kd=at(0x5000))), (B.ERR_SHAPE, dict(kd=at(0x5000), n=0)), (B.ERR_SHAPE, dict(new=0x7000, lens=0x7000)), (B.ERR_SHAPE, dict(new=0x8100)), (B.ERR_SHAPE, dict(new=0x8000)),
])
def test_commit_refuses(status, kw):
    assert commit(**kw) == status


@pytest.mark.parametrize("status,kw", [
    (B.ERR_SHAPE, dict(tokens=-1)), (B.ERR_SHAPE, dict(recent=0)), (B.ERR_SHAPE, dict(recent=65)),
    (B.ERR_SHAPE, dict(recent=61, c=cfg(start_size=4).c())), (B.ERR_NULL, dict(acc=None)), (B.ERR_SHAPE, dict(acc=0x8002)),
    (B.ERR_SHAPE, dict(gone=0x8001)), (B.ERR_NULL, dict(q=NULL)), (B.ERR_NULL, dict(kn=NULL)), (B.ERR_NULL, dict(kc=NULL)),
    (B.ERR_NULL, dict(vc=NULL)), (B.ERR_NULL, dict(out=NULL)), (B.ERR_SHAPE, dict(kn=at(0x5000))), (B.ERR_SHAPE, dict(vn=at(0x6000))),
    (B.ERR_SHAPE, dict(out=at())), (B.ERR_WORKSPACE, dict(ws=None)), (B.ERR_WORKSPACE, dict(size=16)),
    (B.ERR_UNSUPPORTED, dict(c=cfg(head_dim=96).c())), (B.ERR_SHAPE, dict(kc=at(0x5000, s=1 << 27))),
])
def test_bounded_decoding_refuses(status, kw):
    assert evict(**kw) == status


def test_no_configuration():
    lib = B._lib()
    assert lib.citrus_tree_attn(None, at(), at(), at(), 1, 0x8000, 1, at(), at(), 1, None, at(), None, 0x1000, BIG, None) == B.ERR_NULL
    assert lib.citrus_tree_commit(None, at(), at(), 1, 0x8000, 1, 0x8000, at(), at(), 1, None, None, None) == B.ERR_NULL
    assert lib.citrus_decode_evict_step(None, at(), at(), at(), at(), at(), 0x8000, 1, 1, at(), None, 0x1000, BIG, None) == B.ERR_NULL
    assert lib.citrus_generation_workspace_bytes(None, 1) == 0


def test_workspace_grows_with_what_it_serves():
    """A block for a tree of 64 nodes and the capacity serves every smaller call."""
    for kw in (dict(), dict(dtype=B.BF16, q_heads=64, kv_heads=8, head_dim=128), dict(dtype=B.BF16, batch=1, q_heads=40, kv_heads=1)):
        sizes = [api.generation_workspace_bytes(cfg(**kw, cache_capacity=5000), t) for t in range(1, 65)]
        assert sizes[0] > 0 and sizes == sorted(sizes)
        by_budget = [api.generation_workspace_bytes(cfg(**kw, **{"budget": k, "cache_capacity": 50000})) for k in range(64, 40000, 611)]
        assert by_budget == sorted(by_budget)
    assert api.generation_workspace_bytes(cfg(), 0) == api.generation_workspace_bytes(cfg(), 65) == 0
    assert api.generation_workspace_bytes(cfg(head_dim=96), 1) == 0
    with pytest.raises(api.CitrusError):
        api.alloc_generation_workspace(cfg(), 65, "cpu")


def test_the_binding_refuses_tensors_that_do_not_fit(monkeypatch):
    c = cfg(cache_capacity=80)
    f = lambda *shape, **kw: torch.zeros(shape, **kw)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    good = dict(q=f(2, 1, 4, 8, 64), k_draft=f(2, 1, 2, 8, 64), v_draft=f(2, 1, 2, 8, 64), ancestors=torch.zeros((2, 8), dtype=torch.int64),
                k_cache=f(2, 1, 2, 80, 64), v_cache=f(2, 1, 2, 80, 64), cache_len=16)
    with pytest.raises(ValueError, match="host"):
        api.citrus_tree_attn(c, **good)
    monkeypatch.setattr(B, "_stream_on", lambda device, stream: 0)  # from here on the shapes are looked at
    for name, bad in (("k_draft", f(2, 1, 2, 7, 64)), ("v_draft", f(2, 1, 4, 8, 64)), ("k_cache", f(2, 1, 2, 15, 64)),
                      ("v_cache", f(2, 1, 2, 80, 64, dtype=torch.bfloat16)), ("q", f(2, 1, 4, 8, 128)), ("ancestors", i32(2, 8)),
                      ("ancestors", torch.zeros((2, 7), dtype=torch.int64)), ("ancestors", torch.zeros((8, 2), dtype=torch.int64).t()),
                      ("cache_lens", i32(3)), ("cache_lens", torch.zeros(2)), ("lse", f(2, 1, 4, 9)), ("out", f(2, 1, 4, 8, 64).half())):
        with pytest.raises(ValueError, match=name):
            api.citrus_tree_attn(c, **{**good, name: bad})
    with pytest.raises(ValueError, match="contiguous last axis"):
        api.citrus_tree_attn(c, **{**good, "k_cache": f(2, 1, 2, 64, 80).transpose(3, 4)})
    with pytest.raises(api.CitrusError):
        api.citrus_tree_attn(c, **good, stream=0)  # no workspace
    commit_args = dict(k_draft=good["k_draft"], v_draft=good["v_draft"], path=i32(2, 4), accepted=i32(2), k_cache=good["k_cache"],
                       v_cache=good["v_cache"], cache_len=16)
    for name, bad in (("path", i32(2)), ("path", i32(3, 4)), ("accepted", i32(4)), ("k_cache", f(2, 1, 2, 79, 64)), ("new_lens", i32(1))):
        with pytest.raises(ValueError, match=name):
            api.citrus_tree_commit(c, **{**commit_args, name: bad})
    evict_args = dict(q=f(2, 1, 4, 1, 64), k_new=f(2, 1, 2, 1, 64), v_new=f(2, 1, 2, 1, 64), k_cache=good["k_cache"], v_cache=good["v_cache"],
                      acc=f(2, 1, 2, 80), tokens=70, recent=8)
    for name, bad in (("q", f(2, 1, 4, 2, 64)), ("k_new", f(2, 1, 4, 1, 64)), ("k_cache", f(2, 1, 2, 63, 64)), ("acc", f(2, 1, 2, 64)),
                      ("acc", f(2, 1, 2, 80).double()), ("evicted", i32(2, 1, 1))):
        with pytest.raises(ValueError, match=name):
            api.citrus_decode_evict_step(c, **{**evict_args, name: bad})
    with pytest.raises(api.CitrusError):
        api.citrus_decode_evict_step(c, **{**evict_args, "recent": 65}, stream=0)


def test_caches_of_unrotated_keys_are_refused():
    """With position_shift the caches hold keys without rotation: no attention over them as they are.  The commit copies any."""
    shift = cfg(position_shift=1).c()
    assert tree(c=shift) == B.ERR_UNSUPPORTED and evict(c=shift) == B.ERR_UNSUPPORTED
    assert commit(c=shift, path=None) == B.ERR_NULL
    assert api.generation_workspace_bytes(cfg(position_shift=1), 8) == api.generation_workspace_bytes(cfg(), 8)


ROW = 64 * 4


@pytest.mark.parametrize("kw", [
    dict(kd=at(0x5000 + 16 * ROW)), dict(vd=at(0x6000 + 16 * ROW)),          # behind the cached rows, where a draft may be read
    dict(kd=at(0x5000 + 60 * ROW)), dict(kd=at(0x5000 - 7 * ROW)),           # its first rows in the cache, its last one
    dict(kd=at(0x6000 + 2 * ROW), vc=at(0x6000)), dict(vd=at(0x5000 + 63 * ROW)),  # K in V's cache and the other way
    dict(kd=at(0x5000 + 0x8000 + 30 * ROW)), dict(vd=at(0x6000 + 0x40000 + 1)),   # of the next head, of the next document
    dict(kd=at(0x5000 - 0x8000 + 30 * ROW)),
])
def test_a_commit_refuses_a_view_of_the_cache(kw):
    kw = {k: B.CTensor(t.ptr // 16 * 16, t.stride_b, t.stride_l, t.stride_h, t.stride_s) for k, t in kw.items()}
    assert commit(**kw) == B.ERR_SHAPE


@pytest.mark.parametrize("kw", [
    dict(kn=at(0x5000 + 16 * ROW)), dict(vn=at(0x6000 + 63 * ROW)), dict(kn=at(0x6000 + 5 * ROW)), dict(vn=at(0x5000 + 5 * ROW)),
    dict(tokens=20, kn=at(0x5000 + 19 * ROW)), dict(tokens=20, vn=at(0x5000 + 20 * ROW)), dict(tokens=20, kn=at(0x5000 + 0x8000 + 20 * ROW)),
])
def test_bounded_decoding_refuses_a_view_of_the_cached_states(kw):
    assert evict(**kw) == B.ERR_SHAPE


# ---- what the checks of long caches can see ----
def states(seed, n, d, heads=2, nodes=3):
    rng = np.random.default_rng(seed)
    bf16 = lambda x: torch.from_numpy(x).bfloat16().double().numpy()
    return [bf16(rng.normal(size=s) * f) for s, f in (((heads, nodes, d), 1.0), ((nodes, d), 0.5), ((nodes, d), 1.0), ((n, d), 0.5), ((n, d), 1.0))]


def test_rows_in_64_bits_are_the_oracles():
    q, kd, vd, kc, vc = states(1, 70, 16, nodes=6)
    words = [0b1, 0b11, 0b101, 0, 0b10001, 0b100001]
    for got, want in zip(rows_in_64(q, kd, vd, words, kc, vc, 0.3), orc.tree_attn(q, kd[None], vd[None], words, kc[None], vc[None], 0.3)):
        np.testing.assert_allclose(got, want, rtol=1e-12, atol=1e-13)
    out, lse, _ = rows_in_64(q, kd, vd, words, kc[:0], vc[:0])
    assert np.array_equal(out[:, 0], np.broadcast_to(vd[0], (2, 16))) and (out[:, 3] == 0).all() and (lse[:, 3] == -np.inf).all()


@pytest.mark.parametrize("n,d", [(9001, 128), (40000, 64), (131007, 128), (130000, 64)])
def test_a_count_without_one_state_is_rejected(n, d):
    words = [1, 3]
    for only, lost in ((None, range(64, 96)), (0, [n // 64 * 64 - 64]), (31, [31]), (63, [n // 128 * 64 - 1])):
        counts = Counts(d, only)
        ref, total = counts.rows(n, 3, words)
        right = ref.bfloat16()
        check_counts(right, torch.log(total).float(), ref, total, "bf16")
        v = counts.cached(n, 3)
        wrong = ((ref * total[:, None] - v[list(lost)].sum(0)) / total[:, None]).bfloat16()  # its V was zero
        with pytest.raises(AssertionError):
            check_counts(wrong, None, ref, total, "bf16")
        with pytest.raises(AssertionError):  # not seen at all, any one
            check_counts(right, torch.log(total - 1).float(), ref, total, "bf16")
        if only is not None:
            moved = (ref * total[:, None] - v[lost[0]] + torch.roll(v[lost[0]], 1)) / total[:, None]  # another state's V
            with pytest.raises(AssertionError):
                check_counts(moved.bfloat16(), None, ref, total, "bf16")
    ref, total = Counts(d).rows(n, 0, [1, 0])
    assert (ref[1] == 0).all() and total[1] == 0


@pytest.mark.parametrize("n,d", [(3000, 64), (9001, 128), (131007, 128)])
def test_heavy_states_are_missed(n, d):
    """Any one of them lost, or with the V of its neighbour."""
    q, kd, vd, kc, vc = states(2, n, d)
    words, c, places, scale = [1, 3, 5], d // 2 - 3, heavy_places(n, 10), d ** -0.5
    q[..., c], kc[:, c], kd[:, c] = 4.0, 0.0, 0.0
    kc[places, c] = torch.tensor(14.0 * d ** 0.5 / 4.0).bfloat16().item()
    ref, _, mag = rows_in_64(q, kd, vd, words, kc, vc, scale)
    error = weight_error(q, np.concatenate([kc, kd]), n + 3, scale)
    rounded = lambda x: torch.from_numpy(x).bfloat16().double().numpy()
    check_rows(rounded(ref), ref, mag, error, "bf16")
    for j in places:
        others = np.arange(n) != j
        with pytest.raises(AssertionError):
            check_rows(rounded(rows_in_64(q, kd, vd, words, kc[others], vc[others], scale)[0]), ref, mag, error, "bf16")
        shifted = vc.copy()
        shifted[j] = vc[j - 1]
        with pytest.raises(AssertionError):
            check_rows(rounded(rows_in_64(q, kd, vd, words, kc, shifted, scale)[0]), ref, mag, error, "bf16")


# ---- pins of the oracle ----
def test_a_chain_is_causal_attention_and_a_step_a_decoding_step():
    rng = np.random.default_rng(1)
    q, kd, vd = rng.normal(size=(4, 6, 8)), rng.normal(size=(2, 6, 8)), rng.normal(size=(2, 6, 8))
    kc, vc = rng.normal(size=(2, 9, 8)), rng.normal(size=(2, 9, 8))
    out, lse, _ = orc.tree_attn(q, kd, vd, [(1 << t + 1) - 1 for t in range(6)], kc, vc)
    ref, ref_lse, _ = orc.chunk_attn(q, np.concatenate([kc, kd], 1), np.concatenate([vc, vd], 1), 9)
    np.testing.assert_allclose(out, ref, atol=1e-13)
    np.testing.assert_allclose(lse, ref_lse, atol=1e-13)
    out, sums, evicted, k, v, acc = orc.decode_evict_step(q[:, 0], kd[:, 0], vd[:, 0], kc, vc, np.ones((2, 9)), 9, 20, 3)
    ref, k_all, v_all = orc.decode_step(q[:, 0], kd[:, 0], vd[:, 0], kc, vc)
    np.testing.assert_allclose(out, ref, atol=1e-13)
    assert evicted is None and np.array_equal(k, k_all) and np.array_equal(v, v_all)
    np.testing.assert_allclose(sums.sum(1), 9 + 2, atol=1e-12)  # a head's weights add up to 1, two heads a group


def test_a_window_keeps_the_first_and_the_newest_states():
    """No rows between the first and the recent ones: whatever the weights, what is left are the first two and the last three."""
    rng, k, acc = np.random.default_rng(2), np.zeros((1, 0, 4)), np.zeros((1, 0))
    states = rng.normal(size=(40, 1, 4))
    for t in range(40):
        _, _, gone, k, _, acc = orc.decode_evict_step(rng.normal(size=(2, 4)), states[t], states[t], k, k, acc, t, 5, 3, start_size=2)
        assert gone is None if t < 5 else gone[0] == 2 + (t - 5) % 3
    left = sorted(int(np.where((states[:, 0] == row).all(1))[0][0]) for row in k[0])
    assert left == [0, 1, 37, 38, 39]


def test_a_sum_that_is_no_number_is_never_the_smallest():
    """Of the oldest recent state (row 3) neither; where no other is smaller it goes."""
    nan, inf, k = float("nan"), float("inf"), np.zeros((1, 5, 2))
    for acc, row in (([9.0, 2.0, 3.0, nan, 1.0], 1), ([nan, 7.0, nan, nan, 1.0], 1), ([nan, nan, nan, nan, 0.0], 3), ([nan, nan, nan, 5.0, 0.0], 3),
                     ([nan, 4.0, 4.0, 5.0, 0.0], 1), ([inf, inf, nan, nan, 0.0], 0), ([9.0, 9.0, 9.0, 9.0, 0.0], 0)):
        for mode in (orc.SELECT_PER_KV_HEAD, orc.SELECT_PER_LAYER):
            _, _, gone, _, _, _ = orc.decode_evict_step(np.zeros((1, 2)), np.zeros((1, 2)), np.zeros((1, 2)), k, k, np.array([acc]), 5, 5, 2,
                                                        select_mode=mode)
            assert gone[0] == row, (acc, gone)


def test_the_least_attended_state_goes_and_the_oldest_recent_one_takes_its_row():
    k = np.array([[[4.0], [0.0], [-9.0], [1.0], [2.0]]])  # 4 of 5 rows may go with recent = 2: 0 .. 2 and the older recent one
    _, sums, gone, after, _, acc = orc.decode_evict_step([[1.0]], [[0.5]], [[0.5]], k, k, np.zeros((1, 5)), 5, 5, 2, scale=1.0)
    w = np.exp([4.0, 0.0, -9.0, 1.0, 2.0, 0.5])
    np.testing.assert_allclose(sums[0], w / w.sum(), rtol=1e-14)
    assert gone[0] == 2 and after[0, :, 0].tolist() == [4.0, 0.0, 1.0, 0.5, 2.0]
    np.testing.assert_allclose(acc[0], (w / w.sum())[[0, 1, 3, 5, 4]], rtol=1e-14)
    # in the next step row 4 is the oldest recent one
    _, _, gone, after, _, _ = orc.decode_evict_step([[1.0]], [[0.1]], [[0.1]], after, after, np.array([[9.0, 9.0, 9.0, 0.0, 5.0]]), 6, 5, 2)
    assert gone[0] == 4 and after[0, :, 0].tolist() == [4.0, 0.0, 1.0, 0.5, 0.1]
