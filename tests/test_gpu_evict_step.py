"""Decoding in bounded memory, with eviction by accumulated attention weight, against the 64-bit oracle, step by step on the states
that the GPU left; ties, sums that are no numbers, windows, graphs, and generation as a whole.  Needs an MI355X."""

import numpy as np
import pytest
import torch

import paper_2406_12018_amd as api
from generation import DEV, Rand, as_tensor, check_rows, config, f64, same_bits, tree_words, weight_error
from oracle import citrus_oracle as orc

pytestmark = pytest.mark.gpu


class Run:
    """A bounded cache and its sums; step() feeds it one token and checks what comes back."""

    def __init__(self, seed, B, L, Hq, Hkv, d, budget, recent, start=0, per_layer=False, dtype="bf16", cap=None, tokens=0, **kw):
        self.cfg = config(B, L, Hq, Hkv, d, cap or budget, dtype, budget=budget, start_size=start,
                          select_mode=api.SELECT_PER_LAYER if per_layer else api.SELECT_PER_KV_HEAD, **kw)
        self.make, self.dtype, self.recent, self.tokens = Rand(seed, dtype), dtype, recent, tokens
        rows = self.cfg.cache_capacity
        self.k, self.v = self.make(B, L, Hkv, rows, d, scale=0.6), self.make(B, L, Hkv, rows, d)
        g = torch.Generator().manual_seed(seed + 1)
        self.acc = torch.exp(torch.randn((B, L, Hkv, rows), generator=g)).to(DEV) * (0.3 * Hq / Hkv)
        self.ws = api.alloc_generation_workspace(self.cfg)

    def token(self):
        c = self.cfg
        return (self.make(c.batch, c.layers, c.q_heads, 1, c.head_dim), self.make(c.batch, c.layers, c.kv_heads, 1, c.head_dim, scale=0.6),
                self.make(c.batch, c.layers, c.kv_heads, 1, c.head_dim))

    def call(self, q, k, v, **kw):
        self.evicted = torch.full((self.cfg.batch, self.cfg.layers, self.cfg.sel_heads), -9, dtype=torch.int32, device=DEV)
        out = api.citrus_decode_evict_step(self.cfg, q, k, v, self.k, self.v, self.acc, self.tokens, self.recent,
                                           **{**dict(evicted=self.evicted, workspace=self.ws), **kw})
        self.tokens += 1
        return out

    def step(self, token=None):
        c, tokens = self.cfg, self.tokens
        n = min(tokens, c.budget)
        q, kn, vn = token or self.token()
        k0, v0, acc0 = self.k.clone(), self.v.clone(), self.acc.clone()
        out = self.call(q, kn, vn)
        torch.cuda.synchronize()
        scale = c.softmax_scale or c.head_dim ** -0.5
        gone = self.evicted.cpu().numpy()
        layers = range(c.layers) if c.batch * c.layers <= 6 else sorted({0, c.layers // 2, c.layers - 1})  # the oracle is slow
        pick = torch.tensor(list(layers), device=DEV)
        Q, KN, VN, K0, V0, A0, O, A, K1, V1 = (f64(t[:, pick]) for t in (q, kn, vn, k0, v0, acc0, out, self.acc, self.k, self.v))
        gone = gone[:, list(layers)]
        for b in range(c.batch):
            for l in range(len(layers)):
                chosen = np.broadcast_to(gone[b, l], (c.kv_heads,))
                forced = chosen if tokens >= c.budget else None
                ref, sums, best, k, v, acc = orc.decode_evict_step(Q[b, l, :, 0], KN[b, l, :, 0], VN[b, l, :, 0], K0[b, l, :, :n], V0[b, l, :, :n],
                                                                   A0[b, l, :, :n], tokens, c.budget, self.recent, c.start_size, c.select_mode,
                                                                   scale, forced)
                error = weight_error(Q[b, l], np.concatenate([K0[b, l, :, :n], KN[b, l]], axis=1), n + 1, scale)
                group = c.q_heads // c.kv_heads
                absolute = np.concatenate([np.abs(V0[b, l, :, :n]), np.abs(VN[b, l])], axis=1)
                keys = np.concatenate([K0[b, l, :, :n], KN[b, l]], axis=1)
                mag = np.stack([orc.softmax_rows((keys[h // group] @ Q[b, l, h, 0] * scale)[None])[0][0] @ absolute[h // group]
                                for h in range(c.q_heads)])
                check_rows(O[b, l, :, 0], ref, mag, error, self.dtype, f"step {tokens}, document {b}, layer {l}")
                rows = acc.shape[1]
                weight = sums[:, :n + 1] - np.concatenate([A0[b, l, :, :n], np.zeros((c.kv_heads, 1))], axis=1)
                slack = weight.max() * (error + 2.0 ** -22) + 2.0 ** -23 * np.abs(sums).max()  # group sums and one addition to a sum
                np.testing.assert_allclose(A[b, l, :, :rows], acc, rtol=0, atol=slack)
                assert np.array_equal(A[b, l, :, rows:], A0[b, l, :, rows:])
                if tokens >= c.budget:
                    oldest = c.budget - self.recent + (tokens - c.budget) % self.recent
                    free = list(range(c.start_size, c.budget - self.recent)) + [oldest]
                    rank = np.broadcast_to(sums.sum(0), sums.shape) if c.select_mode == api.SELECT_PER_LAYER else sums
                    for g in range(c.kv_heads):
                        assert chosen[g] in free
                        assert rank[g, chosen[g]] <= rank[g, free].min() + 2 * slack * c.kv_heads
                else:
                    assert (chosen == -1).all()
                assert np.array_equal(K1[b, l, :, :rows], k) and np.array_equal(V1[b, l, :, :rows], v)
        assert torch.equal(self.k[:, :, :, max(n, min(n + 1, c.budget)):], k0[:, :, :, max(n, min(n + 1, c.budget)):])
        return out


CASES = {  # seed, B, L, Hq, Hkv, d, budget, recent, ...
    "one_row": dict(B=1, L=1, Hq=2, Hkv=1, d=64, budget=1, recent=1),
    "two_rows": dict(B=2, L=1, Hq=2, Hkv=2, d=128, budget=2, recent=1),
    "window": dict(B=1, L=2, Hq=4, Hkv=2, d=64, budget=6, recent=4, start=2),
    "small": dict(B=1, L=2, Hq=6, Hkv=2, d=128, budget=9, recent=3, start=2),
    "tile_edges": dict(B=1, L=1, Hq=8, Hkv=2, d=128, budget=33, recent=8, start=4),
    "per_layer": dict(B=2, L=2, Hq=12, Hkv=3, d=64, budget=40, recent=7, start=1, per_layer=True),
    "spare_capacity": dict(B=1, L=3, Hq=8, Hkv=8, d=64, budget=30, recent=5, cap=77),
    "scale": dict(B=1, L=1, Hq=8, Hkv=1, d=128, budget=31, recent=31, softmax_scale=0.2),
    "many_heads": dict(B=1, L=1, Hq=40, Hkv=1, d=128, budget=36, recent=2),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(CASES))
def test_from_an_empty_cache_until_it_has_turned_over(name, dtype):
    run = Run(40, **CASES[name], dtype=dtype)
    for _ in range(2 * run.cfg.budget + 5 if run.cfg.budget < 20 else run.cfg.budget + 12):
        run.step()


LARGE = {
    "one_layer": dict(B=1, L=1, Hq=32, Hkv=8, d=128, budget=768, recent=64, start=4),
    "many_units": dict(B=2, L=70, Hq=8, Hkv=4, d=64, budget=300, recent=20, start=4),
    "long": dict(B=1, L=1, Hq=8, Hkv=2, d=128, budget=9001, recent=500, start=4),
    "long_per_layer": dict(B=1, L=2, Hq=8, Hkv=4, d=64, budget=5000, recent=1, per_layer=True),
    "layers_of_two_waves": dict(B=1, L=33, Hq=32, Hkv=8, d=128, budget=1025, recent=100),
    "group_of_8": dict(B=2, L=40, Hq=64, Hkv=8, d=128, budget=2047, recent=300),
    "group_of_33": dict(B=1, L=2, Hq=33, Hkv=1, d=64, budget=700, recent=3),
    "one_round": dict(B=1, L=32, Hq=32, Hkv=8, d=128, budget=1024, recent=128, start=4),          # within the launch, logits in LDS
    "one_round_global": dict(B=1, L=32, Hq=64, Hkv=8, d=128, budget=2000, recent=100, start=1),   # ... in the workspace
    "one_round_64": dict(B=2, L=32, Hq=32, Hkv=8, d=64, budget=900, recent=64),
    "one_round_64_global": dict(B=2, L=32, Hq=40, Hkv=8, d=64, budget=1500, recent=7),
    "unit_kernel_at_its_end": dict(B=1, L=1, Hq=5, Hkv=1, d=64, budget=8191, recent=10),
    "ranges_from_here": dict(B=1, L=1, Hq=5, Hkv=1, d=64, budget=8192, recent=10, start=4),
    "layer_kernel_at_its_end": dict(B=1, L=2, Hq=16, Hkv=4, d=64, budget=2047, recent=90, per_layer=True),
    "layer_ranges_from_here": dict(B=1, L=2, Hq=16, Hkv=4, d=64, budget=2048, recent=90, per_layer=True, start=4),
    "layer_of_many_heads": dict(B=2, L=2, Hq=24, Hkv=6, d=128, budget=333, recent=20, per_layer=True),
    "layer_of_one_wide_group": dict(B=1, L=1, Hq=37, Hkv=1, d=64, budget=130, recent=20, per_layer=True),
    "chip_full_wide_group": dict(B=1, L=260, Hq=16, Hkv=1, d=64, budget=1600, recent=3),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(LARGE))
def test_full_caches_of_real_sizes(name, dtype):
    run = Run(50, **LARGE[name], dtype=dtype)
    run.tokens = run.cfg.budget + 17
    for _ in range(2):
        run.step()


MANY_SHORT = {  # units that fill the chip more than once, with few states each
    "one_state": dict(B=2, L=70, Hq=4, Hkv=2, d=128, budget=1, recent=1),
    "tile_end": dict(B=1, L=140, Hq=4, Hkv=2, d=128, budget=63, recent=9, start=1),
    "group_of_8": dict(B=2, L=66, Hq=16, Hkv=2, d=128, budget=130, recent=20, start=4),
    "group_of_32": dict(B=1, L=300, Hq=32, Hkv=1, d=128, budget=65, recent=64),
    "several_rounds": dict(B=2, L=700, Hq=2, Hkv=1, d=128, budget=257, recent=30, start=4),
    "head_dim_64": dict(B=3, L=100, Hq=6, Hkv=2, d=64, budget=300, recent=77),
    "head_dim_64_rounds": dict(B=1, L=2100, Hq=3, Hkv=1, d=64, budget=40, recent=5, cap=50),
    "per_layer": dict(B=1, L=300, Hq=6, Hkv=2, d=128, budget=90, recent=10, start=2, per_layer=True),
    "per_layer_64": dict(B=2, L=40, Hq=32, Hkv=8, d=64, budget=30, recent=10, per_layer=True),
}


@pytest.mark.parametrize("name", list(MANY_SHORT))
def test_many_units_of_few_states(name):
    run = Run(60, **MANY_SHORT[name])
    for tokens in (0, run.cfg.budget - 1, run.cfg.budget, run.cfg.budget + 17):
        run.tokens = tokens
        run.step()
        run.step()


def test_equal_sums_the_lowest_row_goes():
    """Zero queries: every weight is the same number; sums of 1: the first row behind the start, then the next, as each eviction moves
    the oldest recent state, with a larger sum, into it."""
    for per_layer in (False, True):
        run = Run(60, 1, 2, 4, 2, 64, 200, 10, start=3, per_layer=per_layer, tokens=200)
        run.acc.fill_(1.0)
        run.acc[..., 190:] = 2.0
        q, k, v = run.token()
        for i in range(4):
            run.call(torch.zeros_like(q), k, v)
            assert (run.evicted == 3 + i).all()


def test_sums_that_are_no_numbers():
    """NaN is never the smallest; where nothing is smaller than infinity the oldest recent state goes."""
    run = Run(61, 1, 1, 2, 2, 64, 64, 8, start=2, tokens=64)
    run.acc[..., 2:56] = float("nan")
    run.call(*run.token())
    assert (run.evicted == 56).all()
    run.acc.fill_(float("nan"))
    run.call(*run.token())
    assert (run.evicted == 57).all()
    run.acc.fill_(float("inf"))
    run.acc[..., 30] = -float("inf")
    run.call(*run.token())
    assert (run.evicted == 30).all()


@pytest.mark.parametrize("name", ["window", "tile_edges", "per_layer", "many_heads"])
def test_a_token_in_the_row_that_becomes_its_own(name):
    """While the cache grows the token's state may be written there before the step; the bits are those of one that comes from elsewhere."""
    a, b = (Run(95, **CASES[name]) for _ in range(2))
    for n in range(a.cfg.budget):
        q, k, v = a.token()
        b.k[:, :, :, n:n + 1], b.v[:, :, :, n:n + 1] = k, v
        same_bits(a.call(q, k, v), b.call(q, b.k[:, :, :, n:n + 1], b.v[:, :, :, n:n + 1]))
        for x, y in ((a.k, b.k), (a.v, b.v), (a.acc, b.acc)):
            same_bits(x, y)


@pytest.mark.parametrize("name", ["one_layer", "long", "many_units", "long_per_layer"])
def test_captured_steps_replay(name):
    """Three steps in a graph; every replay, from the same start, leaves the bits that eager steps leave."""
    run = Run(70, **LARGE[name])
    run.tokens = run.cfg.budget + 5
    start = [t.clone() for t in (run.k, run.v, run.acc)]
    tokens = [run.token() for _ in range(3)]
    outs = [torch.zeros_like(t[0]) for t in tokens]

    def steps():
        run.tokens = run.cfg.budget + 5
        for t, o in zip(tokens, outs):
            api.citrus_decode_evict_step(run.cfg, *t, run.k, run.v, run.acc, run.tokens, run.recent, out=o, workspace=run.ws)
            run.tokens += 1

    def reset():
        for t, s in zip((run.k, run.v, run.acc), start):
            t.copy_(s)
        for o in outs:
            o.zero_()

    steps()
    torch.cuda.synchronize()
    want = [t.clone() for t in (run.k, run.v, run.acc, *outs)]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        steps()
    for _ in range(3):
        reset()
        run.ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((run.k, run.v, run.acc, *outs), want):
            same_bits(a, b)


def test_strided_caches_give_the_same_bits():
    a, b = (Run(80, 2, 2, 8, 2, 128, 150, 20, start=4, tokens=150) for _ in range(2))
    wide = torch.full((2, 150, 2, 2, 3 * 128), float("nan"), dtype=torch.bfloat16, device=DEV)
    for name, at in (("k", 0), ("v", 256)):
        view = wide[..., at:at + 128].permute(0, 2, 3, 1, 4)
        view.copy_(getattr(b, name))
        setattr(b, name, view)
    for _ in range(3):
        q, k, v = a.token()
        out = a.call(q, k, v)
        rows = torch.full((2, 2, 8, 1, 256), 3.0, dtype=torch.bfloat16, device=DEV)[..., :128]
        same_bits(out, b.call(q, k.transpose(1, 2).contiguous().transpose(1, 2), v, out=rows))
        for x, y in ((a.k, b.k), (a.v, b.v), (a.acc, b.acc), (a.evicted, b.evicted)):
            same_bits(x, y)
    assert torch.isnan(wide[..., 128:256]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,L,cap", [(8, 2, 1, 9000), (8, 8, 40, 300), (64, 1, 1, 5000), (2, 2, 1, 1)])
def test_nothing_is_written_outside_the_workspace(Hq, Hkv, L, cap, dtype):
    guard = 1 << 16
    run = Run(90, 1, L, Hq, Hkv, 64, cap, 1, dtype=dtype)
    size = api.generation_workspace_bytes(run.cfg, 1)
    buf = torch.full((size + 2 * guard,), 0xA5, dtype=torch.uint8, device=DEV)
    run.ws = buf[guard:guard + size]
    for tokens in sorted({0, 1, cap // 2, cap - 1, cap, cap + 3}):
        run.tokens = tokens
        run.call(*run.token())
        assert bool((buf[:guard] == 0xA5).all()) and bool((buf[guard + size:] == 0xA5).all()), tokens


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_generation_as_a_whole(dtype):
    """A document through the chunk loop with accumulated scores; two drafted trees verified and their accepted paths committed; then
    bounded steps on the cache and the sums, until rows of the drafts have gone too."""
    L, Hq, Hkv, d, budget, cap, T = 2, 8, 2, 64, 96, 104, 10
    cfg = api.Config(batch=1, layers=L, q_heads=Hq, kv_heads=Hkv, head_dim=d, chunk_len=64, budget=budget, instr_len=8,
                     dtype=api.F32 if dtype == "f32" else api.BF16, cache_capacity=cap, score_mode=api.SCORE_ACCUMULATED, start_size=4)
    make = Rand(7, dtype)
    doc, qi = [make(1, L, h, 300, d, scale=s) for h, s in ((Hq, 1.0), (Hkv, 0.6), (Hkv, 1.0))], make(1, L, Hq, 8, d)
    state = api.DocumentState.allocate(cfg)
    api.citrus_process_document(cfg, state, api.alloc_workspace(cfg), doc=api.resident_doc(cfg, *doc, qi, torch.empty_like(doc[0])))
    assert state.cache_len == budget
    kc, vc, acc = state.k_cache[state.buffer_index], state.v_cache[state.buffer_index], state.acc_score[state.buffer_index]
    acc[..., budget:] = 0  # sums of the states to come
    ws = api.alloc_generation_workspace(cfg, T)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    lens, n = dev([budget]), budget
    for i, path in enumerate(([0, 2, 5], [0, 1])):
        q, kd, vd, words = make(1, L, Hq, T, d), make(1, L, Hkv, T, d, scale=0.6), make(1, L, Hkv, T, d), tree_words(i, T)
        out = api.citrus_tree_attn(cfg, q, kd, vd, as_tensor(words), kc, vc, cap, cache_lens=lens, workspace=ws)
        ref_k, ref_v = f64(kc), f64(vc)
        for l in range(L):
            ref, _, mag = orc.tree_attn(f64(q)[0, l], f64(kd)[0, l], f64(vd)[0, l], words, ref_k[0, l, :, :n], ref_v[0, l, :, :n])
            error = weight_error(f64(q)[0, l], np.concatenate([ref_k[0, l, :, :n], f64(kd)[0, l]], axis=1), n + T, d ** -0.5)
            check_rows(f64(out)[0, l], ref, mag, error, dtype)
        lens = api.citrus_tree_commit(cfg, kd, vd, dev([path + [0] * (4 - len(path))]), dev([len(path)]), kc, vc, cap, cache_lens=lens)
        same_bits(kc[:, :, :, n:n + len(path)], kd[:, :, :, path])
        n += len(path)
        assert lens.tolist() == [n]
    # the cache now holds 101 states; it is kept at that size
    run = Run(8, 1, L, Hq, Hkv, d, n, 5, start=4, dtype=dtype, cap=cap, tokens=n)
    run.k, run.v, run.acc = kc, vc, acc
    for _ in range(12):
        run.step()
