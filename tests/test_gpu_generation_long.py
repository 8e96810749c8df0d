"""Generation over long caches, where every state counts: results that count the states, heavy states at the edges of tiles, documents of
different lengths over several ranges of keys, long streams within a workgroup, and what a bounded step adds to every sum.  Needs an MI355X."""

import numpy as np
import pytest
import torch

import paper_2406_12018_amd as api
from generation import (DEV, TORCH, Counts, as_tensor, check_counts, check_rows, config, f64, heavy_places, rows_in_64, same_bits, tree_words,
                        weight_error)
from oracle import citrus_oracle as orc
from test_gpu_evict_step import CASES, LARGE, Run
from test_gpu_tree_attn import Case

pytestmark = pytest.mark.gpu

# B, L, Hq, Hkv, d, T, n, type, workgroups' ranges of keys: one, or how many at least
LONG = [
    (1, 32, 32, 8, 128, 1, 8000, "bf16", 1), (2, 16, 32, 8, 128, 13, 8000, "bf16", 1), (1, 32, 32, 8, 128, 24, 8000, "bf16", 1),
    (1, 64, 32, 8, 128, 24, 4000, "bf16", 1), (1, 32, 32, 8, 128, 40, 8000, "bf16", 1), (1, 32, 64, 8, 128, 40, 4100, "bf16", 1),
    (2, 32, 16, 8, 64, 1, 8000, "bf16", 1), (1, 64, 32, 8, 64, 13, 6000, "bf16", 1), (1, 32, 32, 8, 64, 24, 8000, "bf16", 1),
    (1, 100, 32, 8, 64, 40, 3000, "bf16", 1), (1, 32, 16, 8, 128, 2, 3000, "f32", 1), (1, 2, 32, 8, 128, 1, 130000, "bf16", 2),
    (1, 2, 32, 8, 128, 13, 130001, "bf16", 2), (1, 1, 32, 8, 128, 40, 131007, "bf16", 2), (1, 2, 8, 8, 64, 5, 130000, "bf16", 2),
    (1, 1, 40, 8, 64, 40, 70000, "bf16", 2), (1, 1, 8, 4, 64, 3, 60000, "f32", 2), (1, 1, 1, 1, 64, 1, 40000, "bf16", 30),
    (1, 1, 1, 1, 128, 3, 40000, "bf16", 30), (1, 1, 8, 1, 128, 7, 40000, "bf16", 30), (1, 1, 8, 1, 64, 33, 40000, "bf16", 30),
    (1, 1, 1, 1, 128, 1, 8192, "bf16", 30), (1, 1, 1, 1, 64, 2, 40000, "f32", 30),
]
# documents of these lengths over several ranges, trees of other sizes: rows up to 32, 64, 128, 256 and beyond
LENS = [0, 1, 33, 129, 2999, 3000]
RAGGED = [(Hq, d, T, dtype) for d in (64, 128) for Hq, T in ((1, 1), (4, 8), (4, 16), (3, 40), (4, 64), (5, 64)) for dtype in ("bf16", "f32")
          if dtype == "bf16" or T <= 16]


def trees(T):
    return [T, 1, max(1, T - 3), max(1, T // 2), T, max(1, T - 1)]


class Big:
    """Inputs of a call, made on the GPU."""

    def __init__(self, seed, B, L, Hq, Hkv, d, T, n, dtype, lens=None, sizes=None):
        self.cfg, self.T, self.n, self.dtype = config(B, L, Hq, Hkv, d, n, dtype), T, n, dtype
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.q, self.kd, self.vd = (self.randn(h, T) for h in (Hq, Hkv, Hkv))
        self.kc, self.vc = self.randn(Hkv, n), self.randn(Hkv, n)
        for k in (self.kd, self.kc):
            k.mul_(0.5)
        self.lens = lens or [n] * B
        self.given = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.words = [tree_words(seed + b, t) + [0] * (T - t) for b, t in enumerate(sizes or [T] * B)]
        self.ws = api.alloc_generation_workspace(self.cfg, T)

    def randn(self, heads, rows):
        c = self.cfg
        return torch.randn((c.batch, c.layers, heads, rows, c.head_dim), generator=self.gen, dtype=TORCH[self.dtype], device=DEV)

    def run(self):
        lse = torch.full(self.q.shape[:4], 7.0, dtype=torch.float32, device=DEV)
        self.ws.fill_(0xFF)
        out = api.citrus_tree_attn(self.cfg, self.q, self.kd, self.vd, as_tensor(self.words), self.kc, self.vc, self.n, cache_lens=self.given,
                                   out=torch.full_like(self.q, 7.0), lse=lse, workspace=self.ws)
        torch.cuda.synchronize()
        return out, lse

    def units(self):
        c = self.cfg
        return [(b, l, g, (b * c.layers + l) * c.kv_heads + g) for b in range(c.batch) for l in range(c.layers) for g in range(c.kv_heads)]

    def count(self, only):
        c, counts = self.cfg, Counts(self.cfg.head_dim, only)
        cached, draft = (f(r, 0, self.vc.dtype, DEV) for f, r in ((counts.cached, self.n), (counts.draft, self.T)))
        for b, l, g, unit in self.units():
            self.vc[b, l, g] = torch.roll(cached, 5 * unit, 1)
            self.vd[b, l, g] = torch.roll(draft, 3 * unit, 1)
        out, lse = self.run()
        group = c.q_heads // c.kv_heads
        rows = [counts.rows(self.lens[b], unit, self.words[b]) for b, _, _, unit in self.units()]
        ref, total = (torch.stack([r[i] for r in rows]).to(DEV) for i in (0, 1))
        ref = ref.reshape(c.batch, c.layers, c.kv_heads, 1, self.T, c.head_dim).expand(-1, -1, -1, group, -1, -1)
        total = total.reshape(c.batch, c.layers, c.kv_heads, 1, self.T).expand(-1, -1, -1, group, -1)
        check_counts(out.reshape(ref.shape), lse.reshape(total.shape), ref, total, self.dtype)

    def check(self, out, lse, units):
        scale, group = self.cfg.head_dim ** -0.5, self.cfg.q_heads // self.cfg.kv_heads
        for b, l, g, _ in units:
            n, heads = self.lens[b], slice(g * group, (g + 1) * group)
            q, kd, vd = (f64(t) for t in (self.q[b, l, heads], self.kd[b, l, g], self.vd[b, l, g]))
            kc, vc = f64(self.kc[b, l, g, :n]), f64(self.vc[b, l, g, :n])
            ref, ref_lse, mag = rows_in_64(q, kd, vd, self.words[b], kc, vc, scale)
            real = np.isfinite(ref_lse)
            error = weight_error(q[real][:, None], np.concatenate([kc, kd]), n + self.T, scale)
            got, got_lse = f64(out[b, l, heads]), f64(lse[b, l, heads])
            assert (got_lse[~real] == -np.inf).all() and (got[~real] == 0).all(), "padding"
            check_rows(got[real], ref[real], mag[real], error, self.dtype, f"document {b} layer {l} head {g}")
            assert np.abs(got_lse[real] - ref_lse[real]).max(initial=0) <= error + 2.0 ** -22 * np.abs(ref_lse[real]).max(initial=1)


def name(s):
    return "x".join(map(str, s))


@pytest.mark.parametrize("shape", LONG, ids=name)
def test_every_state_counts_once(shape):
    big = Big(1, *shape[:8])
    big.q.zero_()
    for only in (None, 0, 31, 32, 63):
        big.count(only)


def heavy(big, strength=14.0):
    """A few states of every document outweigh the others, for every query."""
    d, c = big.cfg.head_dim, big.cfg.head_dim // 2 - 3
    big.q[..., c], big.kc[..., c], big.kd[..., c] = 4.0, 0.0, 0.0
    for b, n in enumerate(big.lens):
        big.kc[b, :, :, heavy_places(n, 10 + b), c] = strength * d ** 0.5 / 4.0


@pytest.mark.parametrize("shape", LONG, ids=name)
def test_heavy_states_at_edges_and_in_between(shape):
    big = Big(2, *shape[:8])
    heavy(big)
    units = big.units()
    out, lse = big.run()
    big.check(out, lse, [units[0], units[len(units) // 2 + 1]] if len(units) > 2 else units)
    for a, b in zip(big.run(), (out, lse)):
        same_bits(a, b)


@pytest.mark.parametrize("Hq,d,T,dtype", RAGGED)
def test_ragged_documents_over_several_ranges(Hq, d, T, dtype):
    big = Big(3, len(LENS), 1, Hq, 1, d, T, 3000, dtype, lens=LENS, sizes=trees(T))
    clean = big.run()
    big.check(*clean, big.units())
    heavy(big)
    clean = big.run()
    big.check(*clean, big.units())
    kept = [t.clone() for t in (big.q, big.kd, big.vd, big.kc, big.vc)]
    for b, (n, t) in enumerate(zip(LENS, trees(T))):
        for x in (big.kc, big.vc):
            x[b, :, :, n:] = float("nan")
        for x in (big.q, big.kd, big.vd):
            x[b, :, :, t:] = float("nan")
    for a, b in zip(big.run(), clean):
        same_bits(a, b)
    for t, x in zip((big.q, big.kd, big.vd, big.kc, big.vc), kept):
        t.copy_(x)
    big.q.zero_()
    for only in (None, 0, 32, 55):  # 2999 = 46 * 64 + 55
        big.count(only)


@pytest.mark.parametrize("dtype,d,T,n", [("bf16", 128, 1, 700), ("bf16", 64, 20, 90), ("f32", 128, 5, 130), ("bf16", 128, 64, 2100)])
def test_two_lengths_against_64_bits(dtype, d, T, n):
    """The shapes whose strides are varied elsewhere."""
    case = Case(21, 2, 3, 8, 2, d, T, n, dtype, lens=[n, n // 2])
    case.check(*case.run())


BOUNDED = {  # budget, ...: within the launch, a workgroup per unit, per layer, in ranges
    "in_the_launch": dict(B=1, L=32, Hq=32, Hkv=8, d=128, budget=4500, recent=100, start=4),
    "in_the_launch_64": dict(B=2, L=32, Hq=16, Hkv=8, d=64, budget=5001, recent=33),
    "many_units": dict(B=1, L=160, Hq=16, Hkv=8, d=128, budget=700, recent=33, start=1),
    "a_unit": dict(B=1, L=1, Hq=33, Hkv=1, d=128, budget=8190, recent=500, start=4),
    "ranges": dict(B=1, L=1, Hq=8, Hkv=2, d=128, budget=20001, recent=700, start=4),
    "ranges_64": dict(B=1, L=3, Hq=3, Hkv=1, d=64, budget=12288, recent=1),
    "layer": dict(B=2, L=2, Hq=12, Hkv=4, d=128, budget=2000, recent=77, start=4, per_layer=True),
    "layer_ranges": dict(B=1, L=2, Hq=32, Hkv=8, d=128, budget=9000, recent=300, start=4, per_layer=True),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(BOUNDED))
def test_a_bounded_step_counts_every_state(name, dtype):
    """A zero query: every sum grows by G / (n + 1), the result counts the states, and the smallest of sums that are all different goes."""
    c = BOUNDED[name]
    B, L, Hq, Hkv, d, n, recent, start = (c.get(x, 0) for x in ("B", "L", "Hq", "Hkv", "d", "budget", "recent", "start"))
    cfg = config(B, L, Hq, Hkv, d, n, dtype, budget=n, start_size=start,
                 select_mode=api.SELECT_PER_LAYER if c.get("per_layer") else api.SELECT_PER_KV_HEAD)
    gen = torch.Generator(device=DEV).manual_seed(5)
    zeros = lambda heads, rows: torch.zeros((B, L, heads, rows, d), dtype=TORCH[dtype], device=DEV)
    q, kc, vc, kn, vn = zeros(Hq, 1), zeros(Hkv, n), zeros(Hkv, n), zeros(Hkv, 1), zeros(Hkv, 1)
    kc.copy_(torch.randn(kc.shape, generator=gen, dtype=kc.dtype, device=DEV))
    ws, group, tokens = api.alloc_generation_workspace(cfg), Hq // Hkv, n + recent // 2
    for only in (None, 0, 31, 63):
        counts = Counts(d, only)
        cached = counts.cached(n, 0, vc.dtype, DEV)
        units = [(b, l, g, (b * L + l) * Hkv + g) for b in range(B) for l in range(L) for g in range(Hkv)]
        for b, l, g, unit in units:
            vc[b, l, g] = torch.roll(cached, 5 * unit, 1)
            vn[b, l, g] = counts.draft(1, unit, vn.dtype, DEV)
        acc = torch.stack([torch.randperm(n, generator=gen, device=DEV) for _ in units]).reshape(B, L, Hkv, n) / n
        before, v0 = acc.clone(), vc.clone()
        evicted = torch.full((B, L, cfg.sel_heads), -9, dtype=torch.int32, device=DEV)
        ws.fill_(0xFF)
        out = api.citrus_decode_evict_step(cfg, q, kn, vn, kc, vc, acc, tokens, recent, evicted=evicted, workspace=ws)
        ref = torch.stack([counts.rows(n, unit, [1])[0] for *_, unit in units]).to(DEV).reshape(B, L, Hkv, 1, 1, d)
        check_counts(out.reshape(B, L, Hkv, group, 1, d), None, ref.expand(-1, -1, -1, group, -1, -1), None, dtype)
        weight, oldest = group / (n + 1), n - recent + (tokens - n) % recent
        slots = torch.tensor([*range(start, n - recent), oldest], device=DEV)
        if cfg.select_mode == api.SELECT_PER_KV_HEAD:  # sums that differ by 1 / n at least: no rounding changes their order
            assert torch.equal(evicted.long(), slots[before[..., slots].argmin(3)])
        gone = evicted.long().expand(B, L, Hkv)[..., None]
        rank = before.double().sum(2, keepdim=True) if cfg.sel_heads == 1 else before.double()
        # each of Hkv sums is off by two roundings of numbers up to Hkv
        assert bool((rank.gather(3, gone[:, :, :rank.shape[2]]) <= rank[..., slots].amin(3, keepdim=True) + 2.0 ** -22 * Hkv * Hkv).all())
        want = before.double() + weight
        want.scatter_(3, gone, want[..., oldest:oldest + 1].clone())
        want[..., oldest] = weight
        # a weight is off by an exponential and a logarithm near log2 n, as many of them are added as there are heads in the group
        assert bool(((acc.double() - want).abs() <= 2.0 ** -24 * (want + weight * (group + 64))).all())
        v0.scatter_(3, gone[..., None].expand(-1, -1, -1, 1, d), v0[:, :, :, oldest:oldest + 1].clone())
        v0[:, :, :, oldest] = vn[:, :, :, 0]
        same_bits(vc, v0)


@pytest.mark.parametrize("name", ["window", "many_units", "one_layer", "long", "layer_kernel_at_its_end", "long_per_layer"])
def test_sums_that_are_no_numbers_in_every_kernel(name):
    """NaN, of the oldest recent state too, and infinity: the oracle's choice.  All sums of a row are the same number plus the same weight."""
    nan, inf = float("nan"), float("inf")
    run = Run(62, **{**CASES, **LARGE}[name])
    c, n = run.cfg, run.cfg.budget
    q, k, v = run.token()
    last = n - run.recent - 1  # the last row that may go in front of the recent ones
    for others, special, oldest_sum in ((5.0, {last: 4.0}, nan), (5.0, {c.start_size: nan, last: 5.0}, 6.0), (nan, {last: 7.0}, nan), (nan, {}, 3.0),
                                        (nan, {}, nan), (inf, {last: nan}, nan), (5.0, {}, 4.0), (5.0, {last: -inf}, nan)):
        run.tokens = n + 1
        oldest = n - run.recent + 1 % run.recent
        run.acc.fill_(others)
        for row, value in special.items():
            if row >= c.start_size:
                run.acc[..., row] = value
        run.acc[..., oldest] = oldest_sum
        sums = f64(run.acc[0, 0, :, :n])
        none = np.zeros((c.kv_heads, n, 1))  # keys of any values: the queries are zero
        *_, want, _, _, _ = orc.decode_evict_step(np.zeros((c.q_heads, 1)), none[:, 0], none[:, 0], none, none, sums, run.tokens, n, run.recent,
                                                  c.start_size, c.select_mode)
        run.call(torch.zeros_like(q), k, v)
        want = torch.from_numpy(want[:c.sel_heads]).to(DEV)
        assert bool((run.evicted == want).all()), (others, special, oldest_sum, want.tolist(), run.evicted[0, 0].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,d,budget,per_layer", [(1024, 64, 70, False), (1000, 128, 300, True)])
def test_the_widest_groups(Hq, d, budget, per_layer, dtype):
    """Up to 1024 query heads to a KV head: 32 blocks of rows, whose logits one workgroup adds up."""
    run = Run(63, 1, 1, Hq, 1, d, budget, 9, start=2, per_layer=per_layer, dtype=dtype)
    for run.tokens in (0, budget - 1, budget + 4):
        run.step()
    tree = Case(64, 1, 1, Hq, 1, d, 2, budget, dtype)
    tree.check(*tree.run())
