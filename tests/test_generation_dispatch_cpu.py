"""Generation over a retained cache without a GPU: which kernels a call launches, that every launch fits a grid, and what a failed launch
leaves.  The calls run in a child process behind the stand-in for the HIP runtime; this file is the child's program too."""

import ctypes as C
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if __name__ == "__main__":
    sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]

from test_dispatch_cpu import Fake, Recorder  # noqa: E402


# ---- in the child ----
def fakes(api):
    import torch

    class Tensor(Fake):
        dtype = torch.bfloat16

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

    def make(kind, *shape, at=1 << 20):
        t = Tensor(*shape, at=at)
        t.dtype = kind
        return t

    api.binding._stream_on = lambda device, stream: 0
    return make, torch


def tree(api, launches, cases):
    make, torch = fakes(api)
    out = []
    for B, L, Hq, Hkv, d, T, n, f32, fail in cases:
        kind = torch.float32 if f32 else torch.bfloat16
        cfg = api.Config(batch=B, layers=L, q_heads=Hq, kv_heads=Hkv, head_dim=d, chunk_len=1, budget=1, instr_len=1,
                         dtype=api.F32 if f32 else api.BF16, cache_capacity=max(n, 1))
        q, draft, cache = (make(kind, B, L, h, s, d, at=(i + 1) << 24) for i, (h, s) in enumerate(((Hq, T), (Hkv, T), (Hkv, max(n, 1)))))
        ws = make(torch.uint8, api.generation_workspace_bytes(cfg, T), at=1 << 30)
        ws.nbytes = ws.numel()
        words, status = make(torch.int64, T), [0]

        def call():
            try:
                api.citrus_tree_attn(cfg, q, draft, draft, words, cache, cache, n, out=make(kind, B, L, Hq, T, d, at=1 << 40), workspace=ws)
            except api.CitrusError as e:
                status[0] = e.status

        got = [x for x in launches(call, fail) if x[0] != "lds"]
        out.append([status[0], got])
    return out


def evict(api, launches, cases):
    make, torch = fakes(api)
    out = []
    for B, L, Hq, Hkv, d, n, f32, per_layer, fail in cases:
        kind = torch.float32 if f32 else torch.bfloat16
        cfg = api.Config(batch=B, layers=L, q_heads=Hq, kv_heads=Hkv, head_dim=d, chunk_len=1, budget=n, instr_len=1,
                         dtype=api.F32 if f32 else api.BF16, cache_capacity=n, select_mode=per_layer)
        q, state, cache = (make(kind, B, L, h, s, d, at=(i + 1) << 24) for i, (h, s) in enumerate(((Hq, 1), (Hkv, 1), (Hkv, n))))
        ws = make(torch.uint8, api.generation_workspace_bytes(cfg, 1), at=1 << 30)
        ws.nbytes = ws.numel()
        acc, status = make(torch.float32, B, L, Hkv, n), [0]

        def call():
            try:
                api.citrus_decode_evict_step(cfg, q, state, state, cache, cache, acc, n + 3, 1, out=make(kind, B, L, Hq, 1, d, at=1 << 40), workspace=ws)
            except api.CitrusError as e:
                status[0] = e.status

        got = [x for x in launches(call, fail) if x[0] != "lds"]
        out.append([status[0], got])
    return out


def joins(api, launches, cases):
    """Calls whose new states lie beside the caches' rows or in their own place: the launches of each."""
    make, torch = fakes(api)
    dtype, out = torch.float32, []
    L, H, cap, T, d, ROW = 3, 4, 64, 8, 64, 256

    def view(at, **kw):  # [2, L, H, rows, d] with the strides of a cache, in bytes
        st = {**dict(b=L * H * 80 * ROW, l=H * 80 * ROW, h=80 * ROW, s=ROW), **kw}
        return api.binding.CTensor(at, *(st[x] // 4 for x in "blhs"))

    cfg = api.Config(batch=2, layers=L, q_heads=H, kv_heads=H, head_dim=d, chunk_len=1, budget=cap, instr_len=1, dtype=api.F32, cache_capacity=cap)
    lib, cc, kc, vc, apart = api.binding._lib(), cfg.c(), 1 << 24, 2 << 24, 5 << 24
    for kind, k_at, v_at, tokens, interleaved in cases:
        kw = dict(s=3 * ROW, h=80 * 3 * ROW, l=H * 80 * 3 * ROW, b=L * H * 80 * 3 * ROW) if interleaved else {}
        kc_t, vc_t = view(kc, **kw), view(kc + 2 * ROW if interleaved else vc, **kw)
        k, v = (view(apart + i * (1 << 24) if x is None else x, **kw) for i, x in enumerate((k_at, v_at)))
        status = [0]

        def call():
            if kind == "commit":
                status[0] = lib.citrus_tree_commit(C.byref(cc), k, v, T, 1 << 30, 4, 1 << 31, kc_t, vc_t, 16, None, None, None)
            else:
                status[0] = lib.citrus_decode_evict_step(C.byref(cc), view(8 << 24), k, v, kc_t, vc_t, 1 << 30, tokens, 1, view(9 << 24), None,
                                                         1 << 32, 1 << 40, None)

        got = [x for x in launches(call) if x[0] != "lds"]
        out.append([status[0], len(got)])
    return out


# ---- in the test ----
def in_child(body, tmp_path, **kw):
    shim = str(tmp_path / "fake_hip.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-o", shim, os.path.join(ROOT, "tests", "fake_hip.cpp")])
    done = subprocess.run([sys.executable, os.path.abspath(__file__), shim, body.__name__, json.dumps(kw)], cwd=ROOT, stdout=subprocess.PIPE,
                          stderr=subprocess.PIPE, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-3000:]
    return json.loads(done.stdout.splitlines()[-1])


def names(launches):
    return [x[0].split("<")[0] for x in launches]


def test_forms_of_the_attention(tmp_path):
    """By rows of a KV head: private tiles up to 32, waves that share stages beyond, row groups from 257 on; ranges of keys where few units
    have many; another launch only to join these."""
    wants = {(1, 32, 32, 8, 128, 8, 900): ["few_rows_kernel<128, 4, 4"], (1, 32, 32, 8, 128, 9, 900): ["few_rows_kernel<128, 4, 2"],
             (1, 32, 32, 8, 128, 17, 900): ["few_rows_kernel<128, 8, 2"], (1, 32, 32, 8, 128, 33, 900): ["few_rows_kernel<128, 8, 1"],
             (1, 32, 64, 8, 128, 64, 900): ["few_rows_kernel<128, 8, 1"], (1, 1, 32, 8, 64, 1, 9000): ["few_rows_kernel<64, 4, 4", "join_ranges_kernel"],
             (1, 1, 8, 8, 64, 1, 20): ["few_rows_kernel<64, 4, 4"]}
    got = in_child(tree, tmp_path, cases=[[*c, False, -1] for c in wants])
    for (case, want), (status, launches) in zip(wants.items(), got):
        assert status == 0 and len(launches) == len(want), (case, launches)
        for launch, name in zip(launches, want):
            assert launch[0].startswith(name), (case, launches)
    assert [x[1][0][1] for x in got[:5]] == [[1, 8, 32]] * 4 + [[2, 8, 32]]


def test_a_unit_to_a_wave_where_many_have_few_keys(tmp_path):
    wants = {(1, 64, 32, 8, 128, 1, 130): "128, 1, 1", (1, 32, 32, 8, 128, 1, 130): "128, 4, 4", (1, 160, 32, 8, 128, 1, 900): "128, 4, 4",
             (1, 96, 32, 8, 64, 4, 130): "64, 1, 1", (1, 64, 32, 8, 64, 4, 130): "64, 4, 4", (1, 160, 32, 8, 64, 4, 1200): "64, 4, 4"}
    got = in_child(tree, tmp_path, cases=[[*c, False, -1] for c in wants])
    for (case, want), (status, launches) in zip(wants.items(), got):
        assert status == 0 and len(launches) == 1 and launches[0][0].startswith(f"few_rows_kernel<{want},"), (case, launches)
    wants = {(1, 160, 16, 8, 128, 130, False, 0): ["128, 1, 1"], (1, 32, 16, 8, 128, 130, False, 0): ["128, 4, 4"],
             (1, 160, 16, 8, 128, 1000, False, 0): ["128, 4, 4"], (1, 160, 16, 8, 64, 130, False, 0): ["64, 1, 1"],
             (1, 160, 16, 8, 128, 130, False, 1): ["128, 1, 1", "evict_layer_kernel"]}
    got = in_child(evict, tmp_path, cases=[[*c, -1] for c in wants])
    for (case, want), (status, launches) in zip(wants.items(), got):
        assert status == 0 and len(launches) == len(want) and launches[0][0].startswith(f"few_rows_kernel<{want[0]},"), (case, launches)
        assert names(launches)[1:] == want[1:]


def test_four_waves_of_a_block_each_where_units_are_many(tmp_path):
    wants = {(1, 64, 32, 8, 128, 24, 130): ("128, 4, 1", 1), (1, 64, 64, 8, 128, 32, 130): ("128, 4, 1", 2), (1, 64, 64, 8, 128, 32, 900): ("128, 8, 1", 1),
             (1, 64, 64, 8, 128, 20, 130): ("128, 8, 1", 1), (1, 16, 32, 8, 128, 24, 130): ("128, 8, 2", 1), (1, 64, 32, 8, 64, 24, 130): ("64, 4, 1", 1),
             (1, 16, 64, 8, 64, 32, 70): ("64, 4, 1", 2), (1, 16, 32, 8, 64, 24, 130): ("64, 8, 2", 1)}
    got = in_child(tree, tmp_path, cases=[[*c, False, -1] for c in wants])
    for (case, (want, groups)), (status, launches) in zip(wants.items(), got):
        assert status == 0 and len(launches) == 1 and launches[0][0].startswith(f"few_rows_kernel<{want},"), (case, launches)
        assert launches[0][1][0] == groups


def test_largest_configurations_fit_a_grid(tmp_path):
    """The most heads, the widest groups, and the longest caches that a configuration may have."""
    cases = [[1, 65535, 64, 64, 64, 1, 5, f32, -1] for f32 in (False, True)]
    cases += [[1, 8, 65535, 1, 64, 64, 70, f32, -1] for f32 in (False, True)] + [[1, 1, 65535, 65535, 128, 64, 3, f32, -1] for f32 in (False, True)]
    cases += [[1, 1, 8, 1, 128, 64, (1 << 31) // 512 - 1, f32, -1] for f32 in (False, True)]
    for case, (status, launches) in zip(cases, in_child(tree, tmp_path, cases=cases)):
        assert status == 0 and launches, (case, status)
    cases = [[1, 65535, 64, 64, 64, 5, f32, p, -1] for f32 in (False, True) for p in (0, 1)] + [[1, 1, 1024, 1, 64, 70, f32, 0, -1] for f32 in (False, True)]
    cases += [[1, 1, 8, 1, 128, (1 << 31) // 512 - 1, f32, p, -1] for f32 in (False, True) for p in (0, 1)]
    for case, (status, launches) in zip(cases, in_child(evict, tmp_path, cases=cases)):
        assert status == 0 and launches, (case, status)


def test_forms_of_the_eviction(tmp_path):
    """Within the launch that attends where the units fill the chip once; behind it a workgroup per unit, or per layer of few heads; ranges
    of keys for long caches and for layers of many heads."""
    wants = {(1, 32, 32, 8, 128, 1024, False, 0): ["few_rows_kernel"], (1, 1, 32, 8, 128, 2000, False, 0): ["few_rows_kernel", "evict_unit_kernel"],
             (1, 1, 33, 1, 128, 700, False, 0): ["few_rows_kernel", "evict_unit_kernel"],
             (1, 1, 8, 8, 128, 9000, False, 0): ["few_rows_kernel", "grow_sums_kernel", "make_room_kernel"],
             (1, 4, 16, 4, 128, 2000, False, 1): ["few_rows_kernel", "evict_layer_kernel"],
             (1, 4, 32, 8, 128, 2000, False, 1): ["few_rows_kernel", "grow_sums_kernel", "make_room_kernel"],
             (2, 128, 8, 2, 64, 200, True, 0): ["few_rows_f32_kernel"], (1, 4, 16, 4, 64, 500, True, 1): ["few_rows_f32_kernel", "evict_layer_kernel"]}
    got = in_child(evict, tmp_path, cases=[[*c, -1] for c in wants])
    for (case, want), (status, launches) in zip(wants.items(), got):
        assert status == 0 and names(launches) == want, (case, launches)


def ranges_of(case, launch):
    """Key ranges of an attention's launch: its workgroups in x but for the row groups."""
    _, _, Hq, Hkv, _, T, *_ = case
    waves, kh = (4, 4) if "f32" in launch[0] else (int(x) for x in launch[0].split("<")[1].split(",")[1:3])
    rows = 32 * waves // kh
    groups = (Hq // Hkv * T + rows - 1) // rows
    assert launch[1][0] % groups == 0
    return launch[1][0] // groups


def test_ranges_of_the_long_caches_that_are_checked(tmp_path):
    """The GPU's tests of long streams within a workgroup, of many ranges, and of ragged documents over several, are what they say."""
    from test_gpu_generation_long import LENS, LONG, RAGGED
    cases = [[*c[:7], c[7] == "f32", -1] for c in LONG]
    cases += [[len(LENS), 1, Hq, 1, d, T, max(LENS), dtype == "f32", -1] for Hq, d, T, dtype in RAGGED]
    wants = [c[8] for c in LONG] + [2] * len(RAGGED)
    got, forms = in_child(tree, tmp_path, cases=cases), {}
    for case, want, (status, launches) in zip(cases, wants, got):
        have = ranges_of(case, launches[0])
        assert status == 0 and (have == 1 if want == 1 else have >= want), (case, have, launches)
        forms.setdefault(launches[0][0].split("<")[0] + launches[0][0].split("<")[1][:9], set()).add(want)
    # one range and several of every form but the single wave's, which has one range of a few keys, and these
    both, one = {1, 2}, {1}
    assert {k: v & both for k, v in forms.items() if "f32" not in k} == {
        "few_rows_kernel128, 4, 4": both, "few_rows_kernel128, 4, 2": both, "few_rows_kernel128, 8, 2": both, "few_rows_kernel128, 8, 1": both,
        "few_rows_kernel128, 4, 1": one, "few_rows_kernel64, 4, 4,": both, "few_rows_kernel64, 4, 2,": both, "few_rows_kernel64, 8, 2,": both,
        "few_rows_kernel64, 4, 1,": both}


def test_kernels_of_the_bounded_steps_that_are_counted(tmp_path):
    from test_gpu_generation_long import BOUNDED
    wants = {"in_the_launch": [], "in_the_launch_64": [], "many_units": [], "a_unit": ["evict_unit_kernel"], "layer": ["evict_layer_kernel"]}
    cases = [[*(c[x] for x in ("B", "L", "Hq", "Hkv", "d", "budget")), f32, int(c.get("per_layer", 0)), -1] for f32 in (False, True)
             for c in BOUNDED.values()]
    for name, (status, launches) in zip([*BOUNDED] * 2, in_child(evict, tmp_path, cases=cases)):
        assert status == 0 and names(launches)[1:] == wants.get(name, ["grow_sums_kernel", "make_room_kernel"]), (name, launches)


def test_states_beside_the_cached_rows_are_taken(tmp_path):
    """Memory that K, V and drafts share row by row, rows behind the capacity, and a token in the row that becomes its own."""
    ROW, kc, vc = 256, 1 << 24, 2 << 24
    cases = [["commit", None, None, 0, False], ["commit", kc + 64 * ROW, vc + 64 * ROW, 0, False], ["commit", kc - 8 * ROW, vc + 64 * ROW, 0, False],
             ["commit", kc + ROW, None, 0, True], ["commit", None, kc + 3 * ROW * 70 + 2 * ROW, 0, True], ["evict", None, None, 70, False], ["evict", kc + 64 * ROW, vc + 64 * ROW, 70, False],
             ["evict", kc + 20 * ROW, vc + 20 * ROW, 20, False], ["evict", kc, vc, 0, False], ["evict", kc + ROW, None, 70, True]]
    refused = [["commit", kc + 56 * ROW, None, 0, False], ["commit", kc + 3 * ROW * 20, None, 0, True],
               ["evict", kc + 63 * ROW, None, 70, False], ["evict", vc + 20 * ROW, kc + 20 * ROW, 20, False]]
    got = in_child(joins, tmp_path, cases=cases + refused)
    assert all(status == 0 and launches for status, launches in got[:len(cases)]), got
    assert all(x == [2, 0] for x in got[len(cases):]), got


def test_failed_launches_are_reported(tmp_path):
    from paper_2406_12018_amd import binding as B
    got = in_child(tree, tmp_path, cases=[[1, 1, 32, 8, 128, 8, 4000, False, at] for at in (0, 1, 2)])
    assert [(x[0], len(x[1])) for x in got] == [(B.ERR_DEVICE, 0), (B.ERR_DEVICE, 1), (0, 2)]
    got = in_child(evict, tmp_path, cases=[[1, 1, 8, 8, 128, 9000, False, 0, at] for at in (0, 1, 2, 3)])
    assert [(x[0], len(x[1])) for x in got] == [(B.ERR_DEVICE, 0), (B.ERR_DEVICE, 1), (B.ERR_DEVICE, 2), (0, 3)]


if __name__ == "__main__":
    fake = C.CDLL(sys.argv[1], C.RTLD_GLOBAL)  # before anything that loads the real runtime
    import paper_2406_12018_amd as api_

    print(json.dumps(globals()[sys.argv[2]](api_, Recorder(fake, api_.binding._lib()), **json.loads(sys.argv[3]))))
