"""Generation over a retained cache, as cases that can be measured and compared: attention of a tree of drafted tokens,
the commit of its accepted path, and decoding steps that evict by accumulated attention weight.

A case is a dict of plain values.  `kind` says what one pass is:

  tree     citrus_tree_attn: every node of a drafted tree attends over its document's cache and its own ancestors.
           `ragged`: documents have lengths of their own, and smaller trees are padded.
  commit   citrus_tree_commit: the accepted path's states move behind the cache, another number for every document.
  bounded  citrus_decode_evict_step: a token attends over the full cache and itself, the weights join the states' sums, and
           the state with the smallest sum makes room.

With `own` false the operators run in elementary torch operations in 32 bits; `exact` is written apart from that, in 64 bits.

Inputs follow what attention meets: q, k, v are normal, every key carries an importance of its own that all queries share
(one channel with an offset in q: attention's heavy hitters, log-normal weights), the first four states are attention sinks
and one state in fifty is heavier still.  Sums of weights are log-normal.  All from the seed.
"""

from __future__ import annotations

import math

import torch

own = False


def _tree(name=None, *, dtype="bf16", batch=1, layers=1, q_heads=32, kv_heads=8, head_dim=128, states=768, nodes=8, ragged=False):
    return _named(name, kind="tree", dtype=dtype, batch=batch, layers=layers, q_heads=q_heads, kv_heads=kv_heads,
                  head_dim=head_dim, states=states, nodes=nodes, ragged=ragged)


def _commit(name=None, *, dtype="bf16", batch=1, layers=1, kv_heads=8, head_dim=128, states=768, nodes=8, path=4):
    return _named(name, kind="commit", dtype=dtype, batch=batch, layers=layers, q_heads=kv_heads, kv_heads=kv_heads,
                  head_dim=head_dim, states=states, nodes=nodes, path=path)


def _bounded(name=None, *, dtype="bf16", batch=1, layers=1, q_heads=32, kv_heads=8, head_dim=128, budget=768, start=4, recent=64,
             per_layer=False):
    return _named(name, kind="bounded", dtype=dtype, batch=batch, layers=layers, q_heads=q_heads, kv_heads=kv_heads,
                  head_dim=head_dim, budget=budget, start=start, recent=recent, per_layer=per_layer)


def _named(name, **case):
    if name is not None:
        case["name"] = name
    return case


def listed():
    return [
        # one layer of the Mistral-7B shape, as a model that calls its layers one after the other verifies eight tokens
        _tree("tree_one_layer", states=832, nodes=8),
        # all layers of that shape in one call, a tree of usual size
        _tree("tree_all_layers", layers=32, states=1280, nodes=24),
        # seven requests with lengths and trees of their own, the layers with 64 query heads
        _tree("tree_batch_ragged", batch=7, layers=8, q_heads=64, states=4352, nodes=61, ragged=True),
        # one request whose whole document stayed in the cache
        _tree("tree_long_cache", layers=2, states=131072, nodes=13),
        # no draft at all: decoding steps of a batch with lengths of its own, multi-head attention, head dimension 64
        _tree("tokens_ragged_head_dim_64", batch=16, layers=4, kv_heads=32, head_dim=64, states=2048, nodes=1, ragged=True),
        # the f32 mode: checks of a small model
        _tree("tree_f32", dtype="f32", batch=2, layers=2, q_heads=8, kv_heads=2, head_dim=64, states=640, nodes=12, ragged=True),
        # what follows tree_one_layer
        _commit("commit_one_layer", states=832, nodes=8, path=4),
        # many requests of a multi-head model, all layers: the most that a commit moves
        _commit("commit_batch", batch=16, layers=32, kv_heads=32, states=512, nodes=64, path=16),
        # one layer at a time, the budget of the headline workload
        _bounded("bounded_one_layer", budget=768),
        # all layers of the Mistral-7B shape in one call
        _bounded("bounded_all_layers", layers=32, budget=1024, recent=256),
        # four requests over the largest layers and their budget
        _bounded("bounded_batch_large", batch=4, layers=20, q_heads=64, budget=4096, recent=1024),
        # the f32 mode, one choice for all heads of a layer, an odd budget
        _bounded("bounded_f32_per_layer", dtype="f32", batch=2, layers=4, q_heads=12, kv_heads=4, head_dim=64, budget=501,
                 recent=33, per_layer=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operators and types in the proportions they are used in, sizes spread over their ranges.  A case that
    would cost more than the largest listed one is made smaller."""
    kind = rng.choice(["tree", "tree", "bounded", "bounded", "commit"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    kv_heads, group = rng.choice([1, 2, 4, 8, 8, 16, 32]), rng.choice([1, 2, 3, 4, 4, 7, 8])
    while kv_heads * group > 64:
        kv_heads //= 2
    common = dict(dtype=dtype, batch=rng.choice([1, 1, 2, 3, 4, 8, 13]), layers=_log(rng, 1, 40), kv_heads=kv_heads,
                  head_dim=64 if rng.random() < 0.3 else 128)
    if kind == "tree":
        case = _tree(q_heads=kv_heads * group, states=_log(rng, 1, 40000), nodes=_log(rng, 1, 64), ragged=rng.random() < 0.5, **common)
    elif kind == "commit":
        nodes = _log(rng, 1, 64)
        case = _commit(states=_log(rng, 1, 4000), nodes=nodes, path=rng.randint(1, min(nodes, 16)), **common)
    else:
        budget = _log(rng, 24, 20000)
        case = _bounded(q_heads=kv_heads * group, budget=budget, start=rng.choice([0, 1, 4]), recent=max(1, int(budget * rng.uniform(0.02, 0.5))),
                        per_layer=rng.random() < 0.25, **common)
    most_flops = 2e10 if dtype == "f32" else 2e11
    while work(case)["bytes"] > 1e9 or work(case)["flops"] > most_flops or _scores(case) > 4e8:
        for key in ("layers", "batch", "states", "budget"):
            if case.get(key, 1) > (1 if key in ("layers", "batch") else 64):
                case[key] = max(1, case[key] * 2 // 3)
                break
        else:
            case["nodes"] = case["nodes"] // 2
        if kind == "bounded":
            case["recent"] = min(case["recent"], case["budget"] // 2)
    return case


def _scores(case):
    """How many attention weights there are."""
    keys = case["budget"] if case["kind"] == "bounded" else case["states"]
    return case["batch"] * case["layers"] * case["q_heads"] * case.get("nodes", 1) * keys


def _lengths(case):
    """States in the cache, nodes and accepted nodes of every document."""
    batch, states, nodes = case["batch"], case["states"], case["nodes"]
    back = [5 * b % batch / batch for b in range(batch)] if case.get("ragged") or case["kind"] == "commit" else [0.0] * batch
    lens = [max(1, states - int(0.75 * states * x)) for x in back]
    trees = [max(1, nodes - int(0.5 * nodes * x)) for x in back]
    return lens, trees, [1 + 3 * b % case.get("path", 1) for b in range(batch)]


class _Inputs:
    """Seeded tensors of one case on the GPU."""

    def __init__(self, case, seed):
        self.case, self.gen = case, torch.Generator(device="cuda").manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)
        self.dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        self.d, self.units = case["head_dim"], (case["batch"], case["layers"])
        self.channel = self.d // 2 - 1

    def values(self, rows, heads=None):
        shape = (*self.units, heads or self.case["kv_heads"], rows, self.d)
        return torch.randn(shape, generator=self.gen, dtype=self.dtype, device="cuda")

    def queries(self, rows):
        q = self.values(rows, self.case["q_heads"])
        q[..., self.channel] = 4.0
        return q

    def keys(self, rows):
        k = self.values(rows)
        importance = k[..., self.channel] * (self.d ** 0.5 / 4.0)  # logit part ~ N(0, 1) for every query
        k *= 0.35                                                  # the part that depends on the query
        boost = torch.rand((self.case["batch"], 1, 1, rows), generator=self.gen, device="cuda") < 0.02
        boost[..., :4] = True
        k[..., self.channel] = importance + boost * (2.0 * self.d ** 0.5 / 4.0)
        return k

    def parents(self, nodes):
        """A random tree: a node hangs on one of the eight before it."""
        up = torch.rand(nodes, generator=self.host).tolist()
        return [-1] + [max(0, t - 1 - int(8 * up[t])) for t in range(1, nodes)]


def _words(parents, nodes):
    """Every node's ancestors and itself as the bits of a word (as torch's signed numbers); padding: 0."""
    words = []
    for t, p in enumerate(parents):
        words.append((words[p] if p >= 0 else 0) | 1 << t)
    return [w - (1 << 64) if w >> 63 else w for w in words] + [0] * (nodes - len(words))


def prepare(case, seed):
    make = _Inputs(case, seed)
    state = {"kind": case["kind"], "case": dict(case)}
    if case["kind"] == "bounded":
        rows = case["budget"]
        state.update(q=make.queries(1), k_new=make.keys(1), v_new=make.values(1), k_cache=make.keys(rows), v_cache=make.values(rows),
                     tokens=rows + seed % 1000)
        sums = torch.randn((*make.units, case["kv_heads"], rows), generator=make.gen, device="cuda")
        state["acc"] = torch.exp(sums) * (case["q_heads"] // case["kv_heads"] * 50.0 / rows)
    else:
        lens, trees, accepted = _lengths(case)
        nodes, rows = case["nodes"], case["states"] + case.get("path", 0)
        words = [_words(make.parents(n), nodes) for n in trees]
        ints = lambda x, t: torch.tensor(x, dtype=t, device="cuda")
        state.update(k_draft=make.keys(nodes), v_draft=make.values(nodes), k_cache=make.keys(rows), v_cache=make.values(rows),
                     lens=ints(lens, torch.int32) if case["kind"] == "commit" or case["ragged"] else None,
                     words=ints(words, torch.int64))
        if case["kind"] == "tree":
            state["q"] = make.queries(nodes)
        else:
            paths = [sorted(torch.randperm(nodes, generator=make.host)[:case["path"]].tolist()) for _ in lens]
            state.update(path=ints(paths, torch.int32), accepted=ints(accepted, torch.int32))
    if own:
        state["plan"] = _plan(case, state)
    return state


def _plan(case, state):
    """What a program that generates keeps between its calls: the configuration, a workspace, the tensors that results go to."""
    import paper_2406_12018_amd as api

    rows = state["k_cache"].shape[3]
    bounded = case["kind"] == "bounded"
    cfg = api.Config(batch=case["batch"], layers=case["layers"], q_heads=case["q_heads"], kv_heads=case["kv_heads"],
                     head_dim=case["head_dim"], chunk_len=64, budget=case["budget"] if bounded else 1, instr_len=1,
                     dtype=api.F32 if case["dtype"] == "f32" else api.BF16, cache_capacity=rows,
                     start_size=case["start"] if bounded else 0,
                     select_mode=api.SELECT_PER_LAYER if bounded and case["per_layer"] else api.SELECT_PER_KV_HEAD)
    plan = {"api": api, "cfg": cfg}
    device = state["k_cache"].device
    if case["kind"] == "commit":
        plan["lens"] = torch.empty(case["batch"], dtype=torch.int32, device=device)
        return plan
    plan["workspace"] = api.alloc_generation_workspace(cfg, case.get("nodes", 1), device)
    plan["out"] = torch.empty_like(state["q"])
    if bounded:
        plan["evicted"] = torch.empty((case["batch"], case["layers"], cfg.sel_heads), dtype=torch.int32, device=device)
    else:
        plan["lse"] = torch.empty(state["q"].shape[:4], dtype=torch.float32, device=device)
    return plan


# ---- the framework's calls ----
def _own_tree(s):
    p = s["plan"]
    p["api"].citrus_tree_attn(p["cfg"], s["q"], s["k_draft"], s["v_draft"], s["words"], s["k_cache"], s["v_cache"],
                              s["case"]["states"], cache_lens=s["lens"], out=p["out"], lse=p["lse"], workspace=p["workspace"])
    return {"out": p["out"], "lse": p["lse"]}


def _own_commit(s):
    p = s["plan"]
    p["api"].citrus_tree_commit(p["cfg"], s["k_draft"], s["v_draft"], s["path"], s["accepted"], s["k_cache"], s["v_cache"],
                                s["case"]["states"], cache_lens=s["lens"], new_lens=p["lens"])
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": p["lens"]}


def _own_bounded(s):
    p = s["plan"]
    p["api"].citrus_decode_evict_step(p["cfg"], s["q"], s["k_new"], s["v_new"], s["k_cache"], s["v_cache"], s["acc"], s["tokens"],
                                      s["case"]["recent"], out=p["out"], evicted=p["evicted"], workspace=p["workspace"])
    s["tokens"] += 1
    return {"out": p["out"], "evicted": p["evicted"], "acc": s["acc"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ---- the plain forms ----
def _grouped(q, kv_heads):
    """[B, L, Hq, T, d] -> [B, L, Hkv, G * T, d] in 32 bits, scaled."""
    b, l, hq, t, d = q.shape
    return q.float().reshape(b, l, kv_heads, hq // kv_heads * t, d) * d ** -0.5


def _plain_tree(s):
    q, n = s["q"], s["case"]["states"]
    nodes, kv_heads = q.shape[3], s["case"]["kv_heads"]
    k = torch.cat((s["k_cache"][:, :, :, :n], s["k_draft"]), 3).float()
    v = torch.cat((s["v_cache"][:, :, :, :n], s["v_draft"]), 3).float()
    at = torch.arange(nodes, device=q.device)
    bits = (s["words"][:, :, None] >> at & 1).bool()                      # [B, node, other node]
    real = bits & torch.eye(nodes, dtype=torch.bool, device=q.device)
    real = real.any(2)                                                    # [B, node]: not padding
    j = torch.arange(n, device=q.device)
    cached = j < s["lens"][:, None] if s["lens"] is not None else (j < n).expand(q.shape[0], n)
    seen = torch.cat((cached[:, None].expand(-1, nodes, -1), bits), 2) & real[:, :, None]
    scores = _grouped(q, kv_heads) @ k.transpose(3, 4)
    scores = scores.reshape(*q.shape[:2], q.shape[2], nodes, -1).masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(4, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(4, keepdim=True)
    out = (p.reshape(*k.shape[:3], -1, k.shape[3]) @ v).reshape(q.shape) / torch.where(total == 0, 1.0, total)
    return {"out": out.to(q.dtype), "lse": (top + total.log()).squeeze(4)}


def _plain_commit(s):
    rows, path = s["k_cache"].shape, s["path"].long()
    step = torch.arange(path.shape[1], device=path.device)
    taken = (step < s["accepted"][:, None])[:, None, None, :, None]
    spread = lambda i: i[:, None, None, :, None].expand(*rows[:3], -1, rows[4])
    to, of = spread(s["lens"].long()[:, None] + step), spread(path)
    for cache, draft in ((s["k_cache"], s["k_draft"]), (s["v_cache"], s["v_draft"])):
        cache.scatter_(3, to, torch.where(taken, draft.gather(3, of), cache.gather(3, to)))
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "lens": s["lens"] + s["accepted"]}


def _plain_bounded(s):
    q, acc, case = s["q"], s["acc"], s["case"]
    n, recent = case["budget"], case["recent"]
    b, l, hkv = acc.shape[:3]
    k = torch.cat((s["k_cache"], s["k_new"]), 3).float()
    v = torch.cat((s["v_cache"], s["v_new"]), 3).float()
    scores = _grouped(q, hkv) @ k.transpose(3, 4)                         # [B, L, Hkv, G, n + 1]
    p = (scores - scores.amax(4, keepdim=True)).exp()
    total = p.sum(4, keepdim=True)
    out = ((p @ v) / total).reshape(q.shape).to(q.dtype)
    weight = (p / total).sum(3)
    acc += weight[..., :n]
    oldest = n - recent + (s["tokens"] - n) % recent
    slot = torch.arange(n, device=q.device)
    free = (slot >= case["start"]) & (slot < n - recent) | (slot == oldest)
    rank = acc.sum(2, keepdim=True) if case["per_layer"] else acc
    rank = torch.where(free, rank, math.inf)
    evicted = torch.where(rank == rank.amin(3, keepdim=True), slot, n).amin(3, keepdim=True)  # the lowest of equal ones
    to = evicted.expand(b, l, hkv, 1)
    acc.scatter_(3, to, acc[..., oldest:oldest + 1].clone())
    acc[..., oldest] = weight[..., n]
    for cache, new in ((s["k_cache"], s["k_new"]), (s["v_cache"], s["v_new"])):
        cache.scatter_(3, to[..., None].expand(b, l, hkv, 1, q.shape[4]), cache[:, :, :, oldest:oldest + 1].clone())
        cache[:, :, :, oldest] = new[:, :, :, 0]
    s["tokens"] += 1
    return {"out": out, "evicted": evicted.squeeze(3).int(), "acc": acc, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def run(state):
    if own:
        return {"tree": _own_tree, "commit": _own_commit, "bounded": _own_bounded}[state["kind"]](state)
    return {"tree": _plain_tree, "commit": _plain_commit, "bounded": _plain_bounded}[state["kind"]](state)


def work(case):
    """Every input read once and every output written once; two products per query row and state it sees."""
    d, esize, layers = case["head_dim"], 4 if case["dtype"] == "f32" else 2, case["layers"]
    hq, hkv, batch = case["q_heads"], case["kv_heads"], case["batch"]
    row = 2 * d * esize  # a state's key and value
    if case["kind"] == "bounded":
        n, units = case["budget"], batch * layers
        # the sums are read and written; the token's state is read and written, and so is the state that moves
        return {"bytes": units * (hkv * (n * (row + 8) + 3 * row) + 2 * hq * d * esize),
                "flops": 4.0 * units * hq * (n + 1) * d}
    lens, trees, accepted = _lengths(case)
    if case["kind"] == "commit":
        return {"bytes": layers * hkv * 2 * row * sum(accepted), "flops": 0.0}
    rows = sum(trees)
    return {"bytes": layers * (hkv * row * (sum(lens) + rows) + hq * rows * (2 * d * esize + 4)),
            "flops": 4.0 * layers * hq * d * sum(t * (n + 1) for n, t in zip(lens, trees))}


# ---- in 64 bits, from the definitions, document by document ----
def exact(case, seed):
    s = prepare(case, seed)
    return {"tree": _exact_tree, "commit": _exact_commit, "bounded": _exact_bounded}[case["kind"]](case, s)


def _exact_tree(case, s):
    lens, _, _ = _lengths(case)
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:4], -math.inf, dtype=torch.float64, device="cuda")
    words = [[w % (1 << 64) for w in doc] for doc in s["words"].tolist()]
    for b, n in enumerate(lens):
        nodes = [t for t, w in enumerate(words[b]) if w >> t & 1]
        hidden = torch.tensor([[not w >> u & 1 for u in nodes] for w in (words[b][t] for t in nodes)], device="cuda")
        for l in range(case["layers"]):
            for g in range(case["kv_heads"]):
                keys, values = (torch.cat((c[b, l, g, :n], x[b, l, g, nodes])).double()
                                for c, x in ((s["k_cache"], s["k_draft"]), (s["v_cache"], s["v_draft"])))
                heads = slice(g * group, (g + 1) * group)
                logits = s["q"][b, l, heads][:, nodes].double() @ keys.T / math.sqrt(case["head_dim"])
                logits[:, :, n:].masked_fill_(hidden, -math.inf)
                total = torch.logsumexp(logits, 2)
                lse[b, l, heads, :len(nodes)] = total
                out[b, l, heads, :len(nodes)] = torch.exp(logits - total[:, :, None]) @ values
    return {"out": out, "lse": lse}


def _exact_commit(case, s):
    lens, _, accepted = _lengths(case)
    k, v, path = s["k_cache"].clone(), s["v_cache"].clone(), s["path"].tolist()
    for b, (n, m) in enumerate(zip(lens, accepted)):
        for i in range(m):
            k[b, :, :, n + i], v[b, :, :, n + i] = s["k_draft"][b, :, :, path[b][i]], s["v_draft"][b, :, :, path[b][i]]
    return {"k_cache": k, "v_cache": v, "lens": torch.tensor([n + m for n, m in zip(lens, accepted)])}


def _exact_bounded(case, s):
    group, n, recent = case["q_heads"] // case["kv_heads"], case["budget"], case["recent"]
    k, v, acc = s["k_cache"].clone(), s["v_cache"].clone(), s["acc"].double()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    weight = torch.empty((*acc.shape[:3], n + 1), dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        for l in range(case["layers"]):
            for g in range(case["kv_heads"]):
                keys, values = (torch.cat((c[b, l, g], x[b, l, g])).double() for c, x in ((k, s["k_new"]), (v, s["v_new"])))
                heads = slice(g * group, (g + 1) * group)
                p = torch.softmax(s["q"][b, l, heads, 0].double() @ keys.T / math.sqrt(case["head_dim"]), 1)
                out[b, l, heads, 0], weight[b, l, g] = p @ values, p.sum(0)
    acc += weight[..., :n]
    oldest = n - recent + (s["tokens"] - n) % recent
    slots = [j for j in range(n) if case["start"] <= j < n - recent or j == oldest]
    rank = acc[..., slots]
    if case["per_layer"]:
        rank = rank.sum(2, keepdim=True)
    rank = rank.tolist()
    evicted = [[[slots[min(range(len(slots)), key=unit.__getitem__)] for unit in layer] for layer in doc] for doc in rank]
    for b, doc in enumerate(evicted):
        for l, chosen in enumerate(doc):
            for g in range(case["kv_heads"]):
                j = chosen[0 if case["per_layer"] else g]
                for cache, new in ((k, s["k_new"]), (v, s["v_new"])):
                    cache[b, l, g, j] = cache[b, l, g, oldest]
                    cache[b, l, g, oldest] = new[b, l, g, 0]
                acc[b, l, g, j] = acc[b, l, g, oldest]
                acc[b, l, g, oldest] = weight[b, l, g, n]
    return {"out": out, "evicted": torch.tensor(evicted, dtype=torch.int32), "acc": acc, "k_cache": k, "v_cache": v}
