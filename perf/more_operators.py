"""The operators of a speculative decoding step, as cases to measure.

One pass is one call of one of the single operations that ``metro_ops.h``
declares for it: the rows of a QKV product normalised by head, rotated and
appended to the paged cache; attention of a tree of drafted tokens (or of one
token) over such a cache; the sampled choice of a token at every row of logits;
and the move of the accepted drafts' keys and values to the slots behind their
context, in all layers.  The widths are those of ``synth`` (Llama-3-8B and 70B
layers, the tiny test model) and the lengths those of the agents' calls.

The cache's pages hold 16 keys, K and V^T in the order that ``metro_ops.h``
states.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
PAGE = 16
N_POS = 16384  # rows of the rotation's table
BF16 = torch.bfloat16


def listed():
    return [
        # One agent's next token: nothing but latency.
        dict(name="append_1", kind="append", items=1, lo=1, hi=1, pad=0, nq=32, nkv=8, hd=128, norm=False, bf16=False),
        # Trees of drafted tokens of the benchmark's 25 agents in a batch padded for a graph, with norms, from an 8-bit product.
        dict(name="append_drafts_25", kind="append", items=25, lo=9, hi=17, pad=11, nq=32, nkv=8, hd=128, norm=True, bf16=True),
        # A prefill forward of sixteen chunks of about 512 tokens.
        dict(name="append_prefill_16", kind="append", items=16, lo=500, hi=524, pad=0, nq=32, nkv=8, hd=128, norm=True, bf16=False),
        # One agent's next token over its history.
        dict(name="tree_1", kind="tree", items=1, lo=1, hi=1, ctx_lo=1311, ctx_hi=1311, nq=32, nkv=8, hd=128, tree=False),
        # The benchmark's 25 agents, each with a tree of drafted tokens.
        dict(name="tree_25", kind="tree", items=25, lo=9, hi=17, ctx_lo=256, ctx_hi=4096, nq=32, nkv=8, hd=128, tree=True),
        # Wide trees over long histories, heads of a 70B layer.
        dict(name="tree_long_2", kind="tree", items=2, lo=57, hi=64, ctx_lo=20000, ctx_hi=30000, nq=64, nkv=8, hd=128, tree=True),
        # The median ready batch of a 1000-agent simulation with drafted trees.
        dict(name="tree_123", kind="tree", items=123, lo=8, hi=32, ctx_lo=256, ctx_hi=4096, nq=32, nkv=8, hd=128, tree=True),
        # One agent's next token, nucleus sampling.
        dict(name="sample_1", kind="sample", rows=1, vocab=128256, how="top_p"),
        # The benchmark's agents, each with settings of its own.
        dict(name="sample_25", kind="sample", rows=25, vocab=128256, how="mixed"),
        # A choice at every node of the drafted trees of 25 agents.
        dict(name="sample_325", kind="sample", rows=325, vocab=128256, how="top_k"),
        # One agent's accepted drafts, and those of 25, in every layer of an 8B model.
        dict(name="move_1", kind="move", seqs=1, lo=3, hi=3, layers=32, nkv=8, hd=128),
        dict(name="move_25", kind="move", seqs=25, lo=2, hi=7, layers=32, nkv=8, hd=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (nq, nkv, hd): 8B, 70B, tiny; no groups, groups of 2, small heads
_HEADS = [(32, 8, 128), (32, 8, 128), (64, 8, 128), (4, 2, 64), (16, 16, 64), (12, 6, 128), (40, 5, 64)]


def draw(rng):
    kind = rng.choice(["append", "append", "tree", "tree", "tree", "sample", "sample", "move"])
    nq, nkv, hd = rng.choice(_HEADS)
    if kind == "append":
        most = int(8192 * 6144 / ((nq + 2 * nkv) * hd))
        items = _log_int(rng, 1, 200)
        hi = _log_int(rng, 1, max(1, min(most // items, 2048)))
        return dict(kind=kind, items=items, lo=max(1, hi // 2), hi=hi, pad=rng.choice([0, 0, 1, 7]), nq=nq, nkv=nkv, hd=hd,
                    norm=rng.random() < 0.5, bf16=rng.random() < 0.5)
    if kind == "tree":
        items = _log_int(rng, 1, 123)
        hi = rng.choice([1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
        most = 123 * 1300 * 20 * 32 * 128 // (items * max(hi, 8) * nq * hd)  # (keys, by the largest listed case's work)
        ctx_hi = _log_int(rng, 1, max(2, min(30000, most, 123 * 1300 * 8 * 128 // (items * nkv * hd))))
        return dict(kind=kind, items=items, lo=max(1, hi // 2), hi=hi, ctx_lo=ctx_hi // rng.choice([1, 2, 8]), ctx_hi=ctx_hi,
                    nq=nq, nkv=nkv, hd=hd, tree=hi > 1 and rng.random() < 0.8)
    if kind == "sample":
        vocab = rng.choice([4096, 32000, 50257, 100003, 128256, 128256])
        return dict(kind=kind, rows=_log_int(rng, 1, 325 * 128256 // max(vocab, 32000)), vocab=vocab,
                    how=rng.choice(["plain", "top_k", "top_p", "min_p", "mixed", "mixed"]))
    lo = rng.choice([1, 2, 3])
    return dict(kind=kind, seqs=_log_int(rng, 1, 25), lo=lo, hi=lo + rng.choice([0, 2, 5]), layers=rng.choice([1, 2, 8, 32]),
                nkv=nkv, hd=hd)


# --- sizes (the same for every seed) --------------------------------------------


def _sizes(case, n, lo, hi):
    r = np.random.Generator(np.random.PCG64([n, lo, hi, len(case["kind"])]))
    return r.integers(lo, hi + 1, n)


def _contexts(case):
    """Keys before each item's queries: lognormal around the agents' 1200 tokens where the range allows it."""
    n, lo, hi = case["items"], case["ctx_lo"], case["ctx_hi"]
    r = np.random.Generator(np.random.PCG64([n, lo, hi, 7]))
    if lo < 1200 < hi:
        return np.clip(np.rint(1200 * np.exp(0.5 * r.standard_normal(n))), lo, hi).astype(np.int64)
    return r.integers(lo, hi + 1, n)


def _parents(n, salt):
    """Parent of each drafted token (the root's is -1), breadth first as a drafter lists them."""
    r = np.random.Generator(np.random.PCG64([n, salt, 11]))
    return np.array([-1] + [int(r.integers(max(0, (j - 1) // 3 - 2), (j - 1) // 2 + 1)) for j in range(1, n)])


def _ancestors(n, salt):
    """[n, n] truth values: node j is node r or above it."""
    up = np.eye(n, dtype=bool)
    for r, p in enumerate(_parents(n, salt)):
        if p >= 0:
            up[r] |= up[p]
    return up


def _seen(case):
    """For each item (keys before it, [n, n] drafted keys that each query sees)."""
    ns = _sizes(case, case["items"], case["lo"], case["hi"])
    return [(int(c), _ancestors(int(n), i) if case["tree"] else np.tril(np.ones((n, n), dtype=bool)))
            for i, (c, n) in enumerate(zip(_contexts(case), ns))]


def work(case):
    kind = case["kind"]
    if kind == "append":
        T = int(_sizes(case, case["items"], case["lo"], case["hi"]).sum()) + case["pad"]
        n = T * (case["nq"] + 2 * case["nkv"]) * case["hd"]
        return {"bytes": n * (2 if case["bf16"] else 4) + 2 * n + T * (8 + 4 * case["hd"]), "flops": n * (9 if case["norm"] else 5)}
    if kind == "tree":
        seen = _seen(case)
        rows, keys = sum(len(m) for _, m in seen), sum(c + len(m) for c, m in seen)
        pairs = sum(c * len(m) + int(m.sum()) for c, m in seen)
        return {"bytes": keys * 4 * case["nkv"] * case["hd"] + rows * 4 * case["nq"] * case["hd"],
                "flops": 4 * pairs * case["nq"] * case["hd"]}
    if kind == "sample":
        n = case["rows"] * case["vocab"]
        return {"bytes": 4 * n + 28 * case["rows"], "flops": 10 * n}
    moves = int(_sizes(case, case["seqs"], case["lo"], case["hi"]).sum())
    return {"bytes": moves * (8 + case["layers"] * 8 * case["nkv"] * case["hd"]), "flops": moves * case["layers"]}


# --- inputs -----------------------------------------------------------------------


def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + salt)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _pool(g, pages, nkv, hd):
    return _normal(g, pages, 2 * nkv * PAGE * hd).to(BF16)


def _rope(hd):
    angle = torch.arange(N_POS, dtype=torch.float64, device=DEV).unsqueeze(1) * torch.pow(
        torch.tensor(500000.0, dtype=torch.float64, device=DEV), -2.0 * torch.arange(hd // 2, device=DEV).double() / hd)
    return torch.stack([torch.cos(angle), torch.sin(angle)], dim=2).float().contiguous()


def _prepare_append(case, g, r):
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    ns = _sizes(case, case["items"], case["lo"], case["hi"])
    # any place in a page, the same for every seed: the pages touched are the case's size
    first = _sizes(case, case["items"], 0, PAGE - 1) + PAGE * r.integers(0, (N_POS - int(ns.max())) // PAGE, case["items"])
    need = [int(f % PAGE + n + PAGE - 1) // PAGE for f, n in zip(first, ns)]
    pages = r.permutation(sum(need) + 3)
    pos, slot, at = [], [], 0
    for f, n, p in zip(first, ns, need):
        o = f % PAGE + np.arange(n)
        slot.append(pages[at + o // PAGE] * PAGE + o % PAGE)
        pos.append(f + np.arange(n))
        at += p
    slot.append(np.full(case["pad"], -1))
    pos.append(np.zeros(case["pad"], dtype=np.int64))
    T = int(ns.sum()) + case["pad"]
    qkv = _normal(g, T, (nq + 2 * nkv) * hd) * torch.exp2(torch.randint(-2, 2, (T, 1), generator=g, device=DEV).float())
    gain = [(1.0 + 0.1 * _normal(g, hd)).to(BF16) for _ in range(2)] if case["norm"] else [None, None]
    return dict(T=T, nq=nq, nkv=nkv, hd=hd, qkv=qkv.to(BF16) if case["bf16"] else qkv, q_gain=gain[0], k_gain=gain[1],
                rope=_rope(hd), pos=_ints(np.concatenate(pos)), slot=_ints(np.concatenate(slot)), n_pages=len(pages),
                kv=_pool(g, len(pages), nkv, hd), q=torch.empty(T, nq * hd, dtype=BF16, device=DEV))


def _prepare_tree(case, g, r):
    nq, nkv, hd = case["nq"], case["nkv"], case["hd"]
    seen = _seen(case)
    need = [-(-(c + len(m)) // PAGE) for c, m in seen]
    pages = r.permutation(sum(need) + 3)
    ldb, max_q = max(need), max(len(m) for _, m in seen)
    tables, at = np.zeros((len(seen), ldb), dtype=np.int64), 0
    for i, p in enumerate(need):
        tables[i, :p] = pages[at:at + p]
        at += p
    ldm = -(-max_q // 32)
    bits = np.zeros((sum(len(m) for _, m in seen), ldm * 32), dtype=np.uint8)
    cu = np.concatenate([[0], np.cumsum([len(m) for _, m in seen])])
    for i, (_, m) in enumerate(seen):
        bits[cu[i]:cu[i + 1], :len(m)] = m
    mask = torch.from_numpy(np.packbits(bits, axis=1, bitorder="little").view(np.int32)).to(DEV)
    rows = int(cu[-1])
    s = dict(nq=nq, nkv=nkv, hd=hd, items=len(seen), rows=rows, max_q=max_q, max_keys=max(c + len(m) for c, m in seen),
             cu_host=[int(c) for c in cu], ctx_host=[c for c, _ in seen], need=need,
             seen=[torch.from_numpy(m).to(DEV) for _, m in seen], cu=_ints(cu), ctx=_ints([c for c, _ in seen]),
             mask=mask if case["tree"] else None, ldm=ldm, tables=_ints(tables), ldb=ldb, n_pages=len(pages),
             kv=_pool(g, len(pages), nkv, hd), q=(1.5 * _normal(g, rows, nq * hd)).to(BF16),
             out=torch.empty(rows, nq * hd, dtype=BF16, device=DEV), ws=None)
    if own:
        from paper_2411_03519_amd import metro
        n = metro.op_attn_tree_workspace(nq, nkv, hd, s["items"], rows, max_q, s["max_keys"])
        s["ws"] = torch.empty(max(n // 4, 4), device=DEV)
    return s


def _prepare_sample(case, g, r):
    rows, vocab, how = case["rows"], case["vocab"], case["how"]
    ldl = -(-vocab // 32) * 32  # as the head's product leaves them
    logits = 2.0 * _normal(g, rows, ldl)
    likely = torch.randint(0, vocab, (rows, 24), generator=g, device=DEV)
    logits.scatter_add_(1, likely, 12.0 * torch.rand(rows, 24, generator=g, device=DEV))
    mixed = how == "mixed"
    pick = lambda values: torch.tensor([values[j] for j in r.integers(0, len(values), rows)], device=DEV)
    s = dict(rows=rows, vocab=vocab, ldl=ldl, logits=logits, u=torch.rand(rows, generator=g, device=DEV),
             temperature=pick([0.0, 0.6, 0.8, 1.0, 1.5] if mixed else [0.7, 1.0]).float(),
             top_k=pick([0, 0, 1, 20, 50, 1000]).int() if mixed else pick([40, 50]).int() if how == "top_k" else None,
             top_p=pick([1.0, 1.0, 0.5, 0.9, 0.95]).float() if mixed else pick([0.9, 0.95]).float() if how == "top_p" else None,
             min_p=pick([0.0, 0.0, 0.02, 0.1]).float() if mixed else pick([0.05, 0.1]).float() if how == "min_p" else None,
             token=torch.empty(rows, dtype=torch.int32, device=DEV), prob=torch.empty(rows, device=DEV), ws=None)
    if own:
        from paper_2411_03519_amd import metro
        s["ws"] = torch.empty(max(metro.op_sample_workspace(rows, vocab), 16), dtype=torch.uint8, device=DEV)
    return s


def _prepare_move(case, g, r):
    nkv, hd, layers = case["nkv"], case["hd"], case["layers"]
    ns = _sizes(case, case["seqs"], case["lo"], case["hi"])
    nodes = 32  # drafted tokens of a sequence
    pages = r.permutation(3 * case["seqs"] + 2)
    src, dst = [], []
    for i, n in enumerate(ns):
        first = int(r.integers(0, PAGE))
        slots = lambda o: pages[3 * i + (first + o) // PAGE] * PAGE + (first + o) % PAGE
        # the root, then an accepted node of each depth, listed behind the path's own length
        path = np.concatenate([[0], np.sort(r.choice(np.arange(n, nodes), n - 1, replace=False))])
        src.append(slots(path))
        dst.append(slots(np.arange(n)))
    return dict(nkv=nkv, hd=hd, layers=layers, n_pages=len(pages), seqs=case["seqs"], moves=int(ns.sum()),
                kv=_pool(g, layers * len(pages), nkv, hd).reshape(layers, len(pages), -1), src=_ints(np.concatenate(src)),
                dst=_ints(np.concatenate(dst)), offsets=_ints(np.concatenate([[0], np.cumsum(ns)])))


_PREPARE = {"append": _prepare_append, "tree": _prepare_tree, "sample": _prepare_sample, "move": _prepare_move}


def prepare(case, seed):
    s = _PREPARE[case["kind"]](case, _gen(seed), np.random.Generator(np.random.PCG64([seed, 3])))
    s["kind"] = case["kind"]
    return s


# --- the operators ------------------------------------------------------------------


def _k_view(kv, nkv, hd):
    """[..., pages, nkv, hd / 32, 4, 16 keys, 8]"""
    return kv.reshape(*kv.shape[:-1], 2, nkv, hd // 32, 4, PAGE, 8).select(-6, 0)


def _v_view(kv, nkv, hd):
    """[..., pages, nkv, hd / 32, 4 (key / 4), 16 (dim % 16), 2 (dim / 16 % 2), 4 (key % 4)]"""
    return kv.reshape(*kv.shape[:-1], 2, nkv, hd // 32, 4, 16, 2, 4).select(-7, 1)


def _run_append(s):
    T, nq, nkv, hd = s["T"], s["nq"], s["nkv"], s["hd"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_rope_append(s["qkv"], T, nq, nkv, hd, s["rope"], N_POS, s["pos"], s["slot"], s["q"], s["kv"], s["n_pages"],
                             q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS)
        return {"q": s["q"], "kv": s["kv"]}
    y = s["qkv"].to(torch.float32).reshape(T, nq + 2 * nkv, hd)
    q, k, v = y[:, :nq], y[:, nq:nq + nkv], y[:, nq + nkv:]
    if s["q_gain"] is not None:
        q, k = [x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * w.to(torch.float32)
                for x, w in ((q, s["q_gain"]), (k, s["k_gain"]))]
    cs = s["rope"][s["pos"].long()].unsqueeze(1)
    c, sn = cs[..., 0], cs[..., 1]

    def turned(x):
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return torch.cat([a * c - b * sn, a * sn + b * c], dim=2).to(BF16)

    here = torch.nonzero(s["slot"] >= 0).squeeze(1)
    slot = s["slot"][here].long()
    page, off = slot // PAGE, slot % PAGE
    kv = s["kv"]
    _k_view(kv, nkv, hd)[page, :, :, :, off] = turned(k)[here].reshape(-1, nkv, hd // 32, 4, 8)
    v = v[here].to(BF16).reshape(-1, nkv, hd // 32, 2, 16).transpose(3, 4)
    _v_view(kv, nkv, hd)[page, :, :, off // 4, :, :, off % 4] = v
    return {"q": turned(q).reshape(T, nq * hd), "kv": kv}


def _run_tree(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_attn_tree(s["q"], s["kv"], s["n_pages"], nq, nkv, hd, s["items"], s["cu"], s["rows"], s["ctx"], s["max_q"],
                           s["max_keys"], s["tables"], s["ldb"], s["out"], mask=s["mask"], ldm=s["ldm"], workspace=s["ws"])
        return s["out"]
    outs = []
    for i in range(s["items"]):
        lo, hi, ctx = s["cu_host"][i], s["cu_host"][i + 1], s["ctx_host"][i]
        n, keys = hi - lo, ctx + hi - lo
        mine = s["kv"][s["tables"][i, :s["need"][i]].long()]
        k = _k_view(mine, nkv, hd).permute(1, 2, 3, 5, 0, 4).reshape(nkv, hd, -1)[:, :, :keys].to(torch.float32)
        v = _v_view(mine, nkv, hd).permute(1, 0, 3, 6, 2, 5, 4).reshape(nkv, -1, hd)[:, :keys].to(torch.float32)
        q = s["q"][lo:hi].to(torch.float32).reshape(n, nkv, nq // nkv, hd).transpose(0, 1).reshape(nkv, -1, hd)
        z = torch.matmul(q, k.contiguous()).reshape(nkv, n, nq // nkv, keys) * (1.0 / math.sqrt(hd))
        ok = torch.cat([torch.ones(n, ctx, dtype=torch.bool, device=DEV), s["seen"][i]], dim=1)
        z = torch.where(ok[None, :, None], z, -math.inf)
        p = torch.exp(z - z.amax(3, keepdim=True))
        o = torch.matmul((p / p.sum(3, keepdim=True)).reshape(nkv, -1, keys), v.contiguous())
        outs.append(o.reshape(nkv, n, -1).transpose(0, 1).reshape(n, nq * hd))
    return torch.cat(outs).to(BF16)


def _run_sample(s):
    rows, vocab = s["rows"], s["vocab"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_sample(s["logits"], rows, vocab, s["u"], s["token"], temperature=s["temperature"], top_k=s["top_k"],
                        top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], ldl=s["ldl"], workspace=s["ws"])
        return {"token": s["token"], "prob": s["prob"]}
    x = s["logits"][:, :vocab].double()  # (cumulated weights next to a border)
    greedy = (s["temperature"] <= 0).unsqueeze(1)
    z = x / torch.where(greedy, 1.0, s["temperature"].double().unsqueeze(1))
    z, index = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp(z - z[:, :1])
    rank = torch.arange(vocab, device=DEV).unsqueeze(0)
    if s["min_p"] is not None:
        w = torch.where(w >= s["min_p"].double().unsqueeze(1), w, 0.0)
    if s["top_k"] is not None:
        k = s["top_k"].long().unsqueeze(1)
        w = torch.where((k <= 0) | (rank < k), w, 0.0)
    upto = torch.cumsum(w, dim=1)
    if s["top_p"] is not None:
        share = s["top_p"].double().unsqueeze(1)
        w = torch.where((share >= 1) | (upto - w < share * upto[:, -1:]) | (rank == 0), w, 0.0)
        upto = torch.cumsum(w, dim=1)
    w = torch.where(greedy & (rank > 0), 0.0, w)
    upto = torch.where(greedy, 1.0, upto)
    at = (upto <= s["u"].double().unsqueeze(1) * upto[:, -1:]).sum(1, keepdim=True)
    return {"token": torch.gather(index, 1, at).squeeze(1).to(torch.int32),
            "prob": (torch.gather(w, 1, at) / upto[:, -1:]).squeeze(1).to(torch.float32)}


def _run_move(s):
    nkv, hd, kv = s["nkv"], s["hd"], s["kv"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_kv_move(kv, s["layers"], s["n_pages"], nkv, hd, s["src"], s["dst"], s["offsets"], s["seqs"], s["moves"])
        return kv
    src, dst = s["src"].long(), s["dst"].long()
    k, v = _k_view(kv, nkv, hd), _v_view(kv, nkv, hd)
    k[:, dst // PAGE, :, :, :, dst % PAGE] = k[:, src // PAGE, :, :, :, src % PAGE]
    v[:, dst // PAGE, :, :, dst % PAGE // 4, :, :, dst % 4] = v[:, src // PAGE, :, :, src % PAGE // 4, :, :, src % 4]
    return kv


_RUN = {"append": _run_append, "tree": _run_tree, "sample": _run_sample, "move": _run_move}


def run(state):
    return _RUN[state["kind"]](state)


# --- the definitions in 64 bits --------------------------------------------------------


def _places(hd):
    """Where (key of the page, dim) lies within a head's K tile and its V^T tile, [16, hd] each."""
    r, e = torch.meshgrid(torch.arange(PAGE, device=DEV), torch.arange(hd, device=DEV), indexing="ij")
    k = ((e // 32 * 4 + (e // 8) % 4) * 16 + r) * 8 + e % 8
    v = ((e // 32 * 4 + r // 4) * 16 + e % 16) * 8 + ((e // 16) % 2) * 4 + r % 4
    return k, v


def _exact_append(s):
    T, nq, nkv, hd = s["T"], s["nq"], s["nkv"], s["hd"]
    y = s["qkv"].double().reshape(T, nq + 2 * nkv, hd)
    heads = []
    for h in range(nq + 2 * nkv):
        x, gain = y[:, h], s["q_gain"] if h < nq else s["k_gain"]
        if h < nq + nkv:
            if gain is not None:
                x = x / torch.sqrt(torch.sum(x ** 2, dim=1, keepdim=True) / hd + EPS) * gain.double()
            turn = torch.view_as_complex(s["rope"].double())[s["pos"].long()]
            pair = torch.complex(x[:, :hd // 2].contiguous(), x[:, hd // 2:].contiguous()) * turn
            x = torch.cat([pair.real, pair.imag], dim=1)
        heads.append(x)
    kv = s["kv"].double().reshape(s["n_pages"], 2, nkv, PAGE * hd)
    places = _places(hd)
    rows = [t for t, at in enumerate(s["slot"].tolist()) if at >= 0]
    slot = s["slot"].long()[rows]
    for c in range(2):
        at = places[c][slot % PAGE]
        for h in range(nkv):
            kv[(slot // PAGE).unsqueeze(1), c, h, at] = heads[nq + c * nkv + h][rows]
    return {"q": torch.cat(heads[:nq], dim=1), "kv": kv.reshape(s["n_pages"], -1)}


def _exact_tree(s):
    nq, nkv, hd = s["nq"], s["nkv"], s["hd"]
    places = _places(hd)
    out = torch.zeros(s["rows"], nq, hd, dtype=torch.float64, device=DEV)
    for i in range(s["items"]):
        lo, hi, ctx = s["cu_host"][i], s["cu_host"][i + 1], s["ctx_host"][i]
        mine = s["kv"].reshape(-1, 2, nkv, PAGE * hd)[s["tables"][i, :s["need"][i]].long()]
        unseen = torch.zeros(hi - lo, ctx + hi - lo, dtype=torch.float64, device=DEV)
        unseen[:, ctx:] = torch.where(s["seen"][i], 0.0, -math.inf)
        for h in range(nkv):
            k, v = [mine[:, c, h][:, places[c]].double().reshape(-1, hd)[:ctx + hi - lo] for c in range(2)]
            for j in range(h * (nq // nkv), (h + 1) * (nq // nkv)):
                z = torch.mm(s["q"][lo:hi, j * hd:(j + 1) * hd].double(), k.t()) / hd ** 0.5 + unseen
                out[lo:hi, j] = torch.mm(torch.softmax(z, dim=1), v)
    return out.reshape(s["rows"], nq * hd)


def _exact_sample(s):
    host = {k: (s[k].cpu().numpy() if s[k] is not None else None) for k in ("logits", "u", "temperature", "top_k", "top_p", "min_p")}
    tokens, probs = [], []
    for r in range(s["rows"]):
        x, T = host["logits"][r, :s["vocab"]].astype(np.float64), float(host["temperature"][r])
        if T <= 0:
            tokens.append(int(np.argmax(x)))
            probs.append(1.0)
            continue
        order = np.argsort(-x, kind="stable")
        w = np.exp((x[order] - x[order[0]]) / T)
        if host["min_p"] is not None:
            w = w[:np.count_nonzero(w >= float(host["min_p"][r]))]
        if host["top_k"] is not None and host["top_k"][r] > 0:
            w = w[:host["top_k"][r]]
        if host["top_p"] is not None and host["top_p"][r] < 1:
            w = w[:int(np.searchsorted(np.cumsum(w), float(host["top_p"][r]) * w.sum(), side="left")) + 1]
        upto = np.cumsum(w)
        at = int(np.searchsorted(upto, float(host["u"][r]) * upto[-1], side="right"))
        tokens.append(int(order[at]))
        probs.append(w[at] / upto[-1])
    return {"token": _ints(tokens), "prob": torch.tensor(probs, dtype=torch.float64, device=DEV)}


def _exact_move(s):
    nkv, hd, layers = s["nkv"], s["hd"], s["layers"]
    was = s["kv"].reshape(layers, s["n_pages"], 2, nkv, PAGE * hd)
    now = was.double()
    places = _places(hd)
    for a, b in zip(s["src"].tolist(), s["dst"].tolist()):
        for c in range(2):
            now[:, b // PAGE, c, :, places[c][b % PAGE]] = was[:, a // PAGE, c, :, places[c][a % PAGE]].double()
    return now.reshape(s["kv"].shape)


def exact(case, seed):
    return {"append": _exact_append, "tree": _exact_tree, "sample": _exact_sample, "move": _exact_move}[case["kind"]](prepare(case, seed))
