"""The operators of the 8-bit feed-forward block, dense and by experts, as cases to measure.

One pass is one call of one of the single operations that ``metro_ops.h``
declares for it: the RMSNorm that adds a projection's bf16 rows to the residual
and writes 8-bit rows, the block-scaled product of 8-bit rows and weights (to
bf16 rows, or with SwiGLU behind it to 8-bit rows), the router of tokens to
experts, the same product with each expert's rows, and the weighted sum that
adds the experts' rows to their tokens' residual.  The widths are those of ``synth``
(Llama-3-8B and 70B layers, the tiny test model), the row counts those of the
agents' calls.

8-bit rows are e4m3 codes with one power of two for each 128 consecutive values
(the smallest that brings them within 448, as an E8M0 byte).
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
GROUP = 128
E4M3_MAX = 448.0
F8, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def listed():
    return [
        # One agent's next token: the norm before its projections, nothing but latency.
        dict(name="norm_1", kind="norm", rows=1, d=4096, delta=True, bf16=False),
        # All prompts of the benchmark's 25 agents in one forward, with the bf16 rows that a router's product reads.
        dict(name="norm_31527", kind="norm", rows=31527, d=4096, delta=True, bf16=True),
        # The benchmark's decode batch through the widest product of an 8B layer.
        dict(name="gate_up_25", kind="gemm", M=25, N=28672, K=4096, epilogue=2),
        # A large ready batch, an odd number of rows, through the attention's projections.
        dict(name="qkv_301", kind="gemm", M=301, N=6144, K=4096, epilogue=0),
        # A 70B layer's feed-forward back to the model's width at its benchmark batch.
        dict(name="down_70b_128", kind="gemm", M=128, N=8192, K=28672, epilogue=0),
        # A prefill forward of sixteen 512-token chunks.
        dict(name="gate_up_8192", kind="gemm", M=8192, N=28672, K=4096, epilogue=2),
        # The router of a decode batch: softmax over eight experts, two for each token.
        dict(name="route_25", kind="route", T=25, E=8, scoring=0, bias=False, groups=1, top_groups=1, k=2, renorm=True),
        # The router of the benchmark's prefill with many small experts: sigmoid, balance bias, groups.
        dict(name="route_31527", kind="route", T=31527, E=128, scoring=1, bias=True, groups=8, top_groups=4, k=8, renorm=True),
        # A decode batch through eight experts of an 8B layer's feed-forward: a few rows each, every weight read once.
        dict(name="experts_up_25", kind="experts", T=25, E=8, k=2, N=28672, K=4096, epilogue=2),
        # A prefill forward's rows back from the experts, ragged counts.
        dict(name="experts_down_4096", kind="experts", T=4096, E=8, k=2, N=4096, K=14336, epilogue=0),
        # The weighted sums behind them, at both ends.
        dict(name="combine_25", kind="combine", T=25, k=2, d=4096),
        dict(name="combine_16001", kind="combine", T=16001, k=2, d=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (N, K, epilogue) of a layer's products: 8B QKV, gate/up, down; 70B gate/up, down; tiny gate/up, down; odd ones
_PRODUCTS = [(6144, 4096, 0), (28672, 4096, 2), (4096, 14336, 0), (57344, 8192, 2), (8192, 28672, 0), (1376, 256, 2),
             (256, 768, 0), (1056, 640, 0), (2080, 1408, 2), (4000, 896, 0)]


def draw(rng):
    kind = rng.choice(["norm", "gemm", "gemm", "gemm", "route", "experts", "experts", "combine"])
    if kind == "norm":
        d = rng.choice([256, 688, 1000, 4096, 4096, 5120, 8192])
        return dict(kind=kind, rows=_log_int(rng, 1, min(31527, 31527 * 4096 // d)), d=d, delta=rng.random() < 0.7,
                    bf16=rng.random() < 0.3)
    if kind == "gemm":
        N, K, epilogue = rng.choice(_PRODUCTS)
        return dict(kind=kind, M=_log_int(rng, 1, min(8192, 8192 * 28672 * 4096 // (N * K))), N=N, K=K, epilogue=epilogue)
    if kind == "route":
        E, groups, top_groups = rng.choice([(8, 1, 1), (8, 2, 1), (16, 1, 1), (60, 1, 1), (64, 8, 3), (128, 8, 4), (256, 8, 4)])
        return dict(kind=kind, T=_log_int(rng, 1, 31527 * 128 // max(E, 128)), E=E, scoring=rng.choice([0, 1]),
                    bias=rng.random() < 0.5, groups=groups, top_groups=top_groups, k=rng.choice([1, 2, 4]),
                    renorm=rng.random() < 0.7)
    if kind == "experts":
        N, K, epilogue, E, k = rng.choice([(28672, 4096, 2, 8, 2), (4096, 14336, 0, 8, 2), (2816, 2048, 2, 32, 4),
                                           (2048, 1408, 0, 32, 4), (1376, 256, 2, 4, 1), (4096, 1536, 0, 16, 2)])
        return dict(kind=kind, T=_log_int(rng, 1, min(8192, 8192 * 2 * 4096 * 14336 // (N * K * k))), E=E, k=k, N=N, K=K,
                    epilogue=epilogue)
    k, d = rng.choice([1, 2, 4, 8]), rng.choice([256, 1000, 2048, 4096, 8192])
    return dict(kind=kind, T=_log_int(rng, 1, 16001 * 2 * 4096 // (k * d)), k=k, d=d)


# --- sizes ---------------------------------------------------------------------


def _pad(n, to=GROUP):
    return -(-n // to) * to


def _assigned(T, E, k):
    """[T, k] distinct experts of each token, some experts sought more than others (the same for every seed: the
    counts are the case's size)."""
    r = np.random.Generator(np.random.PCG64([T, E, k]))
    want = r.gumbel(size=(T, E)) - 0.5 * np.log1p(np.arange(E))
    return np.argsort(-want, axis=1, kind="stable")[:, :k]


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n, g = case["rows"] * case["d"], case["rows"] * (_pad(case["d"]) // GROUP)
        return {"bytes": n * (4 + 1 + (6 if case["delta"] else 0) + (2 if case["bf16"] else 0)) + g + 2 * case["d"], "flops": 6 * n}
    if kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return {"bytes": 4 * T * E + 4 * T * k * 4 + 4 * (E + 1), "flops": T * E * (8 + k)}
    if kind == "combine":
        n = case["T"] * case["d"]
        return {"bytes": n * (2 * case["k"] + 8) + 8 * case["T"] * case["k"], "flops": 2 * n * case["k"]}
    N, K = case["N"], case["K"]
    weight = N * K + N * (K // GROUP)
    if kind == "gemm":
        M, rows, weights = case["M"], case["M"], 1
    else:
        chosen = _assigned(case["T"], case["E"], case["k"])
        M, rows, weights = chosen.size, case["T"] if case["epilogue"] == 2 else chosen.size, len(np.unique(chosen))
    out = M * (N // 2 + N // 2 // GROUP) if case["epilogue"] == 2 else 2 * M * N
    return {"bytes": weights * weight + rows * (K + K // GROUP) + out, "flops": 2 * M * N * K}


# --- 8-bit rows ------------------------------------------------------------------


def _quantise(v):
    """v [..., n] float32 -> e4m3 codes [..., n padded to 128] and E8M0 bytes [..., groups]."""
    n = v.shape[-1]
    if n % GROUP:
        v = torch.nn.functional.pad(v, (0, _pad(n) - n))
    v = v.reshape(*v.shape[:-1], -1, GROUP)
    frac, e = torch.frexp(v.abs().amax(-1))  # amax = frac * 2^e, 0.5 <= frac < 1; 448 = 0.875 * 2^9
    e = (e + 127 - 9 + (frac > 0.875)).clamp(min=1, max=254).to(torch.int32)
    codes = (v * torch.exp2((127 - e).to(torch.float32)).unsqueeze(-1)).to(F8)
    return codes.reshape(*codes.shape[:-2], -1), e.to(torch.uint8)


def _values(codes, scale):
    """float32 values of e4m3 codes [rows, n] with E8M0 bytes [rows, n / 128]."""
    s = torch.exp2(scale.to(torch.float32) - 127.0)
    return (codes.to(torch.float32).reshape(*scale.shape, GROUP) * s.unsqueeze(-1)).reshape(codes.shape)


def _pack(codes, scale):
    """Codes [N, K] and bytes [N, K / 128] in the weight layout of metro_op_pack_weight_fp8."""
    N, K = codes.shape
    packed = codes.view(torch.uint8).reshape(N // 16, 16, K // 128, 2, 4, 16).permute(0, 2, 3, 4, 1, 5).contiguous()
    q = _pad(K // GROUP, 4)
    s = torch.nn.functional.pad(scale, (0, q - K // GROUP), value=127)
    return packed.reshape(-1), s.reshape(N // 16, 16, q // 4, 4).permute(0, 2, 1, 3).contiguous().reshape(-1)


def _padded_scale(scale):
    """The bytes as the products read them: rows of a multiple of four."""
    groups = scale.shape[-1]
    return torch.nn.functional.pad(scale, (0, _pad(groups, 4) - groups), value=127).contiguous()


# --- inputs --------------------------------------------------------------------


def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 16 + salt)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _rows(g, M, K, epilogue):
    """8-bit rows as a norm leaves them, or (down products) SwiGLU's outputs, most of them small."""
    v = _normal(g, M, K)
    return _quantise(v if epilogue == 2 or K <= 8192 else v * _normal(g, M, K))


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "norm":
        rows, d = case["rows"], case["d"]
        x = _normal(g, rows, d) * torch.exp2(torch.randint(-2, 3, (rows, 1), generator=g, device=DEV).float())
        return dict(kind=kind, x=x, delta=(0.5 * _normal(g, rows, d)).to(torch.bfloat16) if case["delta"] else None,
                    gain=(1.0 + 0.1 * _normal(g, d)).to(torch.bfloat16), rows=rows, d=d,
                    x_out=torch.empty_like(x) if case["delta"] else None,
                    h16=torch.empty(rows, d, dtype=torch.bfloat16, device=DEV) if case["bf16"] else None,
                    h=torch.empty(rows, _pad(d), dtype=torch.uint8, device=DEV),
                    h_scale=torch.full((rows, _pad(_pad(d) // GROUP, 4)), 127, dtype=torch.uint8, device=DEV))
    if kind == "route":
        T, E, k = case["T"], case["E"], case["k"]
        return dict(kind=kind, case=case, logits=2.0 * _normal(g, T, E),
                    bias=0.1 * _normal(g, E) if case["bias"] else None,
                    experts=torch.empty(T, k, dtype=torch.int32, device=DEV), weights=torch.empty(T, k, device=DEV),
                    offsets=torch.empty(E + 1, dtype=torch.int32, device=DEV),
                    src=torch.empty(T * k, dtype=torch.int32, device=DEV),
                    slot=torch.empty(T, k, dtype=torch.int32, device=DEV),
                    ws=torch.empty(-(-T // 64) * E, dtype=torch.int32, device=DEV))
    if kind == "combine":
        T, k, d = case["T"], case["k"], case["d"]
        w = torch.rand(T, k, generator=g, device=DEV) + 0.1
        return dict(kind=kind, y=_normal(g, T * k, d).to(torch.bfloat16), x=_normal(g, T, d), weights=w / w.sum(1, keepdim=True), T=T, k=k, d=d,
                    slot=torch.randperm(T * k, generator=g, device=DEV).to(torch.int32).reshape(T, k),
                    out=torch.empty(T, d, device=DEV))
    N, K, epi = case["N"], case["K"], case["epilogue"]
    if kind == "gemm":
        T = M = case["M"]
        weights = [_quantise(0.02 * _normal(g, N, K))]
        s = dict(kind=kind)
    else:
        T, E, k = case["T"], case["E"], case["k"]
        M = T * k
        order = torch.randperm(T, generator=g, device=DEV)
        chosen = torch.from_numpy(_assigned(T, E, k)).to(DEV)[order].reshape(-1)
        src = torch.argsort(chosen, stable=True) // k
        counts = [int(c) for c in np.bincount(_assigned(T, E, k).ravel(), minlength=E)]
        offsets = [0] + [int(c) for c in np.cumsum(counts)]
        weights = [_quantise(0.02 * _normal(g, N, K)) for _ in range(E)]
        if epi != 2:  # the experts' own rows, in order
            T, src = M, None
        s = dict(kind=kind, E=E, offsets_host=offsets, offsets=torch.tensor(offsets, dtype=torch.int32, device=DEV),
                 src=None if src is None else src.to(torch.int32))
    packed = [_pack(*w) for w in weights]
    x, x_scale = _rows(g, T, K, epi)
    cols = N // 2
    s.update(M=M, T=T, N=N, K=K, epilogue=epi, x=x, x_scale=_padded_scale(x_scale), w=[w[0] for w in weights],
             w_scale=[w[1] for w in weights], packed=torch.cat([p[0] for p in packed]),
             packed_scale=torch.cat([p[1] for p in packed]),
             ws=torch.empty(8 * min(M, 1024) * N, device=DEV))
    if epi == 2:
        s.update(out=torch.empty(M, _pad(cols), dtype=torch.uint8, device=DEV),
                 out_scale=torch.full((M, _pad(_pad(cols) // GROUP, 4)), 127, dtype=torch.uint8, device=DEV))
    else:
        s.update(out=torch.empty(M, N, dtype=torch.bfloat16, device=DEV), out_scale=None)
    return s


# --- the operators ---------------------------------------------------------------


def _gated(y):
    """silu(gate) * up of columns in blocks of 8 gate, then the 8 matching up columns."""
    y = y.reshape(y.shape[0], -1, 2, 8)
    return (y[:, :, 0] * torch.sigmoid(y[:, :, 0]) * y[:, :, 1]).reshape(y.shape[0], -1)


def _eight(codes, scale, n):
    groups = _pad(n) // GROUP
    return {"codes": codes[:, :_pad(n)].view(F8), "scale": scale[:, :groups].contiguous().view(E8)}


def _run_norm(s):
    d = s["d"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_rmsnorm_fp8(s["x"], s["gain"], EPS, s["h"], s["h_scale"], s["rows"], d, delta=s["delta"], x_out=s["x_out"],
                             h_bf16=s["h16"])
        return {"x": s["x_out"], "h16": s["h16"], **_eight(s["h"], s["h_scale"], d)}
    x = s["x"] if s["delta"] is None else s["x"] + s["delta"].to(torch.float32)
    h = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s["gain"].to(torch.float32)
    codes, scale = _quantise(h)
    return {"x": None if s["delta"] is None else x, "h16": None if s["h16"] is None else h.to(torch.bfloat16),
            **_eight(codes, scale, d)}


def _run_route(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_route(s["logits"], T, E, k, s["experts"], s["weights"], s["offsets"], s["src"], s["slot"], bias=s["bias"],
                       scoring=c["scoring"], n_groups=c["groups"], top_groups=c["top_groups"], renormalise=c["renorm"],
                       workspace=s["ws"])
        return {"experts": s["experts"], "weights": s["weights"], "offsets": s["offsets"], "src": s["src"], "slot": s["slot"]}
    logits = s["logits"].double()  # (choices next to a border)
    if c["scoring"]:
        score = 1.0 / (1.0 + torch.exp(-logits))
    else:
        score = torch.exp(logits - logits.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    choice = score if s["bias"] is None else score + s["bias"].double()
    if c["groups"] > 1:
        grouped = choice.reshape(T, c["groups"], -1)
        best = torch.sort(grouped, dim=2, descending=True).values[:, :, :2].sum(2)
        kept = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        mask = torch.zeros_like(best).scatter_(1, kept, 1.0).unsqueeze(2).expand_as(grouped).reshape(T, E)
        choice = torch.where(mask > 0, choice, -math.inf)
    experts = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    w = torch.gather(score, 1, experts)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    flat = experts.reshape(-1)
    order = torch.argsort(flat, stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(T * k, device=DEV)
    counts = (flat.unsqueeze(1) == torch.arange(E, device=DEV)).sum(0)
    offsets = torch.cat([counts.new_zeros(1), torch.cumsum(counts, 0)])
    return {"experts": experts.to(torch.int32), "weights": w.to(torch.float32), "offsets": offsets.to(torch.int32),
            "src": (order // k).to(torch.int32), "slot": slot.to(torch.int32).reshape(T, k)}


def _run_combine(s):
    if own:
        from paper_2411_03519_amd import metro
        metro.op_combine_experts(s["y"], s["T"] * s["k"], s["weights"], s["slot"], s["T"], s["k"], s["d"], s["out"], resid=s["x"])
        return s["out"]
    return s["x"] + (s["weights"].unsqueeze(2) * s["y"][s["slot"].long()].to(torch.float32)).sum(1)


def _run_gemm(s):
    N, K, epi = s["N"], s["K"], s["epilogue"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_gemm_fp8(s["x"], s["x_scale"], s["packed"], s["packed_scale"], s["M"], N, K, epi, s["out"],
                          out_scale=s["out_scale"], workspace=s["ws"])
        return _eight(s["out"], s["out_scale"], N // 2) if epi == 2 else s["out"]
    y = _values(s["x"], s["x_scale"][:, :K // GROUP]) @ _values(s["w"][0], s["w_scale"][0]).t()
    if epi == 2:
        return _eight(*_quantise(_gated(y)), N // 2)
    return y.to(torch.bfloat16)


def _run_experts(s):
    N, K, epi = s["N"], s["K"], s["epilogue"]
    if own:
        from paper_2411_03519_amd import metro
        metro.op_gemm_fp8_experts(s["x"], s["x_scale"], s["T"], s["src"], s["offsets"], s["E"], s["M"], s["packed"],
                                  s["packed_scale"], N, K, epi, s["out"], out_scale=s["out_scale"], workspace=s["ws"])
        return _eight(s["out"], s["out_scale"], N // 2) if epi == 2 else s["out"]
    x = _values(s["x"], s["x_scale"][:, :K // GROUP])
    if s["src"] is not None:
        x = x[s["src"].long()]
    o = s["offsets_host"]
    y = torch.cat([x[o[e]:o[e + 1]] @ _values(s["w"][e], s["w_scale"][e]).t() for e in range(s["E"]) if o[e + 1] > o[e]])
    return _eight(*_quantise(_gated(y)), N // 2) if epi == 2 else y.to(torch.bfloat16)


_RUN = {"norm": _run_norm, "route": _run_route, "combine": _run_combine, "gemm": _run_gemm, "experts": _run_experts}


def run(state):
    return _RUN[state["kind"]](state)


# --- the definitions in 64 bits ----------------------------------------------------


def _exact_eight(v):
    """Rows v (float64) to the nearest e4m3 multiples of each group's power of two, ties to even."""
    rows, n = v.shape
    full = torch.zeros(rows, _pad(n), dtype=torch.float64, device=v.device)
    full[:, :n] = v
    full = full.reshape(rows, -1, GROUP)
    top = full.abs().amax(2)
    power = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 1e-300)) / E4M3_MAX))
    power = torch.where(top > torch.exp2(power) * E4M3_MAX, power + 1, power)
    power = torch.where(top <= torch.exp2(power - 1) * E4M3_MAX, power - 1, power).clamp(min=-126)
    scaled = full / torch.exp2(power).unsqueeze(2)
    size = torch.floor(torch.log2(scaled.abs().clamp(min=2.0 ** -6)))  # 3 bits after the leading one, steps of 2^-9 at least
    step = torch.exp2(size - 3)
    return {"codes": (torch.round(scaled / step) * step).reshape(rows, -1), "scale": torch.exp2(power)}


def _exact_values(codes, scale):
    rows, n = codes.shape
    groups = scale[:, :n // GROUP].double()
    return codes.to(torch.float32).double() * torch.repeat_interleave(torch.pow(2.0, groups - 127.0), GROUP, dim=1)


def _exact_swiglu(y):
    columns = torch.arange(y.shape[1] // 2, device=y.device)
    gate = 16 * (columns // 8) + columns % 8
    z = y[:, gate]
    return z / (1.0 + torch.exp(-z)) * y[:, gate + 8]


def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        x = s["x"].double()
        if s["delta"] is not None:
            x = x + s["delta"].double()
        h = x / torch.sqrt(torch.sum(x ** 2, dim=1, keepdim=True) / case["d"] + EPS) * s["gain"].double()
        return {"x": x if s["delta"] is not None else None, "h16": h if s["h16"] is not None else None, **_exact_eight(h)}
    if kind == "route":
        T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
        z = s["logits"].cpu().numpy().astype(np.float64)
        p = 1.0 / (1.0 + np.exp(-z)) if case["scoring"] else np.exp(z - z.max(1, keepdims=True))
        if not case["scoring"]:
            p /= p.sum(1, keepdims=True)
        want = p + s["bias"].cpu().numpy().astype(np.float64) if s["bias"] is not None else p.copy()
        if G > 1:
            by_group = np.sort(want.reshape(T, G, E // G), axis=2)[:, :, -2:].sum(2)
            rank = np.argsort(np.argsort(-by_group, axis=1, kind="stable"), axis=1, kind="stable")
            want[np.repeat(rank >= case["top_groups"], E // G, axis=1)] = -np.inf
        chosen = np.argsort(-want, axis=1, kind="stable")[:, :k]
        w = np.take_along_axis(p, chosen, axis=1)
        if case["renorm"]:
            w = w / w.sum(1, keepdims=True)
        tokens = [np.nonzero((chosen == e).any(1))[0] for e in range(E)]
        offsets = np.concatenate([[0], np.cumsum([len(t) for t in tokens])])
        slot = np.zeros((T, k), np.int64)
        for e, t in enumerate(tokens):
            slot[t, np.argmax(chosen[t] == e, axis=1)] = offsets[e] + np.arange(len(t))
        return {"experts": chosen, "weights": w, "offsets": offsets, "src": np.concatenate(tokens), "slot": slot}
    if kind == "combine":
        out = s["x"].double()
        for j in range(s["k"]):
            out += s["weights"][:, j:j + 1].double() * s["y"][s["slot"][:, j].long()].double()
        return out
    x = _exact_values(s["x"], s["x_scale"])
    if kind == "gemm":
        y = torch.matmul(x, _exact_values(s["w"][0], s["w_scale"][0]).t())
    else:
        y = torch.zeros(s["M"], case["N"], dtype=torch.float64, device=DEV)
        for e in range(s["E"]):
            lo, hi = s["offsets_host"][e], s["offsets_host"][e + 1]
            mine = x[s["src"][lo:hi].long()] if s["src"] is not None else x[lo:hi]
            y[lo:hi] = torch.matmul(mine, _exact_values(s["w"][e], s["w_scale"][e]).t())
    return _exact_eight(_exact_swiglu(y)) if case["epilogue"] == 2 else y
