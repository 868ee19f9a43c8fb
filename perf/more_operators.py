"""Cases that time the operators of a generated token's step between and behind the attention: the residual's addition with the
norm and an output in 8 bits, products of few rows with 4-bit weights, and the choice of a token from logits.

A case is a dict of plain values; its "kind" names the pass:

  norm    sum = x + delta, its norm, and the norm's result in 8 bits with scales
  w4      Y = epilogue(X W^T) with 4-bit W, a scale (and a zero point) for each group of the reduction
  sample  tokens from rows of logits by temperature, top-k, top-p and min-p, each row with its own, and a given random number

`own` chooses between the plain form, elementary torch operations, and the library's calls.  Widths are those of the workloads in
cascade_inputs/configs.py and of the benchmark's LM head, or odd.
"""
import math

import numpy as np
import torch

own = False

_INT8_MAX, _E4M3_MAX = 127.0, 448.0
_LEAST_SCALE = 2.0 ** -100


def _norm(rows, width, dtype="bf16", norm="rms", delta=True, y=True, q="none", q_group=0, bias=False):
    return {"kind": "norm", "rows": rows, "width": width, "dtype": dtype, "norm": norm, "delta": delta, "y": y, "q": q,
            "q_group": q_group, "bias": bias}


def _w4(rows, k, n, dtype="bf16", group=128, zeros=False, x="same", x_group=0, epilogue="none", bias=False, residual=False):
    return {"kind": "w4", "rows": rows, "k": k, "n": n, "dtype": dtype, "group": group, "zeros": zeros, "x": x, "x_group": x_group,
            "epilogue": epilogue, "bias": bias, "residual": residual}


def _sample(rows, vocab, dtype="bf16", settings="mixed", spread=2.5):
    return {"kind": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "settings": settings, "spread": spread}


def listed():
    return [
        # one generated token between two layers: the smallest call
        {"name": "norm_token", **_norm(1, 4096, q="e4m3", y=False)},
        # a batch of generated tokens, scales for groups of columns
        {"name": "norm_batch_groups", **_norm(64, 8192, q="e4m3", q_group=128, y=False)},
        # a long prompt, one scale for a row
        {"name": "norm_prompt_int8", **_norm(8192, 4096, q="int8", y=False)},
        # fp32, odd width, layer norm with biases
        {"name": "norm_odd_f32", **_norm(1021, 1601, dtype="f32", norm="layer", bias=True)},
        # one token through a square projection: latency
        {"name": "w4_token", **_w4(1, 4096, 4096)},
        # gate and up projections of a few tokens, zero points
        {"name": "w4_gate_up", **_w4(4, 4096, 14336, group=64, zeros=True, epilogue="swiglu")},
        # a batch of tokens whose rows come in 8 bits
        {"name": "w4_batch_int8", **_w4(32, 8192, 28672, x="int8", x_group=0)},
        # the projection back, with the residual, for a full batch
        {"name": "w4_down_full_batch", **_w4(64, 14336, 4096, residual=True)},
        # fp32, small groups, sizes that end inside every tile
        {"name": "w4_odd_f32", **_w4(5, 1056, 1777, dtype="f32", group=32, epilogue="gelu", bias=True)},
        # one token from a large vocabulary: latency
        {"name": "sample_token", **_sample(1, 128256, settings="usual")},
        # a batch of requests, each with its own settings
        {"name": "sample_batch", **_sample(256, 128256)},
        # fp32 logits, an odd vocabulary, temperature alone
        {"name": "sample_whole_f32", **_sample(32, 50257, dtype="f32", settings="temperature")},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "w4", "w4", "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "norm":
        q = rng.choice(["none", "int8", "e4m3", "e4m3"])
        width = rng.choice([_log_int(rng, 64, 16384), 32 * _log_int(rng, 4, 512), 256 * _log_int(rng, 1, 64)])
        q_group = rng.choice([0, 0] + [g for g in (32, 64, 128, 256) if width % g == 0]) if q != "none" else 0
        return _norm(min(_log_int(rng, 1, 8192), (1 << 25) // width), width, dtype, rng.choice(["rms", "rms", "layer"]),
                     rng.random() < 0.8, q == "none" or rng.random() < 0.4, q, q_group, rng.random() < 0.3)
    if kind == "w4":
        group = rng.choice([32, 64, 128, 128])
        rows, k = _log_int(rng, 1, 64), group * _log_int(rng, 2, 14336 // group)
        epilogue = rng.choice(["none", "none", "gelu", "gelu_tanh", "swiglu"])
        n = _log_int(rng, 16, min(28672, (1 << 27) // k))
        x = rng.choice(["same", "same", "int8", "e4m3"])
        return _w4(rows, k, n, dtype, group, rng.random() < 0.4, x, rng.choice([0, 0, 32, 64, 128]) if x != "same" and k % 128 == 0 else 0,
                   epilogue, epilogue != "swiglu" and rng.random() < 0.4, rng.random() < 0.4)
    rows, vocab = _log_int(rng, 1, 256), _log_int(rng, 100, 131072)
    return _sample(min(rows, (1 << (24 if dtype == "bf16" else 23)) // vocab), vocab, dtype, rng.choice(["mixed", "mixed", "usual", "temperature"]), rng.uniform(1.0, 4.0))


# ---------------------------------------------------------------------------- inputs
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _settings(case, rng):
    """temperature, top_k, top_p, min_p of every row, as requests bring them; 0 turns a top_k or min_p off, 1 a top_p."""
    n, how = case["rows"], case["settings"]
    temperature = rng.choice([0.6, 0.7, 0.8, 1.0, 1.3], n)
    if how == "temperature":
        return temperature, np.zeros(n), np.ones(n), np.zeros(n)
    if how == "usual":
        return temperature, np.full(n, 50), np.full(n, 0.95), np.zeros(n)
    temperature = np.where(rng.random(n) < 0.1, 0.0, temperature)            # a greedy request among the others
    top_k = np.where(rng.random(n) < 0.5, np.exp(rng.uniform(0, math.log(2000), n)).astype(int), 0)
    top_p = np.where(rng.random(n) < 0.5, rng.uniform(0.3, 0.99, n), 1.0)
    min_p = np.where(rng.random(n) < 0.3, rng.uniform(0.01, 0.3, n), 0.0)
    return temperature, top_k, top_p, min_p


def _in_8_bits(x, how, group):
    """x [rows, k] as 8-bit values and the scales of its groups (0: of a row), as a norm before has left them."""
    rows, k = x.shape
    x = x.float().view(rows, -1, group or k)
    most = _INT8_MAX if how == "int8" else _E4M3_MAX
    scale = x.abs().amax(-1, keepdim=True) / most
    q = x / scale
    q = q.round().to(torch.int8) if how == "int8" else q.to(torch.float8_e4m3fn)
    return q.view(rows, k), scale.view(rows, -1)


def prepare(case, seed):
    """What a program has in hand: rows, weights, settings, the tensors it writes to; with the library, its handles and workspace."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, dtype = case["kind"], _dtype(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    st = {"case": case}
    if kind == "norm":
        rows, D = case["rows"], case["width"]
        st["x"] = (2.0 * normal(rows, D)).to(dtype)
        st["delta"] = normal(rows, D).to(dtype) if case["delta"] else None
        st["gain"] = (1.0 + 0.1 * normal(D)).to(dtype)
        st["bias"] = (0.1 * normal(D)).to(dtype) if case["bias"] else None
        st["sum"] = torch.empty_like(st["x"]) if case["delta"] else None
        st["y"] = torch.empty_like(st["x"]) if case["y"] else None
        st["q"] = st["scale"] = None
        if case["q"] != "none":
            st["q"] = torch.empty((rows, D), device="cuda", dtype=torch.int8 if case["q"] == "int8" else torch.float8_e4m3fn)
            st["scale"] = torch.empty((rows, D // (case["q_group"] or D)), device="cuda")
            if case["q"] == "int8":
                st["values"] = torch.empty((rows, D), device="cuda", dtype=torch.bfloat16)
        return st
    if kind == "w4":
        rows, k, n, group = case["rows"], case["k"], case["n"], case["group"]
        x = normal(rows, k)
        st["x"], st["x_scale"] = (x.to(dtype), None) if case["x"] == "same" else _in_8_bits(x, case["x"], case["x_group"])
        st["weights"] = []
        for _ in range(2 if case["epilogue"] == "swiglu" else 1):
            codes = torch.randint(0, 16, (n, k), device="cuda", generator=g, dtype=torch.uint8)
            scales = ((0.5 + torch.rand((n, k // group), device="cuda", generator=g)) / (4.6 * math.sqrt(k))).to(dtype)
            zeros = torch.randint(5, 12, (n, k // group), device="cuda", generator=g, dtype=torch.uint8) if case["zeros"] else None
            st["weights"].append((codes, scales, zeros))
        st["bias"] = (0.5 * normal(n)).to(dtype) if case["bias"] else None
        st["residual"] = normal(rows, n).to(dtype) if case["residual"] else None
        st["y"] = torch.empty((rows, n), device="cuda", dtype=dtype)
        if own:
            import paper_2507_05228_amd as cas
            st["w4"] = [cas.make_w4_weights(*w) for w in st["weights"]]
            st["ws"] = cas.new_workspace(cas.cascade_w4_gemm_workspace_bytes(st["w4"][0], st["x"], st["w4"][1] if len(st["w4"]) > 1 else None))
        return st
    rng, rows, V = np.random.default_rng(seed), case["rows"], case["vocab"]
    logits = case["spread"] * normal(rows, V)
    peaks = torch.randint(0, V, (rows, 12), device="cuda", generator=g)      # what the context makes likely
    logits.scatter_add_(1, peaks, case["spread"] * (2.0 + 1.5 * normal(rows, 12).abs()))
    st["logits"] = logits.to(dtype)
    for name, values in zip(("temperature", "top_k", "top_p", "min_p"), _settings(case, rng)):
        st[name] = torch.from_numpy(values.astype(np.int32 if name == "top_k" else np.float32)).cuda()
    st["uniform"] = torch.rand(rows, device="cuda", generator=g)
    st["token"], st["prob"] = torch.empty(rows, device="cuda", dtype=torch.int32), torch.empty(rows, device="cuda")
    if own:
        import paper_2507_05228_amd as cas
        st["ws"] = cas.new_workspace(cas.cascade_sample_workspace_bytes(rows, V, st["logits"].dtype))
    return st


# ---------------------------------------------------------------------------- one pass, by the library's calls
def _run_own(st, case):
    import paper_2507_05228_amd as cas
    kind = case["kind"]
    if kind == "norm":
        cas.cascade_add_norm(st["x"], st["gain"], cas.NORM_RMSNORM if case["norm"] == "rms" else cas.NORM_LAYERNORM, 1e-5,
                             delta=st["delta"], bias=st["bias"], sum=st["sum"], y=st["y"], q=st["q"], q_scale=st["scale"])
        if case["q"] == "int8":
            torch.mul(st["q"].view(len(st["q"]), -1, case["q_group"] or case["width"]), st["scale"][..., None],
                      out=st["values"].view(len(st["q"]), -1, case["q_group"] or case["width"]))
    elif kind == "w4":
        flags = {"none": 0, "gelu": cas.EPI_GELU_ERF, "gelu_tanh": cas.EPI_GELU_TANH, "swiglu": cas.EPI_SWIGLU}[case["epilogue"]]
        flags |= (cas.EPI_BIAS if case["bias"] else 0) | (cas.EPI_RESIDUAL if case["residual"] else 0)
        cas.cascade_w4_gemm(st["w4"][0], st["x"], st["y"], x_scale=st["x_scale"], weights_up=st["w4"][1] if len(st["w4"]) > 1 else None,
                            bias=st["bias"], residual=st["residual"], epilogue=flags, workspace=st["ws"])
    else:
        cas.cascade_sample(st["logits"], st["uniform"], st["token"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"],
                           min_p=st["min_p"], prob=st["prob"], workspace=st["ws"])
    return _outputs(st, case)


def _outputs(st, case):
    names = {"norm": ("sum", "y", "scale") + {"none": (), "int8": ("values",), "e4m3": ("q",)}[case.get("q", "none")],
             "w4": ("y",), "sample": ("token", "prob")}[case["kind"]]
    return {k: st[k] for k in names if st[k] is not None}


# ---------------------------------------------------------------------------- one pass, in elementary operations
def _norm_plain(st, case):
    s = st["x"].float()
    if case["delta"]:
        s = s + st["delta"].float()
        st["sum"].copy_(s)
    if case["norm"] == "layer":
        s = s - s.mean(-1, keepdim=True)
    y = s / (s.square().mean(-1, keepdim=True) + 1e-5).sqrt() * st["gain"].float()
    if case["bias"]:
        y = y + st["bias"].float()
    if case["y"]:
        st["y"].copy_(y)
    if case["q"] != "none":
        group = case["q_group"] or case["width"]
        y = y.view(len(y), -1, group)
        scale = (y.abs().amax(-1, keepdim=True) / (_INT8_MAX if case["q"] == "int8" else _E4M3_MAX)).clamp_min(_LEAST_SCALE)
        st["scale"].copy_(scale[..., 0])
        if case["q"] == "int8":
            st["values"].view(y.shape).copy_((y / scale).round() * scale)
        else:
            st["q"].view(y.shape).copy_((y / scale).clamp(-_E4M3_MAX, _E4M3_MAX))


def _product_plain(st, case, weights):
    codes, scales, zeros = weights
    n, k = codes.shape
    w = codes.view(n, -1, case["group"]).float() - (8.0 if zeros is None else zeros.float()[..., None])
    x = st["x"].float()
    if st["x_scale"] is not None:
        x = (x.view(len(x), -1, case["x_group"] or k) * st["x_scale"][..., None]).view(len(x), k)
    return x @ (w * scales.float()[..., None]).view(n, k).t()


def _w4_plain(st, case):
    y = _product_plain(st, case, st["weights"][0])
    if case["bias"]:
        y = y + st["bias"].float()
    if case["epilogue"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
    elif case["epilogue"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
    elif case["epilogue"] == "swiglu":
        y = y / (1.0 + torch.exp(-y)) * _product_plain(st, case, st["weights"][1])
    if case["residual"]:
        y = y + st["residual"].float()
    st["y"].copy_(y)


def _sample_plain(st, case):
    """Sums of many weights decide between neighbouring tokens: 64 bits."""
    logits, index = st["logits"].float().sort(stable=True, dim=-1, descending=True)
    V = logits.shape[1]
    t = st["temperature"].double()[:, None]
    w = ((logits.double() - logits[:, :1].double()) / torch.where(t > 0, t, 1.0)).exp()
    place = torch.arange(V, device="cuda")
    top_k = st["top_k"][:, None]
    w = torch.where((top_k <= 0) | (place < top_k), w, 0.0)
    running = w.cumsum(-1)
    top_p = st["top_p"].double()[:, None]
    kept = (top_p >= 1) | (running - w < top_p * running[:, -1:])
    kept &= w >= st["min_p"].double()[:, None]
    w = torch.where(kept | (place == 0), w, 0.0)
    running = w.cumsum(-1)
    total = running[:, -1:]
    at = (running <= st["uniform"].double()[:, None] * total).sum(-1, keepdim=True).clamp_max(V - 1)
    at = torch.where(t > 0, at, 0)
    st["token"].copy_(index.gather(1, at)[:, 0])
    st["prob"].copy_(torch.where(t > 0, w.gather(1, at) / total, 1.0)[:, 0])


def run(st):
    case = st["case"]
    if own:
        return _run_own(st, case)
    {"norm": _norm_plain, "w4": _w4_plain, "sample": _sample_plain}[case["kind"]](st, case)
    return _outputs(st, case)


# ---------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    es, rows = (2 if case["dtype"] == "bf16" else 4), case["rows"]
    if case["kind"] == "norm":
        D = case["width"]
        each = es * (1 + 2 * case["delta"] + case["y"]) + (case["q"] != "none")
        scales = rows * D // (case["q_group"] or D) * 4 if case["q"] != "none" else 0
        return {"bytes": rows * D * each + scales + D * es * (1 + case["bias"]), "flops": 8.0 * rows * D}
    if case["kind"] == "w4":
        k, n, groups = case["k"], case["n"], case["k"] // case["group"]
        matrices = 2 if case["epilogue"] == "swiglu" else 1
        x = rows * k * es if case["x"] == "same" else rows * (k + 4 * (k // (case["x_group"] or k)))
        return {"bytes": matrices * n * (k / 2 + groups * (es + case["zeros"])) + x + rows * n * es * (1 + case["residual"]) + n * es * case["bias"],
                "flops": 2.0 * matrices * rows * n * k}
    return {"bytes": rows * (case["vocab"] * es + 28), "flops": 2.0 * rows * case["vocab"]}


# ---------------------------------------------------------------------------- the same results in 64 bits
def exact(case, seed):
    global own
    was, own = own, False                                    # the inputs, without handles of the library
    try:
        st = prepare(case, seed)
    finally:
        own = was
    return {"norm": _norm_exact, "w4": _w4_exact, "sample": _sample_exact}[case["kind"]](st, case)


def _norm_exact(st, case):
    s = st["x"].double() + (st["delta"].double() if case["delta"] else 0)
    out = {"sum": s} if case["delta"] else {}
    if case["norm"] == "rms":
        y = s * (s.pow(2).sum(-1, keepdim=True) / case["width"] + 1e-5).pow(-0.5)
    else:
        var, mean = torch.var_mean(s, -1, correction=0, keepdim=True)
        y = (s - mean) * (var + 1e-5).pow(-0.5)
    y = torch.addcmul(st["bias"].double() if case["bias"] else y.new_zeros(()), y, st["gain"].double())
    if case["y"]:
        out["y"] = y
    if case["q"] == "none":
        return out
    parts = y.unflatten(-1, (-1, case["q_group"] or case["width"]))
    scale = torch.maximum(parts.amax(-1), -parts.amin(-1)) / (_INT8_MAX if case["q"] == "int8" else _E4M3_MAX)
    scale = scale.clamp_min(_LEAST_SCALE)
    q = (parts / scale[..., None]).flatten(1)
    out["scale"] = scale
    if case["q"] == "int8":
        out["values"] = (torch.round(q).unflatten(-1, parts.shape[1:]) * scale[..., None]).flatten(1)
    else:                                                   # steps of an eighth of the power of two below, 2^-9 at the least
        step = torch.exp2(torch.floor(torch.log2(q.abs().clamp_min(2.0 ** -6))) - 3)
        out["q"] = torch.round(q / step) * step
    return out


def _w4_exact(st, case):
    x = st["x"].double()
    if st["x_scale"] is not None:
        x = x * st["x_scale"].double().repeat_interleave(case["k"] // st["x_scale"].shape[1], 1)
    ys = []
    for codes, scales, zeros in st["weights"]:
        y = torch.zeros(len(x), case["n"], device="cuda", dtype=torch.float64)
        for j in range(0, case["k"], case["group"]):
            part = slice(j, j + case["group"])
            w = codes[:, part].double() - (8 if zeros is None else zeros[:, j // case["group"], None].double())
            y += (x[:, part] @ w.t()) * scales[:, j // case["group"]].double()
        ys.append(y)
    y = ys[0] + (st["bias"].double() if case["bias"] else 0)
    if case["epilogue"] == "gelu":
        y = y * torch.special.ndtr(y)
    elif case["epilogue"] == "gelu_tanh":
        y = y * torch.sigmoid(math.sqrt(8 / math.pi) * (y + 0.044715 * y.pow(3)))
    elif case["epilogue"] == "swiglu":
        y = y * torch.sigmoid(y) * ys[1]
    return {"y": y + (st["residual"].double() if case["residual"] else 0)}


def _sample_exact(st, case):
    """Row by row, in numpy; tokens are whole numbers."""
    if case["rows"] * case["vocab"] > 1 << 25:
        return None
    prob = []
    logits = st["logits"].double().cpu().numpy()
    t, k, p, least, u = (st[n].double().cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p", "uniform"))
    for r, l in enumerate(logits):
        if not t[r] > 0:
            prob.append(1.0)
            continue
        w = np.exp((np.sort(l)[::-1] - l.max()) / t[r])
        w = w[:int(k[r])] if k[r] > 0 else w
        if p[r] < 1:
            w = w[:np.searchsorted(np.cumsum(w), p[r] * w.sum()) + 1]
        w = w[:max(1, int((w >= least[r]).sum()))]
        running = np.cumsum(w)
        at = min(np.searchsorted(running, u[r] * running[-1], side="right"), len(w) - 1)
        prob.append(w[at] / running[-1])
    return {"token": None, "prob": torch.tensor(prob, device="cuda", dtype=torch.float64)}
