"""Performance cases of the operators around 4-bit weights and routed experts.

`operator` is what a case calls:
  "quantise"  rows to 4-bit floating point with a scale per 32 elements and back (fff_mx4_quantize, fff_mx4_dequantize)
  "product"   act(A W^T + b) with W in 4 bits (fff_mx4_product); A in bf16, or quantised to 4 bits first
  "experts"   the leaf networks in 4 bits that each token is routed to, mixed (fff_leaf_forward_mx4)
  "route"     choice of k experts, mixture weights, counts and balance losses (fff_moe_route), with `train` the gradient
              of the logits too (fff_moe_route_backward)
`listed()` names the cases, `draw(rng)` gives others of the same ranges, `prepare` makes the tensors a caller holds, `run` is
one pass: in plain torch, or with `own` through the framework.  `exact` is the definition in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 32


def listed():
    return [
        # activations of a few sequences of a 4096-wide model, to be fed to a 4-bit product
        {"name": "quantise_activations", "operator": "quantise", "batch": 1, "rows": 8192, "cols": 4096, "dtype": "bf16",
         "transpose": False},
        # expert weights as a checkpoint holds them ([neuron][output]), laid out for the product that sums over the neurons; odd sizes
        {"name": "quantise_expert_weights", "operator": "quantise", "batch": 8, "rows": 1027, "cols": 777, "dtype": "f32",
         "transpose": True},
        # one token through a projection: the bytes of the weights count
        {"name": "product_one_token", "operator": "product", "T": 1, "K": 4096, "N": 4096, "a": "bf16", "out": "bf16", "act": "none"},
        # a few thousand tokens through the first matrix of a feedforward block, activations as they are
        {"name": "product_bf16_rows", "operator": "product", "T": 4096, "K": 4096, "N": 4096, "a": "bf16", "out": "bf16", "act": "gelu"},
        # a long prompt with both sides in 4 bits: the matrix rate counts
        {"name": "product_4bit_rows", "operator": "product", "T": 8192, "K": 4096, "N": 4096, "a": "mx4", "out": "bf16", "act": "none"},
        # nothing is a whole tile, rows are not whole pieces, single-precision results
        {"name": "product_ragged", "operator": "product", "T": 333, "K": 1000, "N": 777, "a": "mx4", "out": "f32", "act": "relu"},
        # the latency experiment's layer: 256 rows of 768, leaves of 32 neurons, one leaf a token
        {"name": "experts_narrow_256", "operator": "experts", "T": 256, "k": 1, "E": 512, "D": 768, "O": 768, "width": 32, "act": "gelu"},
        # serving: eight tokens, each through two wide experts of 64
        {"name": "experts_decode", "operator": "experts", "T": 8, "k": 2, "E": 64, "D": 4096, "O": 4096, "width": 1024, "act": "gelu"},
        # a long prompt through a mixture of 16 experts of a BERT-wide model
        {"name": "experts_prefill", "operator": "experts", "T": 8192, "k": 2, "E": 16, "D": 768, "O": 768, "width": 2048, "act": "gelu"},
        # choosing experts while serving a small batch: what a call costs before it computes anything
        {"name": "route_serve", "operator": "route", "T": 64, "E": 64, "k": 4, "dtype": "f32", "train": False},
        # a training step's routing at the vision transformer's batch, losses and gradients
        {"name": "route_train", "operator": "route", "T": 50432, "E": 128, "k": 2, "dtype": "bf16", "train": True},
        # the same for many experts and a large k
        {"name": "route_train_512", "operator": "route", "T": 32768, "E": 512, "k": 8, "dtype": "f32", "train": True},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("quantise", "product", "experts", "route"))
    if op == "quantise":
        c = {"operator": op, "batch": 1, "rows": _log_int(rng, 1, 16384), "cols": _log_int(rng, 16, 8192),
             "dtype": rng.choice(("bf16", "f32")), "transpose": rng.random() < 0.4}
        if c["transpose"]:
            c["batch"] = _log_int(rng, 1, 32)
        limit = 8192 * 4096 if c["dtype"] == "bf16" else 8192 * 2048
        while c["batch"] * c["rows"] * c["cols"] > limit // (2 if c["transpose"] else 1):
            c["rows"] = max(1, c["rows"] * 3 // 4)
        return c
    if op == "product":
        c = {"operator": op, "T": _log_int(rng, 1, 8192), "K": _log_int(rng, 32, 8192), "N": _log_int(rng, 16, 8192),
             "a": rng.choice(("bf16", "mx4")), "out": "bf16", "act": rng.choice(("none", "relu", "gelu"))}
        if rng.random() < 0.75:
            c["K"], c["N"] = max(32, c["K"] // 32 * 32), max(16, c["N"] // 16 * 16)
        if c["a"] == "mx4" and rng.random() < 0.3:
            c["out"] = "f32"
        while c["T"] * c["K"] * c["N"] > (1 << 36):
            c["T"] = c["T"] * 3 // 4
        return c
    if op == "experts":
        E = _log_int(rng, 1, 512)
        step = 8 if rng.random() < 0.8 else 1
        c = {"operator": op, "T": _log_int(rng, 1, 8192), "k": min(E, rng.choice((1, 1, 2, 2, 4, 8))), "E": E,
             "D": step * _log_int(rng, 64 // step, 4096 // step), "O": 0, "width": _log_int(rng, 16, 2048),
             "act": rng.choice(("relu", "gelu"))}
        c["O"] = c["D"] if rng.random() < 0.6 else step * _log_int(rng, 64 // step, 4096 // step)
        while c["E"] * c["width"] * (c["D"] + c["O"]) > 64 * 1024 * 8192 // 2:
            c["width"] = max(16, c["width"] // 2)
            if c["width"] == 16:
                c["E"] = max(1, c["E"] // 2)
                c["k"] = min(c["k"], c["E"])
        while c["T"] * c["k"] * c["width"] * (c["D"] + c["O"]) > 8192 * 2 * 2048 * 1536:
            c["T"] = c["T"] * 3 // 4
        return c
    E = _log_int(rng, 2, 512)
    c = {"operator": op, "T": _log_int(rng, 1, 65536), "E": E, "k": min(E, rng.choice((1, 2, 2, 4, 6, 8))),
         "dtype": rng.choice(("bf16", "f32")), "train": rng.random() < 0.7}
    while c["T"] * c["E"] > 32768 * 512:
        c["T"] = c["T"] * 3 // 4
    return c


# ---- what a pass needs -----------------------------------------------------------------------------------


def _mx4_bytes(rows, cols):
    return rows * ((cols + BLOCK - 1) // BLOCK) * 17


def work(case):
    """One pass: inputs read once, outputs written once; of the experts those that are met by a token."""
    op = case["operator"]
    if op == "quantise":
        n, es = case["batch"] * case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        r, c = (case["cols"], case["rows"]) if case["transpose"] else (case["rows"], case["cols"])
        return {"bytes": 2 * n * es + case["batch"] * _mx4_bytes(r, c), "flops": 4 * n}
    if op == "product":
        T, K, N = case["T"], case["K"], case["N"]
        return {"bytes": 2 * T * K + _mx4_bytes(N, K) + T * N * (2 if case["out"] == "bf16" else 4) + 2 * N, "flops": 2 * T * K * N}
    if op == "experts":
        T, k, E, D, O, w = (case[i] for i in ("T", "k", "E", "D", "O", "width"))
        met = E * (1 - (1 - 1 / E) ** (T * k)) if E > 1 else 1
        return {"bytes": int(2 * T * (D + O) + 8 * T * k + met * (_mx4_bytes(w, D) + _mx4_bytes(O, w) + 2 * (w + O))),
                "flops": 2 * T * k * w * (D + O)}
    T, E, k, es = case["T"], case["E"], case["k"], 2 if case["dtype"] == "bf16" else 4
    rows = T * E * es
    return {"bytes": (3 * rows + 20 * T * k + T if case["train"] else rows + 8 * T * k), "flops": (20 if case["train"] else 8) * T * E}


# ---- inputs ----------------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["operator"]

    def normal(shape, scale=1.0, dtype=torch.bfloat16):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def weights(shape, scale):      # a matrix in 4 bits, made piece by piece
        codes = empty(shape[:-1] + (16 * ((shape[-1] + 31) // 32),), torch.uint8)
        scales = empty(shape[:-1] + ((shape[-1] + 31) // 32,), torch.uint8)
        for i in range(shape[0]):
            codes[i], scales[i] = _plain_quantise(normal(shape[1:], scale).float())
        return codes, scales

    s = {"case": case}
    if op == "quantise":
        shape = (case["batch"], case["rows"], case["cols"])
        # rows of unlike size, and some large elements, as activations and weights have them
        x = normal(shape, 1.0, torch.float32) * torch.exp(torch.randn(shape[:2] + (1,), generator=g, device="cuda"))
        x = x * torch.where(torch.rand(shape, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        s["x"] = x.to(DTYPES[case["dtype"]])
        r, c = shape[:0:-1] if case["transpose"] else shape[1:]
        blocks = (c + BLOCK - 1) // BLOCK
        s["codes"], s["scales"] = empty((shape[0], r, 16 * blocks), torch.uint8), empty((shape[0], r, blocks), torch.uint8)
        s["values"] = empty((shape[0], r, c), DTYPES[case["dtype"]])
    elif op == "product":
        T, K, N = case["T"], case["K"], case["N"]
        dt = DTYPES[case["out"]]
        s["a"] = normal((T, K))
        codes, scales = weights((1, N, K), K ** -0.5)
        s["w"], s["ws"] = codes[0], scales[0]
        s["bias"] = normal((N,), 0.1, dt)
        s["out"] = empty((T, N), dt)
        if case["a"] == "mx4":
            s["ac"], s["as"] = empty((T, 16 * ((K + 31) // 32)), torch.uint8), empty((T, (K + 31) // 32), torch.uint8)
    elif op == "experts":
        T, k, E, D, O, w = (case[i] for i in ("T", "k", "E", "D", "O", "width"))
        s["x"] = normal((T, D))
        s["w1"], s["s1"] = weights((E, w, D), D ** -0.5)
        s["w2"], s["s2"] = weights((E, O, w), w ** -0.5)
        s["b1"], s["b2"] = normal((E, w), 0.1), normal((E, O), 0.1)
        # some experts are asked more often than others; one token in fifty asks none
        score = torch.rand((T, E), generator=g, device="cuda").clamp_min(1e-9).log().neg().log().neg() + \
            torch.randn((E,), generator=g, device="cuda") * 0.5
        idx = score.topk(k, dim=1).indices.to(torch.int32)
        none = torch.rand((T, 1), generator=g, device="cuda") < 0.02
        s["idx"] = torch.where(none, -1, idx).to(torch.int32).contiguous()
        s["weight"] = torch.softmax(torch.randn((T, k), generator=g, device="cuda"), 1).contiguous()
        s["out"] = empty((T, O), torch.bfloat16)
    else:
        T, E, k, dt = case["T"], case["E"], case["k"], DTYPES[case["dtype"]]
        s["logits"] = (torch.randn((T, E), generator=g, device="cuda") * 1.5 + torch.randn((E,), generator=g, device="cuda") * 0.5).to(dt)
        s["idx"], s["weight"] = empty((T, k), torch.int32), empty((T, k), torch.float32)
        if case["train"]:
            # sequences padded to one length: the tails take no part
            s["mask"] = (torch.rand((T,), generator=g, device="cuda") < 0.9).to(torch.uint8)
            s["count"], s["prob_mean"] = empty((E + 1,), torch.int32), empty((E,), torch.float32)
            s["loss"] = empty((2,), torch.float32)
            s["dweight"] = torch.randn((T, k), generator=g, device="cuda") / T
            s["dloss"] = torch.tensor([1e-2, 1e-3], device="cuda")
            s["dlogits"] = empty((T, E), dt)
    return s


# ---- one pass --------------------------------------------------------------------------------------------


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2308_14711_amd as F
    case = s["case"]
    op = case["operator"]
    if op == "quantise":
        F.fff_mx4_quantize(s["x"], s["codes"], s["scales"], transpose=case["transpose"])
        F.fff_mx4_dequantize(s["codes"], s["scales"], s["values"])
        return s["values"]
    act = {"none": F.ACT_NONE, "relu": F.ACT_RELU, "gelu": F.ACT_GELU}[case.get("act", "none")]
    if op == "product":
        if case["a"] == "mx4":
            F.fff_mx4_quantize(s["a"], s["ac"], s["as"])
            F.fff_mx4_product(s["ac"], s["w"], s["ws"], s["out"], a_scales=s["as"], bias=s["bias"], act=act)
        else:
            F.fff_mx4_product(s["a"], s["w"], s["ws"], s["out"], bias=s["bias"], act=act)
        return s["out"]
    if op == "experts":
        F.fff_leaf_forward_mx4(s["x"], s["w1"], s["s1"], s["b1"], s["w2"], s["s2"], s["b2"], s["idx"], s["weight"], act, s["out"])
        return s["out"]
    if not case["train"]:
        F.fff_moe_route(s["logits"], case["k"], s["idx"], s["weight"])
        return s["idx"], s["weight"]
    F.fff_moe_route(s["logits"], case["k"], s["idx"], s["weight"], s["count"], s["prob_mean"], s["loss"], token_mask=s["mask"])
    F.fff_moe_route_backward(s["logits"], s["idx"], s["count"], s["dlogits"], dweight=s["dweight"], dloss=s["dloss"],
                             token_mask=s["mask"])
    return s["idx"], s["weight"], s["count"], s["prob_mean"], s["loss"], s["dlogits"]


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _plain_quantise(x):
    """Rows of fp32 to codes (two a byte, the first in the low four bits) and scale bytes."""
    pad = -x.shape[-1] % BLOCK
    if pad:
        x = torch.cat([x, x.new_zeros(x.shape[:-1] + (pad,))], -1)
    v = x.reshape(x.shape[:-1] + (-1, BLOCK))
    size = v.abs().amax(-1, keepdim=True)
    # frexp: size = m 2^e with m in [1/2, 1), so floor(log2 size) = e - 1; the largest element is 1.5 * 2^2
    shift = (torch.frexp(size).exponent - 3).clamp(-127, 127)
    shift = torch.where(size == 0, -127, shift)
    half = -shift // 2
    q = torch.ldexp(torch.ldexp(v, half), -shift - half).abs()
    # between neighbours: halfway goes to the even code
    code = ((q > 0.25).int() + (q >= 0.75).int() + (q > 1.25).int() + (q >= 1.75).int() + (q > 2.5).int() + (q >= 3.5).int() +
            (q > 5.0).int())
    code = (code + 8 * torch.signbit(v).int()).reshape(x.shape).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), (shift + 127).squeeze(-1).to(torch.uint8)


def _plain_values(codes, scales, cols):
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    v = grid[code].reshape(scales.shape + (BLOCK,))
    return torch.ldexp(v, scales.int().unsqueeze(-1) - 127).flatten(-2)[..., :cols]


def _plain_act(v, act):
    if act == "relu":
        return v.clamp_min(0)
    return 0.5 * v * (1 + torch.erf(v * 0.5 ** 0.5)) if act == "gelu" else v


def _run_plain(s):
    case = s["case"]
    op = case["operator"]
    if op == "quantise":
        x = s["x"].float()
        if case["transpose"]:
            x = x.transpose(1, 2)
        codes, scales = _plain_quantise(x.contiguous())
        return _plain_values(codes, scales, x.shape[-1]).to(s["x"].dtype)
    if op == "product":
        a = s["a"].float()
        if case["a"] == "mx4":
            a = _plain_values(*_plain_quantise(a), a.shape[-1])
        w = _plain_values(s["w"], s["ws"], a.shape[-1])
        return _plain_act(a @ w.T + s["bias"].float(), case["act"]).to(s["out"].dtype)
    if op == "experts":
        x, out = s["x"].float(), torch.zeros(s["out"].shape, device="cuda")
        for e in range(case["E"]):
            t, i = torch.nonzero(s["idx"] == e, as_tuple=True)
            if len(t) == 0:
                continue
            w1 = _plain_values(s["w1"][e], s["s1"][e], case["D"])
            w2 = _plain_values(s["w2"][e], s["s2"][e], case["width"])
            h = _plain_act(x[t] @ w1.T + s["b1"][e].float(), case["act"])
            out[t] += s["weight"][t, i, None] * (h @ w2.T + s["b2"][e].float())
        return out.to(torch.bfloat16)
    logits, k = s["logits"].float(), case["k"]
    T, E = logits.shape
    idx = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    size = torch.exp(logits - logits.amax(1, keepdim=True))
    p = size / size.sum(1, keepdim=True)
    chosen = p.gather(1, idx)
    weight = chosen / chosen.sum(1, keepdim=True)
    if not case["train"]:
        return idx.to(torch.int32), weight
    on = s["mask"] != 0
    n = on.sum()
    hit = (idx[:, :, None] == torch.arange(E, device="cuda")).sum(1) * on[:, None]
    count = hit.sum(0)
    p = p * on[:, None]
    prob_mean = p.sum(0) / n
    lse = (size.sum(1).log() + logits.amax(1)) * on
    share = count.float() / (n * k)
    loss = torch.stack([E * (share * prob_mean).sum(), (lse * lse).sum() / n])
    pull = s["dloss"][0] * E * share / n
    d = p * (pull - (p * pull).sum(1, keepdim=True)) + s["dloss"][1] * 2 * lse[:, None] * p / n
    dw = weight * (s["dweight"] - (weight * s["dweight"]).sum(1, keepdim=True)) * on[:, None]
    d = d.scatter_add(1, idx, dw)
    idx = torch.where(on[:, None], idx, -1)
    return (idx.to(torch.int32), weight * on[:, None], torch.cat([count, n[None]]).to(torch.int32), prob_mean, loss,
            d.to(s["logits"].dtype))


# ---- the definition in 64 bits ---------------------------------------------------------------------------


def _exact_read(codes, scales, cols):
    """Elements as sign, two exponent bits and one mantissa bit; scales as powers of two."""
    c = torch.empty(codes.shape + (2,), dtype=torch.float64, device=codes.device)
    for n, nibble in enumerate((codes % 16, codes // 16)):
        sign, e, m = nibble // 8, nibble // 2 % 4, (nibble % 2).double()
        v = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e.double() - 1))
        c[..., n] = torch.where(sign == 1, -v, v)
    c = c.flatten(-2)
    power = 2.0 ** (scales.double() - 127)
    return (c * power.repeat_interleave(BLOCK, -1))[..., :cols]


def _exact_round(x):
    """The nearest multiple of the block's scale that four bits hold."""
    cols = x.shape[-1]
    wide = torch.zeros(x.shape[:-1] + ((cols + BLOCK - 1) // BLOCK * BLOCK,), dtype=torch.float64, device=x.device)
    wide[..., :cols] = x
    v = wide.unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1, keepdim=True)
    power = torch.ones_like(top)
    for step in (128.0, 64.0, 32.0, 16.0, 8.0, 4.0, 2.0, 1.0):      # the largest power of two that is no larger than the top
        up, down = 2.0 ** step, 2.0 ** -step
        power = torch.where(power * up <= top, power * up, power)
        power = torch.where(power > top, torch.where(power * down * 2 > top, power * down, power), power)
    power = torch.where(power > top, power / 2, power) / 4
    power = power.clamp_min(2.0 ** -127)
    q = v.abs() / power
    # spacing 1/2 below 2, 1 below 4, 2 above; torch.round takes halves to the even multiple
    step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0)).to(q.dtype)
    q = (torch.round(q / step) * step).clamp_max(6.0)
    return (torch.sign(v) * q * power).flatten(-2)[..., :cols]


def _exact_act(v, act):
    if act == "relu":
        return torch.maximum(v, torch.zeros_like(v))
    return v * torch.special.ndtr(v) if act == "gelu" else v


def exact(case, seed):
    s = prepare(case, seed)
    op = case["operator"]
    if op == "quantise":
        x = s["x"].double()
        return _exact_round(x.permute(0, 2, 1) if case["transpose"] else x)
    if op == "product":
        a = s["a"].double()
        a = _exact_round(a) if case["a"] == "mx4" else a
        return _exact_act(torch.addmm(s["bias"].double(), a, _exact_read(s["w"], s["ws"], case["K"]).t().contiguous()), case["act"])
    if op == "experts":
        x = s["x"].double()
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        for e in torch.unique(s["idx"]).tolist():
            if e < 0:
                continue
            # (an expert is asked at most once by a token)
            asked = (s["idx"] == e)
            t = asked.any(1).nonzero()[:, 0]
            share = (s["weight"].double() * asked).sum(1)[t]
            h = _exact_act(x[t].mm(_exact_read(s["w1"][e], s["s1"][e], case["D"]).t().contiguous()) + s["b1"][e].double(), case["act"])
            y = h.mm(_exact_read(s["w2"][e], s["s2"][e], case["width"]).t().contiguous()) + s["b2"][e].double()
            out[t] = out[t] + share[:, None] * y
        return out
    l, k = s["logits"].double(), case["k"]
    T, E = l.shape
    left = l.clone()
    idx = torch.empty((T, k), dtype=torch.int64, device="cuda")
    place = torch.arange(E, device="cuda")
    for i in range(k):      # the lowest index among the largest that are left
        best = left.max(1, keepdim=True).values
        idx[:, i] = torch.where(left == best, place, E).min(1).values
        left[torch.arange(T, device="cuda"), idx[:, i]] = -math.inf
    p = torch.exp(l - torch.logsumexp(l, 1, keepdim=True))
    w = torch.softmax(l.gather(1, idx), 1)
    if not case["train"]:
        return idx.to(torch.int32), w
    rows = s["mask"].nonzero()[:, 0]
    n = len(rows)
    count = torch.bincount(idx[rows].flatten(), minlength=E)
    mean = p[rows].mean(0) if n else torch.zeros((E,), dtype=torch.float64, device="cuda")
    lse = torch.logsumexp(l, 1)
    n1 = max(n, 1)
    share = count.double() / (n1 * k)
    loss = torch.stack([E * (share * mean).sum(), lse[rows].pow(2).sum() / n1])
    g = s["dloss"].double()
    pull = g[0] * E * share / n1
    d = p * (pull[None] - (p * pull[None]).sum(1, keepdim=True) + 2 * g[1] / n1 * lse[:, None])
    up = s["dweight"].double()
    d.scatter_add_(1, idx, w * (up - (w * up).sum(1, keepdim=True)))
    off = s["mask"] == 0
    d[off], w[off], idx[off] = 0, 0, -1
    return idx.to(torch.int32), w, torch.cat([count, torch.tensor([n], device="cuda")]).to(torch.int32), mean, loss, d
