"""Values of the operators on four-bit matrices and routed experts where a launch could read them otherwise than the definition: NaN and
infinity through activations, the tails of GELU, the roundings on the way, every scale byte, many tokens of few leaves."""
import math

import numpy as np
import pytest

import operators_reference as R
from test_gpu_operators import _bytes, _leaf_case, _matrix, _up, _within

pytestmark = pytest.mark.gpu


# ---- NaN and infinity through the activations ---------------------------------------------------------------

# blocks of 16, 32 and 64 rows, then 64 and 128 rows through LDS
PRODUCTS = [(5, 100, 40), (31, 100, 3100), (64, 100, 3100), (700, 1024, 1100), (3000, 264, 3200)]


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("kind", ["bf16", "mx4", "mx4-f32"])
@pytest.mark.parametrize("size", PRODUCTS, ids=lambda s: "x".join(map(str, s)))
def test_product_hands_on_nan_and_infinity(size, kind, act):
    import torch
    import paper_2308_14711_amd as F
    T, K, N = size
    rng = np.random.default_rng(T)
    x = rng.normal(size=(T, K))
    x[1, K - 1], x[3, 0] = np.nan, np.inf
    rows, a = _up(x, "bf16")
    wc, ws, _ = _matrix(rng, (N, K), 1.0)
    ws[7, -1] = 255
    w, kw, out_kind = R.values(wc, ws, K), {}, "f32" if kind == "mx4-f32" else "bf16"
    if kind != "bf16":
        ac, asc = R.quantise(a)
        rows, kw, a = _bytes(ac), {"a_scales": _bytes(asc)}, R.values(ac, asc, K)
    out = torch.empty((T, N), dtype=torch.float32 if out_kind == "f32" else torch.bfloat16, device="cuda")
    F.fff_mx4_product(rows, _bytes(wc), _bytes(ws), out, act={"none": F.ACT_NONE, "relu": F.ACT_RELU, "gelu": F.ACT_GELU}[act], **kw)
    some = np.unique(np.r_[0:5, T // 2, T - 2:T])
    with np.errstate(invalid="ignore"):
        want, tol = R.product(a[some], w, None, act, out_kind)
    assert np.isnan(want[:, 7]).all() and np.isnan(want[1]).all() and np.isfinite(np.delete(want[[0, 2, 4]], 7, 1)).all()
    _within(out[some.tolist()], want, tol, "product %s %s %s [%s]" % (size, kind, act, F.fff_last_launch()))


# a block a token; few pairs of wide leaves; tiles of 16, 32 and 64 rows; of 64 and 128 through LDS
LEAVES = [(20, 1, 8, 64, 40, 32), (5, 2, 4, 1096, 521, 601), (60, 1, 4, 520, 1024, 700), (40, 2, 3, 96, 40, 36), (150, 1, 3, 160, 130, 257),
          (700, 2, 5, 296, 136, 300), (4100, 8, 2, 136, 1032, 1100)]


@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("case", LEAVES, ids=lambda c: "-".join(map(str, c)))
def test_leaves_hand_on_nan_and_infinity(case, act):
    import torch
    import paper_2308_14711_amd as F
    T, k, E, D, O, width = case
    rng = np.random.default_rng(T + width)
    dev, (x, w1, b1, w2, b2, idx, weight) = _leaf_case(rng, *case, True, none=0.0)
    dev = list(dev)
    x[2, D - 1], x[1, 0] = np.nan, np.inf
    dev[0] = _up(x, "bf16")[0]
    # a block of a neuron of leaf 1, a block of an output of leaf 0; token 0 meets neither
    c1, s1, c2, s2 = (dev[i].cpu().numpy() for i in (1, 2, 4, 5))
    s1[1, 3, -1] = s2[0, 4, 0] = 255
    w1, w2 = R.values(c1, s1, D), R.values(c2, s2, width)
    idx[0] = E - 1 if E > 2 else -1
    idx[3] = 1
    dev[2], dev[5], dev[7] = _bytes(s1), _bytes(s2), _bytes(idx)
    out = torch.full((T, O), -7.0, dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(*dev, {"relu": F.ACT_RELU, "gelu": F.ACT_GELU}[act], out)
    some = np.unique(np.r_[0:min(T, 20), T // 2, T - 2:T])
    with np.errstate(invalid="ignore"):
        want, tol = R.leaves(x[some], w1, b1, w2, b2, idx[some], weight[some], act)
    assert np.isnan(want[2]).all() and np.isnan(want[3]).all() and np.isfinite(want[0]).all()
    _within(out[some.tolist()], want, tol, "leaves %s %s" % (case, act))


# ---- GELU over its whole range -------------------------------------------------------------------------------

# every bf16 value from 2^-10 to 8, and from -2^-10 to -13
GRID = np.array([s * 2.0 ** e * (1 + m / 128) for s in (1, -1) for e in range(-10, 4) for m in range(128)])
GRID = GRID[(GRID <= 8) & (GRID >= -13)]


def _gelu(v):
    return np.array([0.5 * x * math.erfc(-x / math.sqrt(2)) for x in v.ravel()]).reshape(v.shape)


def _gelu_tol(v, kind):
    """bf16: the kernels' own, relative to the value (2^-15 above -7, 2^-12 above -11, 2^-10 below), and half a step of the type.  fp32: the argument of
    erfc rounded twice, which its square in the exponent carries 2 v^2 / 2 times on, and a few steps.  Values below the normal numbers may be zeros."""
    y = np.abs(_gelu(v))
    if kind == "f32":
        return (3 * v * v + 32) * 2.0 ** -24 * y + 2.0 ** -122
    own = np.where(v >= -7, 2.0 ** -15, np.where(v >= -11, 2.0 ** -12, 2.0 ** -10))
    return y * (own + R.HALF["bf16"] * (1 + own)) + 2.0 ** -122


@pytest.mark.parametrize("kind", ["bf16", "mx4", "mx4-f32"])
@pytest.mark.parametrize("T", [3, 4096])
def test_gelu_of_products(T, kind):
    """Rows of zeros and a bias: the activation of the bias, through the small and the large launches."""
    import torch
    import paper_2308_14711_amd as F
    out_kind = "f32" if kind == "mx4-f32" else "bf16"
    v = GRID if out_kind == "bf16" else np.random.default_rng(0).uniform(-13, 8, size=4096).astype(np.float32).astype(np.float64)
    N, u8 = len(v), torch.uint8
    bias, back = _up(v, out_kind)
    assert np.array_equal(back, v)
    a, kw = torch.zeros((T, 32), dtype=torch.bfloat16, device="cuda"), {}
    if kind != "bf16":
        a, kw = torch.zeros((T, 16), dtype=u8, device="cuda"), {"a_scales": torch.full((T, 1), 127, dtype=u8, device="cuda")}
    out = torch.empty((T, N), dtype=bias.dtype, device="cuda")
    F.fff_mx4_product(a, torch.zeros((N, 16), dtype=u8, device="cuda"), torch.full((N, 1), 127, dtype=u8, device="cuda"), out, bias=bias, act=F.ACT_GELU, **kw)
    assert (out == out[:1]).all()
    _within(out[0], _gelu(v), _gelu_tol(v, out_kind), "gelu [%s]" % F.fff_last_launch())


# a block a token; few pairs of wide leaves; tiles of rows; tiles through LDS
@pytest.mark.parametrize("T,D", [(28, 32), (28, 4096), (224, 32), (11200, 1024)])
def test_gelu_of_hidden_activations(T, D):
    """Tokens of zeros, a hidden bias, and a last matrix of ones on the diagonal: each leaf's activations are its outputs."""
    import torch
    import paper_2308_14711_amd as F
    E, L, u8 = 28, 128, torch.uint8
    v = np.resize(GRID, E * L).reshape(E, L)
    b1, _ = _up(v, "bf16")
    c2, s2 = R.quantise(np.broadcast_to(np.eye(L), (E, L, L)))
    idx = np.arange(T, dtype=np.int32) % E
    out = torch.empty((T, L), dtype=torch.bfloat16, device="cuda")
    nb = R.blocks(D)
    F.fff_leaf_forward_mx4(torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((E, L, 16 * nb), dtype=u8, device="cuda"),
                           torch.full((E, L, nb), 127, dtype=u8, device="cuda"), b1, _bytes(c2), _bytes(s2), torch.zeros((E, L), dtype=torch.bfloat16, device="cuda"),
                           _bytes(idx), None, F.ACT_GELU, out)
    assert (out.view(-1, E, L) == out[:E]).all()
    # (a rounded activation times one, plus zeros)
    _within(out[:E], _gelu(v), _gelu_tol(v, "bf16"), "gelu of %d tokens" % T)


# ---- where the leaves' values are rounded ----------------------------------------------------------------------


# a block a token; few pairs of wide leaves; tiles of rows; tiles through LDS
@pytest.mark.parametrize("T,D,k", [(20, 32, 1), (6, 32, 4), (20, 4096, 1), (7, 4096, 3), (300, 32, 2), (6000, 1024, 2)])
def test_mixture_weights_meet_sums_not_activations(T, D, k):
    """Hidden activations that bf16 holds exactly, pairs of which almost cancel: a weight that met them before their rounding would leave an
    error of their size, not of the difference's."""
    import torch
    import paper_2308_14711_amd as F
    E, L, O, u8 = 6, 128, 64, torch.uint8
    rng = np.random.default_rng(T + k)
    h = rng.integers(128, 256, size=(E, L)) / 128.0                       # 1 to 2 in steps of 2^-7
    w2 = np.zeros((E, O, L))
    w2[:, np.arange(O), np.arange(O)], w2[:, np.arange(O), np.arange(O) + O] = 1, -1
    c2, s2 = R.quantise(w2)
    idx = rng.integers(0, E, size=(T, k)).astype(np.int32)
    weight = rng.normal(size=(T, k)).astype(np.float32)
    out, nb = torch.empty((T, O), dtype=torch.bfloat16, device="cuda"), R.blocks(D)
    F.fff_leaf_forward_mx4(torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((E, L, 16 * nb), dtype=u8, device="cuda"),
                           torch.full((E, L, nb), 127, dtype=u8, device="cuda"), _up(h, "bf16")[0], _bytes(c2), _bytes(s2),
                           torch.zeros((E, O), dtype=torch.bfloat16, device="cuda"), _bytes(idx), _bytes(weight), F.ACT_RELU, out)
    parts = weight.astype(np.float64)[:, :, None] * (h[:, :O] - h[:, O:])[idx]
    want, size = parts.sum(1), np.abs(parts).sum(1)
    # the differences are exact; k products and sums in single precision, half a step of bf16
    tol = 2 * k * 2.0 ** -24 * size
    _within(out, want, tol + R.HALF["bf16"] * (np.abs(want) + tol), "mixture of %d tokens" % T)


@pytest.mark.parametrize("T,D,k", [(20, 32, 1), (6, 32, 4), (20, 4096, 1), (7, 4096, 3), (60, 32, 1), (300, 32, 2), (1500, 1024, 2), (6000, 1024, 2)])
def test_hidden_activations_hold_more_bits_than_bf16(T, D, k):
    """Activations a little above 1 to 2, whose small parts are what the differences of their pairs are made of: an activation rounded to bf16 is off by 2^-8."""
    import torch
    import paper_2308_14711_amd as F
    E, L, O = 6, 128, 64
    rng = np.random.default_rng(T + k)
    b1 = np.tile(rng.integers(128, 256, size=(E, O)) / 128.0, (1, 2))
    w1 = np.zeros((E, L, D))
    w1[:, :, 0] = rng.choice(R.GRID, size=(E, L)) * 2.0 ** -12
    w2 = np.zeros((E, O, L))
    w2[:, np.arange(O), np.arange(O)], w2[:, np.arange(O), np.arange(O) + O] = 1, -1
    c1, s1 = R.quantise(w1)
    c2, s2 = R.quantise(w2)
    w1 = R.values(c1, s1, D)
    x = np.zeros((T, D))
    x[:, 0] = rng.choice([1.0, -1.0, 0.5], size=T)
    idx = rng.integers(0, E, size=(T, k)).astype(np.int32)
    weight = rng.normal(size=(T, k)).astype(np.float32)
    out = torch.empty((T, O), dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(_up(x, "bf16")[0], _bytes(c1), _bytes(s1), _up(b1, "bf16")[0], _bytes(c2), _bytes(s2),
                           torch.zeros((E, O), dtype=torch.bfloat16, device="cuda"), _bytes(idx), _bytes(weight), F.ACT_RELU, out)
    h = x[:, 0][:, None, None] * w1[idx][:, :, :, 0] + b1[idx]
    g = np.abs(weight.astype(np.float64))[:, :, None]
    want = (weight.astype(np.float64)[:, :, None] * (h[:, :, :O] - h[:, :, O:])).sum(1)
    # an activation within 2^-15 of its value (and its sum of two terms within 2^-24), sums and products in single precision, half a step of bf16
    size = (g * (np.abs(h[:, :, :O]) + np.abs(h[:, :, O:]))).sum(1)
    tol = (2.0 ** -15 + (2 * k + 4) * 2.0 ** -24) * size
    _within(out, want, tol + R.HALF["bf16"] * (np.abs(want) + tol), "differences of %d tokens" % T)


# ---- every scale byte ------------------------------------------------------------------------------------------


def _every_code():
    """[256 scale bytes x 16 codes] rows of one block whose first element is the code, and the element's value."""
    c, s = np.zeros((256, 16, 16), np.uint8), np.zeros((256, 16, 1), np.uint8)
    c[:, :, 0], s[:, :, 0] = np.arange(16), np.arange(256)[:, None]
    c, s = c.reshape(4096, 16), s.reshape(4096, 1)
    return c, s, R.values(c, s, 1)[:, 0]


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_values_of_every_scale_byte_and_code(kind):
    """Values of 2^128 and more (4 and 6 at byte 253; 2, 3, 4 and 6 at 254) are infinities in either type; all others are exact, 255 is NaN."""
    import torch
    import paper_2308_14711_amd as F
    c, s, v = _every_code()
    for cols in (1, 8, 32):
        out = torch.empty((4096, cols), dtype=torch.float32 if kind == "f32" else torch.bfloat16, device="cuda")
        F.fff_mx4_dequantize(_bytes(c), _bytes(s), out)
        want = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
        got = out.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got[:, 0], want, equal_nan=True)
        assert np.isnan(got[4080:]).all() and not got[:4080, 1:].any()


@pytest.mark.parametrize("power", [-120, -60, 0, 60, 120])
@pytest.mark.parametrize("kind", ["bf16", "mx4"])
@pytest.mark.parametrize("T", [3, 4096])
def test_products_of_every_scale_byte_and_code(T, kind, power):
    """A power of two in every row against every code at every scale, through the small and the large launches.  bf16 rows meet the value as
    bf16 holds it, infinities included; rows of codes meet scale and code as they are."""
    import torch
    import paper_2308_14711_amd as F
    c, s, v = _every_code()
    if kind == "bf16":
        a, kw = torch.zeros((T, 32), dtype=torch.bfloat16, device="cuda"), {}
        a[:, 0] = 2.0 ** power
        v = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
    else:
        a, kw = torch.zeros((T, 16), dtype=torch.uint8, device="cuda"), {"a_scales": torch.full((T, 1), 127 + power, dtype=torch.uint8, device="cuda")}
        a[:, 0] = 2                                       # 1.0
    out = torch.empty((T, 4096), dtype=torch.bfloat16, device="cuda")
    F.fff_mx4_product(a, _bytes(c), _bytes(s), out, **kw)
    assert torch.equal(out.view(torch.int16), out[:1].view(torch.int16).expand(T, -1))
    want = v * 2.0 ** power
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    # exact, but for results below the normal numbers, which may be zeros
    _within(out[0], want, np.where(np.abs(want) < 2.0 ** -126, 2.0 ** -126, 0.0), "2^%d [%s]" % (power, F.fff_last_launch()))


# ---- routing: shares far below the largest ---------------------------------------------------------------------


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("E", [2, 60, 130, 600, 1500])
def test_shares_far_below_the_largest(E, normalise):
    """Differences of logits that single precision holds exactly: only the exponential is rounded, whose error does not grow with the difference."""
    import torch
    import paper_2308_14711_amd as F
    gap = np.arange(1, 641) / 8.0                                  # up to 80
    T = len(gap)
    l = np.full((T, E), -np.inf)
    l[:, E // 2] = 3.0
    l[:, E - 1 if E > 2 else 0] = 3.0 - gap
    logits, lv = _up(l)
    assert np.array_equal(lv, l)
    idx, w = torch.empty((T, 2), dtype=torch.int32, device="cuda"), torch.empty((T, 2), device="cuda")
    count = torch.empty((E + 1,), dtype=torch.int32, device="cuda")
    F.fff_moe_route(logits, 2, idx, w, count, normalise=normalise)
    want = R.route(l, 2, None, normalise)
    assert np.array_equal(idx.cpu().numpy(), want[0])
    # the exponential (two steps of 2^-23, and the product before it carried in two parts: one), a sum and a division
    few = 8 * 2.0 ** -24
    _within(w, want[1], few * want[1], "weights")
    # the gradient of the smaller weight: w0 w1 at both, through as many roundings again
    dw = np.zeros((T, 2), np.float32)
    dw[:, 1] = 1
    d = torch.empty((T, E), device="cuda")
    F.fff_moe_route_backward(logits, idx, count, d, dweight=_bytes(dw), normalise=normalise)
    g, size = R.route_backward(l, want[0], want[2], dw, None, None, normalise)
    _within(d, g, 3 * few * size, "dlogits")


# ---- many tokens of few leaves ---------------------------------------------------------------------------------


@pytest.mark.parametrize("E,T,k", [(1, 5000, 1), (1, 131072, 1), (1, 131073, 1), (2, 50001, 2), (3, 200003, 1), (16, 65536, 2), (16, 65537, 2), (64, 131071, 1),
                                   (130, 65000, 1), (125, 66000, 1)])
def test_many_tokens_of_few_leaves(E, T, k):
    """Matrices of zeros: a token is the mixture of its leaves' last biases, whichever launches group the pairs."""
    import torch
    import paper_2308_14711_amd as F
    D, L, O = 32, 16, 16
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, D), generator=g, device="cuda").bfloat16()
    b2 = torch.randn((E, O), generator=g, device="cuda").bfloat16()
    idx = torch.randint(-1, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    weight = torch.rand((T, k), generator=g, device="cuda")
    out = torch.full((T, O), -7.0, dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(x, z(E, L, 16), z(E, L, 1), torch.zeros((E, L), dtype=torch.bfloat16, device="cuda"), z(E, O, 16), z(E, O, 1), b2, idx, weight,
                           F.ACT_RELU, out)
    # 128 blocks of 1024 pairs are the most of which each adds up all counts (work that grows with their square), 8192 counts in all
    two = T * k <= 1 << 17 and -(-T * k // 1024) * E <= 8192
    assert ("group_spread_kernel" in F.fff_last_launch()) == two, F.fff_last_launch()
    parts = weight.double()[:, :, None] * torch.where(idx[:, :, None] < 0, 0.0, b2.double()[idx.clamp_min(0).long()])
    want, size = parts.sum(1).cpu().numpy(), parts.abs().sum(1).cpu().numpy()
    # k products and sums in single precision, half a step of bf16
    tol = 2 * k * 2.0 ** -24 * size
    _within(out, want, tol + R.HALF["bf16"] * (np.abs(want) + tol), "biases")


def test_a_token_s_activations_that_fill_a_block_s_lds():
    """32 leaves a token, 470 neurons of two values each: 60 KB, in one launch."""
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(60)
    dev, ref = _leaf_case(rng, 3, 32, 40, 20, 1, 470, True)
    out = torch.full((3, 1), -7.0, dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(*dev, F.ACT_GELU, out)
    assert F.fff_last_launch().endswith("mx4_token_kernel"), F.fff_last_launch()
    want, tol = R.leaves(*ref, "gelu")
    _within(out, want, tol, "leaves")
