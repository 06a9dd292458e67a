"""GPU parity of the operators on four-bit matrices and routed experts with their 64-bit forms (operators_reference.py), at the sizes,
values and masks where they can go wrong; and a run of them together."""
import numpy as np
import pytest

import operators_reference as R

pytestmark = pytest.mark.gpu
TYPES = ("bf16", "f32")


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _up(a, name="f32"):
    """A numpy array on the GPU, rounded to the type; and the values it then holds."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(_dt(name)).cuda()
    return t, t.float().cpu().numpy().astype(np.float64)


def _bytes(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _guarded(shape, dtype, fill):
    """A tensor with a row's worth of `fill` before and behind it, and a check that those stay."""
    import torch
    n, pad = int(np.prod(shape)), 64
    whole = torch.full((n + 2 * pad,), fill, dtype=dtype, device="cuda")
    t = whole[pad:pad + n].view(shape)

    def intact():
        edge = torch.cat([whole[:pad], whole[pad + n:]])
        return bool((edge == fill).all())
    return t, intact


def _within(got, want, tol, what):
    got = got.float().cpu().numpy().astype(np.float64)
    assert got.shape == want.shape
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        err, tol = np.where(same, 0, np.abs(got - want)), np.where(same, 0, tol)
    assert not np.isnan(err).any(), what + ": NaN where the definition has none, or the other way round"
    worst = np.unravel_index(np.argmax(err - tol), err.shape)
    assert (err <= tol).all(), "%s: %r off by %.3e, tolerance %.3e" % (what, worst, err[worst], np.broadcast_to(tol, err.shape)[worst])


# ---- quantisation ------------------------------------------------------------------------------------------


def _hard_rows(rng, shape, kind):
    x = rng.normal(size=shape) * np.exp(3 * rng.normal(size=shape[:-1] + (1,)))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.5])
    at = rng.random(shape) < 0.2
    x = np.where(at, rng.choice(ties, shape) * rng.choice([-1, 1], shape) * 4.0, x)
    flat = x.reshape(-1, shape[-1])
    for i, v in enumerate((0.0, -0.0, np.inf, -np.inf, np.nan, 3.3e38, 1.2e-38, 1e-40, -1e-44)):
        r = (7 * i) % len(flat)
        flat[r, (11 * i) % shape[-1]] = v
        if abs(v) < 1e-30:
            flat[r] = v      # a whole row of zeros, or of tiny values
    return x


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 3, 31), (1, 5, 32), (2, 33, 70), (1, 130, 257), (3, 7, 1000), (1, 1, 4096), (2, 129, 65), (1, 2000, 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_quantise(shape, transpose, kind):
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(sum(shape) + transpose)
    src, x = _up(_hard_rows(rng, shape, kind), kind)
    want_c, want_s = R.quantise(x.transpose(0, 2, 1) if transpose else x)
    codes, ok_c = _guarded(want_c.shape, torch.uint8, 0xA5)
    scales, ok_s = _guarded(want_s.shape, torch.uint8, 0xA5)
    F.fff_mx4_quantize(src, codes, scales, transpose=transpose)
    torch.cuda.synchronize()
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.array_equal(codes.cpu().numpy(), want_c)
    assert ok_c() and ok_s()
    for out_kind in TYPES:
        out, ok = _guarded(want_c.shape[:2] + (shape[1] if transpose else shape[2],), _dt(out_kind), -7.0)
        F.fff_mx4_dequantize(codes, scales, out)
        torch.cuda.synchronize()
        want = R.values(want_c, want_s, out.shape[-1])
        got = out.float().cpu().numpy().astype(np.float64)
        assert np.array_equal(got, want, equal_nan=True) and ok()


def test_rows_at_any_element_are_quantised_too():
    """A source that starts at any element and rows of odd length, and a value for every scale."""
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(3)
    for kind, start, cols in (("bf16", 1, 37), ("bf16", 3, 64), ("f32", 1, 33), ("f32", 3, 256)):
        whole, w = _up(rng.normal(size=(12 * cols + start,)), kind)
        src, x = whole[start:].view(12, cols), w[start:].reshape(12, cols)
        want_c, want_s = R.quantise(x)
        codes, scales = torch.empty(want_c.shape, dtype=torch.uint8, device="cuda"), torch.empty(want_s.shape, dtype=torch.uint8, device="cuda")
        F.fff_mx4_quantize(src, codes, scales)
        assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    x = np.ldexp(rng.uniform(1, 2, size=(277, 32)), np.arange(-149, 128)[:, None]).astype(np.float32)
    src, x = _up(x)
    want_c, want_s = R.quantise(x)
    codes, scales = torch.empty(want_c.shape, dtype=torch.uint8, device="cuda"), torch.empty(want_s.shape, dtype=torch.uint8, device="cuda")
    F.fff_mx4_quantize(src, codes, scales)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)


# ---- product -----------------------------------------------------------------------------------------------


def _matrix(rng, shape, scale):
    """A random matrix in four bits: codes, scales, values."""
    c, s = R.quantise((rng.normal(size=shape) * scale * np.exp(rng.normal(size=shape[:-1] + (1,)))).astype(np.float32).astype(np.float64))
    return c, s, R.values(c, s, shape[-1])


SIZES = [(1, 32, 16), (1, 8192, 64), (130, 4160, 140), (150, 8230, 40), (3000, 264, 3200), (2050, 100, 4100),
         (700, 1024, 1100), (900, 1030, 1000), (150, 4096, 4100), (1200, 40, 900), (1, 4096, 256), (3, 31, 5), (16, 128, 64), (17, 100, 33), (31, 160, 48), (33, 1000, 77), (64, 96, 130), (65, 257, 31),
         (129, 512, 257), (200, 777, 129), (257, 2048, 96), (300, 64, 515), (513, 320, 256)]


@pytest.mark.parametrize("kind", ["bf16", "mx4", "mx4-f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_product(size, kind):
    import torch
    import paper_2308_14711_amd as F
    T, K, N = size
    rng = np.random.default_rng(T + K + N)
    act = ("none", "relu", "gelu")[(T + N) % 3]
    out_kind = "f32" if kind == "mx4-f32" else "bf16"
    wc, ws, w = _matrix(rng, (N, K), K ** -0.5)
    bias, b = _up(rng.normal(size=N), out_kind)
    rows, a = _up(rng.normal(size=(T, K)), "bf16")
    a_scales = None
    if kind != "bf16":
        ac, asc = R.quantise(a)
        rows, a_scales, a = _bytes(ac), _bytes(asc), R.values(ac, asc, K)
    if (T + K) % 5 == 0:
        bias = b = None
    out, ok = _guarded((T, N), _dt(out_kind), -7.0)
    F.fff_mx4_product(rows, _bytes(wc), _bytes(ws), out, a_scales=a_scales, bias=bias,
                      act={"none": F.ACT_NONE, "relu": F.ACT_RELU, "gelu": F.ACT_GELU}[act])
    torch.cuda.synchronize()
    want, tol = R.product(a, w, b, act, out_kind)
    _within(out, want, tol, "product %s %s %s [%s]" % (size, kind, act, F.fff_last_launch()))
    assert ok()


@pytest.mark.parametrize("kind", ["bf16", "mx4"])
def test_product_rows_do_not_meet(kind):
    """NaN and infinity in one row of A reach that row alone; a NaN block of W one column alone; and huge values nothing else."""
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(8)
    for T, K, N in ((5, 100, 40), (150, 328, 140)):
        x = rng.normal(size=(T, K))
        x[1, K - 1] = np.nan
        x[3, 0] = np.inf
        rows, a = _up(x, "bf16")
        wc, ws, w = _matrix(rng, (N, K), 1.0)
        ws[7, -1] = 255
        w = R.values(wc, ws, K)
        kw = {}
        if kind == "mx4":
            ac, asc = R.quantise(a)
            rows, kw, a = _bytes(ac), {"a_scales": _bytes(asc)}, R.values(ac, asc, K)
        out = torch.empty((T, N), dtype=torch.bfloat16, device="cuda")
        F.fff_mx4_product(rows, _bytes(wc), _bytes(ws), out, **kw)
        got = out.float().cpu().numpy()
        odd = np.zeros((T, N), bool)
        odd[[1, 3]] = True
        odd[:, 7] = True
        assert np.isfinite(got[~odd]).all() and np.isnan(got[:, 7]).all() and np.isnan(got[1]).all() and not np.isfinite(got[3]).any()
        clean = np.delete(a, [1, 3], 0)
        want, tol = R.product(clean, np.delete(w, 7, 0), None, "none", "bf16")
        _within(torch.from_numpy(np.delete(np.delete(got, [1, 3], 0), 7, 1)), want, tol, "rows beside odd ones")


def test_product_of_misaligned_rows_and_results():
    """bf16 rows that start off a piece of 16 bytes are copied first; results may start at any element; the bias is optional."""
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(12)
    for T, K, N in ((4, 64, 24), (140, 136, 132)):
        whole, v = _up(rng.normal(size=T * K + 3), "bf16")
        a = v[3:].reshape(T, K)
        wc, ws, w = _matrix(rng, (N, K), K ** -0.5)
        big = torch.full((T * N + 6,), -7.0, dtype=torch.bfloat16, device="cuda")
        F.fff_mx4_product(whole[3:].view(T, K), _bytes(wc), _bytes(ws), big[1:1 + T * N].view(T, N))
        want, tol = R.product(a, w, None, "none", "bf16")
        _within(big[1:1 + T * N].view(T, N), want, tol, "misaligned")
        assert float(big[0]) == -7 and (big[1 + T * N:] == -7).all()


# ---- leaf networks -----------------------------------------------------------------------------------------

LEAVES = [
    # T,  k, E,  D,   O,   width, weights
    (1,   1, 1,  8,   1,   1,   False),
    (1,   2, 8,  256, 128, 64,  True),
    (7,   4, 4,  100, 36,  33,  True),
    (16,  2, 64, 136, 72,  40,  True),
    (33,  1, 5,  64,  40,  32,  False),
    (64,  2, 3,  96,  30,  17,  True),
    (90,  3, 16, 77,  51,  70,  True),
    (130, 1, 512, 64, 64,  32,  True),
    (300, 2, 2,  128, 264, 100, True),
    (260, 1, 1,  72,  136, 129, False),
    (400, 8, 8,  40,  24,  48,  True),
    # few pairs with leaves too large for a block a token
    (1,   1, 2,  1024, 520, 600, True),
    (3,   2, 4,  1096, 521, 601, True),
    (5,   6, 9,  2000, 264, 333, False),
    (2,   3, 3,  333, 4100, 128, True),
    # grouped: tiles of 16, 32 and 64 rows, and of 64 and 128 through LDS
    (60,  1, 4,  520, 1024, 700, True),
    (40,  2, 3,  96,  40,  36,  True),
    (150, 1, 3,  160, 130, 257, True),
    (700, 2, 5,  296, 136, 300, True),
    (4100, 8, 2, 136, 1032, 1100, True),
    (900, 2, 3, 1024, 640, 900, True),
    # more pairs, or leaves, than one block groups
    (4200, 8, 8, 40,  24,  16,  True),
    (5001, 8, 4100, 32, 16, 8,  True),
    (5003, 8, 700, 32, 16, 8,   False),
    (2100, 2, 40, 32, 16, 8,    True),
    (4700, 8, 9000, 32, 16, 8,  True),
]


def _leaf_case(rng, T, k, E, D, O, width, weighted, none=0.1):
    x, xv = _up(rng.normal(size=(T, D)), "bf16")
    c1, s1, w1 = _matrix(rng, (E, width, D), D ** -0.5)
    c2, s2, w2 = _matrix(rng, (E, O, width), width ** -0.5)
    b1, b1v = _up(0.2 * rng.normal(size=(E, width)), "bf16")
    b2, b2v = _up(0.2 * rng.normal(size=(E, O)), "bf16")
    idx = rng.integers(0, E, size=(T, k)).astype(np.int32)
    idx[rng.random((T, k)) < none] = -1
    if T > 5:
        idx[4] = -1                      # a token without a leaf
        idx[5, 0] = E                    # no leaf either
        idx[3] = idx[3, 0]               # the same leaf k times
    weight = rng.normal(size=(T, k)).astype(np.float32) if weighted else None
    dev = (x, _bytes(c1), _bytes(s1), b1, _bytes(c2), _bytes(s2), b2, _bytes(idx), None if weight is None else _bytes(weight))
    return dev, (xv, w1, b1v, w2, b2v, idx, None if weight is None else weight.astype(np.float64))


@pytest.mark.parametrize("case", LEAVES, ids=lambda c: "-".join(map(str, c)))
def test_leaves(case):
    import torch
    import paper_2308_14711_amd as F
    T, k, E, D, O, width, weighted = case
    rng = np.random.default_rng(sum(case[:6]))
    dev, ref = _leaf_case(rng, *case)
    act = ("relu", "gelu")[(T + width) % 2]
    out, ok = _guarded((T, O), torch.bfloat16, -7.0)
    F.fff_leaf_forward_mx4(*dev, {"relu": F.ACT_RELU, "gelu": F.ACT_GELU}[act], out)
    torch.cuda.synchronize()
    want, tol = R.leaves(*ref, act)
    _within(out, want, tol, "leaves %s %s [%s]" % (case, act, F.fff_last_launch()))
    assert ok()
    first = out.clone()
    for _ in range(3):                   # the same bits whatever order the grouping's atomics take
        F.fff_leaf_forward_mx4(*dev, {"relu": F.ACT_RELU, "gelu": F.ACT_GELU}[act], out)
        assert torch.equal(out.view(torch.int16), first.view(torch.int16))


def test_leaves_a_vector_of_indices_and_no_token_with_a_leaf():
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(77)
    for T in (20, 200):
        dev, ref = _leaf_case(rng, T, 1, 6, 64, 48, 40, False)
        out = torch.full((T, 48), -7.0, dtype=torch.bfloat16, device="cuda")
        F.fff_leaf_forward_mx4(*dev[:7], dev[7][:, 0].contiguous(), None, F.ACT_RELU, out)
        want, tol = R.leaves(*ref, "relu")
        _within(out, want, tol, "vector of indices")
        for k in (1, 3):
            out.fill_(-7.0)
            F.fff_leaf_forward_mx4(*dev[:7], torch.full((T, k), -1, dtype=torch.int32, device="cuda"), None, F.ACT_RELU, out)
            assert not out.any()


@pytest.mark.parametrize("E,T", [(4090, 60), (8000, 60), (4001, 1500), (3999, 2000), (20000, 90)])
def test_leaves_few_tokens_of_many_wide_leaves(E, T):
    """More leaves than the small groupings' tables hold.  Matrices of zeros: a token is the mixture of its leaves' last biases."""
    import torch
    import paper_2308_14711_amd as F
    D, L, O, k = 2048, 260, 520, 2
    if T > 1000:
        D, L, O, k = 64, 8, 16, 16       # (narrow leaves, more than four pairs a leaf)
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(E)
    x = torch.randn((T, D), generator=g, device="cuda").bfloat16()
    b1 = torch.randn((E, L), generator=g, device="cuda").bfloat16()
    b2 = torch.randn((E, O), generator=g, device="cuda").bfloat16()
    idx = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    idx[3] = E - 1
    weight = torch.rand((T, k), generator=g, device="cuda")
    out = torch.full((T, O), -7.0, dtype=torch.bfloat16, device="cuda")
    nb = R.blocks
    F.fff_leaf_forward_mx4(x, z(E, L, 16 * nb(D)), z(E, L, nb(D)), b1, z(E, O, 16 * nb(L)), z(E, O, nb(L)), b2, idx, weight, F.ACT_RELU, out)
    want = (weight.double()[:, :, None] * b2.double()[idx.long()]).sum(1).cpu().numpy()
    size = (weight.double()[:, :, None] * b2.double()[idx.long()].abs()).sum(1).cpu().numpy()
    # k products and sums in single precision, half a step of bf16
    _within(out, want, 2 * k * 2.0 ** -24 * size + R.HALF["bf16"] * (np.abs(want) + 2 * k * 2.0 ** -24 * size), "biases")


def test_leaves_with_more_results_than_a_launch_has_threads():
    """Rows of an odd number of columns are mixed a column a thread, here in two launches.  Matrices of zeros: mixtures of the last biases."""
    import torch
    import paper_2308_14711_amd as F
    T, D, L, O, k = (1 << 20) + 24, 32, 16, 4099, 2
    z = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    b2 = torch.randn((2, O), device="cuda").bfloat16()
    idx = torch.randint(0, 2, (T, k), device="cuda", dtype=torch.int32)
    weight = torch.rand((T, k), device="cuda")
    out = torch.full((T, O), -7.0, dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(torch.zeros((T, D), dtype=torch.bfloat16, device="cuda"), z(2, L, 16), z(2, L, 1), torch.zeros((2, L), dtype=torch.bfloat16, device="cuda"),
                           z(2, O, 16), z(2, O, 1), b2, idx, weight, F.ACT_RELU, out)
    split = (((1 << 24) - 1) * 256) // O
    assert split < T
    for rows in (slice(0, 30), slice(split - 30, split + 30), slice(T - 30, T)):
        parts = weight[rows].double()[:, :, None] * b2.double()[idx[rows].long()]
        want, size = parts.sum(1).cpu().numpy(), parts.abs().sum(1).cpu().numpy()
        # k products and sums in single precision, half a step of bf16
        _within(out[rows], want, 2 * k * 2.0 ** -24 * size + R.HALF["bf16"] * (np.abs(want) + 2 * k * 2.0 ** -24 * size), "mixtures")


def test_leaves_all_tokens_in_one_of_many():
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(78)
    dev, ref = _leaf_case(rng, 300, 2, 40, 64, 32, 32, True, none=0.0)
    ref[5][:] = 17
    dev[7].fill_(17)
    out = torch.full((300, 32), -7.0, dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(*dev, F.ACT_GELU, out)
    want, tol = R.leaves(*ref, "gelu")
    _within(out, want, tol, "one leaf")


# ---- routing -----------------------------------------------------------------------------------------------

ROUTES = [
    # T,  E,   k, type,  normalise, mask
    (1,   1,   1, "f32", True,  False),
    (5,   3,   2, "f32", False, True),
    (64,  8,   8, "bf16", True, False),
    (70,  7,   3, "bf16", True, True),
    (300, 16,  2, "f32", True,  True),
    (257, 24,  6, "bf16", False, False),
    (513, 64,  4, "f32", True,  False),
    (100, 100, 5, "bf16", True, True),
    (333, 128, 2, "bf16", True, True),
    (129, 512, 8, "f32", False, True),
    (50,  513, 32, "f32", True, False),
    (40,  1000, 7, "bf16", True, True),
    (33,  2047, 9, "bf16", False, False),
    (21,  2048, 2, "f32", True, True),
    (17,  4096, 32, "f32", True, False),
    (9,   4095, 3, "bf16", True, True),
    (5000, 60, 2, "f32", True,  True),
    (40000, 8, 2, "bf16", True, True),
]


def _logits(rng, T, E, kind, odd=True):
    l = rng.normal(size=(T, E)) * 2 + rng.normal(size=E)
    if odd and T > 12:
        l[0] = -np.inf                               # nothing to choose
        l[1] = np.nan
        l[2, : max(1, E // 2)] = -np.inf             # (for large k, fewer than k to choose)
        l[3] = 1.5                                   # all equal
        l[4] = -3e38                                 # the lowest values: a row like another
        l[5, E // 2] = np.nan
        l[6, E - 1] = 80.0
        l[7] = rng.choice([0.0, -0.0, 1.0], E)       # ties of both zeros
        l[8, 1:] = -np.inf
    return _up(l, kind)


def _rtol(l, E):
    """Shares of a softmax in single precision: the difference to the maximum (half a step of it), the exponential (4 steps), a sum of E
    positive terms along the registers of a lane and over the lanes (72 additions at most), a division; twice that."""
    d = np.where(np.isfinite(l), l, 0)
    spread = min(float((d.max(1) - d.min(1)).max()), 110.0)
    return 2 * (spread + 8 + 72 + 2) * 2.0 ** -24


@pytest.mark.parametrize("case", ROUTES, ids=lambda c: "-".join(map(str, c)))
def test_route(case):
    import torch
    import paper_2308_14711_amd as F
    T, E, k, kind, normalise, masked = case
    rng = np.random.default_rng(T + E + k)
    logits, l = _logits(rng, T, E, kind)
    mask = (rng.random(T) < 0.8) if masked else None
    d_mask = None if mask is None else (_bytes(mask) if T % 2 else _bytes(mask.astype(np.uint8)))
    idx, ok_i = _guarded((T, k), torch.int32, -9)
    weight, ok_w = _guarded((T, k), torch.float32, -9.0)
    count, ok_c = _guarded((E + 1,), torch.int32, -9)
    mean, ok_m = _guarded((E,), torch.float32, -9.0)
    loss, ok_l = _guarded((2,), torch.float32, -9.0)
    want = R.route(l, k, mask, normalise)
    rtol = _rtol(l, E)

    def check():
        torch.cuda.synchronize()
        assert np.array_equal(idx.cpu().numpy(), want[0])
        # (shares below the smallest normal number may be flushed: exp(-88))
        _within(weight, want[1], rtol * want[1] + 1e-37, "weight")
        assert ok_i() and ok_w()
    F.fff_moe_route(logits, k, idx, weight, token_mask=d_mask, normalise=normalise)
    check()
    idx.fill_(-9), weight.fill_(-9)
    F.fff_moe_route(logits, k, idx, weight, count, mean, loss, token_mask=d_mask, normalise=normalise)
    check()
    assert np.array_equal(count.cpu().numpy(), want[2])
    # sums over the tokens: along a lane, over groups, waves and blocks, fewer than 400 additions of positive terms
    sums = rtol + 400 * 2.0 ** -24
    _within(mean, want[3], sums * want[3] + 1e-37, "prob_mean")
    # (a token of the lowest values has lse = -3e38 and lse^2 = 9e76: infinity is what single precision rounds such a mean to)
    want_loss = np.where(want[4] > np.finfo(np.float32).max, np.inf, want[4])
    _within(loss, want_loss, np.where(np.isinf(want_loss), 0, 3 * sums * np.abs(want[4])) + 1e-37, "loss")
    assert ok_c() and ok_m() and ok_l()
    only = torch.empty_like(loss)
    F.fff_moe_route(logits, k, idx, weight, loss=only, token_mask=d_mask, normalise=normalise)
    assert torch.equal(only.view(torch.int32), loss.view(torch.int32))       # always in the same order


@pytest.mark.parametrize("case", ROUTES, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("parts", ["both", "weights", "losses", "none"])
def test_route_backward(case, parts):
    import torch
    import paper_2308_14711_amd as F
    T, E, k, kind, normalise, masked = case
    rng = np.random.default_rng(T + E + k + 1)
    logits, l = _logits(rng, T, E, kind)
    mask = (rng.random(T) < 0.8) if masked else None
    d_mask = None if mask is None else _bytes(mask)
    idx, _, count, *_ = R.route(l, k, mask, normalise)
    dw = rng.normal(size=(T, k)).astype(np.float32) if parts in ("both", "weights") else None
    dl = np.array([0.3, -0.02], np.float32) if parts in ("both", "losses") else None
    if dw is not None:
        dw[idx < 0] = np.nan                         # slots without an expert are not read
    d, ok = _guarded((T, E), _dt(kind), -9.0)
    F.fff_moe_route_backward(logits, _bytes(idx), _bytes(count.astype(np.int32)), d, dweight=None if dw is None else _bytes(dw),
                             dloss=None if dl is None else _bytes(dl), token_mask=d_mask, normalise=normalise)
    torch.cuda.synchronize()
    want, size = R.route_backward(l, idx, count, dw, dl, mask, normalise)
    # every term carries a share (_rtol) or two and a handful of roundings; bf16 results half a step more
    tol = 3 * _rtol(l, E) * size + R.HALF[kind] * np.abs(want) + 1e-36
    _within(d, want, tol, "dlogits")
    assert ok()
    # rows that take no part, and logits of minus infinity or NaN, have no gradient
    got = d.float().cpu().numpy()
    assert not got[~R.route(l, 1, mask)[7]].any() and not got[np.isnan(l) | (l == -np.inf)].any()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("E,k", [(65, 3), (128, 6), (129, 12), (250, 7), (256, 32), (260, 24), (512, 8), (700, 25), (1024, 31), (1300, 6), (2048, 32), (4096, 20)])
def test_route_chooses_among_few_and_many_that_are_equal(E, k, kind):
    """Rows with any number of finite logits, all of them equal or all but a few: whether choices are taken one by one or at once, ties
    go to the lower index."""
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(E * k)
    there = [0, 1, 2, k - 1, k, k + 1, 31, 32, 33, 60, 63, 64, 65, 66, 80, E - 1, E]
    T = 4 * len(there)
    l = np.full((T, E), -np.inf)
    for t in range(T):
        n = min(there[t // 4], E)
        at = rng.permutation(E)[:n]
        l[t, at] = rng.normal() * 4                       # one value for all
        if t % 4 == 1:
            l[t, at] = rng.normal(size=n)
        if t % 4 == 2:
            l[t, at[: n // 2]] += 1.0                     # two
        if t % 4 == 3:
            few = at[: min(n, k - 1)]
            l[t, few] += rng.integers(1, 4, len(few))     # fewer above than are to be chosen
    order = rng.permutation(T)                            # rows of all kinds share a wave
    logits, l = _up(l[order], kind)
    idx, w = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda")
    count = torch.empty((E + 1,), dtype=torch.int32, device="cuda")
    want = R.route(l, k)
    for stats in (None, count):
        F.fff_moe_route(logits, k, idx, w, stats)
        assert np.array_equal(idx.cpu().numpy(), want[0])
        _within(w, want[1], _rtol(l, E) * want[1] + 1e-37, "weight")
    assert np.array_equal(count.cpu().numpy(), want[2])


def test_route_logits_of_plus_infinity_share_the_token():
    import torch
    import paper_2308_14711_amd as F
    l = np.zeros((14, 10))
    l[9, [2, 7]] = np.inf
    logits, lv = _up(l)
    idx, w = torch.empty((14, 3), dtype=torch.int32, device="cuda"), torch.empty((14, 3), device="cuda")
    loss = torch.empty((2,), device="cuda")
    F.fff_moe_route(logits, 3, idx, w, loss=loss)
    assert idx[9].tolist() == [2, 7, 0] and w[9].tolist() == [0.5, 0.5, 0.0] and loss[1] == float("inf") and torch.isfinite(loss[0])


def test_route_without_tokens():
    import torch
    import paper_2308_14711_amd as F
    for T, mask in ((0, None), (6, torch.zeros(6, dtype=torch.bool, device="cuda"))):
        logits = torch.randn((T, 300), device="cuda")
        idx, w = torch.full((T, 2), 5, dtype=torch.int32, device="cuda"), torch.full((T, 2), 5.0, device="cuda")
        count, mean, loss = torch.full((301,), 5, dtype=torch.int32, device="cuda"), torch.full((300,), 5.0, device="cuda"), torch.full((2,), 5.0, device="cuda")
        F.fff_moe_route(logits, 2, idx, w, count, mean, loss, token_mask=mask)
        assert not count.any() and not mean.any() and not loss.any() and (idx == -1).all() and not w.any()
        d = torch.full((T, 300), 5.0, device="cuda")
        F.fff_moe_route_backward(logits, idx, count, d, dweight=w, dloss=torch.ones(2, device="cuda"), token_mask=mask)
        assert not d.any()


def test_route_backward_ignores_indices_out_of_range_and_adds_repeated_ones():
    import torch
    import paper_2308_14711_amd as F
    rng = np.random.default_rng(9)
    logits, l = _up(rng.normal(size=(40, 12)))
    idx = rng.integers(0, 12, size=(40, 4)).astype(np.int32)
    idx[:, 1] = idx[:, 0]
    idx[3:9, 2] = 12
    idx[5:7, 3] = -5
    count = np.append(np.bincount(idx[(idx >= 0) & (idx < 12)], minlength=12), 40).astype(np.int32)
    dw = rng.normal(size=(40, 4)).astype(np.float32)
    for normalise in (True, False):
        d = torch.empty((40, 12), device="cuda")
        F.fff_moe_route_backward(logits, _bytes(idx), _bytes(count), d, dweight=_bytes(dw), normalise=normalise)
        want, size = R.route_backward(l, idx, count, dw, None, None, normalise)
        _within(d, want, 3 * _rtol(l, 12) * size + 1e-36, "dlogits")


# ---- far offsets ---------------------------------------------------------------------------------------------


def test_rows_beyond_four_gigabytes():
    """Offsets that pass 32 bits: the last rows of large matrices, against the 64-bit forms of these rows."""
    import torch
    import paper_2308_14711_amd as F
    n64 = lambda t: t.float().cpu().numpy().astype(np.float64)
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(4)
    T, D, tail = 540000, 4100, 70
    x = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")         # 4.4 GB
    for part in x.split(60000):
        part.normal_()
    nb = R.blocks(D)
    codes, scales, back = u8(T, 16 * nb), u8(T, nb), torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    F.fff_mx4_quantize(x, codes, scales)
    F.fff_mx4_dequantize(codes, scales, back)
    c, s = R.quantise(n64(x[-tail:]))
    assert np.array_equal(codes[-tail:].cpu().numpy(), c) and np.array_equal(scales[-tail:].cpu().numpy(), s)
    assert np.array_equal(n64(back[-tail:]), R.values(c, s, D))
    del back
    # products: codes, bf16 rows that are copied (4100 is no multiple of 8), and bf16 rows as they are
    wc, ws, w = _matrix(rng, (40, D), D ** -0.5)
    out = torch.empty((T, 40), dtype=torch.bfloat16, device="cuda")
    F.fff_mx4_product(codes, _bytes(wc), _bytes(ws), out, a_scales=scales)
    want, tol = R.product(R.values(c, s, D), w, None, "none", "bf16")
    _within(out[-tail:], want, tol, "codes")
    del codes, scales
    F.fff_mx4_product(x, _bytes(wc), _bytes(ws), out)
    want, tol = R.product(n64(x[-tail:]), w, None, "none", "bf16")
    _within(out[-tail:], want, tol, "copied rows")
    rows = x.view(-1)[:539000 * 4104].view(539000, 4104)
    wc, ws, w = _matrix(rng, (40, 4104), 4104 ** -0.5)
    F.fff_mx4_product(rows, _bytes(wc), _bytes(ws), out[:539000])
    want, tol = R.product(n64(rows[-tail:]), w, None, "none", "bf16")
    _within(out[539000 - tail:539000], want, tol, "rows as they are")
    # leaves: tokens gathered from all over
    T, D = rows.shape
    c1, s1, w1 = _matrix(rng, (3, 32, D), D ** -0.5)
    c2, s2, w2 = _matrix(rng, (3, 24, 32), 32 ** -0.5)
    b1, b1v = _up(rng.normal(size=(3, 32)), "bf16")
    b2, b2v = _up(rng.normal(size=(3, 24)), "bf16")
    idx = torch.randint(0, 3, (T,), device="cuda", dtype=torch.int32)
    y = torch.empty((T, 24), dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(rows, _bytes(c1), _bytes(s1), b1, _bytes(c2), _bytes(s2), b2, idx, None, F.ACT_RELU, y)
    for at in (slice(0, tail), slice(T - tail, T)):
        want, tol = R.leaves(n64(rows[at]), w1, b1v, w2, b2v, idx[at].cpu().numpy()[:, None], None, "relu")
        _within(y[at], want, tol, "leaves")
    del x, rows
    torch.cuda.empty_cache()
    # routing: 2^31 and more elements
    T, E, k = (1 << 22) + 5, 520, 2
    logits = torch.empty((T, E), dtype=torch.bfloat16, device="cuda")
    for part in logits.split(1 << 19):
        part.normal_()
    idx, weight, d = torch.empty((T, k), dtype=torch.int32, device="cuda"), torch.empty((T, k), device="cuda"), torch.empty_like(logits)
    count = torch.empty((E + 1,), dtype=torch.int32, device="cuda")
    F.fff_moe_route(logits, k, idx, weight, count)
    assert int(count[E]) == T and int(count[:E].sum()) == T * k
    dw = torch.randn((T, k), device="cuda")
    F.fff_moe_route_backward(logits, idx, count, d, dweight=dw)
    l = n64(logits[-tail:])
    want = R.route(l, k)
    assert np.array_equal(idx[-tail:].cpu().numpy(), want[0])
    _within(weight[-tail:], want[1], _rtol(l, E) * want[1], "weight")
    g, size = R.route_backward(l, want[0], count.cpu().numpy(), n64(dw[-tail:]), None)
    _within(d[-tail:], g, 3 * _rtol(l, E) * size + R.HALF["bf16"] * np.abs(g) + 1e-36, "dlogits")


# ---- together ----------------------------------------------------------------------------------------------


def _mixture(rng, T, E, k, D, O, width):
    """Everything a mixture holds and works in."""
    import torch
    e = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")
    s = {"x": _up(rng.normal(size=(T, D)), "bf16")[0], "gate": _up(rng.normal(size=(E, D)) * D ** -0.5)[0],
         "w1": _up(rng.normal(size=(E, width, D)) * D ** -0.5, "bf16")[0], "w2": _up(rng.normal(size=(E, width, O)) * width ** -0.5, "bf16")[0],
         "b1": _up(0.1 * rng.normal(size=(E, width)), "bf16")[0], "b2": _up(0.1 * rng.normal(size=(E, O)), "bf16")[0],
         "logits": e(T, E), "idx": e(T, k, dtype=torch.int32), "weight": e(T, k), "count": e(E + 1, dtype=torch.int32), "loss": e(2),
         "out": e(T, O, dtype=torch.bfloat16), "dweight": _up(rng.normal(size=(T, k)))[0], "dloss": _up(np.array([0.01, 0.001]))[0],
         "dlogits": e(T, E)}
    nb = R.blocks
    u8 = torch.uint8
    s["c1"], s["s1"] = e(E, width, 16 * nb(D), dtype=u8), e(E, width, nb(D), dtype=u8)
    s["c2"], s["s2"] = e(E, O, 16 * nb(width), dtype=u8), e(E, O, nb(width), dtype=u8)
    return s


def _mixture_pass(F, s, k, stream=None):
    F.fff_moe_route(s["logits"], k, s["idx"], s["weight"], s["count"], None, s["loss"], stream=stream)
    F.fff_leaf_forward_mx4(s["x"], s["c1"], s["s1"], s["b1"], s["c2"], s["s2"], s["b2"], s["idx"], s["weight"], F.ACT_GELU, s["out"], stream=stream)
    F.fff_moe_route_backward(s["logits"], s["idx"], s["count"], s["dlogits"], dweight=s["dweight"], dloss=s["dloss"], stream=stream)


@pytest.mark.parametrize("T", [3, 150])
def test_a_mixture_of_experts_from_logits_to_gradients(T):
    """Weights quantised, experts chosen, their networks mixed, the logits' gradient: against the 64-bit forms throughout; then the same
    pass captured into a graph and replayed on other inputs beside eager calls."""
    import torch
    import paper_2308_14711_amd as F
    E, k, D, O, width = 6, 2, 72, 40, 50
    rng = np.random.default_rng(T)
    s = _mixture(rng, T, E, k, D, O, width)
    F.fff_mx4_quantize(s["w1"], s["c1"], s["s1"])
    F.fff_mx4_quantize(s["w2"], s["c2"], s["s2"], transpose=True)
    n64 = lambda t: t.float().cpu().numpy().astype(np.float64)

    def check():
        torch.cuda.synchronize()
        l = n64(s["logits"])
        idx, w, count, _, loss, *_ = R.route(l, k)
        assert np.array_equal(s["idx"].cpu().numpy(), idx) and np.array_equal(s["count"].cpu().numpy(), count)
        q1, q2 = R.quantise(n64(s["w1"])), R.quantise(n64(s["w2"]).transpose(0, 2, 1))
        want, tol = R.leaves(n64(s["x"]), R.values(*q1, D), n64(s["b1"]), R.values(*q2, width), n64(s["b2"]), idx, n64(s["weight"]), "gelu")
        _within(s["out"], want, tol, "mixture")
        _within(s["weight"], w, _rtol(l, E) * w, "weight")
        _within(s["loss"], loss, 3 * (_rtol(l, E) + 400 * 2.0 ** -24) * loss, "loss")
        d, size = R.route_backward(l, idx, count, n64(s["dweight"]), n64(s["dloss"]))
        _within(s["dlogits"], d, 3 * _rtol(l, E) * size + 1e-36, "dlogits")
    torch.mm(s["x"].float(), s["gate"].t().contiguous(), out=s["logits"])
    _mixture_pass(F, s, k)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _mixture_pass(F, s, k)
    for i in range(3):
        s["x"].normal_()
        torch.mm(s["x"].float(), s["gate"].t().contiguous(), out=s["logits"])
        for name in ("out", "dlogits", "weight", "loss"):
            s[name].fill_(float("nan"))
        graph.replay()
        check()
        other = torch.empty_like(s["out"])       # eager work of its own between the replays
        F.fff_leaf_forward_mx4(s["x"], s["c1"], s["s1"], s["b1"], s["c2"], s["s2"], s["b2"], s["idx"], s["weight"], F.ACT_GELU, other)
        assert torch.equal(other.view(torch.int16), s["out"].view(torch.int16))


def test_two_streams_and_two_graphs_at_once():
    """Scratch is of the call's own: calls on two streams, and replays of two graphs, do not meet."""
    import torch
    import paper_2308_14711_amd as F
    E, k, D, O, width, T = 5, 2, 64, 96, 64, 500
    rng = np.random.default_rng(1)
    both = [_mixture(np.random.default_rng(i), T, E, k, D, O, width) for i in range(2)]
    want = []
    for s in both:
        F.fff_mx4_quantize(s["w1"], s["c1"], s["s1"])
        F.fff_mx4_quantize(s["w2"], s["c2"], s["s2"], transpose=True)
        s["logits"].copy_(torch.from_numpy(rng.normal(size=(T, E)).astype(np.float32)))
        _mixture_pass(F, s, k)
        torch.cuda.synchronize()
        want.append({n: s[n].clone() for n in ("out", "loss", "dlogits", "count")})
    streams = [torch.cuda.Stream() for _ in both]
    graphs = [torch.cuda.CUDAGraph() for _ in both]
    for s, g in zip(both, graphs):
        with torch.cuda.graph(g):
            _mixture_pass(F, s, k)

    def same():
        torch.cuda.synchronize()
        for s, w in zip(both, want):
            for n, t in w.items():
                assert torch.equal(s[n].view(torch.uint8), t.view(torch.uint8)), n
                s[n].zero_()
        torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(both, streams):
            _mixture_pass(F, s, k, stream=st)
    same()
    for _ in range(5):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    same()


def test_a_tree_with_four_bit_leaves():
    """The descent's indices and the leaves in four bits: an FFF, as fff_forward_hard runs it in bf16."""
    import torch
    import fff_workloads as W
    import paper_2308_14711_amd as F
    from fff_testlib import to_device
    w = W.make_layer("mx4_tree", 700, 128, 64, 4, 32, W.ACT_GELU, W.DTYPE_BF16, seed=2)
    dev = to_device(w)
    idx = torch.empty((w.T,), dtype=torch.int32, device="cuda")
    F.fff_descend(dev["x"], dev["node_w"], dev["node_b"], w.depth, idx)
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    c1, s1, c2, s2 = u8(16, 32, 64), u8(16, 32, 4), u8(16, 64, 16), u8(16, 64, 1)
    F.fff_mx4_quantize(dev["leaf_w1"], c1, s1)
    F.fff_mx4_quantize(dev["leaf_w2"], c2, s2, transpose=True)
    out = torch.empty((w.T, w.O), dtype=torch.bfloat16, device="cuda")
    F.fff_leaf_forward_mx4(dev["x"], c1, s1, dev["leaf_b1"], c2, s2, dev["leaf_b2"], idx, None, w.act, out)
    n64 = lambda t: t.float().cpu().numpy().astype(np.float64)
    w1 = R.values(*R.quantise(n64(dev["leaf_w1"])), w.D)
    w2 = R.values(*R.quantise(n64(dev["leaf_w2"]).transpose(0, 2, 1)), 32)
    want, tol = R.leaves(n64(dev["x"]), w1, n64(dev["leaf_b1"]), w2, n64(dev["leaf_b2"]), idx.cpu().numpy()[:, None], None, "gelu")
    _within(out, want, tol, "tree")
