"""Host-side checks of the operators on four-bit matrices and routed experts: what is refused before any HIP call, what sizes of
scratch are, what the binding checks; and the reference's own gradient against differences."""
import ctypes

import numpy as np
import pytest

import operators_reference as R

OK, NULL, SHAPE, DTYPE, RANGE, UNSUP, WORKSPACE, ALIAS = 0, 1, 2, 3, 4, 5, 6, 8
F32, BF16 = 0, 1
P = ctypes.c_void_p
BIG = 1 << 40      # addresses far apart, never followed


@pytest.fixture(scope="module")
def L():
    import paper_2308_14711_amd as F
    return F.lib()


def test_route_refusals(L):
    def call(**kw):
        a = dict(logits=P(BIG), mask=None, E=8, k=2, idx=P(2 * BIG), weight=P(3 * BIG), count=None, mean=None, loss=None, T=4, dtype=F32,
                 scratch=None, bytes=0)
        a.update(kw)
        return L.fff_moe_route(a["logits"], a["mask"], a["E"], a["k"], 1, a["idx"], a["weight"], a["count"], a["mean"], a["loss"], None,
                               a["T"], a["dtype"], a["scratch"], a["bytes"])
    assert call(T=0) == OK
    assert call(logits=None) == NULL and call(idx=None) == NULL and call(weight=None) == NULL
    assert call(dtype=2) == DTYPE
    assert call(E=0) == RANGE and call(E=4097) == RANGE and call(k=0) == RANGE and call(k=9) == RANGE
    assert call(E=64, k=33) == RANGE and call(T=-1) == RANGE and call(T=1 << 31) == RANGE
    assert call(T=1 << 30, k=2) == RANGE                              # slots beyond 32-bit indices
    assert call(T=1 << 30, E=4096, k=1) == SHAPE
    need = L.fff_route_scratch_bytes(4, 8)
    assert need > 0
    assert call(loss=P(5 * BIG)) == NULL                              # statistics need scratch
    assert call(loss=P(5 * BIG), scratch=P(6 * BIG + 128), bytes=need) == WORKSPACE
    assert call(loss=P(5 * BIG), scratch=P(6 * BIG), bytes=need - 1) == WORKSPACE
    assert call(idx=P(BIG + 64)) == ALIAS and call(weight=P(2 * BIG + 16)) == ALIAS
    assert call(mask=P(2 * BIG)) == ALIAS
    assert call(count=P(5 * BIG), scratch=P(5 * BIG), bytes=need) == ALIAS
    assert L.fff_route_scratch_bytes(-1, 8) == 0 and L.fff_route_scratch_bytes(4, 5000) == 0
    assert L.fff_route_scratch_bytes(100, 64) <= L.fff_route_scratch_bytes(100000, 64)


def test_route_backward_refusals(L):
    def call(**kw):
        a = dict(logits=P(BIG), idx=P(2 * BIG), count=P(3 * BIG), dweight=P(4 * BIG), dloss=P(5 * BIG), dlogits=P(6 * BIG), E=8, k=2, T=4, dtype=BF16)
        a.update(kw)
        return L.fff_moe_route_backward(a["logits"], None, a["E"], a["k"], 1, a["idx"], a["count"], a["dweight"], a["dloss"], a["dlogits"], None,
                                        a["T"], a["dtype"])
    assert call(T=0) == OK
    assert call(logits=None) == NULL and call(dlogits=None) == NULL and call(idx=None) == NULL and call(count=None) == NULL
    assert call(dtype=7) == DTYPE and call(E=5000) == RANGE and call(k=0) == RANGE
    assert call(dlogits=P(BIG)) == ALIAS and call(dlogits=P(4 * BIG + 8)) == ALIAS


def test_quantise_refusals(L):
    def q(**kw):
        a = dict(src=P(BIG), codes=P(2 * BIG), scales=P(3 * BIG), t=0, batch=1, rows=4, cols=64, dtype=F32)
        a.update(kw)
        return L.fff_mx4_quantize(a["src"], a["codes"], a["scales"], a["t"], None, a["batch"], a["rows"], a["cols"], a["dtype"])
    assert q(batch=0) == OK
    assert q(src=None) == NULL and q(codes=None) == NULL and q(scales=None) == NULL
    assert q(dtype=5) == DTYPE and q(batch=-1) == RANGE
    assert q(rows=0) == SHAPE and q(cols=0) == SHAPE and q(rows=1 << 30, cols=1 << 20) == SHAPE
    assert q(rows=1 << 38, cols=1) == SHAPE                           # blocks of 32 count whole
    assert q(batch=1 << 32, rows=1, cols=1, t=1) == SHAPE
    assert q(codes=P(2 * BIG + 8)) == UNSUP
    assert q(codes=P(BIG + 16)) == ALIAS and q(scales=P(2 * BIG + 4)) == ALIAS

    def d(**kw):
        a = dict(codes=P(2 * BIG), scales=P(3 * BIG), out=P(BIG), rows=4, cols=64, dtype=F32)
        a.update(kw)
        return L.fff_mx4_dequantize(a["codes"], a["scales"], a["out"], None, a["rows"], a["cols"], a["dtype"])
    assert d(rows=0) == OK
    assert d(codes=None) == NULL and d(out=None) == NULL and d(scales=None) == NULL
    assert d(cols=0) == SHAPE and d(rows=-1) == RANGE and d(rows=1 << 39) == SHAPE and d(dtype=3) == DTYPE
    assert d(codes=P(2 * BIG + 4)) == UNSUP and d(out=P(2 * BIG)) == ALIAS


def test_product_refusals(L):
    def call(**kw):
        a = dict(a=P(BIG), s=None, w=P(2 * BIG), ws=P(3 * BIG), bias=None, act=2, out=P(4 * BIG), T=4, K=64, N=16, dtype=BF16, scratch=None, bytes=0)
        a.update(kw)
        return L.fff_mx4_product(a["a"], a["s"], a["w"], a["ws"], a["bias"], a["act"], a["out"], None, a["T"], a["K"], a["N"], a["dtype"],
                                 a["scratch"], a["bytes"])
    assert call(T=0) == OK
    assert call(a=None) == NULL and call(w=None) == NULL and call(ws=None) == NULL and call(out=None) == NULL
    assert call(act=3) == UNSUP and call(dtype=F32) == UNSUP and call(dtype=9) == DTYPE
    assert call(T=-1) == RANGE and call(K=0) == SHAPE and call(N=0) == SHAPE and call(K=(1 << 22) + 1) == SHAPE
    assert call(T=1 << 30, N=1 << 12) == SHAPE
    assert call(w=P(2 * BIG + 8)) == UNSUP and call(a=P(BIG + 8), s=P(5 * BIG)) == UNSUP
    assert call(K=60) == NULL and call(a=P(BIG + 2)) == NULL          # rows that are copied need scratch
    need = L.fff_mx4_product_scratch_bytes(4, 60)
    assert need >= 4 * 64 * 2
    assert call(K=60, scratch=P(6 * BIG), bytes=need - 1) == WORKSPACE and call(K=60, scratch=P(6 * BIG + 16), bytes=need) == WORKSPACE
    assert call(K=60, scratch=P(4 * BIG), bytes=need) == ALIAS
    assert call(out=P(BIG)) == ALIAS and call(out=P(2 * BIG)) == ALIAS and call(bias=P(4 * BIG)) == ALIAS
    assert L.fff_mx4_product_scratch_bytes(-1, 60) == 0


def test_leaf_refusals(L):
    need = L.fff_leaf_mx4_scratch_bytes(4, 64, 32, 8, 2, 40)
    assert need > 0

    def call(**kw):
        a = dict(x=P(BIG), w1=P(2 * BIG), s1=P(3 * BIG), b1=P(4 * BIG), w2=P(5 * BIG), s2=P(6 * BIG), b2=P(7 * BIG), idx=P(8 * BIG), weight=None,
                 E=8, k=2, width=40, act=1, out=P(9 * BIG), T=4, D=64, O=32, dtype=BF16, scratch=P(10 * BIG), bytes=need)
        a.update(kw)
        return L.fff_leaf_forward_mx4(a["x"], a["w1"], a["s1"], a["b1"], a["w2"], a["s2"], a["b2"], a["idx"], a["weight"], a["E"], a["k"],
                                      a["width"], a["act"], a["out"], None, a["T"], a["D"], a["O"], a["dtype"], a["scratch"], a["bytes"])
    assert call(T=0) == OK
    for name in ("x", "w1", "s1", "b1", "w2", "s2", "b2", "idx", "out", "scratch"):
        assert call(**{name: None}) == NULL, name
    assert call(k=0) == RANGE and call(k=33) == RANGE and call(E=0) == RANGE and call(E=65537) == RANGE
    assert call(width=0) == RANGE and call(width=65537) == RANGE and call(T=-1) == RANGE
    assert call(D=0) == SHAPE and call(O=0) == SHAPE and call(E=65536, width=65536, D=4096) == SHAPE
    assert call(dtype=F32) == UNSUP and call(dtype=4) == DTYPE and call(act=2) == UNSUP
    assert call(w1=P(2 * BIG + 4)) == UNSUP and call(w2=P(5 * BIG + 8)) == UNSUP
    assert call(bytes=need - 1) == WORKSPACE and call(scratch=P(10 * BIG + 8)) == WORKSPACE
    assert call(out=P(BIG)) == ALIAS and call(scratch=P(BIG)) == ALIAS and call(out=P(10 * BIG)) == ALIAS
    assert L.fff_leaf_mx4_scratch_bytes(4, 64, 32, 8, 0, 40) == 0 and L.fff_leaf_mx4_scratch_bytes(0, 64, 32, 8, 2, 40) == 0


def test_refusals_of_sizes_that_no_launch_takes(L):
    """A launch ends at 2^32 threads."""
    q = lambda t, batch, rows, cols: L.fff_mx4_quantize(P(BIG), P(2 * BIG), P(3 * BIG), t, None, batch, rows, cols, BF16)
    assert q(1, 1 << 24, 1, 1) == SHAPE and q(1, 1 << 23, 129, 1) == SHAPE and q(1, 1 << 23, 1, 65) == SHAPE
    assert q(0, 1, 1, (1 << 34) + 1) == SHAPE
    assert L.fff_mx4_dequantize(P(BIG), P(2 * BIG), P(3 * BIG), None, 1, (1 << 34) + 1, BF16) == SHAPE
    m = lambda T, N: L.fff_mx4_product(P(BIG), None, P(2 * BIG), P(3 * BIG), None, 2, P(4 * BIG), None, T, 32, N, BF16, None, 0)
    assert m((1 << 31) - 1, 1) == RANGE and m(1 << 30, 129) == SHAPE           # (2^31 - 1024 tokens are the most of any call)
    assert L.fff_leaf_mx4_scratch_bytes(1 << 30, 32, 32, 4, 1, 16) == 0 and L.fff_leaf_mx4_scratch_bytes(1 << 20, 32, 129, 4, 16, 2000) > 0
    assert L.fff_leaf_mx4_scratch_bytes(1 << 26, 32, 32, 4, 8, 4097) == 0


def test_binding_checks_every_extent():
    import torch
    import paper_2308_14711_amd as F
    z = torch.zeros
    u8, i32, bf = torch.uint8, torch.int32, torch.bfloat16

    def refuses(status, f, *args, **kw):
        with pytest.raises(F.FffError) as e:
            f(*args, **kw)
        assert e.value.status == status

    def reaches_the_device_check(f, *args, **kw):
        with pytest.raises(ValueError, match="GPU"):
            f(*args, **kw)

    logits, idx, w = z(5, 8), z(5, 2, dtype=i32), z(5, 2)
    reaches_the_device_check(F.fff_moe_route, logits, 2, idx, w)
    refuses(SHAPE, F.fff_moe_route, logits[0], 2, idx, w)
    refuses(SHAPE, F.fff_moe_route, logits, 3, idx, w)
    refuses(DTYPE, F.fff_moe_route, logits, 2, idx.long(), w)
    refuses(SHAPE, F.fff_moe_route, logits, 2, idx, w, count=z(8, dtype=i32))
    refuses(SHAPE, F.fff_moe_route, logits, 2, idx, w, prob_mean=z(9))
    refuses(SHAPE, F.fff_moe_route, logits, 2, idx, w, loss=z(3))
    refuses(DTYPE, F.fff_moe_route, logits, 2, idx, w, token_mask=z(5, dtype=i32))
    refuses(SHAPE, F.fff_moe_route, logits, 2, idx, w, token_mask=z(4, dtype=torch.bool))
    count = z(9, dtype=i32)
    reaches_the_device_check(F.fff_moe_route_backward, logits, idx, count, z(5, 8))
    refuses(DTYPE, F.fff_moe_route_backward, logits, idx, count, z(5, 8, dtype=bf))
    refuses(SHAPE, F.fff_moe_route_backward, logits, idx, count[:8], z(5, 8))
    refuses(SHAPE, F.fff_moe_route_backward, logits, idx, count, z(5, 8), dweight=z(5, 3))
    refuses(DTYPE, F.fff_moe_route_backward, logits, idx, count, z(5, 8), dloss=z(2, dtype=torch.float64))

    src = z(3, 5, 70)
    reaches_the_device_check(F.fff_mx4_quantize, src, z(3, 5, 48, dtype=u8), z(3, 5, 3, dtype=u8))
    reaches_the_device_check(F.fff_mx4_quantize, src, z(3, 70, 16, dtype=u8), z(3, 70, 1, dtype=u8), transpose=True)
    refuses(SHAPE, F.fff_mx4_quantize, src, z(3, 5, 40, dtype=u8), z(3, 5, 3, dtype=u8))
    refuses(DTYPE, F.fff_mx4_quantize, src, z(3, 5, 48), z(3, 5, 3, dtype=u8))
    refuses(SHAPE, F.fff_mx4_dequantize, z(5, 48, dtype=u8), z(5, 2, dtype=u8), z(5, 70))
    with pytest.raises(ValueError):
        F.fff_mx4_dequantize(z(5, 48, dtype=u8), z(5, 3, dtype=u8), z(5, 70))

    a, wc, ws, out = z(4, 70, dtype=bf), z(6, 48, dtype=u8), z(6, 3, dtype=u8), z(4, 6, dtype=bf)
    reaches_the_device_check(F.fff_mx4_product, a, wc, ws, out)
    reaches_the_device_check(F.fff_mx4_product, z(4, 48, dtype=u8), wc, ws, z(4, 6), a_scales=z(4, 3, dtype=u8))
    refuses(DTYPE, F.fff_mx4_product, a.float(), wc, ws, out)
    refuses(SHAPE, F.fff_mx4_product, a, wc[:, :32], ws, out)
    refuses(SHAPE, F.fff_mx4_product, a, wc, ws, out, bias=z(5, dtype=bf))
    refuses(SHAPE, F.fff_mx4_product, z(4, 32, dtype=u8), wc, ws, out, a_scales=z(4, 3, dtype=u8))

    def leaf(**kw):
        t = dict(x=z(4, 70, dtype=bf), w1=z(3, 40, 48, dtype=u8), s1=z(3, 40, 3, dtype=u8), b1=z(3, 40, dtype=bf), w2=z(3, 6, 32, dtype=u8),
                 s2=z(3, 6, 2, dtype=u8), b2=z(3, 6, dtype=bf), idx=z(4, 2, dtype=i32), weight=z(4, 2), out=z(4, 6, dtype=bf))
        t.update(kw)
        F.fff_leaf_forward_mx4(t["x"], t["w1"], t["s1"], t["b1"], t["w2"], t["s2"], t["b2"], t["idx"], t["weight"], 0, t["out"])
    reaches_the_device_check(leaf)
    reaches_the_device_check(leaf, idx=z(4, dtype=i32), weight=None)
    for name, t in (("w1", z(3, 40, 32, dtype=u8)), ("s1", z(3, 40, 2, dtype=u8)), ("w2", z(3, 40, 32, dtype=u8)), ("s2", z(3, 6, 1, dtype=u8)),
                    ("b2", z(2, 6, dtype=bf)), ("idx", z(5, 2, dtype=i32)), ("weight", z(4, 1)), ("out", z(5, 6, dtype=bf))):
        refuses(SHAPE, leaf, **{name: t})
    refuses(DTYPE, leaf, idx=z(4, 2))
    refuses(DTYPE, leaf, b1=z(3, 40))


@pytest.mark.parametrize("normalise", [True, False])
def test_the_reference_gradient_against_differences(normalise):
    rng = np.random.default_rng(5)
    T, E, k = 9, 11, 3
    l = rng.normal(size=(T, E)) * 2
    l[4, 3] = -np.inf
    mask = np.ones(T, np.uint8)
    mask[2] = 0
    idx, _, count, *_ = R.route(l, k, mask, normalise)
    dw, dl = rng.normal(size=(T, k)), np.array([0.7, -0.3])

    def value(l):
        """The losses with the choice and the counts held fixed."""
        _, _, _, mean, loss, p, _, on = R.route(l, k, mask, normalise)
        q = np.where(idx >= 0, np.take_along_axis(p, np.maximum(idx, 0), 1), 0)
        w = q / np.where(q.sum(1) > 0, q.sum(1), 1)[:, None] if normalise else q
        n = count[E]
        return (w * dw).sum() + dl[0] * E * (count[:E] / (n * k) * mean).sum() + dl[1] * loss[1]
    got, _ = R.route_backward(l, idx, count, dw, dl, mask, normalise)
    h = 1e-5
    for t in range(T):
        for e in range(E):
            if l[t, e] == -np.inf:
                assert got[t, e] == 0
                continue
            up, down = l.copy(), l.copy()
            up[t, e] += h
            down[t, e] -= h
            # (central differences: truncation ~ h^2, rounding ~ 1e-16 / h)
            assert abs((value(up) - value(down)) / (2 * h) - got[t, e]) < 1e-8


def test_the_reference_quantisation_on_known_blocks():
    x = np.zeros((5, 32))
    x[0, :8] = [6, 5, 2.5, 1.75, 0.25, 0.75, -1.25, 7.9]      # scale 1: halves go to the even code, 7.9 is limited
    x[1, 0] = 2.0 ** -140
    x[2, 3] = np.inf
    x[3, 31] = np.nan
    c, s = R.quantise(x)
    assert s.tolist() == [[127], [0], [255], [255], [0]]
    assert R.values(c, s, 32)[0, :8].tolist() == [6, 4, 2, 2, 0, 1, -1, 6]
    assert not c[2].any() and np.isnan(R.values(c, s, 32)[2]).all() and not c[1].any()
