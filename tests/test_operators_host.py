"""The calls around the layer refuse what they cannot take before anything is launched.  No GPU needed."""
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def usl():
    lib = os.path.join(ROOT, "paper_2306_03725_amd", "libusl.so")
    if not os.path.exists(lib):
        from paper_2306_03725_amd import build
        build.build(force=True)
    from paper_2306_03725_amd import usl as u
    return u


P, Q = 4096, 8192    # never dereferenced


def refused(usl, status, call):
    with pytest.raises(usl.UslError) as e:
        call()
    assert e.value.status == status and str(e.value), str(e.value)


def test_layer_norm_refuses(usl):
    L = usl.Layer(64, 16, 4, 8)
    for h, x in ((None, P), (P, None)):
        refused(usl, usl.USL_EINVAL, lambda: L.layer_norm(h, P, P, 1e-5, x, P, P, 1))
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        refused(usl, usl.USL_EINVAL, lambda: L.layer_norm(P, P, P, eps, P, P, P, 1))
    refused(usl, usl.USL_EINVAL, lambda: L.layer_norm(P, P, P, 1e-5, P, P, P, 0))
    refused(usl, usl.USL_ESHAPE, lambda: L.layer_norm(P, P, P, 1e-5, P, P, P, 9))
    ok = dict(grad_x=P, h=P, gamma=P, mean=P, rstd=P, grad_h=Q, grad_gamma=P, grad_beta=P, b=8)
    for name in ("grad_x", "h", "mean", "rstd", "grad_h"):
        refused(usl, usl.USL_EINVAL, lambda: L.layer_norm_backward(**dict(ok, **{name: None})))
    refused(usl, usl.USL_EINVAL, lambda: L.layer_norm_backward(**dict(ok, grad_h=P)))             # an input
    refused(usl, usl.USL_EINVAL, lambda: L.layer_norm_backward(**dict(ok, grad_x=3 * P, grad_h=P)))
    refused(usl, usl.USL_ESHAPE, lambda: L.layer_norm_backward(**dict(ok, b=9)))
    L.close()


def test_mx4_refuses(usl):
    L = usl.Layer(64, 16, 4, 8)
    for i in range(3):
        args = [P, P, P]
        args[i] = None
        refused(usl, usl.USL_EINVAL, lambda: L.quantize_mx4(*args))
        refused(usl, usl.USL_EINVAL, lambda: L.dequantize_mx4(*args))
    for i in range(5):
        args = [P] * 5
        args[i] = None
        refused(usl, usl.USL_EINVAL, lambda: L.forward_mx4(*args, 1))
    refused(usl, usl.USL_EINVAL, lambda: L.forward_mx4(P, P, P, P, P, -1))
    refused(usl, usl.USL_ESHAPE, lambda: L.forward_mx4(P, P, P, P, P, 9))
    L.close()


def test_adjustments_refuse(usl):
    L = usl.Layer(64, 16, 4, 8)
    calls = (lambda a, b=2: L.adjust_scores(P, a, P, b), lambda a, b=2: L.topk_adjusted(P, a, b, 5, P, P))
    nan, inf = float("nan"), float("inf")
    for call in calls:
        for bad in (dict(repeat=0.0), dict(repeat=-1.0), dict(repeat=nan), dict(repeat=inf), dict(presence=nan), dict(presence=-inf),
                    dict(frequency=inf), dict(frequency=nan), dict(shown_off=P), dict(shown_lab=P), dict(allowed=P, allowed_rows=0),
                    dict(allowed=P, allowed_rows=-1)):
            refused(usl, usl.USL_EINVAL, lambda: call(usl.Adjustments(**bad)))
        refused(usl, usl.USL_EINVAL, lambda: call(usl.Adjustments(allowed=P, allowed_rows=2), 3))   # masks for two of three
        refused(usl, usl.USL_EINVAL, lambda: call(usl.Adjustments(), 0))
        refused(usl, usl.USL_ESHAPE, lambda: call(usl.Adjustments(), 9))
    good = usl.Adjustments()
    refused(usl, usl.USL_EINVAL, lambda: L.adjust_scores(None, good, P, 1))
    refused(usl, usl.USL_EINVAL, lambda: L.adjust_scores(P, good, None, 1))
    refused(usl, usl.USL_EINVAL, lambda: L.topk_adjusted(P, good, 1, 0, P, P))
    refused(usl, usl.USL_ESHAPE, lambda: L.topk_adjusted(P, good, 1, 33, P, P))
    refused(usl, usl.USL_ESHAPE, lambda: usl.Layer(4, 16, 4, 8).topk_adjusted(P, good, 1, 5, P, P))
    for args in ((None, 5, P, P), (P, 5, None, P), (P, 5, P, None)):
        refused(usl, usl.USL_EINVAL, lambda: L.topk_adjusted(args[0], good, 1, args[1], args[2], args[3]))
    assert usl._lib.usl_adjust_scores(L._h, P, None, P, 1) == usl.USL_EINVAL
    L.close()


def test_tensors_that_are_not_contiguous_are_refused(usl):
    torch = pytest.importorskip("torch")
    L = usl.Layer(64, 16, 4, 8)
    with pytest.raises(ValueError):
        L.layer_norm(torch.zeros(16, 2).t(), None, None, 1e-5, P, None, None, 2)
    with pytest.raises(ValueError):
        usl.Adjustments(bias=torch.zeros(128)[::2])
    L.close()
