"""The calls in front of the layer and the losses against short lists refuse what they cannot take before anything is launched.  No GPU needed."""
import os
import re

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


A = [4096 * n for n in range(1, 20)]    # never dereferenced
NAN, INF = float("nan"), float("inf")


def refused(usl, status, call):
    with pytest.raises(usl.UslError) as e:
        call()
    assert e.value.status == status and str(e.value), str(e.value)


def each_refused(usl, status, call, good, bad):
    for name, values in bad.items():
        for v in values:
            refused(usl, status, lambda: call(**dict(good, **{name: v})))


def test_gated_block_refuses(usl):
    L = usl.Layer(64, 16, 4, 8)
    good = dict(e=A[0], V_gate=A[1], V_up=A[2], w=5, act=0, x=A[3], gate=A[4], up=A[5], b=8)
    each_refused(usl, usl.USL_EINVAL, L.gated_block, good, dict(e=[None], V_gate=[None], V_up=[None], x=[None, A[0], A[1], A[2], A[4], A[5]], gate=[A[0], A[1], A[5]],
                                                              up=[A[2], A[3]], w=[0, -1], act=[-1, 2], b=[0, -1]))
    each_refused(usl, usl.USL_ESHAPE, L.gated_block, good, dict(w=[65537, 2 ** 31 - 1], b=[9]))
    good = dict(grad_x=A[0], e=A[1], V_gate=A[2], V_up=A[3], gate=A[4], up=A[5], w=5, act=1, grad_e=A[6], grad_V_gate=A[7], grad_V_up=A[8], b=8)
    each_refused(usl, usl.USL_EINVAL, L.gated_block_backward, good,
                 dict(grad_x=[None], e=[None], V_gate=[None], V_up=[None], gate=[None], up=[None], w=[0], act=[2], b=[0], grad_e=[A[0], A[1], A[7]],
                      grad_V_gate=[A[2], A[8]], grad_V_up=[A[3], A[5], A[6]]))
    each_refused(usl, usl.USL_ESHAPE, L.gated_block_backward, good, dict(w=[65537], b=[9]))
    L.gated_block_backward(**dict(good, grad_e=None, grad_V_gate=None, grad_V_up=None))   # nothing is asked for
    L.close()
    L = usl.Layer(4, 2 ** 20 + 1, 1, 8)
    refused(usl, usl.USL_ESHAPE, lambda: L.gated_block_backward(**good))
    L.close()


def test_int8_refuses(usl):
    L = usl.Layer(64, 16, 4, 8, "bf16")
    good = dict(rows=A[0], n=3, w=5, codes=A[1], scales=A[2])
    each_refused(usl, usl.USL_EINVAL, L.quantize_i8, good, dict(rows=[None], codes=[None, A[0], A[2]], scales=[None, A[0]], n=[0, -1], w=[0]))
    each_refused(usl, usl.USL_ESHAPE, L.quantize_i8, good, dict(n=[2 ** 31], w=[65537]))
    good = dict(e_codes=A[0], e_scales=A[1], V_codes=A[2], V_scales=A[3], w=5, h=A[4], b=8)
    each_refused(usl, usl.USL_EINVAL, L.project_i8, good, dict(e_codes=[None], e_scales=[None], V_codes=[None], V_scales=[None], h=[None, A[0], A[3]], w=[0], b=[0]))
    each_refused(usl, usl.USL_ESHAPE, L.project_i8, good, dict(w=[65537], b=[9]))
    good = dict(e_codes=A[0], e_scales=A[1], gate_codes=A[2], gate_scales=A[3], up_codes=A[4], up_scales=A[5], w=5, act=0, x=A[6], b=8)
    each_refused(usl, usl.USL_EINVAL, L.gated_block_i8, good, dict(e_codes=[None], e_scales=[None], gate_codes=[None], gate_scales=[None], up_codes=[None], up_scales=[None],
                                                                 x=[None, A[0], A[5]], act=[3], w=[-5], b=[0]))
    each_refused(usl, usl.USL_ESHAPE, L.gated_block_i8, good, dict(w=[65537], b=[9]))
    L.close()


def test_losses_refuse(usl):
    L = usl.Layer(64, 16, 4, 8)
    good = dict(out=A[0], tea_off=A[1], tea_lab=A[2], tea_logit=A[3], temperature=1.0, scale=1.0, g=A[4], loss=A[5], b=8)
    each_refused(usl, usl.USL_EINVAL, L.distill_loss_grad, good, dict(out=[None], tea_off=[None], tea_lab=[None], tea_logit=[None], loss=[None, A[0], A[3], A[4]], g=[A[1], A[2], A[3]],
                                                                    temperature=[0.0, -1.0, NAN, INF, 1e-40], scale=[NAN, INF, -INF], b=[0]))
    each_refused(usl, usl.USL_ESHAPE, L.distill_loss_grad, good, dict(b=[9]))
    good = dict(out=A[0], act_off=A[1], act_lab=A[2], old_logp=A[3], ref_logp=A[4], advantage=A[5], clip_low=0.2, clip_high=0.2, beta=0.1, scale=1.0, g=A[6], logp=A[7],
                loss=A[8], b=8)
    each_refused(usl, usl.USL_EINVAL, L.policy_loss_grad, good,
                 dict(out=[None], act_off=[None], act_lab=[None], old_logp=[None], ref_logp=[None], advantage=[None], clip_low=[-0.1, 1.1, NAN], clip_high=[-0.1, NAN, INF],
                      beta=[-1.0, NAN, INF], scale=[NAN, INF], g=[A[3], A[5], A[7]], logp=[A[0], A[3], A[4], A[5], A[8]], loss=[None, A[0], A[1], A[6]], b=[0]))
    each_refused(usl, usl.USL_ESHAPE, L.policy_loss_grad, good, dict(b=[9]))
    L.close()


def test_tensors_that_are_not_contiguous_are_refused(usl):
    torch = pytest.importorskip("torch")
    L = usl.Layer(64, 16, 4, 8)
    with pytest.raises(ValueError):
        L.gated_block(torch.zeros(16, 2).t(), A[1], A[2], 16, 0, A[3], None, None, 2)
    with pytest.raises(ValueError):
        L.distill_loss_grad(A[0], A[1], torch.zeros(8, dtype=torch.int32)[::2], A[3], 1.0, 1.0, None, A[5], 2)
    L.close()


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    """The compiler's listings of the kernels whose tiles are loaded to LDS by inline assembly."""
    import subprocess

    from paper_2306_03725_amd import build
    lines = {}
    for name in ("k_gated.hip", "k_gated_grad.hip", "k_int8.hip"):
        out = str(tmp_path_factory.mktemp("listings") / (name + ".s"))
        subprocess.check_call([build._hipcc()] + build.FLAGS + ["--cuda-device-only", "-S", os.path.join(build.CSRC, name), "-o", out], stderr=subprocess.DEVNULL)
        with open(out) as fh:
            lines[name] = fh.read().splitlines()
    return lines


def test_m0_belongs_to_the_tiles(listings):
    """The tiles' loads to LDS write M0 from inline assembly, which the compiler cannot be told: M0 must appear nowhere else in their kernels."""
    for name, lines in listings.items():
        inside, own, other = False, 0, []
        for line in lines:
            if "ASMSTART" in line:
                inside = True
            elif "ASMEND" in line:
                inside = False
            elif re.search(r"\bm0\b", line.split(";")[0]):
                if inside:
                    own += 1
                else:
                    other.append(line.strip())
        assert own > 0 and not other, (name, other[:5])


def test_no_read_of_a_step_crosses_a_barrier(listings):
    """Behind a barrier the tiles' loads overwrite the step before it: a wavefront's reads from LDS have to be there when it comes to the barrier.  In the order of the
    listing, which is that of the loops' bodies."""
    barriers = 0
    for name, lines in listings.items():
        outstanding = False
        for line in lines:
            code = line.split(";")[0]
            if re.match(r"_Z\w+:", code):
                outstanding = False
            if "ds_read" in code:
                outstanding = True
            if re.search(r"s_waitcnt.*lgkmcnt\(0\)", code):
                outstanding = False
            if "s_barrier" in code:
                barriers += 1
                assert not outstanding, (name, line)
    assert barriers > 50
