"""Which kernel makes the scores from 4-bit values, told from its name, with a HIP runtime that launches nothing (stand_in_hip.cpp), on the host: the
forms that test_gpu_mx4_forms.py asks for by hand are the ones it gets, and the sizes it names for the rule itself reach the forms that keep codes."""
import pytest

from test_launches_host import run, stand_in   # noqa: F401  (a fixture)

FORM = """
import os, re
def form(m, d, k, b, storage, **tune):   # (slots, labels of a lane, lanes, instances of a read, two halves)
    for name, value in tune.items(): os.environ["USL_TUNE_" + name] = str(value)
    L = usl.Layer(m, d, k, b, storage)
    hip.stand_in_start(b"")
    L.forward_mx4(P["x"], P["idx"], P["W"], P["m1"], P["g"], b)
    for name in tune: del os.environ["USL_TUNE_" + name]
    found = [f for f in (re.search(r"k_forwardILi(\\d+)ELi(\\d+)ELi(\\d+)E[ft]Li(\\d)ELb(\\d)ELi0ELb(\\d)ELb\\dELb1E", n) for n in hip.stand_in_launched().decode().split()) if f]
    assert len(found) == 1, hip.stand_in_launched()
    return tuple(int(g) for g in found[0].groups())
"""

# (d, b, storage) of test_gpu_mx4_forms.py and their groups of instances, rows in halves
LAYOUTS = [(300, 7, "f32", 4, 0), (15000, 5, "f32", 2, 0), (30000, 3, "f32", 1, 0), (50000, 3, "f32", 1, 1), (300, 7, "bf16", 4, 0), (30001, 5, "bf16", 2, 0),
           (45000, 3, "bf16", 1, 0)]
# labels of a lane and lanes by fan-in and shape, the first for groups of 4 and 2 instances, the second for single ones
ASKED = {(24, 1): ((2, 512), (1, 1024)), (24, 2): ((2, 1024), (2, 1024)), (24, 4): ((5, 1024), (5, 1024)), (32, 2): ((2, 1024), (2, 1024)),
         (32, 4): ((4, 1024), (4, 1024)), (8, 2): ((4, 1024), (4, 1024)), (16, 1): ((4, 512), (1, 1024)), (64, 2): ((2, 512), (2, 512)), (48, 2): ((1, 1024), (1, 1024))}


@pytest.mark.parametrize("K,shape", sorted(ASKED))
def test_forms_asked_for_by_hand(stand_in, K, shape):   # noqa: F811
    run(stand_in, FORM + """
for d, b, storage, q, halves in %r:
    for labels in (224, 8192):   # blocks of equal size, and more than any block takes: full ones
        got = form(6001, d, %d, b, storage, SHAPE=%d, LABELS=labels)
        assert got == (%d,) + %r[q == 1] + (q, halves, int(labels == 224)), (d, b, storage, got)
""" % (LAYOUTS, K, shape, K, ASKED[K, shape]))


@pytest.mark.parametrize("m,d,k,b,storage,form", [(200003, 30000, 32, 64, "f32", (32, 4, 1024, 1, 0, 0)), (262147, 36000, 32, 33, "bf16", (32, 4, 1024, 2, 0, 1)),
                                                  (262147, 50000, 32, 17, "f32", (32, 4, 1024, 1, 1, 1)), (500000, 32768, 32, 256, "f32", (32, 4, 1024, 1, 0, 0)),
                                                  (500000, 32768, 32, 256, "bf16", (32, 4, 1024, 2, 0, 0)), (300007, 30000, 24, 9, "bf16", (24, 5, 512, 2, 0, 0))])
def test_forms_that_keep_codes_by_the_rule(stand_in, m, d, k, b, storage, form):   # noqa: F811
    run(stand_in, FORM + """
assert form(%d, %d, %d, %d, "%s") == %r
""" % (m, d, k, b, storage, form))


def test_no_form_that_no_size_reaches(stand_in):   # noqa: F811
    """512 lanes with four labels of 32 slots each were there and never taken: shape 2 has as many labels to a block and twice the wavefronts."""
    run(stand_in, FORM + """
for d, b, storage, q, halves in %r:
    assert form(6001, d, 32, b, storage, SHAPE=5)[1:3] != (4, 512), (d, b, storage)
""" % LAYOUTS)
