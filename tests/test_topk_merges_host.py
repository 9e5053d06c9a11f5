"""Which kernel merges a row's candidates, told from its name, with a HIP runtime that launches nothing (stand_in_hip.cpp), on the host: no more lanes, and no more
candidates to a lane, than the row has candidates for.  (1024 lanes with 16 each for 3720 candidates, 5 labels: 7.0 us; 512 with 8: 4.0.)"""
import pytest

from test_launches_host import run, stand_in   # noqa: F401  (a fixture)

# labels, labels asked for: one row of kk candidates from every 2048 scores
MERGES = [(2048 * 256, 1, "k_topk_merge_few"), (2048 * 257, 1, "k_topk_merge_rowILi256ELi4E"), (2048 * 204, 5, "k_topk_merge_rowILi256ELi4E"), (500000, 5, "k_topk_merge_rowILi256ELi8E"),
          (2048 * 420, 5, "k_topk_merge_rowILi512ELi8E"), (1522105, 5, "k_topk_merge_rowILi512ELi8E"), (500000, 32, "k_topk_merge_rowILi512ELi16E"),
          (2048 * 512, 32, "k_topk_merge_rowILi1024ELi16E"), (2900000, 32, "k_topk_mergeE")]


@pytest.mark.parametrize("m,kk,name", MERGES)
def test_who_merges(stand_in, m, kk, name):   # noqa: F811
    run(stand_in, """
L = usl.Layer(%d, 1, 1, 1)
hip.stand_in_start(b"")
L.topk(P["g"], 1, %d, P["off"], P["lab"])
names = hip.stand_in_launched().decode().split()
assert "k_topk_segments" in names[-2] and "%s" in names[-1], names
""" % (m, kk, name))
