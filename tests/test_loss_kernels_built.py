"""Every kernel of the token loss that is built is one that some size of vocabulary is given; no GPU needed."""
import re

from paper_2111_04007_amd import binding as B


def reached():
    """(waves, pieces of a thread, row stays in registers) of rows of n pieces, as they are dealt out."""
    out = set()
    for n in range(1, 16 * 1024 + 2):
        waves = 1 if n <= 256 else 4 if n <= 2048 else 8 if n <= 8192 else 16
        out.add((waves, -(-n // (64 * waves)), True) if n <= 16 * 1024 else (16, 8, False))
    return out


def test_built_kernels_are_those_that_sizes_reach():
    B.load()
    with open(B.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"cross_entropy_kernelI(f|DF16b)Li(\d+)ELi(\d+)ELb([01])ELi([012])E", f.read()))
    want = reached()
    assert {(t, int(past)) for t, _, _, _, past in names} == {(t, p) for t in (b"f", b"DF16b") for p in range(3)}
    for kind in {(t, past) for t, _, _, _, past in names}:
        assert {(int(w), int(nv), res == b"1") for t, w, nv, res, past in names if (t, past) == kind} == want
