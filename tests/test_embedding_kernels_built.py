"""Every kernel of the embedding that is built is one that some call is given; no GPU needed."""
import re

from paper_2111_04007_amd import binding as B


def test_built_kernels_are_those_that_calls_reach():
    """Entries of a piece, rows in flight, whether they share a position, whether they are written past the caches: outputs beyond the last-level
    cache have four rows in flight where rows move in 16-byte pieces."""
    B.load()
    with open(B.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"embedding_fwd_kernelI(f|DF16b)Li(\d+)ELi(\d+)ELb([01])ELb([01])E", f.read()))
    for kind, wide in ((b"f", 4), (b"DF16b", 8)):
        got = {tuple(int(v) for v in rest) for k, *rest in names if k == kind}
        assert got == {(wide, 1, 0, 0), (wide, 4, 0, 1), (wide, 4, 1, 1), (1, 1, 0, 0), (1, 1, 0, 1)}
