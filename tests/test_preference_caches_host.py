"""Whether the rows of a preference loss with its gradient are read through the caches or past them: both passes alike, on rows of any
alignment (libmimose on the stand-in for the HIP runtime of test_launch_errors, which keeps the kernels' names)."""
import pytest

from test_launch_choice import run
from test_launch_errors import runtime  # noqa: F401

SETUP = """
    at, far = 1 << 20, 1 << 44                          # (aligned addresses that nothing reads)
    def preference(dtype, V, ld, T, x=at, g=far):
        names = launched(lambda: mi.mimose_op_preference_loss(dtype, x, ld, at, at, 9, 0, at, .1, 0., g, at, at, at, at, T, V, at, 1 << 40))
        assert len(names) == 3 and "token_rows_held" in names[0] and "pair_sums" in names[1], names
        # template arguments: of the first pass past the caches and rows on 16 bytes, of the second past the caches
        return [(past, even, second) for past in (0, 1) for even in (0, 1) for second in (0, 1)
                if "Li0ELb%dELb%dEE" % (past, even) in names[0] and "Lb%dELb0EE" % second in names[2]]
"""


@pytest.mark.parametrize("dtype", [0, 1])
def test_beside(runtime, dtype):  # noqa: F811
    run(runtime, SETUP + """
    dtype = int(sys.argv[2])
    size, most = 2 if dtype else 4, 640 << 20
    for V, ld, offset, even in ((50257, 50304, 0, 1), (50257, 50257, 0, 0), (1003, 1003, 0, 0), (1000, 1024, size, 0), (1000, 1000, 0, 1)):
        rows = most // (ld * size)
        for T, past in ((rows, 0), (rows + 1, 1)):
            got = preference(dtype, V, ld, T, at + offset, far)
            assert got == [(past, even, past)], (V, ld, T, got)
    """, dtype)


@pytest.mark.parametrize("dtype", [0, 1])
def test_in_place(runtime, dtype):  # noqa: F811
    run(runtime, SETUP + """
    dtype = int(sys.argv[2])
    size, most = 2 if dtype else 4, 160 << 20
    for V, ld, offset, even in ((50257, 50304, 0, 1), (50257, 50257, 0, 0), (1003, 1003, 0, 0), (1000, 1024, size, 0), (1000, 1000, 0, 1)):
        rows = most // (ld * size)
        for T, past in ((rows, 0), (rows + 1, 1), (rows * 4, 1), (rows * 5, 1)):
            got = preference(dtype, V, ld, T, at + offset, at + offset)
            assert got == [(past, even, past)], (V, ld, T, got)
    """, dtype)
