"""Which kernels a token loss launches for which rows, where results do not show it: libmimose on the stand-in for the HIP
runtime of test_launch_errors, which launches nothing and keeps the names."""
import pytest

from test_launch_choice import run
from test_launch_errors import runtime  # noqa: F401

SETUP = """
    at = 1 << 20                                        # (an aligned address that nothing reads)
    far = 1 << 44
    def logprob(dtype, V, ld, x=at):
        return launched(lambda: mi.mimose_op_token_logprob(dtype, x, ld, at, at, 64, V))
    def policy(dtype, V, ld, x=at, g=far, T=64):
        return launched(lambda: mi.mimose_op_policy_loss(dtype, x, ld, at, at, None, at, None, 1.0, .2, .2, 0., g, at, at, T, V))
    def preference(dtype, V, ld, T, g=far, pairs=2):
        return launched(lambda: mi.mimose_op_preference_loss(dtype, at, ld, at, at, pairs, 0, at, .1, 0., g, at, at, at, at, T, V, at, 1 << 40))
"""


@pytest.mark.parametrize("dtype,letter", [(0, "f"), (1, "t")])
def test_rows(runtime, dtype, letter):  # noqa: F811
    """Waves and chunks a lane by the length of a row, and the variant for rows that begin and end on a 16-byte address."""
    run(runtime, SETUP + """
    dtype, letter = int(sys.argv[2]), sys.argv[3]
    n = 8 if dtype else 4
    for chunks, waves, per_lane in ((1, 1, 1), (64, 1, 1), (65, 1, 2), (128, 1, 2), (129, 1, 4), (257, 1, 9), (576, 1, 9), (577, 2, 9), (1153, 4, 9),
                                    (2305, 8, 9), (4608, 8, 9), (6657, 16, 7), (7168, 16, 7), (7169, 16, 9), (9217, 16, 13), (13313, 16, 16),
                                    (16384, 16, 16)):
        want = "token_rows_held_kernelI%sLi%dELi%dELi" % (letter, waves, per_lane)
        names = logprob(dtype, chunks * n, chunks * n)
        assert len(names) == 1 and want + "0ELb1ELb1E" in names[0], (chunks, names)
        names = policy(dtype, chunks * n, chunks * n)
        assert len(names) == 2 and want + "1ELb1ELb1E" in names[0] and "policy_stats" in names[1], (chunks, names)
    assert "Li8ELi13ELi0E" in logprob(dtype, 6656 * n, 6656 * n)[0]
    assert "Li16ELi7ELi1E" in policy(dtype, 6656 * n, 6656 * n)[0]
    assert "token_rows_long_kernel" in logprob(dtype, 16385 * n, 16385 * n)[0]
    size = 2 if dtype else 4
    for names in (logprob(dtype, 1000, 1001), logprob(dtype, 1000, 1024, at + size), policy(dtype, 1000, 1024, at, far + size)):
        assert "ELb1ELb0E" in names[0], names
    """, dtype, letter)


def test_preference(runtime):  # noqa: F811
    """Rows of up to 640 MB through the caches, more past them; three launches, two where the gradient makes the pairs' sums or a
    block is enough for the loss alone."""
    run(runtime, SETUP + """
    for T, past in ((6670, 0), (6671, 1)):
        names = preference(1, 50257, 50304, T)
        assert len(names) == 3 and "Li8ELi13ELi0ELb%dELb1E" % past in names[0] and "pair_sums" in names[1], names
        assert "pair_grad_kernelItLb%dELb0E" % past in names[2], names
    for V, ld, T, pairs, sums in ((4096, 4096, 3071, 8, 1), (4096, 4096, 3072, 8, 1), (4096, 4096, 3073, 8, 0), (4096, 4096, 100, 9, 0),
                                  (4097, 4104, 1536, 8, 1), (4097, 4104, 1537, 8, 0)):
        names = preference(1, V, ld, T, far, pairs)
        assert len(names) == (2 if sums else 3) and "pair_grad_kernelItLb0ELb%dE" % sums in names[-1], (V, T, pairs, names)
    names = preference(1, 50257, 50304, 100, None)
    assert len(names) == 2 and "few_pairs_kernel" in names[1], names
    names = preference(1, 50257, 50304, 100, None, 9)
    assert len(names) == 3 and "pair_sums" in names[1] and "pair_loss" in names[2], names
    names = preference(1, 50257, 50304, 0)
    assert len(names) == 1 and "few_pairs_kernel" in names[0], names
    """)


def test_update(runtime):  # noqa: F811
    run(runtime, """
    for bits, name in ((8, "adamw8_kernel"), (32, "adamw_kernel")):
        names = launched(lambda: mi.mimose_op_adamw_step(mi.mimose_adamw_table(1 << 20, 3, 5, bits, 0), 1))
        assert len(names) == 1 and name in names[0], names
        assert not launched(lambda: mi.mimose_op_adamw_step(mi.mimose_adamw_table(1 << 20, 3, 0, bits, 0), 1))
    """)
