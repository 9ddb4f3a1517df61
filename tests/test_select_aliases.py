"""Outputs of the choice of candidates may not be its inputs: they are written while tokens of finished hypotheses are still read."""
import pytest

from paper_2510_08666_amd import binding as b

GOOD = [0x1000, b.F32, 9, 1, 2, 9, 0x2000, 0x7000, 2, 0x3000, 0x4000, 0x5000, 0x6000, 1 << 20, None]
SCORE, HOLD, ROW, TOKEN, SCORE_OUT = 6, 7, 9, 10, 11


@pytest.mark.parametrize("out,given", [(ROW, HOLD), (TOKEN, HOLD), (SCORE_OUT, HOLD), (SCORE_OUT, SCORE), (ROW, TOKEN)])
def test_an_output_that_is_another_argument(out, given):
    args = list(GOOD)
    args[out] = args[given]
    assert b.lib.dinfer_beam_select(*args) == -1
    assert b.last_error() == "an output is another argument"
