"""What the marked rows of tests/marked_cases.py tell: a token, or a step of 32, left out or counted twice is beyond the tolerances, wherever it is."""
import math

import pytest
import torch

from marked_cases import kept_as, marks, tolerances, wanted


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("sees,D", [(900, 64), (2049, 128), (20000, 64), (20000, 256), (65537, 128)])
def test_what_is_lost_or_counted_twice_shows(sees, D, dtype):
    out, lse = wanted(sees, D, kept_as(dtype, 4))
    off_out, off_lse = tolerances(out, lse, dtype, 2)
    of = marks(sees, D)
    steps = torch.stack([x.sum(0) for x in of.split(32)])      # [steps, D]
    for times in (-1, 1):
        assert abs(math.log(sees + times) - lse) > off_lse                    # one token
        n = sees + times * steps.sum(1)
        assert ((torch.log(n) - lse).abs() > off_lse).all()
        whole = steps.sum(1) == 32
        assert (((of.sum(0) + times * steps) * kept_as(dtype, 4) / n[:, None] - out).abs() > off_out).any(1)[whole].all()
    swapped = steps[0] - steps[1]                              # a step read twice in another's place
    assert ((swapped * kept_as(dtype, 4) / sees).abs() > off_out).any()
