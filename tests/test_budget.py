"""A budget of tokens a row: what cannot hold is refused where it is made."""
import ast
import inspect

import pytest

from paper_2501_16385_amd import decode_loop
from paper_2501_16385_amd.decode_loop import Budget


def test_a_class_is_defined_once():
    names = [n.name for n in ast.parse(inspect.getsource(decode_loop)).body if isinstance(n, (ast.ClassDef, ast.FunctionDef))]
    assert len(names) == len(set(names))


@pytest.mark.parametrize("bad", [dict(keep=8, first=4, recent=8), dict(keep=8, first=9, recent=0), dict(keep=0), dict(keep=-1, recent=0), dict(keep=8, first=-1), dict(keep=8, recent=-1),
                                 dict(keep=8, decay=1.5), dict(keep=8, decay=-0.1), dict(keep=8, decay=float("nan"))])
def test_budgets_that_no_row_can_keep(bad):
    with pytest.raises(ValueError, match="budget"):
        Budget(**bad)


def test_budgets_that_rows_can_keep():
    for good in (dict(keep=1), dict(keep=0, recent=0), dict(keep=12, first=4, recent=8), dict(keep=8, decay=0.0), dict(keep=8, decay=0.5)):
        assert Budget(**good).keep == good["keep"]
