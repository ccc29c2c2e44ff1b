"""What the binding passes on of a plan whose requests' most new tokens are known."""

import pytest

import paper_2607_08565_gb300 as pkg
from test_kv4_refusals import kv  # noqa: F401 (a fixture)
from test_kv_refusals import on, plan


@pytest.mark.parametrize("max_new,passed", [(None, None), (0, 0), (1, 1), (4, 4), (2 ** 40, 2 ** 40), (2 ** 70, 2 ** 63 - 1), (-5, -1)])
def test_most_new_tokens_come_through(kv, max_new, passed):  # noqa: F811
    kv.plan(*(on(x, 0) for x in plan()), 4, window=7, max_new=max_new)
    assert kv.library.calls == ["smetric_kv_plan" if passed is None else "smetric_kv_plan_up_to"]
    args = kv.library.args
    assert args[8] == 7 and (passed is None or args[9] == passed) and len(args) == (10 if passed is None else 11)


def test_without_a_handle_it_is_refused():
    assert pkg.lib().smetric_kv_plan_up_to(None, None, 0, 0, None, None, 0, 0, 0, 1, None) == pkg.SMETRIC_ERR_INVALID_ARG
