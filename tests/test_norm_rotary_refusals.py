"""Refusals of the head norms' gradient, each by itself: every other argument is valid but for a workspace of no bytes, which is checked
last, so that nothing is launched whatever is let through."""

import pytest
from test_norm_rotary_abi import BAD, backward

CALM = dict(lens=(0, 0), nbytes=0)


def test_nothing_else_is_wrong():
    assert backward(**CALM) == -4
    assert backward(**CALM | dict(lens=(4, 4))) == -4 and backward(**CALM | dict(lens=None)) == -4
    assert backward(**CALM | dict(flags=2)) == -4 and backward(**CALM | dict(dtype=1)) == -4


@pytest.mark.parametrize("kw", BAD, ids=[f"{i}-{'-'.join(kw)}" for i, kw in enumerate(BAD)])
def test_refused(kw):
    assert backward(**CALM | kw) == -1


@pytest.mark.parametrize("kw", [dict(gq=None), dict(gk=None), dict(dqw=None), dict(dkw=None), dict(q=None, qo=None), dict(k=None, ko=None)],
                         ids=lambda kw: "-".join(kw))
def test_rows_and_all_that_belongs_to_them(kw):
    assert backward(**CALM | kw) == -1


def test_one_kind_alone():
    assert backward(**CALM | dict(q=None, qo=None, gq=None, qw=None, dqw=None, hq=0)) == -4
    assert backward(**CALM | dict(k=None, ko=None, gk=None, kw=None, dkw=None, hk=0)) == -4
    assert backward(**CALM | dict(hq=65535, hk=1)) == -2
