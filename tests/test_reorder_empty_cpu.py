"""Calls of sharq_beam_reorder that have nothing to do, or leave arrays out: without a GPU, a launch would show as an
error."""

from test_serve_cpu import EINVAL, FAKE, L, OK, reorder  # noqa: F401


def test_token_ids_without_columns(L):  # noqa: F811
    none = dict(table=None, out=None, copies=None)
    assert reorder(L, **none, id_cols=0) == OK
    assert reorder(L, **none, id_cols=0, ldi=0, ldio=0, ids_out=FAKE) == OK
    assert reorder(L, **none, id_cols=0, parents=None) == EINVAL


def test_strides_of_arrays_that_are_not_given_mean_nothing(L):  # noqa: F811
    ids = dict(ids=None, ids_out=None, tokens=None)
    assert reorder(L, table=None, out=None, copies=None, ldt=3, ldto=5, **ids) == OK
    assert reorder(L, groups=0, table=None, out=None, copies=None, ldt=3, ldto=5) == OK
    assert reorder(L, groups=0, ldi=3, ldio=5, **ids) == OK
    assert reorder(L, groups=0, out=FAKE, ldto=9) == EINVAL and reorder(L, groups=0, ids_out=FAKE, ldio=60) == EINVAL
