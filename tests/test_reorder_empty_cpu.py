"""Calls of sharq_beam_reorder that have nothing to do, or leave arrays out: without a GPU, a launch would show as an
error."""

from test_serve_cpu import EINVAL, FAKE, L, OK, reorder  # noqa: F401


def test_token_ids_without_columns(L):  # noqa: F811
    none = dict(table=None, out=None, copies=None)
    assert reorder(L, **none, id_cols=0) == OK
    assert reorder(L, **none, id_cols=0, ldi=0, ldio=0, ids_out=FAKE) == OK
    assert reorder(L, **none, id_cols=0, parents=None) == EINVAL
