"""Refusals of the serving operators at the limits of their arguments (no GPU needed).

Every call here fails validation or has nothing to do, which returns before any HIP call is made.
"""
import pytest

import libutil
from paper_2607_23265_amd import serve
from test_serve_capi import ALIGN, AT, NULL, OK, append, ragged, turn


@pytest.fixture(scope="module")
def L():
    libutil.ensure_built()
    return serve.lib()


def test_queries_without_a_token_to_store(L):
    """max_tokens = 0: queries are rotated all the same, so their arguments are looked at."""
    none = ragged(max_tokens=0)
    assert append(L, r=none, q=None) == OK
    assert append(L, r=none, out=None) == NULL and append(L, r=none, out=2 * AT + 8) == ALIGN
    assert append(L, r=none, t=turn(positions=None)) == NULL
