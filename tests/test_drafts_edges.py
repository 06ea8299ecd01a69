"""Calls of a decoding step of several drafted tokens at the edge of what they take, as far as the host decides them (handles in host memory only: a call that refuses
nothing ends at the device they were made for)."""
from __future__ import annotations

import pytest

from test_drafts_abi import ALIGN, AT, BUFSIZE, HIP, NULL, SHAPE, verify

NOTHING = dict(rows=0, target=None, target_row=0, vocab=0, tokens=None, parents=None, uniforms=None, finals=None, starts=None, path=None, out=None)


@pytest.mark.parametrize("change, status", [
    (dict(n_seqs=0, accepted=None), 0), (dict(n_seqs=0), 0), (dict(n_seqs=0, v=None), NULL), (dict(n_seqs=-1), SHAPE),
    (dict(n_seqs=3), HIP), (dict(n_seqs=3, starts=AT, finals=AT, vocab=100), HIP), (dict(n_seqs=3, accepted=None), NULL), (dict(n_seqs=3, accepted=AT + 2), ALIGN),
    (dict(n_seqs=4), BUFSIZE)])
def test_verify_without_rows(change, status):
    """Without sequences there is nothing to do; with them, only `accepted` is written."""
    assert verify(**{**NOTHING, **change}) == status
