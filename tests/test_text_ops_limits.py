"""Limits of the attention to an encoder's states at the C boundary.  Every call here ends on the host (no GPU needed): the pointers are never
dereferenced."""
import pytest

from test_text_ops_refusals import ARG, P, SHAPE, UNSUPPORTED, L, _bwd, _fwd, _pack, _shape    # noqa: F401 (L is the library)


def _both(L, **kw):
    return {_fwd(L, **kw), _bwd(L, **kw)}


def test_packed_rows_of_many_sequences(L):
    """What counts is the rows together, not every sequence's longest possible length.  (k missing: the check that comes next.)"""
    packed = dict(kv_offsets=P, k=0, n_seq=9000, n_enc=9000, kv_heads=16, heads=16, q_seq=128000, n_kv=2700000, kv_rows=2700000)
    assert _both(L, os=(128000, 128, 64), **packed) == {ARG}
    assert _both(L, os=(128000, 128, 64), **{**packed, "n_enc": 0x7fffff00, "kv_seq": P}) == {UNSUPPORTED}
    assert _both(L, os=(128000, 128, 64), **{**packed, "kv_offsets": 0}) == {UNSUPPORTED}
