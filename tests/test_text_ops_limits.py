"""Limits of the attention to an encoder's states at the C boundary.  Every call here ends on the host (no GPU needed): the pointers are never
dereferenced."""
import pytest

from test_text_ops_refusals import ARG, P, UNSUPPORTED, L, _bwd, _fwd, _pack    # noqa: F401 (L is the library)


def _both(L, **kw):
    return {_fwd(L, **kw), _bwd(L, **kw)}


def test_packed_rows_of_many_sequences(L):
    """What counts is the rows together, not every sequence's longest possible length.  (k missing: the check that comes next.)"""
    packed = dict(kv_offsets=P, k=0, n_seq=9000, n_enc=9000, kv_heads=16, heads=16, q_seq=128000, n_kv=2700000, kv_rows=2700000)
    assert _both(L, os=(128000, 128, 64), **packed) == {ARG}
    assert _both(L, os=(128000, 128, 64), **{**packed, "n_enc": 0x7fffff00, "kv_seq": P}) == {UNSUPPORTED}
    assert _both(L, os=(128000, 128, 64), **{**packed, "kv_offsets": 0}) == {UNSUPPORTED}


def test_lengths_near_the_end_of_31_bits(L):
    """A state, token or sequence that all share may be named as often as 31 bits hold; kernels that count on in steps would pass them."""
    one = dict(n_seq=1, n_enc=1, heads=1, kv_heads=1, q_seq=0, q_tok=0, k_seq=0, k_tok=0, v_seq=0, v_tok=0)
    wide = dict(os=(1 << 40, 64, 64))
    for n in (0x7fffffff, 0x7fffffc1, 0x7fff0001):
        assert _both(L, n_kv=n, **one) == {UNSUPPORTED}
        assert _both(L, n_kv=n, kv_rows=n, kv_offsets=P, **one) == {UNSUPPORTED}
        assert _both(L, kv_rows=n, kv_offsets=P, **one) == {UNSUPPORTED}
        assert _both(L, n_q=n, **wide, **one) == {UNSUPPORTED}
        assert _both(L, **{**one, "n_seq": n, "kv_seq": P}) == {UNSUPPORTED}
        assert _both(L, **{**one, "n_enc": n, "kv_seq": P}) == {UNSUPPORTED}
        for kw in (dict(n_kv=n), dict(n_q=n)):
            assert L.free_op_cross_attention_workspace_bytes(_pack(**{**one, **kw})) == 0
            assert L.free_op_cross_attention_bwd_workspace_bytes(_pack(**{**one, **kw})) == 0
    assert _both(L, n_kv=0x7fff0000, k=0, **one) == {ARG}          # allowed: the next check is told


def test_scales_whose_exponent_in_base_two_overflows(L):
    assert _both(L, scale=2.4e38) == {ARG} and _both(L, scale=3.4e38) == {ARG}
    assert _fwd(L, scale=2.2e38, n_seq=0) == 0
