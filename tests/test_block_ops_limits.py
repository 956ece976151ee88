"""Sizes and calls at the limits of the block operators.  Every call here ends on the host (no GPU needed): the pointers are
never dereferenced, and the sizes that must be refused would be empty batches if they were cut to 32 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

P = C.c_void_p(4096)
FAR = 1 << 32                                                      # 0 in 32 bits


@pytest.fixture(scope="module")
def L():
    from paper_2511_20390_b200.build import build
    build()
    from paper_2511_20390_b200 import binding
    return binding.lib()


def test_sizes_past_32_bits_are_refused(L):
    with pytest.raises(C.ArgumentError):
        L.free_op_layer_norm(0, 0, 1, FAR, 8, P, 8, None, None, 0, 0, 1e-6, P, 8, None, None)
    with pytest.raises(C.ArgumentError):
        L.free_op_layer_norm_bwd(0, 0, FAR, 1, 8, P, 8, P, 8, P, None, 0, 0, None, 0, P, 8, None, None, 0, None, 0, None)
    with pytest.raises(C.ArgumentError):
        L.free_op_layer_norm_bwd_workspace_bytes(1, FAR + 1000, 1152)
    axes = (C.c_int32 * 1)(8)
    for n, t in ((FAR, 3), (3, FAR)):
        with pytest.raises(C.ArgumentError):
            L.free_op_rope_axes(0, 0, 0, 0, n, t, 1, 8, 1, axes, 1e4, P, 0, P, 8, 8, 8, P, 8, 8, 8, None)
    with pytest.raises(C.ArgumentError):
        L.free_op_gated_linear(1, 0, FAR, 8, 8, P, P, None, P, None, P, None)
    with pytest.raises(C.ArgumentError):
        L.free_op_gated_linear_bwd(1, 0, FAR, 8, 8, P, P, P, P, P, None, None, P, 0, P, None)
    with pytest.raises(C.ArgumentError):
        L.free_op_gated_linear_bwd_workspace_bytes(1, FAR + 64, 64, 64)
    with pytest.raises(C.ArgumentError):
        L.free_op_gated_linear_bwd_workspace_bytes(1, -FAR + 64, 64, 64)
    with pytest.raises(C.ArgumentError):
        L.spec_verify(FAR, 4, 16, P, P, P, P, None, P, None, P, P, None, None)


def test_sizes_of_32_bits_and_integer_types_pass(L):
    want = L.free_op_gated_linear_bwd_workspace_bytes(1, 64, 64, 64)
    assert want > 0 and L.free_op_gated_linear_bwd_workspace_bytes(np.int64(1), np.int32(64), torch.tensor(64), True * 64) == want
    assert L.free_op_gated_linear_bwd_workspace_bytes(0, -(1 << 31), 8, 8) == 0          # negative: an ordinary refusal
    assert L.free_op_gated_linear_bwd_workspace_bytes(0, (1 << 31) - 1, 8, 8) == 0       # above the operator's own limit
    with pytest.raises(C.ArgumentError):
        L.free_op_gated_linear_bwd_workspace_bytes(1, 64.0, 64, 64)


def test_axis_widths_past_32_bits_are_refused():
    import paper_2511_20390_b200 as free
    with pytest.raises(ValueError, match="axis_dims"):
        free.op_rope_axes(torch.zeros(1, 3, 2, 8), torch.zeros(3, 1), (FAR + 8,))
    with pytest.raises(ValueError, match="axis_dims"):
        free.op_rope_axes(torch.zeros(1, 3, 2, 8), torch.zeros(3, 2), (4, 4 - FAR))


def test_threads_that_come_first_share_one_error_word(monkeypatch):
    # a word that is made twice is lost once, with what a kernel reports in it; torch's part is played by fakes
    import contextlib
    import threading
    import time
    from types import SimpleNamespace
    from paper_2511_20390_b200 import binding
    made = []

    def zeros(*args, **kw):
        time.sleep(0.05)
        made.append(torch.empty(1, dtype=torch.int32))
        return made[-1]
    stream = SimpleNamespace(synchronize=lambda: None)
    cuda = SimpleNamespace(device=lambda d: contextlib.nullcontext(), is_current_stream_capturing=lambda: False, current_stream=lambda: stream)
    monkeypatch.setattr(binding, "torch", SimpleNamespace(zeros=zeros, cuda=cuda, int32=torch.int32))
    monkeypatch.setattr(binding, "_ERROR_WORDS", {})
    got = [None] * 4

    def first(i):
        got[i] = binding._error_word(i % 2)
    threads = [threading.Thread(target=first, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(made) == 2 and got[0] is got[2] and got[1] is got[3] and got[0] is not got[1]
    assert binding._ERROR_WORDS == {0: got[0], 1: got[1]}
