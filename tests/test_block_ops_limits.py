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


def test_shared_elements_are_found():
    # against the sets of element addresses, for pairs of views of one buffer as results and inputs are
    from paper_2511_20390_b200.binding import _meet
    rng = np.random.default_rng(3)
    buf = torch.zeros(4000)
    base = buf.data_ptr()

    def addresses(t):
        idx = np.zeros(1, np.int64) + (t.data_ptr() - base)
        for n, s in zip(t.shape, t.stride()):
            idx = (idx[:, None] + np.arange(n) * s * t.element_size()).reshape(-1)
        return set((idx[:, None] + np.arange(t.element_size())).reshape(-1).tolist())
    met = apart = 0
    for _ in range(3000):
        kind = rng.integers(4)
        if kind == 0:                                              # dense matrices anywhere
            M, D = int(rng.integers(1, 12)), int(rng.integers(1, 20))
            a, b = (buf[o:o + M * D].view(M, D) for o in rng.integers(0, 400, 2).tolist())
        elif kind == 1:                                            # rows with gaps, columns beside one another
            M, D, s = int(rng.integers(1, 8)), int(rng.integers(1, 10)), int(rng.integers(10, 30))
            a, b = (buf.as_strided((M, D), (s, 1), o) for o in rng.integers(0, 60, 2).tolist())
        elif kind == 2:                                            # heads inside a packed projection, either order of strides
            n, t, h, d = rng.integers(1, 5, 4).tolist()
            H = 3 * h
            o = rng.integers(0, 2 * h + 1, 2).tolist()
            a, b = (buf[:n * t * H * d].view(n, t, H, d)[:, :, q:q + h] for q in o)
            if rng.random() < 0.5:
                a, b = a.transpose(1, 2), b.transpose(1, 2)
        else:                                                      # dense, of different types
            n, (p, q) = int(rng.integers(1, 50)), rng.integers(0, 120, 2).tolist()
            a, b = buf[p:p + n], buf.view(torch.bfloat16)[2 * q:2 * q + n]
        want = bool(addresses(a) & addresses(b))
        assert _meet(a, b) == want and _meet(b, a) == want, (kind, a.shape, a.stride(), b.shape, b.stride(), a.data_ptr() - base, b.data_ptr() - base)
        met += want; apart += not want
    assert met > 500 and apart > 500
    assert not _meet(buf[:0], buf) and not _meet(buf[:8].view(8, 1)[:, :0], buf[:8].view(8, 1))
    # broadcast inputs, and layouts that cannot be compared: not called shared
    assert _meet(buf[3:4].expand(5), buf[:8].view(8)[3:4].expand(5)) and not _meet(buf.as_strided((3, 2), (5, 1)), buf.as_strided((2, 2), (7, 1), 2))
