"""Calls of several threads at once, of sizes whose launches differ: none is refused, and results are those of calls alone."""
import sys
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _at_once(calls, times):
    """Runs every call (of a stream handle; returns a code) `times` times in a thread and stream of its own, all at once."""
    codes, gate, interval = [set() for _ in calls], threading.Barrier(len(calls)), sys.getswitchinterval()

    def work(i):
        stream = torch.cuda.Stream()
        gate.wait(60)
        for k in range(times):
            codes[i].add(calls[i](stream.cuda_stream))
            if k % 256 == 0:
                stream.synchronize()
        stream.synchronize()
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(calls))]
    torch.cuda.synchronize()
    sys.setswitchinterval(1e-6)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join(120)
    finally:
        sys.setswitchinterval(interval)
    assert codes == [{0}] * len(calls)


def test_attention_with_heads_of_different_size():
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    L, calls, results = binding.lib(), [], []
    for d in (6, 62, 8, 50):
        q, k, v = (torch.randn(1, 9, 1, d, device="cuda") for _ in range(3))
        want, lse = free.op_cross_attention(q, k, v, want_lse=True)
        _, shape = binding._cross_shape(q, k, v, None, None, None, None, None, None)
        out, st = torch.empty_like(q), q.stride()[:3]
        calls.append(lambda s, shape=shape, out=out, st=st, keep=(q, k, v): L.free_op_cross_attention(shape, out.data_ptr(), *st, None, None, 0, None, s))
        results.append((out, want))
        grads = free.op_cross_attention_bwd(q, k, v, want, lse, q)
        got = [torch.empty_like(g) for g in grads]
        need = L.free_op_cross_attention_bwd_workspace_bytes(shape)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        args = [shape, want.data_ptr(), *st, lse.data_ptr(), q.data_ptr(), *st] + [a for g in got for a in (g.data_ptr(), *st)] + [ws.data_ptr(), need, None]
        calls.append(lambda s, args=args, keep=(got, ws, lse): L.free_op_cross_attention_bwd(*args, s))
        results += list(zip(got, grads))
    _at_once(calls, 3000)
    assert all(torch.equal(a, b) for a, b in results)


def test_norm_backward_of_rows_of_different_width():
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    L, calls, results = binding.lib(), [], []
    for D in (2048, 8192, 2560, 6144):
        x, g = torch.randn(2, D, device="cuda"), torch.randn(2, D, device="cuda")
        r = free.op_rms_norm(x, want_rstd=True).rstd
        want, dx = free.op_rms_norm_bwd(x, g, r, want_dweight=False)[0], torch.empty_like(x)
        args = [0, 0, 1, 2, 1, D, x.data_ptr(), D, 0, g.data_ptr(), D, 0, r.data_ptr(), None, 0, 0, None, 0, 0, dx.data_ptr(), D, 0, None, D, None, 0]
        calls.append(lambda s, args=args, keep=(x, g, r): L.free_op_rms_norm_bwd(*args, s))
        results.append((dx, want))
    _at_once(calls, 4000)
    assert all(torch.equal(a, b) for a, b in results)


def test_self_attention_of_different_lengths():
    import paper_2511_20390_b200 as free
    from paper_2511_20390_b200 import binding
    L, calls, results = binding.lib(), [], []
    for n in (8, 2600, 16, 2000):
        qkv = torch.randn(1, n, 48, device="cuda")
        want = free.op_attention(qkv, 1)
        out = torch.empty_like(want)
        need = L.free_op_attention_workspace_bytes(0, 1, n, 1, 16)
        ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        args = [0, 1, n, 1, 16, qkv.data_ptr(), out.data_ptr(), ws.data_ptr(), need]
        calls.append(lambda s, args=args, keep=(qkv, ws): L.free_op_attention(*args, s))
        results.append((out, want))
    _at_once(calls, 2000)
    assert all(torch.equal(a, b) for a, b in results)
