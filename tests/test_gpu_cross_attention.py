"""op_cross_attention and its backward pass against the fp64 definitions.

Tolerances (u = 2^-24, b = 2^-8: half a step of bf16 relative to the value).  A score is a sum of d products: off by at most
(d + 4) u scale sum |q k|, plus 4 u of itself for the scaling and the exponent's argument; that is the relative error of e^S, to
which the exponential adds 8 u.  Call it E (the row's largest).  Sums over n states run in any order: n u of the sum of magnitudes.
In bf16 a probability, and a dS, is rounded once before the product that takes it: b of each term.  A result is rounded once:
eps / 2 of its type.  So
    out   sum_j p |v_j| (2 E + (n + 16) u [+ b]) + half |out|             (E twice: p and the sum that it is divided by)
    lse   E + (n + 16) u + 4 u |lse|
    dv    sum p |g| (E + (rows + 16) u [+ b]) + half |dv|
    dS    an error of (d + 8) u p scale (sum |g v| + sum |g o|) and of dS (E [+ b]), both within  terms (E + (d + 8) u [+ b]), terms as
          the oracle gives it with the products, so that dq and dk are off by at most that sum (+ (rows + 16) u) + half of themselves."""
import math

import numpy as np
import pytest
import torch

import synth
from oracle import block_ops as ob

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _half(dt):
    return torch.finfo(DT[dt]).eps / 2


def _b(dt):
    return 2.0 ** -8 if dt == "bf16" else 0.0


class Case:
    """Inputs of a call on the GPU, in one of the layouts, and what the oracle needs of them."""

    def __init__(self, seed, dt, n_seq, n_enc, n_q, n_kv, heads, kvh, d, lens="ragged", layout="padded", mask=False, seq_of=None, scale=None,
                 junk=True, spread=1.0):
        rng = np.random.default_rng(seed)
        self.dt, self.scale, self.heads, self.kvh, self.d = dt, (d ** -0.5 if scale is None else scale), heads, kvh, d
        if lens == "full":
            n = [n_kv] * n_enc
        elif lens == "ragged":
            n = [n_kv] + [int(v) for v in rng.integers(0, n_kv + 1, n_enc - 1)]
        else:
            n = list(lens)
        self.lens = n
        t = lambda a: torch.from_numpy(np.asarray(a, np.float32)).to(DT[dt])
        q = t(spread * synth.normal(seed, 1, (n_seq, n_q, heads, d)))
        ks = [t(spread * synth.normal(seed, 10 + e, (m, kvh, d))) for e, m in enumerate(n)]
        vs = [t(synth.normal(seed, 110 + e, (m, kvh, d))) for e, m in enumerate(n)]
        self.counts = [np.ones(m, bool) if not mask else rng.random(m) < 0.7 for m in n]
        self.seq_of = None if seq_of is None else list(seq_of)
        self.enc_of = self.seq_of if seq_of is not None else [s // (n_seq // n_enc) for s in range(n_seq)]
        bad = float("nan") if junk else 0.0
        # q inside a packed projection with rubbish around it
        full = torch.full((n_seq, n_q, 3, heads, d), bad, dtype=DT[dt], device="cuda")
        full[:, :, 1] = q.cuda()
        self.q = full[:, :, 1]
        self.kw = {"scale": scale}
        if layout == "padded":
            kv = torch.full((n_enc, n_kv, 2, kvh, d), bad, dtype=DT[dt], device="cuda")
            where = lambda e: kv[e, :n[e]]
            self.kw["kv_lens"] = torch.tensor(n, dtype=torch.int32, device="cuda")
            mk = torch.ones((n_enc, n_kv), dtype=torch.bool, device="cuda")
            mrow = lambda e: mk[e, :n[e]]
            self.span = [(e, slice(0, n[e])) for e in range(n_enc)]
        else:                                                      # rubbish in front of the first sequence and behind the last
            at = np.concatenate([[3], 3 + np.cumsum(n)]).astype(np.int32)
            kv = torch.full((int(at[-1]) + 5, 2, kvh, d), bad, dtype=DT[dt], device="cuda")
            where = lambda e: kv[at[e]:at[e + 1]]
            self.kw["kv_offsets"] = torch.from_numpy(at).cuda()
            mk = torch.ones(len(kv), dtype=torch.bool, device="cuda")
            mrow = lambda e: mk[at[e]:at[e + 1]]
            self.span = [(slice(at[e], at[e + 1]),) for e in range(n_enc)]
        for e in range(n_enc):
            dst = where(e)
            dst[:, 0], dst[:, 1] = ks[e].cuda(), vs[e].cuda()
            if mask:
                mrow(e).copy_(torch.from_numpy(self.counts[e]))
                dst[~torch.from_numpy(self.counts[e]).cuda()] = bad if seed % 2 else float("inf")
        if mask:
            self.kw["kv_mask"] = mk
        self.k, self.v = (kv[:, :, 0], kv[:, :, 1]) if layout == "padded" else (kv[:, 0], kv[:, 1])
        if seq_of is not None:
            self.kw["kv_seq"] = torch.tensor(self.seq_of, dtype=torch.int32, device="cuda")
        self.qf = q.double().numpy()
        self.ksf, self.vsf = [k.double().numpy() for k in ks], [v.double().numpy() for v in vs]
        self.g = t(0.1 * synth.normal(seed, 2, (n_seq, n_q, heads, d))).cuda()

    def spread_of_score(self):
        """E of the header, per sequence, head and token."""
        out = np.zeros((self.qf.shape[0], self.heads, self.qf.shape[1]))
        for s, e in enumerate(self.enc_of):
            use = np.flatnonzero(self.counts[e]) if 0 <= e < len(self.ksf) else []
            for h in range(self.heads):
                if len(use):
                    k = self.ksf[e][use, h // (self.heads // self.kvh)]
                    mag = self.scale * np.abs(self.qf[s, :, h]) @ np.abs(k).T
                    out[s, h] = ((self.d + 4) * U * mag + 4 * U * mag).max(1) + 8 * U
        return out

    def check(self, backward=True):
        import paper_2511_20390_b200 as free
        E = self.spread_of_score()
        En = E.transpose(0, 2, 1)[..., None]                       # [n_seq, n_q, heads, 1]
        n = max([1] + self.lens)
        out, lse = free.op_cross_attention(self.q, self.k, self.v, want_lse=True, **self.kw)
        assert free.op_device_error() == 0
        oo, lo = ob.cross_attention(self.qf, self.ksf, self.vsf, self.counts, self.enc_of, self.scale)
        mag, _ = ob.cross_attention(self.qf, self.ksf, [np.abs(v) for v in self.vsf], self.counts, self.enc_of, self.scale)
        og, lg = out.double().cpu().numpy(), lse.double().cpu().numpy()
        assert np.array_equal(np.isneginf(lg), np.isneginf(lo))
        fine = np.isfinite(lo)
        assert (np.abs(lg[fine] - lo[fine]) <= E[fine] + (n + 16) * U + 4 * U * np.abs(lo[fine])).all()
        assert (np.abs(og - oo) <= mag * (2 * En + (n + 16) * U + _b(self.dt)) + _half(self.dt) * np.abs(oo) * (1 + 1e-3) + 1e-37).all()
        if not backward:
            return
        got = free.op_cross_attention_bwd(self.q, self.k, self.v, out, lse, self.g, **self.kw)
        assert free.op_device_error() == 0
        dq, dk, dv, mq, mk, mv = ob.cross_attention_bwd(self.qf, self.ksf, self.vsf, self.counts, self.enc_of, self.scale, og, lg, self.g.double().cpu().numpy())
        rows = self.qf.shape[0] * self.qf.shape[1] * (self.heads // self.kvh)
        # e^(S - lse) with the lse that was kept (an fp32 number: half a step of it)
        lmag = np.where(fine, np.abs(lo), 0.0)
        R = (E + 2 * U * lmag + 8 * U).max() + (self.d + 8) * U + _b(self.dt)
        close = lambda a, want, m, k: (np.abs(a - want) <= m * (R + (k + 16) * U) + _half(self.dt) * np.abs(want) * (1 + 1e-3) + 1e-37).all()
        assert close(got[0].double().cpu().numpy(), dq, mq, n)
        left_k, left_v = got[1].double().cpu().numpy(), got[2].double().cpu().numpy()
        for e in range(len(self.lens)):
            assert close(left_k[self.span[e]], dk[e], mk[e], rows) and close(left_v[self.span[e]], dv[e], mv[e], rows)
            left_k[self.span[e]] = left_v[self.span[e]] = 0
        assert (left_k == 0).all() and (left_v == 0).all()         # padding, and rows of no sequence
        again = free.op_cross_attention_bwd(self.q, self.k, self.v, out, lse, self.g, **self.kw)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        out2, lse2 = free.op_cross_attention(self.q, self.k, self.v, want_lse=True, **self.kw)
        assert torch.equal(out, out2) and torch.equal(lse, lse2)


SHAPES = [  # n_seq, n_enc, n_q, n_kv, heads, kv_heads, d
    (1, 1, 1, 1, 1, 1, 8), (2, 2, 1, 77, 6, 6, 64), (3, 3, 5, 3, 2, 1, 16), (2, 1, 64, 64, 2, 2, 64), (4, 2, 65, 63, 2, 2, 72), (2, 2, 130, 129, 4, 4, 80),
    (3, 3, 100, 300, 3, 3, 40), (1, 1, 257, 128, 2, 2, 128), (6, 2, 33, 17, 6, 2, 96), (2, 2, 200, 256, 4, 1, 64), (1, 1, 7, 513, 8, 2, 128),
    (5, 5, 128, 120, 1, 1, 32), (2, 2, 300, 77, 12, 4, 24), (1, 1, 384, 640, 1, 1, 112), (2, 2, 3, 1000, 8, 1, 128), (1, 1, 16, 700, 3, 3, 104),
]


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["padded", "packed"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(shape, layout, dt):
    Case(sum(shape), dt, *shape, layout=layout).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["padded", "packed"])
@pytest.mark.parametrize("shape", SHAPES[1:12:2], ids=str)
def test_masks_with_holes(shape, layout, dt):
    """Masked states hold NaN or infinities."""
    for seed in (1, 2):
        Case(seed + sum(shape), dt, *shape, layout=layout, mask=True).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [3, 20, 36, 65, 77, 100, 127])
def test_head_sizes_of_no_tile(dt, d):
    Case(d, dt, 2, 2, 70, 90, 2, 2, d).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["padded", "packed"])
def test_sequences_without_states(layout, dt):
    c = Case(7, dt, 6, 3, 70, 90, 2, 2, 64, lens=[90, 0, 33], layout=layout)
    c.check()
    Case(8, dt, 3, 3, 20, 30, 2, 1, 32, lens=[0, 0, 0], layout=layout).check()
    Case(9, dt, 4, 4, 20, 130, 2, 1, 32, lens=[0, 1, 130, 128], layout=layout).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["padded", "packed"])
def test_sequences_choose_their_states(layout, dt):
    """Any order, some encoder sequences unread, some read often, indices of none."""
    Case(11, dt, 7, 4, 40, 50, 4, 2, 64, layout=layout, seq_of=[3, 0, 3, -1, 0, 4, 3]).check()
    Case(12, dt, 2, 5, 150, 140, 2, 2, 40, layout=layout, seq_of=[4, 4]).check()


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("spread", [0.01, 6.0])
def test_flat_and_sharp_scores(dt, spread):
    """Scores of hundreds: single states take everything; offsets of the running maximum move."""
    Case(13, dt, 2, 2, 140, 400, 2, 2, 64, spread=spread).check()
    Case(14, dt, 1, 1, 70, 300, 2, 1, 72, spread=spread, scale=0.5).check()


@pytest.mark.parametrize("layout", ["padded", "packed"])
@pytest.mark.parametrize("shape,lens", [
    ((16, 4, 520, 300, 12, 12, 72), [300, 1, 0, 257]), ((40, 8, 130, 90, 8, 2, 64), "ragged"), ((30, 30, 33, 140, 10, 5, 128), "ragged"),
    ((200, 1, 5, 130, 4, 1, 40), "full"), ((3, 3, 1500, 520, 16, 16, 48), [520, 512, 513]),
])
def test_more_items_than_sms(shape, lens, layout):
    """CTAs walk over several items each, long and short ones, some without a state."""
    Case(21, "bf16", *shape, lens=lens, layout=layout, mask=shape[0] == 30).check()
