"""Attention of many new rows over the cache against the definition in 64 bits.

Tolerance of an output element: with A the softmax-weighted sum of |v|, the probabilities' rounding to bf16 is off by at most 2^-8 A,
the output's by 2^-8 |out|; the exponentials (3e-6), the fp32 scores (D products and sums of exact bf16 products, |score| up to 10 here
unless a test says more: 1e-5 in the exponent) and the fp32 sums add at most 4e-5 A.  The log-sum-exp is within 1e-4.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2502_20330_b200 as R

LSE_TOL = 1e-4


def _bf(*shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()


def _want(q, k, v, n, window=0, sink=0, all_visible=False, scale=None):
    """Rows q [T, Hq, D] of one sequence over its keys k, v [Hkv, L, D], n of the rows: (out, A, lse) in float64."""
    T, Hq, D = q.shape
    Hkv, L, _ = k.shape
    G = Hq // Hkv
    qd = q[:n].double().view(n, Hkv, G, D)
    pos = torch.arange(L - n, L, device="cuda")[:, None]
    j = torch.arange(L, device="cuda")[None]
    seen = torch.ones(n, L, dtype=torch.bool, device="cuda") if all_visible else j <= pos
    if window:
        seen &= (j > pos - window) | (j < sink)
    out, mag, lse = [], [], []
    for h in range(Hkv):
        s = torch.einsum("rgd,nd->rgn", qd[:, h], k[h].double()) * (D ** -0.5 if scale is None else scale)
        s = s.masked_fill(~seen[:, None], -math.inf)
        w = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(w == -math.inf, 0.0, w)[..., None])
        vd = v[h].double()
        out.append(torch.einsum("rgn,nd->rgd", p, vd))
        mag.append(torch.einsum("rgn,nd->rgd", p, vd.abs()))
        lse.append(w)
    return torch.stack(out, 1).reshape(n, Hq, D), torch.stack(mag, 1).reshape(n, Hq, D), torch.stack(lse, 1).reshape(n, Hq)


def _close(out, lse, want, extra=0.0):
    o, mag, w = want
    off = (out.double() - o).abs()
    tol = (2.0 ** -8 + 4e-5 + extra) * mag + 2.0 ** -8 * o.abs()
    assert (off <= tol).all(), (off - tol).max().item()
    if lse is not None:
        both = torch.where(w == lse.double(), 0.0, (lse.double() - w).abs())
        assert (both <= LSE_TOL).all(), both.max().item()


class _Case:
    """Inputs of a batch; the caches' rows past every sequence's keys hold NaN."""

    def __init__(self, B, T, Hq, Hkv, D, old, block=0, ragged=True, seed=0, slack=37, scale=1.0):
        g = torch.Generator().manual_seed(1000 * seed + B * T + old)
        self.B, self.T, self.Hq, self.Hkv, self.D = B, T, Hq, Hkv, D
        n = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32) if ragged else torch.full((B,), T, dtype=torch.int32)
        n[0] = T
        olds = torch.randint(0, old + 1, (B,), generator=g, dtype=torch.int32)
        olds[0] = old
        self.n, self.ctx = n, n + olds
        self.q = _bf(B, T, Hq, D, seed=seed + 1, scale=scale)
        rows = int(self.ctx.max()) + slack
        self.k, self.v = _bf(B, Hkv, rows, D, seed=seed + 2), _bf(B, Hkv, rows, D, seed=seed + 3)
        for b in range(B):
            self.k[b, :, int(self.ctx[b]):] = math.nan
            self.v[b, :, int(self.ctx[b]):] = math.nan
        self.block, self.table = block, None
        if block:
            per = -(-rows // block)
            order = torch.randperm(B * per + 2, generator=g)
            self.table = order[:B * per].view(B, per).to(torch.int32)
            self.kp, self.vp = (torch.full((B * per + 2, Hkv, block, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            for pool, src in ((self.kp, self.k), (self.vp, self.v)):
                for b in range(B):
                    for i in range(per):
                        part = src[b, :, i * block:(i + 1) * block]
                        pool[int(self.table[b, i]), :, :part.shape[1]] = part
            # entries past the blocks that a sequence uses are never read
            for b in range(B):
                self.table[b, -(-int(self.ctx[b]) // block):] = -7
            self.table = self.table.cuda()
        self.out = torch.full_like(self.q, 3.0)
        self.lse = torch.full((B, T, Hq), 3.0, device="cuda")
        self.o32 = torch.full((B, T, Hq, D), 3.0, device="cuda")
        self.ws = R.new_workspace(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T))

    def run(self, null_counts=False, **params):
        p = R.AttnParams(lse_out=self.lse, out_f32=self.o32, **params)
        n = None if null_counts else self.n.cuda()
        if self.block:
            R.rapid_prefill_attention_paged(self.q, self.kp, self.vp, self.table, self.ctx.cuda(), self.out, self.ws, n_tokens=n, params=p)
        else:
            R.rapid_prefill_attention(self.q, self.k, self.v, self.ctx.cuda(), self.out, self.ws, n_tokens=n, params=p)
        return self

    def check(self, status=0, extra=0.0, **mask):
        assert R.workspace_status(self.ws) == status
        for b in range(self.B):
            n, L = int(self.n[b]), int(self.ctx[b])
            if n:
                want = _want(self.q[b], self.k[b, :, :L], self.v[b, :, :L], n, **mask)
                _close(self.out[b, :n], self.lse[b, :n], want, extra)
                off = (self.o32[b, :n].double() - want[0]).abs()
                assert (off <= (2.0 ** -8 + 4e-5 + extra) * want[1] + 2.0 ** -23 * want[0].abs()).all()
            assert (self.out[b, n:] == 3.0).all() and (self.lse[b, n:] == 3.0).all() and (self.o32[b, n:] == 3.0).all()
        return self


@pytest.mark.parametrize("B,T,Hq,Hkv,D,old", [
    (1, 1, 8, 2, 64, 0), (1, 1, 32, 8, 128, 700), (2, 31, 8, 2, 128, 5), (1, 32, 32, 8, 128, 0), (3, 33, 32, 8, 128, 100), (2, 64, 4, 1, 64, 64),
    (1, 65, 4, 1, 128, 127), (2, 127, 2, 2, 64, 1), (1, 129, 3, 3, 128, 0), (1, 257, 2, 2, 128, 128), (4, 18, 28, 4, 128, 300),
    (1, 37, 28, 4, 128, 90), (2, 50, 15, 5, 64, 33), (2, 25, 10, 2, 128, 2), (1, 9, 64, 1, 128, 40), (1, 3, 128, 1, 64, 10), (2, 2, 100, 1, 128, 511),
    (1, 700, 32, 8, 128, 0), (2, 1000, 8, 2, 64, 77), (7, 40, 16, 2, 128, 1000), (70, 6, 8, 2, 64, 30),
])
@pytest.mark.parametrize("block", [0, 64, 256])
def test_causal(B, T, Hq, Hkv, D, old, block):
    _Case(B, T, Hq, Hkv, D, old, block, seed=B + T).run().check()


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (64, 4), (127, 200), (128, 128), (500, 1), (700, 2000), (4092, 4), (2 ** 31 - 1, 0)])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,old,block", [(2, 300, 8, 2, 128, 900, 0), (1, 1500, 4, 4, 64, 0, 64), (3, 1, 32, 8, 128, 2000, 128), (1, 260, 7, 1, 128, 50, 0)])
def test_window(window, sink, B, T, Hq, Hkv, D, old, block):
    _Case(B, T, Hq, Hkv, D, old, block, seed=7).run(window_keys=window, sink_keys=sink).check(window=window, sink=sink)


@pytest.mark.parametrize("B,T,Hq,Hkv,D,old,block", [(2, 70, 8, 2, 64, 500, 0), (1, 200, 4, 4, 128, 0, 0), (2, 40, 28, 4, 128, 300, 64)])
def test_all_keys_visible(B, T, Hq, Hkv, D, old, block):
    _Case(B, T, Hq, Hkv, D, old, block, seed=9).run(all_keys_visible=True).check(all_visible=True)


def test_units_in_whole_and_in_parts():
    """More units than two for every CTA: most are whole, the last ones cut.  Causal and within a window; all rows present."""
    c = _Case(2, 1200, 32, 8, 128, 40, ragged=False, seed=11).run(null_counts=True).check()
    c.run(null_counts=True, window_keys=300, sink_keys=10).check(window=300, sink=10)
    c = _Case(1, 4100, 8, 8, 64, 0, ragged=False, seed=12).run().check()


@pytest.mark.parametrize("num_ctas", [1, 2, 7, 100, 147, 256])
def test_any_number_of_ctas(num_ctas):
    for case in (_Case(1, 20, 32, 8, 128, 5000, ragged=False, seed=13), _Case(5, 200, 8, 2, 64, 300, seed=14)):
        case.run(num_ctas=num_ctas).check()
        first = case.out.clone()
        case.run(num_ctas=num_ctas)
        assert torch.equal(first, case.out)                    # the order of every sum is fixed


def test_few_rows_over_many_keys():
    _Case(1, 3, 8, 1, 128, 60000, ragged=False, seed=15).run().check()
    _Case(2, 40, 8, 2, 128, 9000, 64, seed=16).run().check()
