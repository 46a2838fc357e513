"""Prefix attention at the ends of bf16's range: keys without weight whose values are the largest there are, and large values under
scores that rise along the keys."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16_MAX = torch.finfo(torch.bfloat16).max


def _rnd(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()


def _lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def _call(q, kp, vp, P, k, v, lens, gamma, **kw):
    """(out, out in fp32, lse), the status having been 0"""
    import paper_2502_20330_b200 as R
    B, rows, Hq, D = q.shape
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, k.shape[1], D, gamma))
    out, o32 = torch.empty_like(q), torch.empty(q.shape, dtype=torch.float32, device="cuda")
    lse = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
    R.rapid_verify_attention_prefix(q, kp, vp, _lens(P), k, v, _lens(*lens), gamma, out, ws,
                                    R.AttnParams(lse_out=lse, out_f32=o32, **kw))
    assert R.workspace_status(ws) == 0
    return out, o32, lse


def _exact(q, kp, vp, P, k, v, lens):
    """(out, sum of p |v|, lse) of every row from the definition in 64 bits."""
    B, R_, Hq, D = q.shape
    Hkv = k.shape[1]
    out, size = torch.empty(2, *q.shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(q.shape[:3], dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        kk, vv = torch.cat([kp[:, :P], k[b, :, :n]], 1).double(), torch.cat([vp[:, :P], v[b, :, :n]], 1).double()
        x = q[b].double().view(R_, Hkv, -1, D).permute(1, 2, 0, 3)                        # [Hkv, G, R, D]
        s = x @ kk[:, None].transpose(2, 3) / D ** 0.5
        lim = P + n - R_ + torch.arange(R_, device="cuda")
        s = s.masked_fill(torch.arange(P + n, device="cuda") > lim[:, None], -float("inf"))
        p = torch.softmax(s, -1)
        for o, val in ((out, vv), (size, vv.abs())):
            o[b] = (p @ val[:, None]).permute(2, 0, 1, 3).reshape(R_, Hq, D)
        lse[b] = torch.logsumexp(s, -1).permute(2, 0, 1).reshape(R_, Hq)
    return out, size, lse


@pytest.mark.parametrize("low", [-float("inf"), -2.0 ** 11])
@pytest.mark.parametrize("D", [64, 128])
def test_keys_without_weight_add_nothing_however_large_their_values(D, low):
    """Every third key's score is -inf, or 2^11 / sqrt(D) below the others (more than 2^-250 in weight), and its V the largest
    finite value.  Tolerance: probabilities and output are rounded to bf16, 2^-8 of sum p |v| each at most."""
    P, n, gamma = 300, 75, 3
    q, kp, vp = _rnd(2, gamma + 1, 4, D, seed=1), _rnd(2, P, D, seed=2), _rnd(2, P, D, seed=3)
    k, v = _rnd(2, 2, n, D, seed=4), _rnd(2, 2, n, D, seed=5)
    q[..., 0] = 1
    for keys, values in ((kp, vp), (k, v)):
        keys[..., ::3, 0] = low
        values[..., ::3, :] = BF16_MAX
    got = _call(q, kp, vp, P, k, v, (n, n), gamma)
    want, size, lse = _exact(q, kp, vp, P, k, v, (n, n))
    assert torch.isfinite(want).all() and size.max() < 100
    assert ((got[0].double() - want).abs() <= 2 * 2 ** -8 * size + 1e-6).all()
    assert (got[2].double() - lse).abs().max() < 1e-4


@pytest.mark.parametrize("D,B,num_ctas", [(64, 2, 1), (128, 2, 1), (128, 12, 1), (128, 12, 3)])
@pytest.mark.parametrize("rise", [12, 36])
def test_large_values_where_scores_rise_along_the_keys(D, B, num_ctas, rise):
    """Later keys weigh 2^rise times the earlier ones and V is around 2^95 everywhere: times the keys 2^106, inside the 2^111 that the
    call allows.  (A CTA takes long runs of tiles here, so that rows come to the later keys with a reference of the earlier.)
    Tolerance: 2^-8 of sum p |v| for the probabilities and for the output, 2^-11 for the scores' fp32 sums: 128 products of at
    most 600 in all, 128 * 2^-24 * 600 / sqrt(128) < 2^-11."""
    P, n, gamma = 640, 400, 4
    q, kp, vp = _rnd(B, gamma + 1, 8, D, seed=10), _rnd(2, P, D, seed=11), _rnd(2, P, D, seed=12)
    k, v = _rnd(B, 2, n, D, seed=13), _rnd(B, 2, n, D, seed=14)
    q[..., 0] = 1
    by = rise * np.log(2) * D ** 0.5
    for keys in (kp, k):
        keys[..., 0] = 0
        keys[..., 64:, 0] = by / 2
        keys[..., 256:, 0] = by
    vp *= 2.0 ** 95
    v *= 2.0 ** 95
    lens = [n - 7 * b for b in range(B)]
    got = _call(q, kp, vp, P, k, v, lens, gamma, num_ctas=num_ctas)
    want, size, _ = _exact(q, kp, vp, P, k, v, lens)
    assert ((got[0].double() - want).abs() <= (2 * 2 ** -8 + 2 ** -11) * size).all()
    assert ((got[1].double() - want).abs() <= (2 ** -8 + 2 ** -11) * size).all()
