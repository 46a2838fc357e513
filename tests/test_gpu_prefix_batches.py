"""Prefix attention over batches of more than a warp of sequences, several pairs of row tiles at both head_dims and over pages, and
every number of warps a merge block has."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import parity


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


MANY = [
    # B, Hq, Hkv, D, gamma, P, longest own
    (33, 32, 8, 128, 0, 1000, 700),       # the 33rd sequence is the first of the second round of lengths
    (48, 32, 8, 128, 0, 2100, 1500),
    (100, 8, 2, 128, 1, 300, 90),         # four rounds
    (64, 32, 8, 64, 4, 700, 300),         # 1,280 rows a KV head, ten row tiles, merged by two warps a block
    (12, 32, 8, 64, 4, 1500, 400),        # 240 rows, one pair, by four
    (40, 16, 4, 64, 4, 513, 200),         # seven row tiles: the last alone
    (37, 7, 1, 64, 8, 129, 140),          # seven heads to a group, 18 of 19 row tiles full
]


@pytest.mark.parametrize("B,Hq,Hkv,D,gamma,P,top", MANY)
def test_batches_of_many_sequences(B, Hq, Hkv, D, gamma, P, top):
    q, kp, vp = _rnd(B, gamma + 1, Hq, D, seed=20), _rnd(Hkv, P, D, seed=21), _rnd(Hkv, P, D, seed=22)
    k, v = _rnd(B, Hkv, top, D, seed=23), _rnd(B, Hkv, top, D, seed=24)
    lens = [gamma + 1 + (37 * b * b) % (top - gamma) for b in range(B)]
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
    want, _, want_lse = _exact(q, kp, vp, P, k, v, lens)
    for num_ctas in (0, 5, 40):
        out, o32, lse = _call(q, kp, vp, P, k, v, lens, gamma, num_ctas=num_ctas)
        parity.check_attention(out.float().cpu().numpy(), want.cpu().numpy())
        parity.check_attention(o32.cpu().numpy(), want.cpu().numpy())
        assert (lse.double() - want_lse).abs().max() < 1e-4


@pytest.mark.parametrize("B,Hq,Hkv,D,gamma,P,top", [MANY[1], MANY[3], MANY[5], (30, 28, 4, 128, 4, 512, 260)])
@pytest.mark.parametrize("bs", [64, 256])
def test_paged_batches_of_many_sequences(B, Hq, Hkv, D, gamma, P, top, bs):
    import paper_2502_20330_b200 as R
    P -= P % bs
    shared, mine = P // bs, -(-top // bs)
    q = _rnd(B, gamma + 1, Hq, D, seed=30)
    pool_k, pool_v = [_rnd(shared + B * mine + 2, Hkv, bs, D, seed=31 + i) for i in range(2)]
    order = torch.randperm(len(pool_k), generator=torch.Generator().manual_seed(33)).int()
    table = torch.cat([order[:shared].expand(B, shared), order[shared:shared + B * mine].view(B, mine)], 1).contiguous().cuda()
    lens = [gamma + 1 + (53 * b * b) % (top - gamma) for b in range(B)]

    def rows(pool, blocks):                                    # [.., blocks] of a table -> [.., Hkv, keys, D]
        return pool[blocks.long()].transpose(-4, -3).flatten(-3, -2)

    kp, vp, k, v = rows(pool_k, table[0, :shared]), rows(pool_v, table[0, :shared]), rows(pool_k, table[:, shared:]), rows(pool_v, table[:, shared:])
    want, _, want_lse = _exact(q, kp, vp, P, k, v, lens)
    ws = R.new_workspace(R.prefix_attention_workspace_bytes(B, Hq, Hkv, D, gamma))
    for num_ctas in (0, 7):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
        R.rapid_verify_attention_prefix_paged(q, pool_k, pool_v, table, _lens(P), _lens(*[P + n for n in lens]), gamma, out, ws,
                                              R.AttnParams(lse_out=lse, num_ctas=num_ctas))
        assert R.workspace_status(ws) == 0
        parity.check_attention(out.float().cpu().numpy(), want.cpu().numpy())
        assert (lse.double() - want_lse).abs().max() < 1e-4
