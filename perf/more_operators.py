"""Cases for the operators that bring a prompt, or the next piece of one, into a cache: the position rotation of queries and
keys (one position axis for text, three for images and video), appending rows to a cache with the rotation applied on the
way, and the attention of many new rows over the cache, causal, within a window with a few first tokens (sinks), or over all keys.

``own`` chooses between the plain torch forms and the library's calls.  Shapes follow the workloads of this repository
(32/8, 28/4, 64/8 and 8/2 heads, head_dim 64 and 128, 32K to 128K contexts, gamma 0 to 8, the drafter's 4 sinks and
4,092 window keys).
"""
import math

import torch

own = False


def listed():
    return [
        # queries and keys of a batch's verify step deep in a long context: what a call costs at all
        dict(name="rope_step", op="rope", B=4, T=5, Hq=28, Hkv=4, D=128, rd=128, axes=1, inter=False, far=100000),
        # two videos' tokens at positions of time, height and width
        dict(name="rope_video", op="rope", B=2, T=20011, Hq=28, Hkv=4, D=128, rd=128, axes=3, inter=False, far=0),
        # a prompt of a model that turns a half of each head, in neighbouring pairs
        dict(name="rope_partial", op="rope", B=3, T=3001, Hq=8, Hkv=2, D=64, rd=32, axes=1, inter=True, far=5000),
        # the rows of one verify step
        dict(name="append_step", op="append", B=1, T=9, ragged=False, Hq=32, Hkv=8, D=128, rd=128, axes=1, inter=False, old=32000, block=0),
        # the rows of a batch's verify step, paged
        dict(name="append_batch", op="append", B=64, T=5, ragged=False, Hq=28, Hkv=4, D=128, rd=128, axes=1, inter=False, old=2000, block=64),
        # three prompts of different lengths with images in them
        dict(name="append_prompts", op="append", B=3, T=24000, ragged=True, Hq=32, Hkv=8, D=128, rd=128, axes=3, inter=False, old=100, block=256),
        # two short questions behind a little text
        dict(name="prefill_short", op="prefill", B=2, T=100, ragged=True, Hq=8, Hkv=2, D=64, old=50, sink=0, window=0, block=0),
        # a drafter's retrieved context
        dict(name="prefill_8k", op="prefill", B=1, T=8192, ragged=False, Hq=32, Hkv=8, D=128, old=0, sink=0, window=0, block=0),
        # a whole document
        dict(name="prefill_32k", op="prefill", B=1, T=32768, ragged=False, Hq=32, Hkv=8, D=128, old=0, sink=0, window=0, block=0),
        # the same document through the streaming drafter's mask
        dict(name="prefill_window_32k", op="prefill", B=1, T=32768, ragged=False, Hq=32, Hkv=8, D=128, old=0, sink=4, window=4092, block=0),
        # the next piece of a prompt, 128K behind it, paged
        dict(name="prefill_piece_128k", op="prefill", B=1, T=500, ragged=False, Hq=32, Hkv=8, D=128, old=130000, sink=0, window=0, block=64),
        # prompts of different lengths at seven heads to a group, behind what their caches hold
        dict(name="prefill_ragged", op="prefill", B=8, T=4001, ragged=True, Hq=28, Hkv=4, D=128, old=3000, sink=0, window=0, block=256),
    ]


_MOST_FLOPS = 8.8e12  # a pass of the largest listed case


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "prefill", "prefill", "prefill"])
    Hq, Hkv, D = rng.choice([(8, 2, 64), (32, 8, 128), (28, 4, 128), (64, 8, 128), (8, 8, 64), (16, 2, 128)])
    c = dict(op=op, Hq=Hq, Hkv=Hkv, D=D)
    if op == "prefill":
        B = _log(rng, 1, 16)
        T = _log(rng, 1, 32768 // B)
        old = rng.choice([0, _log(rng, 1, max(2, 131072 // B - T))])
        while 4 * D * Hq * B * T * (old + T // 2 + 1) > _MOST_FLOPS:
            old, T = old // 2, max(1, 3 * T // 4)
        sink, window = rng.choice([(0, 0), (0, 0), (rng.randint(0, 40), _log(rng, 1, 6000))])
        return dict(c, B=B, T=T, ragged=rng.random() < 0.6, old=old, sink=sink, window=window, block=rng.choice([0, 0, 64, 128, 256]))
    axes = rng.choice([1, 1, 2, 3])
    B = _log(rng, 1, 64)
    T = _log(rng, 1, max(2, 400_000_000 // (D * (Hq + 2 * Hkv)) // B))
    c.update(B=B, T=min(T, 40000), rd=rng.choice([D, D, D // 2]), axes=axes, inter=rng.random() < 0.3)
    if op == "rope":
        return dict(c, far=rng.choice([0, _log(rng, 10, 1000000)]))
    return dict(c, ragged=rng.random() < 0.6, old=rng.choice([0, _log(rng, 1, 4000)]), block=rng.choice([0, 16, 64, 256]))


# ---- inputs -----------------------------------------------------------------------------------------------------


def _counts(case):
    """New rows of every sequence, by the case alone, so that work() knows them; the first sequence has them all."""
    g = torch.Generator().manual_seed(20334 + case["T"] + 131 * case["B"])
    n = torch.randint(case["T"] // 3 + 1, case["T"] + 1, (case["B"],), generator=g, dtype=torch.int32)
    n[0] = case["T"]
    return n if case["ragged"] else torch.full_like(n, case["T"])


def _olds(case):
    """Keys that every cache holds before the new rows; the first sequence has the most."""
    g = torch.Generator().manual_seed(20335 + case["old"] + 131 * case["B"])
    n = torch.randint(case["old"] // 2, case["old"] + 1, (case["B"],), generator=g, dtype=torch.int32)
    n[0] = case["old"]
    return n


def _rows(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _pair_axis(case):
    """The axis that turns each pair: the first share of the pairs goes by time, the next by height, the last by width."""
    n, axes = case["rd"] // 2, case["axes"]
    return sorted([0] * (n - (axes - 1) * (n // axes)) + [a for a in range(1, axes) for _ in range(n // axes)])


def _grid(g, axes, B, T, far):
    """[axes, B, T] positions: a run of text for one axis, frames of rows and columns for more."""
    t = torch.arange(T, device="cuda")
    wide, high = 16, (12 if axes == 3 else T)
    parts = [t // (wide * high), t // wide % high, t % wide]
    parts = [t] if axes == 1 else parts[3 - axes:]
    start = torch.randint(0, far + 1, (B, 1), generator=g, device="cuda")
    return torch.stack([start + p for p in parts]).to(torch.int32).contiguous()


def _table(g, case, rows):
    """A pool's block table: every sequence's blocks in an order of their own, and how many blocks there are."""
    per = -(-rows // case["block"])
    order = torch.randperm(case["B"] * per + 3, generator=g, device="cuda")
    return order[:case["B"] * per].view(case["B"], per).to(torch.int32).contiguous(), case["B"] * per + 3


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    c, s = case, {"case": case}
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    s["q"] = _rows(g, B, T, Hq, D)
    if c["op"] != "prefill":
        s["freq"] = torch.exp2(-math.log2(500000.0) * torch.arange(c["rd"] // 2, device="cuda") / (c["rd"] // 2)).float()
        s["kn"] = _rows(g, B, T, Hkv, D)
        s["qo"] = torch.zeros_like(s["q"])
    if c["op"] == "rope":
        s["pos"] = _grid(g, c["axes"], B, T, c["far"])
        s["ko"] = torch.zeros_like(s["kn"])
    else:
        n, old = _counts(c), _olds(c)
        s["n"] = n.cuda() if c["ragged"] else None
        rows = int((n + old).max())
        if c["block"]:
            s["table"], blocks = _table(g, c, rows)
            s["k"], s["v"] = (_rows(g, blocks, Hkv, c["block"], D) for _ in range(2))
        else:
            s["k"], s["v"] = (_rows(g, B, Hkv, rows, D) for _ in range(2))
        if c["op"] == "append":
            s["vn"] = _rows(g, B, T, Hkv, D)
            s["ctx"] = old.cuda()
            s["lens"] = torch.zeros_like(s["ctx"])
            s["pos"] = _grid(g, c["axes"], B, T, c["old"]) if c["axes"] > 1 else None
        else:
            s["ctx"] = (n + old).cuda()
            s["out"] = torch.zeros_like(s["q"])
            s["lse"] = torch.zeros(B, T, Hq, device="cuda")
    if own:
        import paper_2502_20330_b200 as R
        if c["op"] == "prefill":
            s["params"] = R.AttnParams(lse_out=s["lse"], sink_keys=c["sink"], window_keys=c["window"])
            s["ws"] = R.new_workspace(R.prefill_attention_workspace_bytes(B, Hq, Hkv, D, T))
        else:
            s["rope"] = R.Rope(s["freq"], rotary_dim=c["rd"], interleaved=c["inter"],
                               pair_axis=_pair_axis(c) if c["axes"] > 1 else None)
            s["status"] = R.new_workspace(256)[:4].view(torch.int32)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------


def _turned(x, pos, s, c):
    """x [B, T, H, D] with its first rd columns turned by pos [axes, B, T]; angles in 64 bits, where 32 lose far positions."""
    half = c["rd"] // 2
    axis = torch.tensor(_pair_axis(c), device=pos.device)
    angle = pos[axis].permute(1, 2, 0).double() * s["freq"].double()                  # [B, T, half]
    cos, sin = (f(angle).float()[:, :, None, :] for f in (torch.cos, torch.sin))
    y = x.float()
    head = y[..., :c["rd"]]
    a, b = (head[..., 0::2], head[..., 1::2]) if c["inter"] else (head[..., :half], head[..., half:])
    p, q = a * cos - b * sin, a * sin + b * cos
    head = torch.stack([p, q], -1).flatten(-2) if c["inter"] else torch.cat([p, q], -1)
    return torch.cat([head, y[..., c["rd"]:]], -1).to(torch.bfloat16)


def _rope_plain(s, c):
    return _turned(s["q"], s["pos"], s, c), _turned(s["kn"], s["pos"], s, c)


def _append_plain(s, c):
    i = torch.arange(c["T"], device="cuda")
    at = s["ctx"].long()[:, None] + i                                                 # [B, T]
    pos = s["pos"] if s["pos"] is not None else at[None]
    new = (i < s["n"][:, None]) if s["n"] is not None else torch.ones_like(at, dtype=torch.bool)
    s["qo"].copy_(torch.where(new[:, :, None, None], _turned(s["q"], pos, s, c), s["qo"]))
    b = torch.arange(c["B"], device="cuda")[:, None].expand_as(at)[new]
    at = at[new]
    for rows, cache in ((_turned(s["kn"], pos, s, c), s["k"]), (s["vn"], s["v"])):
        if c["block"]:
            cache[s["table"].long()[b, at // c["block"]], :, at % c["block"]] = rows[new]
        else:
            cache[b, :, at] = rows[new]
    s["lens"].copy_(s["ctx"] + (s["n"] if s["n"] is not None else c["T"]))
    return s["qo"], s["k"], s["v"], s["lens"]


def _whole(s, c, name):
    """A cache as [B, Hkv, keys, D]."""
    if not c["block"]:
        return s[name]
    return s[name][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(c["B"], c["Hkv"], -1, c["D"])


def _prefill_plain(s, c):
    """A run of rows at a time (the scores of all of them would not fit), over the keys that some row of the run sees."""
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    G, dev = Hq // Hkv, s["q"].device
    k, v = _whole(s, c, "k").float(), _whole(s, c, "v").float()
    n = (s["n"] if s["n"] is not None else torch.full_like(s["ctx"], T)).long()
    first = s["ctx"].long() - n                                                       # the position of a sequence's row 0
    lo0, hi0 = (_olds(c).min().item(), _olds(c).max().item())
    v = torch.where((torch.arange(k.shape[2], device=dev) < s["ctx"][:, None])[:, None, :, None], v, 0.0)
    step = max(1, min(T, int(6e8 / (B * Hq * k.shape[2]))))
    for t in range(0, T, step):
        i = torch.arange(t, min(T, t + step), device=dev)
        keys = torch.arange(min(k.shape[2], hi0 + t + len(i)), device=dev)
        if c["window"]:
            keys = keys[(keys < c["sink"]) | (keys > lo0 + t - c["window"])]
        at = first[:, None] + i                                                       # [B, rows]
        q = s["q"][:, t:t + step].float().view(B, len(i), Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * len(i), D)
        a = torch.matmul(q, k[:, :, keys].transpose(2, 3)) / math.sqrt(D)
        seen = keys <= at[:, :, None]
        if c["window"]:
            seen &= (keys < c["sink"]) | (keys > at[:, :, None] - c["window"])
        a = torch.where(seen.repeat(1, G, 1)[:, None], a, -math.inf)
        top = a.amax(-1, keepdim=True)
        a = (a - top).exp()
        total = a.sum(-1, keepdim=True)
        o = (torch.matmul(a, v[:, :, keys]) / total).view(B, Hkv, G, len(i), D).permute(0, 3, 1, 2, 4)
        lse = (top + total.log()).view(B, Hkv, G, len(i)).permute(0, 3, 1, 2)
        new = i < n[:, None]
        s["out"][:, t:t + step][new] = o.reshape(B, len(i), Hq, D)[new].to(torch.bfloat16)
        s["lse"][:, t:t + step][new] = lse.reshape(B, len(i), Hq)[new]
    return s["out"], s["lse"]


def _library(s, c):
    import paper_2502_20330_b200 as R
    if c["op"] == "rope":
        R.rapid_rope_apply(s["q"], s["qo"], s["kn"], s["ko"], s["pos"], s["rope"])
        return s["qo"], s["ko"]
    if c["op"] == "append":
        if c["block"]:
            R.rapid_kv_append_rope_paged(s["q"], s["kn"], s["vn"], s["qo"], s["k"], s["v"], s["table"], s["ctx"], s["lens"],
                                         s["rope"], s["status"], n_tokens=s["n"], positions=s["pos"])
        else:
            R.rapid_kv_append_rope(s["q"], s["kn"], s["vn"], s["qo"], s["k"], s["v"], s["ctx"], s["lens"], s["rope"],
                                   s["status"], n_tokens=s["n"], positions=s["pos"])
        return s["qo"], s["k"], s["v"], s["lens"]
    if c["block"]:
        R.rapid_prefill_attention_paged(s["q"], s["k"], s["v"], s["table"], s["ctx"], s["out"], s["ws"], n_tokens=s["n"],
                                        params=s["params"])
    else:
        R.rapid_prefill_attention(s["q"], s["k"], s["v"], s["ctx"], s["out"], s["ws"], n_tokens=s["n"], params=s["params"])
    return s["out"], s["lse"]


def run(state):
    c = state["case"]
    if own:
        return _library(state, c)
    return {"rope": _rope_plain, "append": _append_plain, "prefill": _prefill_plain}[c["op"]](state, c)


# ---- what a pass cannot do without ------------------------------------------------------------------------------


def _span(c, first, n):
    """Visible (row, key) pairs of one sequence's n rows at positions first .. first + n - 1."""
    if not c["window"]:
        return n * first + n * (n + 1) // 2
    at = torch.arange(first, first + n, dtype=torch.int64)
    lo = (at - c["window"] + 1).clamp(min=0)
    return int((at + 1 - lo + torch.minimum(lo, torch.tensor(c["sink"]))).sum())


def work(case):
    c = case
    if c["op"] == "rope":
        el = c["B"] * c["T"] * (c["Hq"] + c["Hkv"]) * c["D"]
        return {"bytes": 4 * el + 4 * c["axes"] * c["B"] * c["T"], "flops": 3 * el * c["rd"] // c["D"]}
    n, old = _counts(c).tolist(), _olds(c).tolist()
    if c["op"] == "append":
        el = sum(n) * c["D"]
        return {"bytes": 4 * el * (c["Hq"] + 2 * c["Hkv"]), "flops": 3 * el * (c["Hq"] + c["Hkv"]) * c["rd"] // c["D"]}
    keys = 0
    for x, o in zip(n, old):
        lo = max(0, o - c["window"] + 1) if c["window"] else 0
        keys += o + x - lo + min(lo, c["sink"])
    rows = sum(n) * c["Hq"]
    return {"bytes": 4 * c["Hkv"] * c["D"] * keys + rows * (4 * c["D"] + 4),
            "flops": 4 * c["D"] * c["Hq"] * sum(_span(c, o, x) for x, o in zip(n, old))}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------


def _exact_turned(x, pos, s, c):
    """Pairs as complex numbers, turned by exp(i p f)."""
    rd, axis = c["rd"], _pair_axis(c)
    lead = x[..., :rd].double()
    if c["inter"]:
        z = torch.view_as_complex(lead.reshape(*lead.shape[:-1], rd // 2, 2).contiguous())
    else:
        z = torch.complex(lead[..., :rd // 2].contiguous(), lead[..., rd // 2:].contiguous())
    angle = torch.stack([pos[axis[i]].double() * s["freq"][i].double() for i in range(rd // 2)], -1)
    z = z * torch.polar(torch.ones_like(angle), angle)[:, :, None]
    y = x.double().clone()
    y[..., :rd] = torch.view_as_real(z).flatten(-2) if c["inter"] else torch.cat([z.real, z.imag], -1)
    return y


def _exact_append(s, c):
    qo, k, v, lens = s["qo"].double(), s["k"].double(), s["v"].double(), s["ctx"].clone()
    for b in range(c["B"]):
        m = c["T"] if s["n"] is None else int(s["n"][b])
        L = int(s["ctx"][b])
        pos = torch.arange(L, L + m, device="cuda")[None, None] if s["pos"] is None else s["pos"][:, b:b + 1, :m]
        qo[b, :m] = _exact_turned(s["q"][b:b + 1, :m], pos, s, c)[0]
        kr, vr = _exact_turned(s["kn"][b:b + 1, :m], pos, s, c)[0], s["vn"][b, :m].double()
        if c["block"]:
            p = torch.arange(L, L + m, device="cuda")
            page = s["table"][b].long()[p // c["block"]]
            k[page, :, p % c["block"]], v[page, :, p % c["block"]] = kr, vr
        else:
            k[b, :, L:L + m], v[b, :, L:L + m] = kr.transpose(0, 1), vr.transpose(0, 1)
        lens[b] += m
    return qo, k, v, lens


def _exact_prefill(s, c):
    B, T, Hq, Hkv, D = c["B"], c["T"], c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(B):
        L, m = int(s["ctx"][b]), T if s["n"] is None else int(s["n"][b])
        if c["block"]:
            pages = s["table"][b, :-(-L // c["block"])].long()
            k, v = (s[x][pages].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].double() for x in "kv")
        else:
            k, v = (s[x][b, :, :L].double() for x in "kv")
        step = max(1, int(1.5e8 / (G * L)))
        for h in range(Hkv):
            for t in range(0, m, step):
                e = min(m, t + step)
                p = torch.arange(L - m + t, L - m + e, device="cuda")
                hi = L - m + e
                j = torch.arange(hi, device="cuda")
                a = torch.einsum("rgd,nd->rgn", s["q"][b, t:e, h * G:(h + 1) * G].double(), k[h, :hi]) * D ** -0.5
                hidden = j[None] > p[:, None]
                if c["window"]:
                    hidden |= (j[None] >= c["sink"]) & (j[None] <= p[:, None] - c["window"])
                a.masked_fill_(hidden[:, None], -math.inf)
                w = torch.logsumexp(a, -1)
                out[b, t:e, h * G:(h + 1) * G] = torch.einsum("rgn,nd->rgd", torch.exp(a - w[..., None]), v[h, :hi])
                lse[b, t:e, h * G:(h + 1) * G] = w
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_turned(s["q"], s["pos"], s, case), _exact_turned(s["kn"], s["pos"], s, case)
    return {"append": _exact_append, "prefill": _exact_prefill}[case["op"]](s, case)
