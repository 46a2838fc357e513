"""One workspace for a verify plan and for the calls whose scratch takes the plan's place: a call that still names the plan finds
it stale, whatever the scratch left there."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, HQ, D, GAMMA, LMAX = 5, 8, 128, 2, 3000


def _rnd(*shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").bfloat16()


def _lens(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


@pytest.fixture(params=[1, 2, 8])
def step(request):
    """A workspace with a plan, and verify calls over it."""
    import paper_2502_20330_b200 as R
    Hkv = request.param
    k, v = _rnd(B, Hkv, LMAX, D, seed=1), _rnd(B, Hkv, LMAX, D, seed=2)
    q, ctx = _rnd(B, GAMMA + 1, HQ, D, seed=3), _lens(3000, 5, 1700, 300, 2999)
    ws = R.new_workspace(max(R.attention_workspace_bytes(B, HQ, Hkv, D, LMAX, GAMMA),
                             R.prefix_attention_workspace_bytes(B, HQ, Hkv, D, GAMMA), R.kv_fill_workspace_bytes(B, Hkv)))
    out = torch.empty_like(q)

    def verify(plan):
        R.rapid_verify_attention(q, k, v, ctx, GAMMA, out, ws, R.AttnParams(plan=plan))
        return out.clone(), R.workspace_status(ws)

    want, status = verify(R.PLAN_NONE)
    assert status == 0

    def prefix(P):
        kp = _rnd(Hkv, 300, D, seed=4)
        o = torch.empty_like(q)
        R.rapid_verify_attention_prefix(q, kp, kp, _lens(P), k, v, _lens(*[40 * (b + 1) for b in range(B)]), GAMMA, o, ws)

    def plan():
        R.workspace_init(ws)
        R.rapid_attention_plan(ctx, GAMMA, B, HQ, Hkv, D, LMAX, ws)

    return verify, prefix, plan, want, ws, (k, v, Hkv)


@pytest.mark.parametrize("P", [0, 1, 300])
@pytest.mark.parametrize("mode", ["PLAN_READY", "PLAN_SETTLED"])
def test_a_prefix_call_ends_the_plan(step, P, mode):
    import paper_2502_20330_b200 as R
    verify, prefix, plan, want, ws, _ = step
    plan()
    got, status = verify(R.PLAN_READY)
    assert status == 0 and torch.equal(got, want)
    prefix(P)
    got, status = verify(getattr(R, mode))
    assert status == R.STATUS_STALE_PLAN
    plan()
    got, status = verify(R.PLAN_READY)
    assert status == 0 and torch.equal(got, want)


def test_a_paged_prefix_call_ends_the_plan(step):
    import paper_2502_20330_b200 as R
    verify, _, plan, want, ws, (k, _, Hkv) = step
    pool = _rnd(40, Hkv, 64, D, seed=5)
    q, table = _rnd(B, GAMMA + 1, HQ, D, seed=6), torch.arange(20, dtype=torch.int32, device="cuda").view(B, 4)
    for P in (0, 64):
        plan()
        R.rapid_verify_attention_prefix_paged(q, pool, pool, table, _lens(P), _lens(*[200] * B), GAMMA, torch.empty_like(q), ws)
        assert verify(R.PLAN_READY)[1] == R.STATUS_STALE_PLAN
        plan()
        got, status = verify(R.PLAN_READY)
        assert status == 0 and torch.equal(got, want)


@pytest.mark.parametrize("T", [100, 5000])
def test_a_fill_ends_the_plan_or_leaves_it_whole(step, T):
    import paper_2502_20330_b200 as R
    verify, _, plan, want, ws, (_, _, Hkv) = step
    rows = _rnd(B, T, Hkv, D, seed=7)
    cache = [torch.zeros(B, Hkv, T, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros(B, Hkv, device="cuda") for _ in range(2)]
    plan()
    R.kernel_launch_count_reset()
    R.rapid_kv_fill_fp8(rows, rows, None, *cache, *scale, None, ws)
    kernels = R.kernel_launch_count()
    got, status = verify(R.PLAN_READY)
    assert (kernels, status) == ((1, 0) if T == 100 else (2, R.STATUS_STALE_PLAN))
    if status == 0:
        assert torch.equal(got, want)


def test_calls_without_a_plan_share_the_workspace(step):
    import paper_2502_20330_b200 as R
    verify, prefix, _, want, ws, _ = step
    for P in (0, 300, 0):
        prefix(P)
        got, status = verify(R.PLAN_NONE)
        assert status == 0
        assert torch.equal(got, want)


@pytest.mark.parametrize("gamma", [0, 3])
@pytest.mark.parametrize("mode", ["PLAN_READY", "PLAN_SETTLED"])
def test_accepting_and_sampling_end_the_plan(step, gamma, mode):
    import paper_2502_20330_b200 as R
    verify, _, plan, want, ws, _ = step
    V = 512
    logits, draft = torch.randn(B, gamma + 1, V, device="cuda"), torch.randn(B, max(gamma, 1), V, device="cuda")
    tokens, u = torch.zeros(B, gamma, dtype=torch.int32, device="cuda"), torch.rand(B, gamma + 1, device="cuda")
    n, tok, logq = _lens(*[0] * B), _lens(*[0] * B), torch.zeros(B, device="cuda")
    calls = [lambda: R.rapid_accept(logits, draft[:, :gamma].contiguous(), tokens, u, 0.5, n, tok, ws)]
    if gamma == 0:
        calls.append(lambda: R.rapid_draft_sample(draft[:, 0].contiguous(), u[:, 0].contiguous(), 1.0, tok, logq, ws))
    for call in calls:
        plan()
        call()
        assert verify(getattr(R, mode))[1] == R.STATUS_STALE_PLAN
        plan()
        got, status = verify(R.PLAN_READY)
        assert status == 0 and torch.equal(got, want)
