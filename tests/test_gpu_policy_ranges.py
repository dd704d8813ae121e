"""GPU placement policies over the ranges that a call may have: the largest
grids, weights and logits of very different size, rows of every length with a
scenario of their own.  Against the plain 64-bit forms of policy_ref.py."""
import numpy as np
import pytest

import policy_ref as ref
from test_gpu_policy import INF, TYPES, draws, host16, make_logits, mlsim, u16, uniform  # noqa: F401
from paper_2002_06790_amd import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# A launch holds fewer than 2^32 threads, 2^24 blocks of 256.  Each of the four
# below has more blocks.


def test_draws_of_more_blocks_than_a_launch_holds(mlsim):
    """Two policies in turn over 2000001 scenarios: 22 million blocks."""
    P, N, R, S = 2, 42, 3, 2_000_001
    rng = np.random.default_rng(31)
    t, x = make_logits(rng, P, N, R, "float32")
    u = torch.rand((N, S), device="cuda", generator=torch.Generator("cuda").manual_seed(31))
    got = host16(mlsim.Policy(t).sample(u))
    st = ref.settings_of(P)
    for v in range(0, N, 5):
        want = ref.sample(x[:, v:v + 1], u[v:v + 1].cpu().numpy().astype(np.float64), st)
        assert np.array_equal(got[v:v + 1], want), v


def test_logp_of_more_blocks_than_a_launch_holds(mlsim):
    """2^28 + 1000 scenarios of two policies in turn: four a block, and sixteen
    a block where the ops' parts are joined."""
    P, R, S = 2, 9, 2**28 + 1000
    rng = np.random.default_rng(32)
    t, x = make_logits(rng, P, 1, R, "float32", masked=False)
    place = torch.randint(0, R, (1, S), device="cuda", dtype=torch.int16, generator=torch.Generator("cuda").manual_seed(32))
    got = mlsim.Policy(t).logp(place.view(torch.uint16))
    one = [ref.logp(x[p:p + 1], np.arange(R)[None], ref.settings_of(1)) for p in range(P)]
    for p in range(P):
        want, tol = (torch.from_numpy(q).cuda() for q in one[p])
        for s in range(p, S, 2**26):
            a = place[0, s:min(S, s + 2**26):2].int()
            assert ((got[s:min(S, s + 2**26):2].double() - want[a]).abs() <= tol[a]).all(), (p, s)


@pytest.mark.parametrize("more", [0, 4])
def test_rows_of_more_blocks_than_a_launch_holds(mlsim, more):
    """2^26 + 5 policies that share a row, four to a block: one scenario each,
    then a second for some."""
    P, R = 2**26 + 5, 520
    S = P + more
    rng = np.random.default_rng(33)
    t, x = make_logits(rng, 1, 1, R, "bfloat16")
    u = torch.rand((1, S), device="cuda", generator=torch.Generator("cuda").manual_seed(33))
    got = mlsim.Policy(t.expand(P, 1, R)).sample(u)
    C, last = ref.kept_sums(x[0, 0], 1.0, 0, 1.0, 0.0)
    C = torch.from_numpy(C).cuda()
    want = torch.searchsorted(C, u[0].double() * C[-1], right=True).clamp(max=last)
    assert torch.equal(got[0].view(torch.int16).int(), want.int())


def test_gradients_of_more_blocks_than_a_launch_holds(mlsim):
    P, R = 2**26 + 5, 2
    gen = torch.Generator("cuda").manual_seed(34)
    x = torch.randn((P, 1, R), device="cuda", generator=gen).bfloat16()
    w = torch.randn(P, device="cuda", generator=gen)
    a = torch.randint(0, R, (1, P), device="cuda", dtype=torch.int16, generator=gen)
    got = mlsim.Policy(x).grad(a.view(torch.uint16), w)
    for s in range(0, P, 2**24):
        e = min(P, s + 2**24)
        _, _, g, tol = ref.learn_each(x[s:e].double(), a[:, s:e].long(), w[s:e].double(), torch.ones(e - s, device="cuda").double(), "bfloat16")
        assert ((got[s:e].double() - g).abs() <= tol).all(), s


# (policies, ops, resources, scenarios per run, scenarios): long runs, short runs,
# a wavefront a row, and batches split over the scenarios
SHARED = [(2, 5, 40, 16384, 32768), (3, 40, 64, 5000, 15000), (2, 3, 9, 3, 60001), (2, 300, 64, 200, 400), (4, 5, 64, 700, 20011),
          (3, 2, 600, 1, 30001), (2, 2000, 100, 5000, 10000)]


@pytest.mark.parametrize("shape", SHARED, ids=str)
def test_gradients_of_weights_of_different_size(mlsim, shape):
    """Each policy's weights are 10^10 times the next one's: a gradient is as
    exact as if its policy were alone."""
    P, N, R, block, S = shape
    rng = np.random.default_rng(41)
    t, x = make_logits(rng, P, N, R, "float32")
    a = draws(rng, x, S)
    pol = ref.policy_of(np.arange(S), block, 0, P)
    w = (rng.normal(size=S) * 10.0 ** (8 - 10 * pol)).astype(np.float32)
    got = mlsim.Policy(t, block=block).grad(u16(a), torch.from_numpy(w).cuda())
    g, tol = ref.grad_shared(x, a, w, ref.settings_of(P), block)
    ref.near(got.double().cpu().numpy(), g, tol, f"grad {shape}")
    assert ((np.abs(g) > 4 * tol) | (x == -np.inf)).mean() > 0.9  # zeros would not pass


def cancelling(rng, a, w, at):
    """Weights of the scenarios `at` whose large ones cancel place by place: what
    the small ones add depends on the order of the additions, unless all are
    first rounded to a grid (to which the small ones are 0)."""
    n = len(at) // 3 * 3
    x, y, z = at[0:n:3], at[1:n:3], at[2:n:3]
    a[:, y] = a[:, x]
    w[x] = rng.choice([-1, 1], len(x)) * 2.0**60
    w[y], w[z] = -w[x], rng.choice([-1, 1], len(z))
    w[at[n:]] = 0


@pytest.mark.parametrize("shape", SHARED, ids=str)
def test_gradients_beside_weights_that_are_not_finite(mlsim, shape):
    """An infinite weight and a NaN of one policy: its own gradients show them,
    those of the others have the same bits as without, every time."""
    P, N, R, block, S = shape
    rng = np.random.default_rng(42)
    t, x = make_logits(rng, P, N, R, "float32")
    a = draws(rng, x, S)
    pol = ref.policy_of(np.arange(S), block, 0, P)
    w = rng.normal(size=S).astype(np.float32)
    for p in [p for p in range(P) if p != 1]:
        cancelling(rng, a, w, np.flatnonzero(pol == p))
    place = u16(a)
    policy = mlsim.Policy(t, block=block)
    want = policy.grad(place, torch.from_numpy(w).cuda())
    ref.near(want.double().cpu().numpy(), *ref.grad_shared(x, a, w, ref.settings_of(P), block), f"grad {shape}")
    mine = np.flatnonzero(pol == 1)
    w[mine[5]], w[mine[70]] = np.inf, np.nan
    others = [p for p in range(P) if p != 1]
    for _ in range(3):
        got = policy.grad(place, torch.from_numpy(w).cuda())
        assert torch.equal(got[others], want[others])
        assert (~torch.isfinite(got[1]) | torch.isinf(t[1])).all()


@pytest.mark.parametrize("shape", SHARED, ids=str)
def test_gradients_where_weights_that_are_not_finite_have_no_place(mlsim, shape):
    """Infinite and NaN weights of scenarios whose ops mostly have no place: the
    rows where they add nothing have the same bits as without them, the others
    show them with the same bits every time."""
    P, N, R, block, S = shape
    rng = np.random.default_rng(43)
    t, x = make_logits(rng, P, N, R, "float32")
    a = draws(rng, x, S)
    pol = ref.policy_of(np.arange(S), block, 0, P)
    w = np.zeros(S, np.float32)
    for p in range(P):
        at = np.flatnonzero(pol == p)
        cancelling(rng, a, w, at)
        w[at[30:33]] = 0
        a[1:, at[30:33]] = ref.NO_PLACE
    policy = mlsim.Policy(t, block=block)
    want = policy.grad(u16(a), torch.from_numpy(w).cuda())
    for p in range(P):
        at = np.flatnonzero(pol == p)
        w[at[30:33]] = [np.inf, np.nan, -np.inf]
        w.view(np.int32)[at[31]] += 77 * p  # NaN of several bits
    first = None
    for _ in range(3):
        got = policy.grad(u16(a), torch.from_numpy(w).cuda())
        assert torch.equal(got[:, 1:], want[:, 1:])
        assert (~torch.isfinite(got[:, 0]) | torch.isinf(t[:, 0])).all()
        first = got if first is None else first
        assert torch.equal(got.view(torch.int32), first.view(torch.int32))


@pytest.mark.parametrize("P,N,R,block,S", [(1, 2, 5, 1, 300_001), (2, 1, 40, 100_000, 200_003), (1, 1, 700, 1, 70_001), (3, 2, 20, 1, 30_001),
                                           (2, 1, 600, 3, 9_001), (4, 5, 64, 700, 20_011), (1, 30, 17, 1, 16_384), (1, 3, 200, 1, 4_500_001)])
def test_gradients_of_long_batches(mlsim, P, N, R, block, S):
    """Sums to the grid's step: a split of the batch that is lost, or added twice, shows."""
    rng = np.random.default_rng(S)
    t, x = make_logits(rng, P, N, R, "float32")
    a = draws(rng, x, S)
    a[:, ::13] = ref.NO_PLACE
    w = rng.normal(size=S).astype(np.float32)
    for T in (1.0, 0.6):
        got = mlsim.Policy(t, block=block, temperature=T).grad(u16(a), torch.from_numpy(w).cuda())
        g, tol = ref.grad_shared(x, a, w, ref.settings_of(P, T), block)
        ref.near(got.double().cpu().numpy(), g, tol, f"grad {P, N, R, block, S}")
        assert ((np.abs(g) > 20 * tol) | (x == -np.inf)).mean() > 0.9  # zeros would not pass


# (policies, ops, resources): so many rows that a group of lanes takes several, for
# every number of lanes
EACH = [(2048, 300, 5), (4096, 130, 12), (2048, 130, 30), (1024, 70, 48), (1024, 70, 100), (1024, 34, 200), (1024, 18, 400), (1024, 18, 520),
        (1027, 17, 1001), (1024, 16, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", EACH, ids=str)
def test_one_draw_of_every_row(mlsim, shape, dtype):
    P, N, R = shape
    rng = np.random.default_rng(R)
    t, _ = make_logits(rng, P, N, R, dtype)
    t[3, 5] = -INF
    t[4, 6, R // 2], t[5, 7, 0], t[6, 8, R - 1] = float("nan"), -float("nan"), INF
    u = torch.from_numpy(uniform(rng, N, P)).cuda()
    cuts = [dict(), dict(top_k=5), dict(temperature=0.7, top_k=8, top_p=0.9), dict(top_k=16, top_p=0.8), dict(top_p=0.9),
            dict(top_k=20, min_p=0.02), dict(min_p=0.1, temperature=1.5), dict(temperature=0.0)]
    cuts.append(dict(temperature=rng.choice([0.0, 0.5, 1.0, 3.0], P).astype(np.float32), top_k=rng.integers(0, R + 2, P).astype(np.float32),
                     top_p=rng.random(P).astype(np.float32), min_p=(rng.random(P) * 0.2).astype(np.float32)))
    for cut in cuts:
        print(f"each {shape} {dtype} {list(cut)}", flush=True)
        got = mlsim.Policy(t, **cut).sample(u).view(torch.int16).long() & 0xFFFF
        want = ref.sample_each(t.double(), u.double(), torch.from_numpy(ref.settings_of(P, **cut)).cuda())
        assert torch.equal(got, want), (cut, (got != want).nonzero()[:5])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", EACH, ids=str)
def test_one_scenario_of_every_row(mlsim, shape, dtype):
    """Log-probabilities and gradients; most scenarios' places are all allowed."""
    P, N, R = shape
    rng = np.random.default_rng(R + 1)
    t, _ = make_logits(rng, P, N, R, dtype)
    a = torch.from_numpy(rng.integers(0, R, (N, P))).cuda()
    ok = torch.isfinite(t.gather(2, a.T[..., None]))[..., 0].T
    a = torch.where(ok, a, torch.isfinite(t).float().argmax(-1).T)
    a[2, 9], a[N - 1, 11] = R, ref.NO_PLACE
    w = rng.normal(size=P).astype(np.float32)
    T = rng.choice([0.5, 1.0, 3.0], P).astype(np.float32)
    policy, place = mlsim.Policy(t, temperature=T), u16(a.cpu().numpy())
    lp, ltol, g, gtol = ref.learn_each(t.double(), a, torch.from_numpy(w).double().cuda(), torch.from_numpy(T).double().cuda(), dtype)
    assert torch.isfinite(lp).sum() == P - 2 and torch.isfinite(ltol[torch.isfinite(lp)]).all()
    ref.near(policy.logp(place).cpu().numpy(), lp.cpu().numpy(), ltol.cpu().numpy(), "logp")
    ref.near(policy.grad(place, torch.from_numpy(w).cuda()).double().cpu().numpy(), g.cpu().numpy(), gtol.cpu().numpy(), "grad")
    few = mlsim.Policy(t[:30], temperature=T[:30])  # the same bits with fewer policies
    assert torch.equal(few.grad(place.view(torch.int16)[:, :30].contiguous().view(torch.uint16), torch.from_numpy(w[:30]).cuda()),
                       policy.grad(place, torch.from_numpy(w).cuda())[:30])


@pytest.mark.parametrize("S", [3, 12, 900])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_logits_further_apart_than_their_type_s_largest(mlsim, dtype, S):
    """The difference of two logits may be twice the largest number; divided by
    a large temperature it is an ordinary exponent."""
    x = torch.tensor([[[3e38, -3e38, 0, -INF], [-3.3e38, 3.3e38, 1e38, 2e38], [-3e38, -INF, -1e38, -2e38], [1.0, 2.0, -INF, 3.0]]]).to(TYPES[dtype])
    rng = np.random.default_rng(S)
    a = rng.integers(0, 4, (4, S))
    a[:, 0] = [1, 0, 3, 0]
    a[0, a[0] == 3], a[2, a[2] == 1], a[3, a[3] == 2] = 1, 0, 0  # allowed places
    w = (rng.normal(size=S) * 1e10).astype(np.float32)
    ids, y = np.array([[[0, 1, 2], [0, 1, 3], [0, 2, 3], [0, 1, 3]]]), torch.tensor([[[3e38, -3e38, 0.0]] * 4]).to(x.dtype)
    xd, u = x.double().numpy(), uniform(rng, 4, S)
    for T in (8e37, 3e38, 1.0):
        policy, st = mlsim.Policy(x.cuda(), temperature=T), ref.settings_of(1, T)
        lp, ltol = ref.logp(xd, a, st)
        far = np.abs(lp) > 3.39e38  # beyond the largest float32, 3.403e38: the sums here are at most 3.32e38, or 4e38 and more
        assert np.array_equal(host16(policy.sample(torch.from_numpy(u).cuda())), ref.sample(xd, u.astype(np.float64), st))
        assert far.any() == (T == 1.0) and np.isfinite(lp).all()
        got = policy.logp(u16(a)).cpu().numpy()
        assert (got[far] < -3.39e38).all()
        ref.near(got[~far], lp[~far], ltol[~far], "logp")
        ref.near(policy.grad(u16(a), torch.from_numpy(w).cuda()).double().cpu().numpy(), *ref.grad(xd, a, w, st, dtype=dtype), "grad")
        if T > 1:
            loss, grad = policy.distill(u16(ids), y.cuda(), weight=torch.full((1, 4), 1e10, device="cuda"))
            rl, lt, rg, gt = ref.distill(xd, ids, y.double().numpy(), st, np.full((1, 4), 1e10), dtype)
            ref.near(loss.cpu().numpy(), rl, lt, "loss")
            ref.near(grad.double().cpu().numpy(), rg, gt, "distillation's gradient")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,N,R,block,S", [(4, 3, 12, 1, 4), (4, 3, 70, 1, 9), (4, 3, 40, 500, 2000), (4, 2, 600, 9000, 36000)])
def test_weights_that_are_not_finite_leave_masked_logits_at_zero(mlsim, P, N, R, block, S, dtype):
    """The gradient of a logit of -inf is 0 whatever the weight; an invalid row is NaN throughout."""
    rng = np.random.default_rng(S)
    t, x = make_logits(rng, P, N, R, dtype)
    t[..., 0], t[..., 1] = 0.5, -INF
    t[3, 1, 2] = float("nan")
    masked = torch.isinf(t)
    masked[3, 1] = False
    a = np.zeros((N, S), np.int64)
    pol = ref.policy_of(np.arange(S), block, 0, P)
    w = rng.normal(size=S).astype(np.float32)
    for p, bad in enumerate((INF, -INF, float("nan"))):
        w[np.flatnonzero(pol == p)[0]] = bad
    g = mlsim.Policy(t, block=block).grad(u16(a), torch.from_numpy(w).cuda())
    assert (g[masked] == 0).all() and not torch.isfinite(g[:3][~masked[:3]]).any()
    assert torch.isnan(g[3, 1]).all() and torch.isfinite(g[3, 0]).all()
    ids, y = u16(np.zeros((P, N, 2))), torch.zeros((P, N, 2), dtype=t.dtype, device="cuda")
    dw = torch.ones((P, N), device="cuda")
    dw[0], dw[1], dw[2] = INF, -INF, float("nan")
    loss, g = mlsim.Policy(t).distill(ids, y, weight=dw)
    assert (g[masked] == 0).all() and not torch.isfinite(g[:3][~masked[:3]]).any()
    assert torch.isnan(g[3, 1]).all() and torch.isfinite(g[3, 0]).all() and torch.isnan(loss[3, 1]) and torch.isfinite(loss[0]).all()


def test_run_sampled_on_another_stream(mlsim):
    """A draw and replay on a stream that is busy, its inputs dropped at once: what
    takes their memory does not reach the replay."""
    w = W.make_config(1, n_scen=5000)
    rng = np.random.default_rng(51)
    N, S = w.n_ops, w.n_scen
    g = mlsim.Graph.from_workload(w)
    policy = mlsim.Policy(torch.zeros((N, w.n_res), device="cuda"))
    dur_h, u_h = w.durations(), uniform(rng, N, S)
    want = [q.clone() for q in g.run_sampled(policy, torch.from_numpy(dur_h).cuda(), torch.from_numpy(u_h).cuda()) if q is not None]
    side, a = torch.cuda.Stream(), torch.ones((4096, 4096), device="cuda")
    for _ in range(3):
        dur, u = torch.from_numpy(dur_h).cuda(), torch.from_numpy(u_h).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                b = a @ a
        got = [q for q in g.run_sampled(policy, dur, u, stream=side) if q is not None]
        del dur, u
        junk = [torch.ones((N, S), dtype=torch.int32, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        del junk, b
        for x, y in zip(want, got):
            assert torch.equal(x.view(torch.int16) if x.dtype == torch.uint16 else x, y.view(torch.int16) if y.dtype == torch.uint16 else y)
    g.close()


def test_run_sampled_captured_and_replayed(mlsim):
    """A draw and replay in a HIP graph, with new numbers, logits and durations
    in place, and eager calls between the replays."""
    w = W.make_config(1, n_scen=700)
    rng = np.random.default_rng(52)
    N, R, S = w.n_ops, w.n_res, w.n_scen
    g = mlsim.Graph.from_workload(w)
    t = torch.randn((2, N, R), device="cuda")
    policy = mlsim.Policy(t, block=100, top_p=0.9)
    dur, u = torch.from_numpy(w.durations()).cuda(), torch.from_numpy(uniform(rng, N, S)).cuda()
    advantage = torch.randn(S, device="cuda")

    def step():
        makespan, _, status, place = g.run_sampled(policy, dur, u)
        return makespan, status, place.view(torch.int16), policy.logp(place), policy.grad(place, advantage)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        u.copy_(torch.from_numpy(uniform(rng, N, S)))
        t.add_(torch.randn(t.shape, device="cuda") * 0.3)
        dur.add_(int(rng.integers(0, 50)))
        want = [q.clone() for q in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, out)), k
    g.close()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,N,R,K,T", [(3, 40, 12, 9, 1.0), (2, 30, 108, 60, 0.1), (2, 20, 447, 18, 1.0), (1, 9, 1001, 400, 3.0)])
def test_entries_of_a_teacher_far_apart(mlsim, P, N, R, K, T, dtype):
    """Entries down to e^-115 of the best one: probabilities that float32 holds
    with few bits, or not at all."""
    rng = np.random.default_rng(R)
    t, x = make_logits(rng, P, N, R, dtype, masked=False)
    for twice in (False, True):
        ids = rng.integers(0, R, (P, N, K)) if twice else np.argsort(rng.random((P, N, R)), -1)[..., :K]
        y = torch.from_numpy(-rng.uniform(0, 115, (P, N, K)) * T)
        y[..., 0] = 0
        y = y.to(TYPES[dtype])
        policy, st = mlsim.Policy(t, temperature=T), ref.settings_of(P, T)
        loss, grad = policy.distill(u16(ids), y.cuda())
        rl, lt, rg, gt = ref.distill(x, ids, y.double().numpy(), st, None, dtype)
        ref.near(loss.cpu().numpy(), rl, lt, "loss")
        ref.near(grad.double().cpu().numpy(), rg, gt, "grad")


def test_gradients_where_one_policy_has_all_scenarios(mlsim):
    """A thousand policies and a block longer than the batch: one policy's sums
    to the grid's step, zeros for the others."""
    P, N, R, S = 1000, 2, 5, 200_000
    rng = np.random.default_rng(61)
    t, x = make_logits(rng, P, N, R, "float32")
    for scen0 in (0, 7 * 10**9 - 50_000):
        a = draws(rng, x[ref.policy_of(np.arange(0, S, S - 1), 10**9, scen0, P)], S)
        w = (rng.normal(size=S) * 100).astype(np.float32)
        got = mlsim.Policy(t, block=10**9, scen0=scen0).grad(u16(a), torch.from_numpy(w).cuda())
        g, tol = ref.grad_shared(x, a, w, ref.settings_of(P), 10**9, scen0)
        ref.near(got.double().cpu().numpy(), g, tol, "grad")
        assert (np.abs(g) > 20 * tol).any((1, 2)).sum() == (1 if scen0 == 0 else 2)
