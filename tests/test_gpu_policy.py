"""GPU placement policies (Policy.sample / logp / grad / distill and
Graph.run_sampled) against plain 64-bit forms (policy_ref.py): draws equal,
sums within the bounds derived there."""
import os

import numpy as np
import pytest

import oracle
import policy_ref as ref
from paper_2002_06790_amd import workloads as W

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

INF = float("inf")
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


@pytest.fixture(scope="module")
def mlsim():
    import paper_2002_06790_amd as m
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if not os.path.exists(m.LIB_PATH):
        m.build()
    return m


def u16(a):
    """uint16 tensor on the GPU from whole numbers."""
    return torch.from_numpy(np.ascontiguousarray(a).astype(np.uint16).view(np.int16)).cuda().view(torch.uint16)


def host16(t):
    return t.view(torch.int16).cpu().numpy().view(np.uint16).astype(np.int64)


def make_logits(rng, P, N, R, dtype, spread=2.0, masked=True):
    """(tensor on the GPU, the float64 values it holds).  Some ops may not run
    on some resources; some rows hold equal logits."""
    x = rng.normal(size=(P, N, R)) * spread
    if masked and R > 1:
        x[rng.random((P, N, R)) < 0.2] = -np.inf
        x[:, ::5] = np.round(x[:, ::5])  # ties
        x[:, 3::7] = np.where(np.isfinite(x[:, 3::7]), 0.0, x[:, 3::7])
        x[..., 0] = np.where((x == -np.inf).all(-1), 0.5, x[..., 0])
    t = torch.from_numpy(x).to(TYPES[dtype])
    return t.cuda(), t.double().numpy()


def uniform(rng, N, S):
    """Multiples of 2^-24 in [0, 1), the ends among them."""
    u = (rng.integers(0, 2**24, (N, S)) * 2.0**-24).astype(np.float32)
    u.ravel()[:2] = [0.0, 1 - 2.0**-24][:u.size]
    return u


# (policies, ops, resources, scenarios per policy, scen0, scenarios, type)
SHAPES = [
    (1, 1, 1, 1, 0, 1, "float32"),        # the smallest call
    (1, 42, 3, 1, 0, 1, "float32"),       # one scenario of the tiny model
    (1, 42, 3, 1, 0, 1023, "bfloat16"),
    (1, 29, 8, 4096, 0, 4500, "float16"),
    (1, 9, 17, 1000, 7, 1001, "float16"),  # odd row length: no row is aligned
    (3, 10, 16, 37, 50, 333, "bfloat16"),  # policies change inside a wavefront, the first begins inside its block
    (5, 7, 48, 64, 100, 777, "float32"),
    (12, 6, 48, 256, 0, 1024, "bfloat16"),
    (70, 5, 33, 1, 0, 70, "float32"),     # a policy per scenario
    (33, 4, 64, 1, 5, 40, "bfloat16"),    # ... and again after the last policy
    (9, 3, 65, 2, 0, 18, "float32"),
    (2, 5, 100, 500, 0, 999, "float16"),
    (1, 4, 128, 2048, 0, 2048, "float32"),
    (3, 3, 200, 3, 1, 20, "bfloat16"),
    (1, 3, 256, 700, 0, 700, "bfloat16"),
    (1, 3, 257, 1, 0, 5, "float32"),
    (2, 3, 500, 130, 0, 260, "float32"),
    (1, 3, 513, 1, 0, 300, "bfloat16"),
    (3, 2, 1001, 1, 0, 3, "float32"),
    (1, 2, 1024, 600, 0, 600, "float16"),
    (4, 3, 12, 10**17, 3, 65, "float32"),  # one block longer than any scenario index: policy 0 alone
    (3, 3, 12, 2**32, 2**32 - 20, 50, "float32"),  # policies change once, at an index beyond 32 bits
    (3, 2, 70, 2**33, 3 * 2**33 * 5 - 30, 700, "bfloat16"),
    (300, 11, 48, 1, 299, 300, "bfloat16"),  # one scenario each, the last policy first
    (40, 13, 20, 7, 3, 275, "float16"),  # few scenarios each, the first and last policies fewer
    (6, 9, 300, 40, 0, 233, "float32"),
    (2, 300, 7, 90, 11, 180, "float32"),
]
CUTS = [dict(), dict(temperature=0.7, top_k=3), dict(top_p=0.8), dict(min_p=0.1, temperature=1.5),
        dict(temperature=0.9, top_k=20, top_p=0.9, min_p=0.02), dict(temperature=0.0), dict(top_k=1), dict(top_p=0.0)]


def per_policy(rng, P, R):
    return dict(temperature=rng.choice([0.0, 0.5, 1.0, 3.0], P).astype(np.float32),
                top_k=rng.integers(0, R + 2, P).astype(np.float32), top_p=rng.random(P).astype(np.float32),
                min_p=(rng.random(P) * 0.2).astype(np.float32))


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_sample(mlsim, shape):
    P, N, R, block, scen0, S, dtype = shape
    rng = np.random.default_rng(hash(shape[:6]) % 2**32)
    t, x = make_logits(rng, P, N, R, dtype)
    u = uniform(rng, N, S)
    ud = torch.from_numpy(u).cuda()
    for cut in CUTS + [per_policy(rng, P, R)]:
        print(f"sample {shape} {list(cut)}", flush=True)
        got = host16(mlsim.Policy(t, block=block, scen0=scen0, **cut).sample(ud))
        want = ref.sample(x, u.astype(np.float64), ref.settings_of(P, **cut), block, scen0)
        assert np.array_equal(got, want), (cut, np.argwhere(got != want)[:5])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("S", [1, 700])
def test_sample_rows_without_a_distribution(mlsim, dtype, S):
    """Empty rows, NaN, infinities, a type's lowest values; settings out of range."""
    low = float(torch.finfo(TYPES[dtype]).min)
    big = float(torch.finfo(TYPES[dtype]).max)
    nan = float("nan")
    rows = [[-INF] * 6, [nan, 1, 2, 0, 0, 0], [0, 0, nan, -INF, 0, 0], [INF, 0, 0, 0, 0, 0], [0, -INF, INF, 0, 0, nan],
            [low] * 6, [low, low, 0, low, -INF, 1], [big, low, big, 0, 0, 0], [-0.0, 0.0, -0.0, -INF, 0.0, -0.0], [-INF] * 5 + [low]]
    t = torch.tensor([rows], dtype=TYPES[dtype])
    x = t.double().numpy()
    rng = np.random.default_rng(8)
    u = uniform(rng, len(rows), S)
    ud = torch.from_numpy(u).cuda()
    for cut in (dict(), dict(top_k=2), dict(top_p=0.5), dict(temperature=0.0), dict(min_p=0.5)):
        got = host16(mlsim.Policy(t.cuda(), **cut).sample(ud))
        want = ref.sample(x, u.astype(np.float64), ref.settings_of(1, **cut))
        assert np.array_equal(got, want), cut
        assert (got[:5] == ref.NO_PLACE).all() and (got[5:] < 6).all()
    bad = dict(temperature=[-1, nan, INF, 1, 1, 1, 1, 1], top_k=[0, 0, 0, nan, -1, 0, 0, 0],
               top_p=[1, 1, 1, 1, 1, 1.5, -0.1, 1], min_p=[0, 0, 0, 0, 0, 0, 0, 1.5])
    got = host16(mlsim.Policy(t[:, 5:].expand(8, 5, 6).cuda(), block=1, **bad).sample(ud[:5]))
    assert (got[:, :8] == ref.NO_PLACE).all()


@pytest.mark.parametrize("S", [9, 900])
def test_sample_numbers_out_of_range(mlsim, S):
    """u below 0, at and above 1, NaN, the smallest positive."""
    rng = np.random.default_rng(3)
    t, x = make_logits(rng, 1, 4, 70, "float32")
    x[0, :, 0] = x[0, :, -1] = -np.inf
    t = torch.from_numpy(x).float()
    u = np.tile(np.array([-1.0, -0.0, 0.0, 1.0, 2.0, np.inf, -np.inf, np.nan, 1e-45], np.float32), (4, S // 9))
    for cut in (dict(), dict(top_k=5), dict(top_p=0.6)):
        got = host16(mlsim.Policy(t.cuda(), **cut).sample(torch.from_numpy(u).cuda()))
        want = ref.sample(t.double().numpy(), u.astype(np.float64), ref.settings_of(1, **cut))
        assert np.array_equal(got, want), cut


@pytest.mark.parametrize("R", [10, 64, 600])
@pytest.mark.parametrize("S", [3, 2000])
def test_sample_on_the_borders(mlsim, R, S):
    """Untrained rows: every weight is 1, so u and top_p fall exactly on
    borders, which 64 bits hold without rounding."""
    t = torch.zeros((1, 5, R)).cuda()
    rng = np.random.default_rng(R + S)
    u = (rng.integers(0, R, (5, S)) / R).astype(np.float32)
    for cut in (dict(), dict(top_p=0.5), dict(top_p=0.25, top_k=8), dict(min_p=1.0)):
        got = host16(mlsim.Policy(t, **cut).sample(torch.from_numpy(u).cuda()))
        assert np.array_equal(got, ref.sample(np.zeros((1, 5, R)), u.astype(np.float64), ref.settings_of(1, **cut))), cut


def test_sample_far_apart_logits(mlsim):
    """Weights down to where float32, and then float64, holds none."""
    x = np.array([[[0.0, -90.0, -150.0, -700.0, -740.0, -2000.0], [-2000.0, -740.0, -1.0, -90.0, -50.0, 0.0]]])
    t = torch.from_numpy(x).float().cuda()
    u = np.tile(np.array([0.0, 1e-45, 1e-38, 1e-20, 0.3, 1 - 2.0**-24, 1.0], np.float32), (2, 100))
    for cut in (dict(), dict(temperature=2.0), dict(top_k=3), dict(top_p=1 - 2.0**-24)):
        got = host16(mlsim.Policy(t, **cut).sample(torch.from_numpy(u).cuda()))
        assert np.array_equal(got, ref.sample(x, u.astype(np.float64), ref.settings_of(1, **cut))), cut


@pytest.mark.parametrize("P,N,R,block,S", [(1, 3, 12, 1, 1), (1, 3, 70, 1, 6), (1, 2, 40, 1, 900), (9, 4, 33, 1, 9), (3, 2, 600, 2, 6), (1, 2, 600, 1, 700)])
def test_logits_of_large_magnitude(mlsim, P, N, R, block, S):
    """Logits around 10^6, where float32 holds them in steps of 1/16: only
    differences count.  One row of ordinary ones among them."""
    rng = np.random.default_rng(R)
    x = (rng.choice([-1e6, 1e6], (P, N, 1)) + rng.normal(size=(P, N, R)) * 3).astype(np.float32)
    x[0, 0] = rng.normal(size=R)
    t = torch.from_numpy(x).cuda()
    u = uniform(rng, N, S)
    a = rng.integers(0, R, (N, S))
    w = rng.normal(size=S).astype(np.float32)
    x = x.astype(np.float64)
    for cut in (dict(), dict(temperature=0.25, top_k=5, top_p=0.9), dict(temperature=3.0, min_p=0.1), dict(temperature=1e-30)):
        print(f"large {P, N, R, block, S} {cut}", flush=True)
        pol, st = mlsim.Policy(t, block=block, **cut), ref.settings_of(P, **cut)
        got = host16(pol.sample(torch.from_numpy(u).cuda()))
        assert np.array_equal(got, ref.sample(x, u.astype(np.float64), st, block)), cut
        if cut.get("temperature", 1) > 1e-3:
            ref.near(pol.logp(u16(a)).cpu().numpy(), *ref.logp(x, a, st, block), "logp")
            g = pol.grad(u16(a), torch.from_numpy(w).cuda()).double().cpu().numpy()
            ref.near(g, *ref.grad(x, a, w, st, block), "grad")


def test_a_row_does_not_depend_on_its_neighbours(mlsim):
    """The same bits for a row among others and alone."""
    rng = np.random.default_rng(21)
    N, R, S = 40, 30, 5
    t, _ = make_logits(rng, 1, N, R, "float32")
    t[0, 7] += 1e6  # another way of computing, for this row only
    ids, y = u16(rng.integers(0, R, (1, N, 3))), torch.from_numpy(rng.normal(size=(1, N, 3))).float().cuda()
    w = torch.from_numpy(rng.normal(size=S).astype(np.float32)).cuda()
    place = u16(rng.integers(0, R, (N, S)))
    grad = mlsim.Policy(t).grad(place, w)
    loss, dgrad = mlsim.Policy(t).distill(ids, y)
    for v in range(N):
        one = mlsim.Policy(t[:, v:v + 1])
        assert torch.equal(one.grad(place[v:v + 1], w), grad[:, v:v + 1])
        l, g = one.distill(ids[:, v:v + 1], y[:, v:v + 1])
        assert torch.equal(torch.nan_to_num(l), torch.nan_to_num(loss[:, v:v + 1])) and torch.equal(g, dgrad[:, v:v + 1])


def draws(rng, x, S):
    """Placements as a search holds them, some on resources that are not
    allowed or do not exist."""
    P, N, R = x.shape
    a = np.floor(rng.random((N, S)) ** 2 * R).astype(np.int64)
    ok = (x > -np.inf).all(0)
    first = np.argmax(ok, 1)[:, None]
    a = np.where(np.take_along_axis(ok, a, 1), a, first)
    return a


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_logp(mlsim, shape):
    P, N, R, block, scen0, S, dtype = shape
    rng = np.random.default_rng(hash(shape[:6]) % 2**32 + 1)
    t, x = make_logits(rng, P, N, R, dtype)
    a = draws(rng, x, S)
    for T in (1.0, 0.6, rng.choice([0.5, 1.0, 3.0], P).astype(np.float32)):
        print(f"logp {shape}", flush=True)
        got = mlsim.Policy(t, block=block, scen0=scen0, temperature=T, top_k=2).logp(u16(a)).cpu().numpy()
        ref.near(got, *ref.logp(x, a, ref.settings_of(P, T), block, scen0), f"logp {shape}")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_grad(mlsim, shape):
    P, N, R, block, scen0, S, dtype = shape
    rng = np.random.default_rng(hash(shape[:6]) % 2**32 + 2)
    t, x = make_logits(rng, P, N, R, dtype)
    a = draws(rng, x, S)
    a[rng.random(a.shape) < 0.05] = ref.NO_PLACE
    a[rng.random(a.shape) < 0.05] = R - 1  # where the row may not allow it
    w = rng.normal(size=S).astype(np.float32)
    for T in (1.0, 0.6, rng.choice([0.5, 1.0, 3.0], P).astype(np.float32)):
        print(f"grad {shape}", flush=True)
        got = mlsim.Policy(t, block=block, scen0=scen0, temperature=T).grad(u16(a), torch.from_numpy(w).cuda())
        assert got.dtype == TYPES[dtype] and got.shape == t.shape
        ref.near(got.double().cpu().numpy(), *ref.grad(x, a, w, ref.settings_of(P, T), block, scen0, dtype), f"grad {shape}")
        again = mlsim.Policy(t, block=block, scen0=scen0, temperature=T).grad(u16(a), torch.from_numpy(w).cuda())
        assert torch.equal(got, again)  # the same bits every time


@pytest.mark.parametrize("S", [3, 500])
def test_logp_and_grad_of_bad_rows(mlsim, S):
    nan = float("nan")
    x = np.array([[[0, 1, -INF], [-INF] * 3, [0, 1, 2]], [[nan, 0, 0], [0, 0, 0], [INF, 0, 0]], [[0, 1, 2], [1, 1, 1], [0, -INF, -INF]]])
    t = torch.from_numpy(x).float().cuda()
    rng = np.random.default_rng(2)
    a = rng.integers(0, 3, (3, S))
    a[:, 0] = [0, 5, 65535]
    w = rng.normal(size=S).astype(np.float32)
    for T in (1.0, np.array([1.0, 1.0, 0.0], np.float32), np.array([1.0, 2.0, nan], np.float32)):
        st = ref.settings_of(3, T)
        P = mlsim.Policy(t, block=S // 3, temperature=T)
        ref.near(P.logp(u16(a)).cpu().numpy(), *ref.logp(x, a, st, S // 3), "logp")
        ref.near(P.grad(u16(a), torch.from_numpy(w).cuda()).cpu().numpy(), *ref.grad(x, a, w, st, S // 3), "grad")
    zero = mlsim.Policy(t, temperature=0.0)
    assert torch.isnan(zero.logp(u16(a))).all() and torch.isnan(zero.grad(u16(a), torch.from_numpy(w).cuda())).all()


# (policies, ops, resources, entries, type)
TABLES = [(1, 1, 1, 1, "float32"), (1, 42, 3, 2, "float32"), (3, 7, 8, 8, "bfloat16"), (2, 9, 17, 5, "float16"),
          (12, 11, 48, 8, "bfloat16"), (1, 5, 64, 64, "float32"), (2, 3, 65, 3, "float16"), (2, 3, 128, 40, "float32"),
          (1, 3, 250, 16, "bfloat16"), (3, 3, 512, 32, "float32"), (1, 5, 1001, 70, "float32"), (1, 2, 1024, 1024, "bfloat16")]


@pytest.mark.parametrize("shape", TABLES, ids=str)
@pytest.mark.parametrize("twice", [False, True])
def test_distill(mlsim, shape, twice):
    P, N, R, K, dtype = shape
    rng = np.random.default_rng(hash(shape[:4]) % 2**32 + twice)
    t, x = make_logits(rng, P, N, R, dtype)
    if twice:  # a resource named by several entries
        ids = rng.integers(0, max(1, R // 2), (P, N, K))
    else:
        ids = np.argsort(rng.random((P, N, R)), -1)[..., :K]
    y = rng.normal(size=(P, N, K)) * 2
    x_at = np.take_along_axis(x, ids, -1)
    gone = x_at == -np.inf
    gone[:, 1::4] = False  # the teacher names what these rows do not allow
    ids = np.where(gone, ref.NO_PLACE, ids)
    y = np.where(gone, np.nan, y)  # what stands at padded entries is not read
    y[:, 2::4] = np.where(rng.random(y[:, 2::4].shape) < 0.3, -np.inf, y[:, 2::4])
    yt = torch.from_numpy(y).to(TYPES[dtype])
    w = rng.random((P, N)).astype(np.float32)
    for T, wt in ((1.0, None), (0.5, w), (rng.choice([0.5, 1.0, 3.0], P).astype(np.float32), w)):
        print(f"distill {shape}", flush=True)
        pol = mlsim.Policy(t, temperature=T)
        loss, grad = pol.distill(u16(ids), yt.cuda(), weight=None if wt is None else torch.from_numpy(wt).cuda())
        rl, lt, rg, gt = ref.distill(x, ids, yt.double().numpy(), ref.settings_of(P, T), wt, dtype)
        ref.near(loss.cpu().numpy(), rl, lt, "loss")
        ref.near(grad.double().cpu().numpy(), rg, gt, "grad")
        alone, none = pol.distill(u16(ids), yt.cuda(), want_grad=False)
        assert none is None and torch.equal(torch.nan_to_num(alone), torch.nan_to_num(loss))
        again, g2 = pol.distill(u16(ids), yt.cuda(), weight=None if wt is None else torch.from_numpy(wt).cuda())
        assert torch.equal(torch.nan_to_num(g2), torch.nan_to_num(grad))


def test_distill_of_bad_rows(mlsim):
    nan = float("nan")
    x = np.array([[[-INF] * 3, [-INF] * 3, [0, nan, 0], [INF, 0, 0], [0, 1, 2], [0, 1, 2], [0, 1, 2], [0, -INF, 1], [nan, 0, 0]]])
    ids = np.array([[[0, 1], [9, 9], [0, 1], [1, 2], [9, 9], [0, 1], [1, 9], [1, 2], [9, 9]]])
    y = np.array([[[0, 1], [0, 1], [0, 1], [0, 1], [0, 1], [nan, 0], [INF, 0], [0, 1], [0, 0]]])
    t = torch.from_numpy(x).float().cuda()
    for T in (1.0, 0.0):
        loss, grad = mlsim.Policy(t, temperature=T).distill(u16(ids), torch.from_numpy(y).float().cuda())
        rl, lt, rg, gt = ref.distill(x, ids, y, ref.settings_of(1, T))
        ref.near(loss.cpu().numpy(), rl, lt, "loss")
        ref.near(grad.cpu().numpy(), rg, gt, "grad")


def test_strides_and_what_lies_behind(mlsim):
    """Ops-major logits, views that begin at odd elements, shared rows, outputs
    inside larger arrays: the rest of those stays as it was."""
    rng = np.random.default_rng(11)
    P, N, R, S = 3, 6, 20, 50
    t, x = make_logits(rng, P, N, R, "bfloat16")
    u = uniform(rng, N, S)
    st = ref.settings_of(P)
    want = ref.sample(x, u.astype(np.float64), st, 4)
    w = rng.normal(size=S).astype(np.float32)
    by_op = t.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.zeros((P, N, R + 9), dtype=t.dtype, device="cuda")
    wide[:, :, 3:3 + R] = t
    for view in (by_op, wide[:, :, 3:3 + R]):
        ud = torch.full((N, S + 5), float("nan"), device="cuda")
        ud[:, 2:2 + S] = torch.from_numpy(u).cuda()
        out = u16(np.full((N, S + 7), 777))
        pol = mlsim.Policy(view, block=4)
        pol.sample(ud[:, 2:2 + S], out=out[:, 3:3 + S])
        got = host16(out)
        assert np.array_equal(got[:, 3:3 + S], want)
        assert (got[:, :3] == 777).all() and (got[:, 3 + S:] == 777).all()
        place = out[:, 3:3 + S]
        ref.near(pol.logp(place).cpu().numpy(), *ref.logp(x, want, st, 4), "logp")
        buf = torch.full((P, N, R + 9), 7.0, dtype=t.dtype, device="cuda")
        pol.grad(place, torch.from_numpy(w).cuda(), out=buf[:, :, 5:5 + R])
        rg, gt = ref.grad(x, want, w, st, 4, dtype="bfloat16")
        ref.near(buf[:, :, 5:5 + R].double().cpu().numpy(), rg, gt, "grad")
        assert (buf[:, :, :5] == 7).all() and (buf[:, :, 5 + R:] == 7).all()
        gop = torch.full((N, P, R), 7.0, dtype=t.dtype, device="cuda").transpose(0, 1)
        pol.grad(place, torch.from_numpy(w).cuda(), out=gop)
        ref.near(gop.double().cpu().numpy(), rg, gt, "grad, ops outermost")
        big = torch.full((S + 9,), 7.0, device="cuda")
        pol.logp(place, out=big[4:4 + S])
        assert (big[:4] == 7).all() and (big[4 + S:] == 7).all()
    # one row for every policy, each with its own temperature
    T = np.array([0.5, 1.0, 2.0], np.float32)
    shared = mlsim.Policy(t[:1].expand(P, N, R), block=4, temperature=T)
    xs = np.broadcast_to(x[:1], x.shape)
    got = host16(shared.sample(torch.from_numpy(u).cuda()))
    assert np.array_equal(got, ref.sample(xs, u.astype(np.float64), ref.settings_of(P, T), 4))
    rg, gt = ref.grad(xs, got, w, ref.settings_of(P, T), 4, dtype="bfloat16")
    ref.near(shared.grad(u16(got), torch.from_numpy(w).cuda()).double().cpu().numpy(), rg, gt, "grad of shared rows")
    # a teacher's table shared by the policies
    ids, y = rng.integers(0, R, (1, N, 4)), torch.from_numpy(rng.normal(size=(1, N, 4))).to(t.dtype)
    pol = mlsim.Policy(torch.nan_to_num(t, neginf=-3.0))
    loss, grad = pol.distill(u16(ids).expand(P, N, 4), y.cuda().expand(P, N, 4))
    rl, lt, rg, gt = ref.distill(pol.logits.double().cpu().numpy(), np.broadcast_to(ids, (P, N, 4)),
                                 np.broadcast_to(y.double().numpy(), (P, N, 4)), st, None, "bfloat16")
    ref.near(loss.cpu().numpy(), rl, lt, "loss")
    ref.near(grad.double().cpu().numpy(), rg, gt, "grad")


def test_offsets_beyond_32_bits(mlsim):
    """Rows whose elements lie past 2^32, in every array."""
    rng = np.random.default_rng(12)
    N, R, S, far = 2, 9, 70, 2**32 + 24
    t, x = make_logits(rng, 1, N, R, "bfloat16")
    u = uniform(rng, N, S)
    big = torch.empty(far + R, dtype=torch.bfloat16, device="cuda").as_strided((1, N, R), (0, far, 1))
    big.copy_(t)
    ud = torch.empty(far + S, device="cuda").as_strided((N, S), (far, 1))
    ud.copy_(torch.from_numpy(u))
    place = torch.empty(far + S, dtype=torch.int16, device="cuda").view(torch.uint16).as_strided((N, S), (far, 1))
    for block in (1, 100):
        pol = mlsim.Policy(big, block=block)
        pol.sample(ud, out=place)
        got = host16(place.contiguous())
        assert np.array_equal(got, ref.sample(x, u.astype(np.float64), ref.settings_of(1)))
        ref.near(pol.logp(place).cpu().numpy(), *ref.logp(x, got, ref.settings_of(1)), "logp")
        g = torch.empty(far + R, dtype=torch.bfloat16, device="cuda").as_strided((1, N, R), (0, far, 1))
        w = rng.normal(size=S).astype(np.float32)
        pol.grad(place, torch.from_numpy(w).cuda(), out=g)
        ref.near(g.double().cpu().numpy(), *ref.grad(x, got, w, ref.settings_of(1), dtype="bfloat16"), "grad")
        del g


def test_many_scenarios_of_one_row(mlsim):
    """A long batch over few ops, its counts odd: split over the scenarios."""
    rng = np.random.default_rng(13)
    for P, N, R, block, S in ((1, 2, 5, 1, 300_001), (2, 1, 40, 100_000, 200_003), (1, 1, 700, 1, 70_001),
                              (3, 2, 20, 1, 30_001), (2, 1, 600, 3, 9_001), (4, 5, 64, 700, 20_011), (5, 9, 9, 2, 4_003)):
        print(f"many {P} {N} {R} {S}", flush=True)
        t, x = make_logits(rng, P, N, R, "float32")
        u = uniform(rng, N, S)
        st = ref.settings_of(P, 1.0, 0, 0.95)
        pol = mlsim.Policy(t, block=block, top_p=0.95)
        place = pol.sample(torch.from_numpy(u).cuda())
        got = host16(place)
        assert np.array_equal(got, ref.sample(x, u.astype(np.float64), st, block))
        ref.near(pol.logp(place).cpu().numpy(), *ref.logp(x, got, st, block), "logp")
        w = rng.normal(size=S).astype(np.float32)
        ref.near(pol.grad(place, torch.from_numpy(w).cuda()).cpu().numpy(), *ref.grad(x, got, w, st, block), "grad")


def test_many_ops_of_one_scenario(mlsim):
    """One long scenario: split over the ops."""
    rng = np.random.default_rng(14)
    N, R = 5003, 12
    t, x = make_logits(rng, 1, N, R, "float16")
    u = uniform(rng, N, 1)
    pol = mlsim.Policy(t)
    place = pol.sample(torch.from_numpy(u).cuda())
    got = host16(place)
    assert np.array_equal(got, ref.sample(x, u.astype(np.float64), ref.settings_of(1)))
    ref.near(pol.logp(place).cpu().numpy(), *ref.logp(x, got, ref.settings_of(1)), "logp")


def test_gradients_against_differences(mlsim):
    """grad and distill's gradient against central differences of logp and loss
    along one direction, |direction| = 1: the step's h^2 / 6 times the third
    derivative (below 2 for a row's softmax at T = 1, weighted), and the
    outputs' own bounds over the step."""
    rng = np.random.default_rng(15)
    P, N, R, S, h = 2, 4, 6, 20, 2.0**-5
    x = rng.normal(size=(P, N, R)).astype(np.float32)
    d = rng.normal(size=(P, N, R))
    d = (d / np.linalg.norm(d)).astype(np.float32)
    a, w = rng.integers(0, R, (N, S)), rng.normal(size=S).astype(np.float32)
    ids, y = rng.integers(0, R, (P, N, 3)), rng.normal(size=(P, N, 3)).astype(np.float32)
    place, yd, st = u16(a), torch.from_numpy(y).cuda(), ref.settings_of(P)

    def pol(x):
        return mlsim.Policy(torch.from_numpy(x).cuda(), block=3)

    steps = [(x + s * h * d).astype(np.float32) for s in (1, -1)]
    step = float((steps[0].astype(np.float64) - steps[1]).ravel() @ d.ravel().astype(np.float64))
    lp = [pol(z).logp(place).double().cpu().numpy() @ w for z in steps]
    g = pol(x).grad(place, torch.from_numpy(w).cuda()).double().cpu().numpy()
    own = np.abs(w) @ ref.logp(x.astype(np.float64), a, st, 3)[1]
    tol = 2 * h * h / 6 * np.abs(w).sum() + 4 * own / (2 * h)
    assert abs((lp[0] - lp[1]) / step - (g * d).sum()) < tol
    ls = [pol(z).distill(u16(ids), yd, want_grad=False)[0].double().sum().item() for z in steps]
    _, g = pol(x).distill(u16(ids), yd)
    own = ref.distill(x.astype(np.float64), ids, y.astype(np.float64), st)[1].sum()
    assert abs((ls[0] - ls[1]) / step - (g.double().cpu().numpy() * d).sum()) < 2 * h * h / 6 + 4 * own / (2 * h)


def search_step(mlsim, g, pol, dur, u, ids, top):
    """One step of a placement search: draw, replay, learn."""
    mk, _, st, place = g.run_sampled(pol, dur, u)
    adv = torch.where(st == 0, mk.float(), 0.0)
    adv = (adv - adv.mean()) / dur.shape[1]
    lp = pol.logp(place)
    grad = pol.grad(place, adv)
    loss, dgrad = pol.distill(ids, top)
    return dict(makespan=mk, status=st, place=place, adv=adv, logp=lp, grad=grad, loss=loss, dgrad=dgrad)


def test_a_search_step(mlsim):
    """The operators together on a workload's graph, replayed by the oracle; an
    op that may run nowhere is reported by the replay."""
    w = W.make_config(1, n_scen=300)
    rng = np.random.default_rng(16)
    N, R, S = w.n_ops, w.n_res, 300
    dur_h = w.durations()
    t, x = make_logits(rng, 3, N, R, "float32")
    t[1, 7] = -INF
    x[1, 7] = -INF
    u = uniform(rng, N, S)
    ids, y = rng.integers(0, R, (3, N, 2)), rng.normal(size=(3, N, 2)).astype(np.float32)
    g = mlsim.Graph.from_workload(w)
    pol = mlsim.Policy(t, block=50)
    o = search_step(mlsim, g, pol, torch.from_numpy(dur_h).cuda(), torch.from_numpy(u).cuda(), u16(ids), torch.from_numpy(y).cuda())
    st = ref.settings_of(3)
    place = ref.sample(x, u.astype(np.float64), st, 50)
    assert np.array_equal(host16(o["place"]), place)
    omk, _, ost = oracle.run_batch(w.succ_ptr, w.succ_idx, w.op_res, R, dur_h, place=place.astype(np.uint16), want_finish=False)
    assert np.array_equal(o["makespan"].cpu().numpy(), omk) and np.array_equal(o["status"].cpu().numpy(), ost)
    assert (ost == mlsim.SIM_ST_BAD_RES).sum() == 100 and (ost == 0).sum() == 200
    adv = o["adv"].cpu().numpy()
    ref.near(o["logp"].cpu().numpy(), *ref.logp(x, place, st, 50), "logp")
    ref.near(o["grad"].cpu().numpy(), *ref.grad(x, place, adv, st, 50), "grad")
    rl, lt, rg, gt = ref.distill(x, ids, y.astype(np.float64), st)
    ref.near(o["loss"].cpu().numpy(), rl, lt, "loss")
    ref.near(o["dgrad"].cpu().numpy(), rg, gt, "distillation's gradient")
    with pytest.raises(ValueError):
        g.run_sampled(mlsim.Policy(t[:, :5]), torch.from_numpy(dur_h).cuda(), torch.from_numpy(u).cuda())
    with pytest.raises(ValueError):
        g.run_sampled(pol, torch.from_numpy(dur_h).cuda(), torch.from_numpy(u[:, :9].copy()).cuda())
    g.close()


def test_captured_and_replayed(mlsim):
    """A step in a HIP graph, replayed with new inputs in place; eager work and
    a second captured graph in between."""
    rng = np.random.default_rng(17)
    P, N, R, S = 2, 30, 9, 700
    t, _ = make_logits(rng, P, N, R, "float32")
    pol = mlsim.Policy(t, block=200, top_p=0.9)
    u = torch.from_numpy(uniform(rng, N, S)).cuda()
    w = torch.from_numpy(rng.normal(size=S).astype(np.float32)).cuda()
    ids, y = u16(rng.integers(0, R, (P, N, 3))), torch.randn((P, N, 3), device="cuda")

    def step():
        place = pol.sample(u)
        return place, pol.logp(place), pol.grad(place, w), *pol.distill(ids, y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step())
        graphs.append(g)
    for k in range(4):
        u.copy_(torch.from_numpy(uniform(rng, N, S)))
        t.add_(torch.randn(t.shape, device="cuda") * 0.3)
        want = [o.clone() for o in step()]
        graphs[k % 2].replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs[k % 2]):
            assert torch.equal(a.view(torch.int16) if a.dtype == torch.uint16 else torch.nan_to_num(a),
                               b.view(torch.int16) if b.dtype == torch.uint16 else torch.nan_to_num(b)), k


def test_two_streams(mlsim):
    """Calls of one policy on two streams at once, inputs dropped right after."""
    rng = np.random.default_rng(18)
    N, R, S = 200, 20, 3000
    t, x = make_logits(rng, 1, N, R, "float32")
    pol = mlsim.Policy(t)
    u = [uniform(rng, N, S) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for k in range(2):
        ud = torch.from_numpy(u[k]).cuda()
        streams[k].wait_stream(torch.cuda.current_stream())
        place = pol.sample(ud, stream=streams[k])
        del ud
        junk = torch.full((N, S), 0.5, device="cuda")  # may take ud's memory if nothing kept it
        got.append((place, pol.logp(place, stream=streams[k])))
        del junk
    torch.cuda.synchronize()
    for k in range(2):
        want = ref.sample(x, u[k].astype(np.float64), ref.settings_of(1))
        assert np.array_equal(host16(got[k][0]), want)
        ref.near(got[k][1].cpu().numpy(), *ref.logp(x, want, ref.settings_of(1)), "logp")


def test_python_refusals(mlsim):
    t = torch.zeros((2, 4, 3), device="cuda")
    pol = mlsim.Policy(t)
    u, place = torch.zeros((4, 6), device="cuda"), u16(np.zeros((4, 6)))
    w, y, ids = torch.zeros(6, device="cuda"), torch.zeros((2, 4, 2), device="cuda"), u16(np.zeros((2, 4, 2)))
    bad = [lambda: mlsim.Policy(t.double()), lambda: mlsim.Policy(t[..., ::2]), lambda: mlsim.Policy(t[0, 0]),
           lambda: mlsim.Policy(t, temperature=[1.0, 2.0, 3.0]), lambda: mlsim.Policy(t, top_k=1.5),
           lambda: mlsim.Policy(torch.zeros((1, 2, 1025), device="cuda")), lambda: mlsim.Policy(t, temperature=-1.0),
           lambda: mlsim.Policy(t, top_p=2.0), lambda: mlsim.Policy(t, block=0),
           lambda: pol.sample(u.cpu()), lambda: pol.sample(u[:3]), lambda: pol.sample(u.double()), lambda: pol.sample(u.T),
           lambda: pol.sample(None), lambda: pol.sample(u, out=place[:, :5]), lambda: pol.sample(u, out=u),
           lambda: pol.logp(u), lambda: pol.logp(place[:2]), lambda: pol.logp(None), lambda: pol.logp(place, out=w[:5]),
           lambda: pol.logp(place, out=w.double()), lambda: pol.grad(place, w[:5]), lambda: pol.grad(place, w.double()),
           lambda: pol.grad(place, w.cpu()), lambda: pol.grad(place, w, out=t[:1]), lambda: pol.grad(place, w, out=t.half()),
           lambda: pol.grad(place, w, out=t[:1].expand(2, 4, 3)), lambda: pol.distill(ids, y[..., :1]),
           lambda: pol.distill(ids.view(torch.int16), y), lambda: pol.distill(ids, y.half()), lambda: pol.distill(ids[:1], y[:1]),
           lambda: pol.distill(ids[..., :0], y[..., :0]), lambda: pol.distill(ids, y, weight=w),
           lambda: pol.distill(ids, y, loss=torch.zeros((4, 2), device="cuda")), lambda: pol.distill(None, None)]
    for k, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, mlsim.SimError)):
            f()
            print(k)
    # no scenarios, no ops
    assert pol.sample(u[:, :0]).shape == (4, 0) and pol.logp(place[:, :0]).shape == (0,)
    assert (pol.grad(place[:, :0], w[:0]) == 0).all()
    none = mlsim.Policy(t[:, :0])
    assert none.sample(u[:0]).shape == (0, 6) and (none.logp(place[:0]) == 0).all()
    assert none.grad(place[:0], w).shape == (2, 0, 3)


def test_numbers_beyond_the_struct_s(mlsim):
    """Numbers that do not fit the C struct are refused or mean what they say,
    and are never cut off to their low bits."""
    t = torch.randn((1, 4, 3), device="cuda")
    for f in (lambda: mlsim.Policy(t.expand(2**32 + 1, 4, 3)), lambda: mlsim.Policy(t[:, :1].expand(1, 2**32 + 1, 3)),
              lambda: mlsim.Policy(t, block=2**64 + 1), lambda: mlsim.Policy(t, scen0=2**64), lambda: mlsim.Policy(t, scen0=-2**64),
              lambda: mlsim.Policy(t, top_k=-2**32)):
        with pytest.raises((ValueError, mlsim.SimError)):
            f()
    u = torch.rand((4, 500), device="cuda")
    all_kept = host16(mlsim.Policy(t).sample(u))
    for top_k in (2**31, 2**32 + 1, 2.0**40):
        assert np.array_equal(host16(mlsim.Policy(t, top_k=top_k).sample(u)), all_kept)


def test_settings_of_each_kind(mlsim):
    """Numbers, sequences, host and GPU tensors give the same draws, on a stream
    that waits for nothing where the settings come from the host."""
    rng = np.random.default_rng(8)
    t, x = make_logits(rng, 3, 5, 12, "float32")
    u = uniform(rng, 5, 60)
    T, k, p = [0.5, 1.0, 2.0], [3, 0, 5], [0.9, 0.8, 1.0]
    want = ref.sample(x, u.astype(np.float64), ref.settings_of(3, T, k, p, 0.01), 4)
    ug, other = torch.from_numpy(u).cuda(), torch.cuda.Stream()
    torch.cuda.synchronize()
    kinds = [list, tuple, np.array, torch.tensor, lambda v: torch.tensor(v, device="cuda")]
    for i, f in enumerate(kinds):
        pol = mlsim.Policy(t, block=4, temperature=f(T), top_k=f(k), top_p=kinds[(i + 1) % 5](p), min_p=0.01)
        if any(q is kinds[4] for q in (f, kinds[(i + 1) % 5])):
            other.wait_stream(torch.cuda.current_stream())
        got = pol.sample(ug, stream=other)
        other.synchronize()
        assert np.array_equal(host16(got), want), i


def test_run_sampled_draws_nothing_for_bad_durations(mlsim):
    w = W.make_config(1, n_scen=6)
    g = mlsim.Graph.from_workload(w)
    pol = mlsim.Policy(torch.zeros((w.n_ops, w.n_res), device="cuda"))
    u = torch.rand((w.n_ops, 6), device="cuda")
    place = u16(np.full((w.n_ops, 6), 7))
    for dur in (torch.ones((w.n_ops, 6), dtype=torch.int64, device="cuda"), torch.ones((w.n_ops, 6), dtype=torch.int32)):
        with pytest.raises((TypeError, ValueError)):
            g.run_sampled(pol, dur, u, place=place)
    assert (host16(place) == 7).all()
    g.close()


@pytest.mark.parametrize("S", [3, 30, 3000])
def test_the_least_temperature(mlsim, S):
    """At T = 2^-126 a row's best resource has probability 1: its log-probability
    is 0, and so is the gradient where it was taken, however large the weights;
    a positive number below is no temperature."""
    x = np.array([[[0.0, -1.0, -INF], [5.0, 4.0, 3.0], [-1.0, -3.0, -2.0], [-3e38, -INF, -INF]]] * 3)
    t, u = torch.from_numpy(x).float().cuda(), torch.rand((4, S), device="cuda")
    w = torch.full((S,), 1e30, device="cuda")
    for T in (2.0**-126, [2.0**-126] * 3, [2.0**-127, 2.0**-126, 1e-45]):
        pol = mlsim.Policy(t, temperature=T, block=S // 3)
        bad = np.array([isinstance(T, list) and q < 2.0**-126 for q in (T if isinstance(T, list) else [T] * 3)])
        place = pol.sample(u)
        lost = bad[ref.policy_of(np.arange(S), S // 3, 0, 3)]
        assert np.array_equal(host16(place), np.where(lost, ref.NO_PLACE, np.zeros((4, S)))), T
        best = u16(np.zeros((4, S)))
        logp = pol.logp(best).cpu().numpy()
        assert np.isnan(logp[lost]).all() and (logp[~lost] == 0).all(), T
        g = pol.grad(best, w).cpu().numpy()
        assert np.isnan(g[bad]).all() and (g[~bad] == 0).all(), T
        loss, dg = pol.distill(u16(np.zeros((3, 4, 1))), torch.zeros((3, 4, 1), device="cuda"), weight=torch.full((3, 4), 1e30, device="cuda"))
        loss, dg = loss.cpu().numpy(), dg.cpu().numpy()
        assert np.isnan(loss[bad]).all() and (loss[~bad] == 0).all() and np.isnan(dg[bad]).all() and (dg[~bad] == 0).all(), T


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("P,N,R,k", [(2048, 75, 48, 8), (1025, 260, 61, 5), (1024, 150, 100, 8), (4096, 67, 64, 1)])
def test_many_rows_of_one_draw(mlsim, dtype, P, N, R, k):
    """So many rows that a group takes several, with few kept: the same draws as
    for a few policies at a time, and the plain form's.  Zeros of both signs,
    subnormal numbers, ties, empty and invalid rows among them."""
    rng = np.random.default_rng(R + k)
    x = torch.from_numpy(rng.normal(size=(P, N, R)).astype(np.float32) * 2).to(TYPES[dtype])
    x[::3, ::4] = torch.round(x[::3, ::4])
    x[::7, 1] = torch.from_numpy(rng.choice([-1, -0.0, 0.0], (len(range(0, P, 7)), R)).astype(np.float32)).to(x.dtype)
    tiny = torch.finfo(x.dtype).tiny
    x[::5, 2] = (torch.from_numpy(rng.integers(-60, 60, (len(range(0, P, 5)), R))).double() * (tiny / 64)).to(x.dtype)
    x[torch.from_numpy(rng.random((P, N, R)) < 0.1)] = -INF
    x[3, 5] = -INF
    x[4, 6, 7], x[5, 7, 8], x[6, 8, 9], x[7, 9, 10] = float("nan"), -float("nan"), INF, -INF
    knobs = dict(temperature=np.full(P, 1.0, np.float32), top_k=rng.integers(1, k + 1, P).astype(np.float32),
                 top_p=rng.choice([0.5, 0.9, 1.0], P).astype(np.float32), min_p=np.float32(0))
    knobs["top_k"][100:200] = rng.integers(0, R, 100)  # others keep more
    t, u = x.cuda(), uniform(rng, N, P)
    ug = torch.from_numpy(u).cuda()
    got = host16(mlsim.Policy(t, **knobs).sample(ug))
    few = [host16(mlsim.Policy(t[a:a + 64], **{n: v if v.ndim == 0 else v[a:a + 64] for n, v in knobs.items()}).sample(ug[:, a:a + 64]))
           for a in range(0, P, 64)]
    assert np.array_equal(got, np.concatenate(few, 1))
    st = ref.settings_of(P, **knobs)
    for p in [*range(9), 100, 150, 199, *rng.integers(0, P, 10), P - 1]:
        want = ref.sample(x[p:p + 1].double().numpy(), u[:, p:p + 1].astype(np.float64), st[p:p + 1])
        assert np.array_equal(got[:, p:p + 1], want), p
    one = dict(temperature=0.7, top_k=k, top_p=0.9)
    got = host16(mlsim.Policy(t, **one).sample(ug))
    few = [host16(mlsim.Policy(t[a:a + 64], **one).sample(ug[:, a:a + 64])) for a in range(0, P, 64)]
    assert np.array_equal(got, np.concatenate(few, 1))


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("P,N,R", [(2048, 75, 48), (1025, 260, 61), (1024, 40, 600)])
def test_many_rows_of_one_scenario(mlsim, dtype, P, N, R):
    """So many rows that a group takes several: the gradient and the
    log-probabilities have the same bits as for a few policies at a time."""
    rng = np.random.default_rng(R)
    t = (torch.randn((P, N, R), device="cuda") * 2).to(TYPES[dtype])
    t[5, 3] = -INF
    t[6, 4, 5] = float("nan")
    a = u16(rng.integers(0, R + 1, (N, P)))
    w = torch.randn(P, device="cuda")
    g, l = mlsim.Policy(t).grad(a, w), mlsim.Policy(t).logp(a)
    for p in range(0, P, 64):
        some, place = mlsim.Policy(t[p:p + 64]), a.view(torch.int16)[:, p:p + 64].contiguous().view(torch.uint16)
        assert torch.equal(torch.nan_to_num(g[p:p + 64]), torch.nan_to_num(some.grad(place, w[p:p + 64].contiguous())))
        # summed in other chunks: to float32's step
        assert torch.allclose(l[p:p + 64], some.logp(place), rtol=2.0**-22, atol=0, equal_nan=True)
