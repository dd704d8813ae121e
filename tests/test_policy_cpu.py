"""Placement policies on the host: refusals before any HIP call, and the plain
forms that the GPU tests compare with, checked against each other."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2002_06790_amd as mlsim
import policy_ref as ref

FAKE = 4096  # an address that no call below gets to read


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(mlsim.LIB_PATH):
        mlsim.build()
    return mlsim.lib()


def struct(**kw):
    d = dict(logits=FAKE, ld_pol=12, ld_op=3, block=1, scen0=0, settings=None, temperature=1.0, top_k=0, top_p=1.0,
             min_p=0.0, dtype=0, n_pol=2, n_ops=4, n_res=3)
    d.update(kw)
    return mlsim._PolicyStruct(**d)


BAD = [dict(n_pol=0), dict(n_ops=-1), dict(n_res=0), dict(block=0), dict(scen0=-1), dict(dtype=3), dict(dtype=-1),
       dict(ld_pol=-1), dict(ld_op=-3), dict(logits=None), dict(logits=FAKE + 2), dict(logits=FAKE + 1, dtype=1),
       dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1),
       dict(top_p=-0.5), dict(top_p=1.5), dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.1),
       dict(min_p=float("nan")), dict(settings=FAKE + 1), dict(scen0=2**63 - 4), dict(ld_op=2**60), dict(ld_pol=2**62)]


@pytest.mark.parametrize("kw", BAD, ids=str)
def test_bad_policies_are_refused(L, kw):
    p = struct(**kw)
    assert L.sim_policy_work(p, 8) == mlsim.SIM_E_INVAL
    assert L.sim_policy_sample(p, 8, FAKE, 8, FAKE, 8, None) == mlsim.SIM_E_INVAL
    assert L.sim_policy_logp(p, 8, FAKE, 8, FAKE, FAKE, 2**40, None) == mlsim.SIM_E_INVAL
    assert L.sim_policy_grad(p, 8, FAKE, 8, FAKE, FAKE, 12, 3, FAKE, 2**40, None) == mlsim.SIM_E_INVAL
    if kw != dict(scen0=2**63 - 4):  # has no scenarios
        assert L.sim_policy_distill(p, FAKE, 4, 1, FAKE, 4, 1, 1, None, FAKE, None, 0, 0, None) == mlsim.SIM_E_INVAL


def test_limits_are_refused(L):
    assert L.sim_policy_work(struct(n_res=1025, ld_op=1025), 8) == mlsim.SIM_E_LIMIT
    assert L.sim_policy_work(struct(n_ops=2**24 + 1), 8) == mlsim.SIM_E_LIMIT
    assert L.sim_policy_work(struct(), 2**40 + 1) == mlsim.SIM_E_LIMIT
    assert L.sim_policy_work(struct(), -1) == mlsim.SIM_E_INVAL
    assert L.sim_policy_work(None, 1) == mlsim.SIM_E_INVAL
    assert L.sim_policy_work(struct(), 8) >= 0


def test_bad_arrays_are_refused(L):
    p, E = struct(), mlsim.SIM_E_INVAL
    assert L.sim_policy_sample(p, 8, None, 8, FAKE, 8, None) == E
    assert L.sim_policy_sample(p, 8, FAKE, 8, None, 8, None) == E
    assert L.sim_policy_sample(p, 8, FAKE, 7, FAKE, 8, None) == E
    assert L.sim_policy_sample(p, 8, FAKE, 8, FAKE, 7, None) == E
    assert L.sim_policy_sample(p, 8, FAKE + 2, 8, FAKE, 8, None) == E
    assert L.sim_policy_sample(p, 8, FAKE, 8, FAKE + 1, 8, None) == E
    need = L.sim_policy_work(p, 8)
    for place, ld, out, work, size in ((None, 8, FAKE, FAKE, need), (FAKE, 7, FAKE, FAKE, need), (FAKE, 8, None, FAKE, need),
                                       (FAKE, 8, FAKE + 2, FAKE, need), (FAKE + 1, 8, FAKE, FAKE, need)):
        assert L.sim_policy_logp(p, 8, place, ld, out, work, size, None) == E
    if need:
        assert L.sim_policy_logp(p, 8, FAKE, 8, FAKE, FAKE, need - 1, None) == E
        assert L.sim_policy_logp(p, 8, FAKE, 8, FAKE, None, need, None) == E
        assert L.sim_policy_logp(p, 8, FAKE, 8, FAKE, FAKE + 4, need, None) == E
    for place, ld, w, g in ((None, 8, FAKE, FAKE), (FAKE, 7, FAKE, FAKE), (FAKE, 8, None, FAKE), (FAKE, 8, FAKE, None),
                            (FAKE, 8, FAKE + 1, FAKE), (FAKE, 8, FAKE, FAKE + 2)):
        assert L.sim_policy_grad(p, 8, place, ld, w, g, 12, 3, FAKE, need, None) == E
    for ld_pol, ld_op in ((11, 3), (12, 2), (0, 3), (12, 0), (3, 5), (-12, 3), (2**62, 3)):  # rows over one another
        assert L.sim_policy_grad(p, 8, FAKE, 8, FAKE, FAKE, ld_pol, ld_op, FAKE, need, None) == E

    def distill(res=FAKE, top=1, logits=FAKE, loss=FAKE, grad=None, ld=(4, 1, 4, 1), weight=None):
        return L.sim_policy_distill(p, res, ld[0], ld[1], logits, ld[2], ld[3], top, weight, loss, grad, 12, 2, None)

    for kw in (dict(res=None), dict(logits=None), dict(loss=None), dict(top=0), dict(top=1025), dict(ld=(-1, 1, 4, 1)),
               dict(ld=(4, 1, 4, -1)), dict(res=FAKE + 1), dict(logits=FAKE + 2), dict(loss=FAKE + 2), dict(weight=FAKE + 2),
               dict(grad=FAKE)):
        assert distill(**kw) == E, kw


def test_nothing_to_do(L):
    p = struct()
    assert L.sim_policy_sample(p, 0, None, 0, None, 0, None) == mlsim.SIM_OK
    assert L.sim_policy_logp(p, 0, None, 0, None, None, 0, None) == mlsim.SIM_OK
    none = struct(n_ops=0, logits=None)
    assert L.sim_policy_sample(none, 5, None, 0, None, 0, None) == mlsim.SIM_OK
    assert L.sim_policy_grad(none, 5, None, 0, None, None, 0, 0, None, 0, None) == mlsim.SIM_OK
    assert L.sim_policy_distill(none, None, 0, 0, None, 0, 0, 1, None, None, None, 0, 0, None) == mlsim.SIM_OK
    assert L.sim_policy_work(none, 5) == 0


def test_struct_is_the_header_s():
    """Field order and size as a C compiler lays out sim_policy."""
    assert ctypes.sizeof(mlsim._PolicyStruct) == 80
    assert mlsim._PolicyStruct.settings.offset == 40 and mlsim._PolicyStruct.n_res.offset == 76


def test_python_refuses_host_tensors():
    with pytest.raises(TypeError):
        mlsim.Policy(torch.zeros(4, 3))
    with pytest.raises(TypeError):
        mlsim.Policy(np.zeros((4, 3)))


def test_plain_sample_keeps_what_the_settings_say():
    x = np.array([1.0, 3.0, 3.0, -np.inf, 2.0])

    def kept(T=1.0, k=0, p=1.0, m=0.0):
        C, _ = ref.kept_sums(x, T, k, p, m)
        return list(np.flatnonzero(np.diff(np.concatenate([[0.0], C])) > 0))

    assert kept() == [0, 1, 2, 4]
    assert kept(k=2) == [1, 2] and kept(k=1) == [1] and kept(T=0) == [1] and kept(p=0.0) == [1]
    assert kept(k=3) == [1, 2, 4] and kept(m=0.3) == [1, 2, 4] and kept(m=1.0) == [1, 2]
    assert kept(p=0.1) == [1] and kept(p=0.5) == [1, 2] and kept(k=2, p=0.4) == [1]
    for bad in (np.nan, np.inf):
        assert ref.kept_sums(np.array([0.0, bad]), 1.0, 0, 1.0, 0.0) is None
    assert ref.kept_sums(np.full(3, -np.inf), 1.0, 0, 1.0, 0.0) is None


def test_plain_gradients_agree_with_differences():
    rng = np.random.default_rng(4)
    P, N, R, S = 2, 3, 5, 7
    x = rng.normal(size=(P, N, R))
    x[0, 1, 3] = -np.inf
    st = ref.settings_of(P, [0.5, 2.0])
    place = rng.integers(0, 3, (N, S))
    w = rng.normal(size=S)
    g, _ = ref.grad(x, place, w, st, block=2, scen0=3)
    ids, top = rng.integers(0, 3, (P, N, 4)), rng.normal(size=(P, N, 4))
    dw = rng.random((P, N))
    _, _, dg, _ = ref.distill(x, ids, top, st, dw)
    for p, v, r in np.ndindex(P, N, R):
        if x[p, v, r] == -np.inf:
            assert g[p, v, r] == 0 and dg[p, v, r] == 0
            continue
        up, dn = x.copy(), x.copy()
        up[p, v, r] += 1e-5
        dn[p, v, r] -= 1e-5
        f = [(w * ref.logp(y, place, st, 2, 3)[0]).sum() for y in (up, dn)]
        assert abs((f[0] - f[1]) / 2e-5 - g[p, v, r]) < 1e-7
        f = [(dw * ref.distill(y, ids, top, st)[0]).sum() for y in (up, dn)]
        assert abs((f[0] - f[1]) / 2e-5 - dg[p, v, r]) < 1e-7


def test_temperatures_and_numbers_of_scenarios(L):
    """0 and normal float32 numbers are temperatures; up to 2^30 scenarios a call."""
    for T in (0.0, 2.0**-126, 3e38):
        assert L.sim_policy_work(struct(temperature=T), 8) >= 0
    for T in (2.0**-127, 1e-45, -1e-45):
        assert L.sim_policy_work(struct(temperature=T), 8) == mlsim.SIM_E_INVAL
    assert L.sim_policy_work(struct(), 2**30) >= 0
    assert L.sim_policy_work(struct(), 2**30 + 1) == mlsim.SIM_E_LIMIT


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_plain_forms_of_one_scenario_a_policy(dtype):
    """The forms over all rows at once against those row by row."""
    rng = np.random.default_rng(5)
    P, N, R = 9, 8, 11
    x = rng.normal(size=(P, N, R)) * 2
    x[rng.random((P, N, R)) < 0.2] = -np.inf
    x[:, ::3] = np.round(x[:, ::3])
    x[:, 1] = np.where(rng.random((P, R)) < 0.5, 0.0, -0.0)
    x[0, 2], x[1, 2, 3], x[2, 2, 4] = -np.inf, np.nan, np.inf
    u = (rng.integers(0, 2**24, (N, P)) * 2.0**-24)
    u[3, :4] = [-1.0, np.nan, 1.0, 0.0]
    for cut in (dict(), dict(top_k=3), dict(temperature=0.7, top_k=4, top_p=0.8), dict(min_p=0.2), dict(temperature=0.0), dict(top_p=0.0),
                dict(temperature=rng.choice([0.0, 0.5, -1.0, 3.0], P), top_k=rng.integers(-1, R + 2, P), top_p=rng.random(P) * 1.1, min_p=rng.random(P))):
        st = ref.settings_of(P, **cut)
        got = ref.sample_each(torch.from_numpy(x), torch.from_numpy(u), torch.from_numpy(st))
        assert np.array_equal(got.numpy(), ref.sample(x, u, st)), cut
    x[0, 2], x[1, 2, 3], x[2, 2, 4] = 1.0, 0.0, 0.0
    a = rng.integers(0, R + 1, (N, P))
    a[:, :4] = np.argmax(x, -1).T[:, :4]
    w, T = rng.normal(size=P), rng.choice([0.5, 1.0, 3.0], P)
    lp, ltol, g, gtol = (q.numpy() for q in ref.learn_each(torch.from_numpy(x), torch.from_numpy(a), torch.from_numpy(w), torch.from_numpy(T), dtype))
    want, tol = ref.logp(x, a, ref.settings_of(P, T))
    ref.near(lp, want, 1e-12, "logp")
    fine = np.isfinite(want)
    assert np.allclose(ltol[fine], tol[fine], rtol=1e-12, atol=0)
    want, tol = ref.grad(x, a, w, ref.settings_of(P, T), dtype=dtype)
    ref.near(g, want, 1e-12, "grad")
    assert (gtol < 4 * tol + 1e-30).all() and (tol < 4 * gtol + 1e-30).all()


def test_plain_gradients_of_shared_rows():
    """The same values as row by row, and a bound that zeros do not pass."""
    rng = np.random.default_rng(6)
    x, a, w = rng.normal(size=(2, 3, 7)), rng.integers(0, 8, (3, 4001)), rng.normal(size=4001).astype(np.float32)
    x[0, 1, 2] = -np.inf
    st = ref.settings_of(2, [0.5, 2.0])
    for dtype in ("float32", "float16"):
        g, tol = ref.grad_shared(x, a, w, st, 5, 3, dtype)
        ref.near(g, ref.grad(x, a, w.astype(np.float64), st, 5, 3, dtype)[0], 1e-9, "grad")
        assert ((np.abs(g) > 20 * tol) | (x == -np.inf)).mean() > 0.9
    assert ref.grid_of(w, 4001) < 2.0**-36 and ref.grid_of(np.zeros(3, np.float32), 3) == 0
    # the grid: as many of the largest weight as a batch may have add up exactly in float64
    for n in (1, 512, 4001, 2**22, 2**30):
        step, count = ref.grid_of(np.array([1.9], np.float32), n), min(-(-n // 512) * 512, 2**22)
        assert 2.0 * count / step <= 2.0**53
