"""GPU: the optimizer step at the limits of what it takes, for both forms of moments."""
import numpy as np
import pytest

from oracle import optim as O

from gpu_util import torch_cuda
from test_gpu_optim import B1, B2, EPS, TABLES, U, bounds, exact_grads, layout, near, stored, table, typed

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -148                                      # two of the smallest steps of fp32, each off by half


def fresh(torch, plan, n, coded):
    """Zero moments of either form, exponents among them."""
    kind = torch.uint8 if coded else torch.float32
    st = [torch.zeros(n, dtype=kind, device="cuda") for _ in range(2)]
    return st + ([torch.zeros(2 * plan.blocks, dtype=torch.uint8, device="cuda")] if coded else [])


def step_of(plan, coded):
    return plan.adamw_coded if coded else plan.adamw


def held(st, offs, numels, coded):
    """The moments that a state holds, in fp64."""
    a = [x.cpu().numpy() for x in st]
    if not coded:
        return [x.astype(np.float64) for x in a]
    m, v, first, exps = np.zeros(a[0].size), np.zeros(a[0].size), 0, a[2].reshape(-1, 2)
    for o, k in zip(offs, numels):
        c, b = slice(o, o + k), slice(first, first + (k + 127) // 128)
        m[c], v[c] = stored(a[0][c], exps[b, 0], O.OCTAVES_M, True), stored(a[1][c], exps[b, 1], O.OCTAVES_V, False)
        first = b.stop
    return [m, v]


def small_bounds(g, p, m, v, t, lr, beta2, eps):
    """p' in fp64 and what the step in fp32 may be off it where v' may lie below the smallest normal number: v' is off by its
    roundings, absolute ones there; the root by what that makes of it and one unit (2 u), the factor, the eps, their sum
    and the second rounding of the factor's product by u each; reciprocal 2 u, products and the rate 4 u."""
    new = O.step(g, p, m, v, t, lr, B1, beta2, eps, 0.0, 1.0)
    a = np.abs(new[1])
    em = 6 * U * (np.abs(B1 * m) + (1 - B1) * np.abs(g)) + TINY
    ev = 9 * U * new[2] + TINY
    root = 1 / np.sqrt(1 - beta2 ** t)
    side = [np.sqrt(np.maximum(new[2] + e, 0)) * root for e in (-ev, 0.0, ev)]
    den = side[1] + eps
    off = np.maximum(side[2] - side[1], side[1] - side[0]) + 6 * U * den
    assert (off < den).all()
    rate = lr / (1 - B1 ** t)
    return new[0], rate * ((a + em) / (den - off) * (1 + 8 * U) - a / den) + U * np.abs(new[0]) + TINY


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("beta2,eps,smallest", [(0.999, 1e-20, 1e-20), (0.999, 1e-30, 1e-20), (0.999, 1.2e-38, 1e-20), (0.5, 1e-25, 1e-21),
                                                (1 - 1e-7, 1e-16, 1e-17), (1 - 1e-7, 1e-30, 1e-17)])
def test_small_eps(beta2, eps, smallest, coded):
    """Gradients whose squares lie at and below the smallest normal number, under an eps that does not hide their root: three
    steps from zero moments, each against the formula from what the one before left."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES["blocks"])
    rng = np.random.default_rng(21)
    inside = np.zeros(n, bool)
    for o, k in zip(offs, numels):
        inside[o:o + k] = True
    plan = B.Optim(table(B, offs, numels))
    st, dp, step = fresh(torch, plan, n, coded), torch.zeros(n, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    s = B.adamw(lr=1e-3, beta1=B1, beta2=beta2, eps=eps, weight_decay=0.0)
    for t in (1, 2, 3):
        g = (smallest * 10.0 ** rng.uniform(0, 4, n) * rng.choice([-1.0, 1.0], n)).astype(np.float32)
        p, (m, v) = dp.cpu().numpy(), held(st, offs, numels, coded)
        step_of(plan, coded)(s, torch.from_numpy(g).cuda(), dp, *st, step)
        want, tol = small_bounds(g[inside], p[inside], m[inside], v[inside], t, 1e-3, beta2, eps)
        near(dp.cpu().numpy()[inside], want, tol, ("p", t))
    assert int(step) == 3


@pytest.mark.parametrize("coded", [False, True])
def test_gradients_whose_squares_leave_fp32(coded):
    """With the sums a step of finite gradients whose squares do not fit fp32 is left out, as one of gradients that are not
    finite is; at the limit, behind a factor, and clipped it is taken."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([700, 3000], 0, 0)
    rng = np.random.default_rng(22)
    p = rng.standard_normal(n).astype(np.float32)
    plan = B.Optim(table(B, offs, numels))
    for peak, scale, max_norm, taken in ((3e19, 1.0, 0.0, False), (-3e38, 1.0, 0.0, False), (1.31e19, 1.0, 0.0, False), (1.3e19, 1.0, 0.0, True),
                                         (3e19, 0.25, 0.0, True), (3e19, 4.0, 1.0, True), (-3e38, 1.0, 10.0, True), (3e19, 4.0, 1e30, False)):
        g = (rng.standard_normal(n) * 1e-3).astype(np.float32)
        g[3000] = peak
        dg, sums = torch.from_numpy(g).cuda(), torch.zeros(3, dtype=torch.float64, device="cuda")
        plan.norms(dg, sums)
        c = O.clip(float((g[:3700].astype(np.float64) ** 2).sum()), scale, max_norm)
        assert (c * abs(peak) < 2 ** 63.5) == taken
        st = [torch.from_numpy(p).cuda()] + fresh(torch, plan, n, coded)
        old, step = [a.clone() for a in st], torch.zeros(1, dtype=torch.int64, device="cuda")
        step_of(plan, coded)(B.adamw(lr=1e-3, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.0, grad_scale=scale, max_norm=max_norm), dg,
                             *st, step, d_sumsq=sums)
        assert int(step) == taken, peak
        if not taken:
            assert all(torch.equal(a, b) for a, b in zip(old, st)), peak
            continue
        new, tol = bounds(g, p, np.zeros(n), np.zeros(n), 1, 1e-3, 0.0, c)
        near(st[0].cpu().numpy()[:3700], new[0][:3700], tol[0][:3700], ("p", peak))
        assert all(np.isfinite(a).all() for a in held(st[1:], offs, numels, coded))


@pytest.mark.parametrize("coded", [False, True])
def test_the_gradients_factor_is_a_normal_number(coded):
    """Factors that fp32 holds as infinite, as 0 or with a few bits only are refused, and a clipped step that comes to one is left out."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([700, 3000], 0, 0)
    rng = np.random.default_rng(23)
    p = rng.standard_normal(n).astype(np.float32)
    plan = B.Optim(table(B, offs, numels))
    f = step_of(plan, coded)
    least, most = 2.0 ** -126, float(np.finfo(np.float32).max)
    zero = torch.zeros(n, device="cuda")
    for scale in (1e39, 1e300, least * 0.99, 1e-42, 1e-60, 1e-300):
        st, step = [torch.from_numpy(p).cuda()] + fresh(torch, plan, n, coded), torch.zeros(1, dtype=torch.int64, device="cuda")
        with pytest.raises(B.LgrecoError) as e:
            f(B.adamw(lr=1e-3, grad_scale=scale), zero, *st, step)
        assert e.value.status == B.EINVAL
    for scale, size in ((least, 1e37), (most, 1e-38)):
        g = (rng.standard_normal(n) * size).astype(np.float32)
        st, step = [torch.from_numpy(p).cuda()] + fresh(torch, plan, n, coded), torch.zeros(1, dtype=torch.int64, device="cuda")
        f(B.adamw(lr=1e-3, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.0, grad_scale=scale), torch.from_numpy(g).cuda(), *st, step)
        new, tol = bounds(g, p, np.zeros(n), np.zeros(n), 1, 1e-3, 0.0, scale)
        near(st[0].cpu().numpy()[:3700], new[0][:3700], tol[0][:3700], scale)
    g = np.full(n, 1e37, np.float32)
    dg, sums = torch.from_numpy(g).cuda(), torch.zeros(3, dtype=torch.float64, device="cuda")
    plan.norms(dg, sums)
    for max_norm, taken in ((1e-7, False), (7.1, False), (7.2, True), (100.0, True)):
        c = O.clip(float(sums[2]), 1.0, max_norm)
        assert (c >= least) == taken
        st, step = [torch.from_numpy(p).cuda()] + fresh(torch, plan, n, coded), torch.zeros(1, dtype=torch.int64, device="cuda")
        old = [a.clone() for a in st]
        f(B.adamw(lr=1e-3, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.0, max_norm=max_norm), dg, *st, step, d_sumsq=sums)
        assert int(step) == taken, max_norm
        if taken:
            new, tol = bounds(g, p, np.zeros(n), np.zeros(n), 1, 1e-3, 0.0, c)
            near(st[0].cpu().numpy()[:3700], new[0][:3700], tol[0][:3700], max_norm)
        else:
            assert all(torch.equal(a, b) for a, b in zip(old, st)), max_norm


@pytest.mark.parametrize("coded", [False, True])
def test_large_eps(coded):
    """An eps whose reciprocal is a normal number keeps its part of the update; one beyond is refused."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([700, 3000], 0, 0)
    rng = np.random.default_rng(24)
    g = (rng.standard_normal(n) * 1e18).astype(np.float32)
    p = np.zeros(n, np.float32)
    plan = B.Optim(table(B, offs, numels))
    for eps in (1e10, 1e30, 2.0 ** 126, 2.0 ** 126 * (1 + 2.0 ** -23), 2e38, 3.4e38):
        st, step = [torch.from_numpy(p).cuda()] + fresh(torch, plan, n, coded), torch.zeros(1, dtype=torch.int64, device="cuda")
        s = B.adamw(lr=1.0, beta1=B1, beta2=B2, eps=eps, weight_decay=0.0)
        if eps > 2.0 ** 126:
            with pytest.raises(B.LgrecoError) as e:
                step_of(plan, coded)(s, torch.from_numpy(g).cuda(), *st, step)
            assert e.value.status == B.EINVAL
            continue
        step_of(plan, coded)(s, torch.from_numpy(g).cuda(), *st, step)
        new, tol = bounds(g, p, np.zeros(n), np.zeros(n), 1, 1.0, 0.0, 1.0, B1, B2, eps)
        near(st[0].cpu().numpy()[:3700], new[0][:3700], tol[0][:3700], eps)


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_moments_are_rounded_operation_by_operation(kind, coded):
    """m' and v' bit for bit those of fp32 arithmetic that rounds the factors, every product and every sum, over three steps; with 8 bits
    the codes and exponents of exactly those numbers.  The inputs tell a fused product and sum apart."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES["parts"])
    rng = np.random.default_rng(25)
    inside = np.zeros(n, bool)
    for o, k in zip(offs, numels):
        inside[o:o + k] = True
    plan = B.Optim(table(B, offs, numels))
    f32 = np.float32
    b1, r1, b2, r2, c = (f32(x) for x in (B1, 1.0 - B1, B2, 1.0 - B2, 1 / 3))
    s = B.adamw(lr=1e-3, beta1=B1, beta2=B2, eps=EPS, grad_scale=1 / 3)
    st, dp, step = fresh(torch, plan, n, coded), torch.zeros(n, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for t in (1, 2, 3):
        dg = typed(torch, (rng.standard_normal(n) * 10.0 ** rng.uniform(-4, 0, n)).astype(f32), kind)
        old = [a.astype(f32) for a in held(st, offs, numels, coded)]
        step_of(plan, coded)(s, dg, dp, *st, step)
        g = c * exact_grads(torch, dg.float().cpu().numpy(), "f32").astype(f32)
        want = [b1 * old[0] + r1 * g, b2 * old[1] + r2 * (g * g)]
        if t > 1:
            wide = (b1 * old[0].astype(np.float64) + (r1 * g)).astype(f32)          # the first product not rounded
            assert ((wide != want[0]) & inside).any()
            wide = (b2 * old[1].astype(np.float64) + r2 * (g * g)).astype(f32)
            assert ((wide != want[1]) & inside).any()
        got = held(st, offs, numels, coded)
        if not coded:
            for a, w, what in zip(got, want, "mv"):
                assert np.array_equal(a[inside], w[inside]), (what, t)
            continue
        exps, first = st[2].cpu().numpy().reshape(-1, 2), 0
        for o, k in zip(offs, numels):
            for j in range(0, k, 128):
                cut, x = slice(o + j, o + min(j + 128, k)), exps[first]
                first += 1
                for q, octaves in ((0, O.OCTAVES_M), (1, O.OCTAVES_V)):
                    a = np.abs(want[q][cut])
                    assert O.exponent(a) == x[q]
                    keep = O.rounded(a, int(x[q]), octaves)
                    if q:
                        keep = np.where(a > 0, np.maximum(keep, 2.0 ** (int(x[q]) - 127.0 - 14 - 4)), keep)
                    assert np.array_equal(np.abs(got[q][cut]), keep), (q, t, o, j)
                    assert (np.sign(got[q][cut]) * np.sign(want[q][cut]) >= 0).all()
