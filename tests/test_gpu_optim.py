"""GPU: norms, AdamW with fp32 moments and with moments in 8 bits against the step in 64 bits.

Errors are counted in u = 2^-24, half a step of fp32.  With g = c * grad rounded twice (c, the product): 2 u of it.
  m' = b1 * m + r1 * g: b1 and r1, both products and the sum are rounded, so 2 u of b1 m and 4 u of r1 g, and u of the sum:
  at most 6 u (|b1 m| + |r1 g|)
  v' = b2 * v + r2 * (g * g): 2 u of b2 v, 4 + 1 + 1 + 1 u of r2 g^2, and u of the sum: at most 9 u v'
  update m' / (sqrt(v') * root + eps): half of v's 9 u, the root's u, the factor's and the sum's rounding and eps's: 9 u of
  the denominator, u of the quotient, 2 u of the rate and its product
  p' = p - (shrink * p + rate * update): 2 u of the first term, 1 u more of the second, u of p'
(second-order terms: within the factors' slack)."""
import itertools

import numpy as np
import pytest

from oracle import optim as O

from gpu_util import torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8
TYPES = ("none", "bf16", "f16")


def layout(numels, gap, first):
    offs, at = [], first
    for n in numels:
        offs.append(at)
        at += n + gap
    return np.array(offs, np.int64), np.array(numels, np.int64), at + 3


TABLES = {
    "one": ([1], 0, 0),
    "short": ([1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 31, 33, 63, 65], 1, 3),
    "blocks": ([127, 128, 129, 255, 256, 257, 1, 1023, 1025], 0, 1),
    "parts": ([2047, 2048, 2049, 4096, 4099, 2016 + 128], 5, 2),
    "norm_parts": ([16384, 16383, 16385, 40000, 3], 0, 7),
    "aligned": ([4096, 32, 20480, 64], 0, 0),
    "large": ([300007, 1, 131072], 2, 31),
}


def table(B, offs, numels):
    z = np.zeros(len(numels), np.int32)
    return B.layer_table(offs, numels, z, z)


def typed(torch, a, kind):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if kind == "f32" else t.to({"bf16": torch.bfloat16, "f16": torch.float16}[kind])


def exact_grads(torch, a, kind):
    """What the gradient buffer holds, in fp64."""
    return typed(torch, a, kind).double().cpu().numpy()


def values(rng, n, offs, numels):
    """Gradients at layer scales from 1e-6 to 1, zeros and outliers among them; parameters; moments of a running job."""
    g = rng.standard_normal(n).astype(np.float32)
    scale = np.ones(n, np.float32)
    for o, k in zip(offs, numels):
        scale[o:o + k] = 10.0 ** rng.uniform(-6, 0)
    g *= scale
    g[rng.random(n) < 0.02] = 0
    g[rng.random(n) < 0.01] *= 100
    p = (rng.standard_normal(n) * 0.05).astype(np.float32)
    m = (rng.standard_normal(n) * 0.3).astype(np.float32) * scale
    v = ((rng.standard_normal(n) ** 2 + 0.01) * scale.astype(np.float64) ** 2).astype(np.float32)
    return g, p, m, v


def bounds(g, p, m, v, t, lr, decay, scale, beta1=B1, beta2=B2, eps=EPS):
    """(p', m', v') in fp64 and what the fp32 step may be off them."""
    new = O.step(g, p, m, v, t, lr, beta1, beta2, eps, decay, scale)
    p, m = np.asarray(p, np.float64), np.asarray(m, np.float64)
    gs = np.abs(np.asarray(g, np.float64) * scale)
    terms = np.abs(beta1 * m) + (1 - beta1) * gs
    den = np.sqrt(new[2] / (1 - beta2 ** t)) + eps
    rate = lr / (1 - beta1 ** t)
    tiny = 2.0 ** -148                                  # products below the smallest normal number
    em = 6 * U * terms + tiny
    ev = 9 * U * new[2] + tiny
    ep = U * np.abs(new[0]) + 3 * U * lr * decay * np.abs(p) + rate * (em + 14 * U * np.abs(new[1])) / den
    # (v near the smallest numbers: what the absolute part of its error does to the denominator)
    ep = ep + rate * np.abs(new[1]) / den ** 2 * np.sqrt(tiny)
    return new, (ep * 1.001, em * 1.001, ev * 1.001)


def near(got, want, tol, what):
    d = np.abs(np.asarray(got, np.float64) - want)
    k = int(np.argmax(d - tol))
    assert (d <= tol).all(), (what, k, got[k], want[k], tol[k])


def rounded16(x, kind):
    import torch
    return torch.from_numpy(x).to({"bf16": torch.bfloat16, "f16": torch.float16}[kind])


# ------------------------------------------------------------------------------ norms
@pytest.mark.parametrize("name", sorted(TABLES))
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_norms(name, kind):
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES[name])
    g, _, _, _ = values(np.random.default_rng(1), n, offs, numels)
    d = typed(torch, g, kind)
    x = d.double().cpu().numpy().astype(np.longdouble)
    plan = B.Optim(table(B, offs, numels))
    assert plan.blocks == int(((numels + 127) // 128).sum())
    out = torch.full((len(numels) + 2,), -3.0, dtype=torch.float64, device="cuda")
    plan.norms(d, out)
    got = out.cpu().numpy()
    want = np.array([float((x[o:o + k] ** 2).sum()) for o, k in zip(offs, numels)])
    # squares are exact in fp64, and at most 17 + 2 + 6 + 2 sums in a row of a part, 1 + 8 of its layer's parts here
    assert np.all(np.abs(got[:-2] - want) <= 64 * 2.0 ** -53 * want)
    assert abs(got[-2] - want.sum()) <= 80 * 2.0 ** -53 * want.sum()
    assert got[-1] == -3.0
    again = torch.zeros_like(out)
    plan.norms(d, again)
    assert torch.equal(out[:-1], again[:-1])


def test_norms_of_extreme_values():
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    numels = np.array([300, 5, 1000, 2, 4])
    offs = np.array([0, 301, 400, 1500, 1503])
    plan = B.Optim(table(B, offs, numels))
    out = torch.zeros(6, dtype=torch.float64, device="cuda")
    g = np.zeros(1600, np.float32)
    g[0:300] = 3e38                                     # squares beyond fp32
    g[301:306] = 1e-42                                  # denormal numbers
    g[1500] = -0.0
    plan.norms(torch.from_numpy(g).cuda(), out)
    got = out.cpu().numpy()
    big, small = float(np.float32(3e38)) ** 2, float(np.float32(1e-42)) ** 2
    assert abs(got[0] - 300 * big) <= 1e-13 * got[0] and abs(got[1] - 5 * small) <= 1e-13 * got[1]
    assert (got[2:5] == 0).all() and abs(got[5] - 300 * big) <= 1e-13 * got[5]
    for bad in (np.nan, np.inf, -np.inf):
        h = g.copy()
        h[1399] = bad                                   # the last element of layer 2
        plan.norms(torch.from_numpy(h).cuda(), out)
        got = out.cpu().numpy()
        assert np.isfinite(got[[0, 1, 3, 4]]).all() and not np.isfinite(got[[2, 5]]).any()
        h[1399], h[1400], h[300], h[1502] = 0, bad, bad, bad   # in gaps only
        plan.norms(torch.from_numpy(h).cuda(), out)
        assert np.isfinite(out.cpu().numpy()).all()


# ------------------------------------------------------------------------------ fp32 moments
@pytest.mark.parametrize("name", sorted(TABLES))
@pytest.mark.parametrize("kind,copy", list(itertools.product(("f32", "bf16", "f16"), TYPES)))
def test_adamw(name, kind, copy):
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES[name])
    rng = np.random.default_rng(2)
    g, p, m, v = values(rng, n, offs, numels)
    lrs, ds = rng.uniform(0, 2, len(numels)).astype(np.float32), rng.integers(0, 2, len(numels)).astype(np.float32)
    plan = B.Optim(table(B, offs, numels), lrs, ds)
    dg, dp, dm, dv = typed(torch, g, kind), *(torch.from_numpy(a).cuda() for a in (p, m, v))
    dc = None if copy == "none" else torch.full((n,), 7.0, device="cuda").to(torch.bfloat16 if copy == "bf16" else torch.float16)
    step = torch.tensor([41], device="cuda")
    s = B.adamw(lr=2e-3, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.1, grad_scale=0.125)
    plan.adamw(s, dg, dp, dm, dv, step, d_copy=dc)
    assert int(step) == 42
    gp, gm, gv = (a.cpu().numpy() for a in (dp, dm, dv))
    gx = exact_grads(torch, g, kind)
    inside = np.zeros(n, bool)
    for l, (o, k) in enumerate(zip(offs, numels)):
        c = slice(o, o + k)
        inside[c] = True
        new, tol = bounds(gx[c], p[c], m[c], v[c], 42, 2e-3 * float(lrs[l]), 0.1 * float(ds[l]), 0.125)
        for got, want, t, what in zip((gp, gm, gv), new, tol, "pmv"):
            near(got[c], want, t, (what, l))
    for got, old in ((gp, p), (gm, m), (gv, v)):
        assert np.array_equal(got[~inside], old[~inside])
    if dc is not None:
        want = rounded16(gp, copy)
        want[torch.from_numpy(~inside)] = 7.0
        assert torch.equal(dc.cpu(), want)


@pytest.mark.parametrize("t0", [0, 1, 9, 1000, 10 ** 6, 2 ** 32 + 5])
def test_adamw_counts_steps_and_follows_the_rate(t0):
    """Bias corrections from the first step on; a device factor of the rate; three steps in a row."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([1000, 77], 0, 0)
    rng = np.random.default_rng(t0 % 1000)
    _, p, m, v = values(rng, n, offs, numels)
    if t0 == 0:
        m[:], v[:] = 0, 0
    plan = B.Optim(table(B, offs, numels))
    dp, dm, dv = (torch.from_numpy(a).cuda() for a in (p, m, v))
    step, rate = torch.tensor([t0], device="cuda"), torch.tensor([0.5], device="cuda")
    s = B.adamw(lr=1e-2, weight_decay=0.01, beta1=B1, beta2=B2, eps=EPS)
    for k in range(3):
        g, _, _, _ = values(rng, n, offs, numels)
        rate.fill_(0.5 ** k)
        plan.adamw(s, torch.from_numpy(g).cuda(), dp, dm, dv, step, d_lr=rate)
        new, tol = bounds(g, p, m, v, t0 + k + 1, 1e-2 * 0.5 ** k, 0.01, 1.0)
        got = [a.cpu().numpy() for a in (dp, dm, dv)]
        for a, want, e, what in zip(got, new, tol, "pmv"):
            near(a[:1077], want[:1077], e[:1077], (what, k))
        p, m, v = got
    assert int(step) == t0 + 3


@pytest.mark.parametrize("beta1,beta2,eps", [(0.0, 0.0, 1e-8), (0.0, 0.95, 1e-6), (0.95, 0.0, 1.0), (0.999999, 0.9999999, 1e-12)])
def test_adamw_settings(beta1, beta2, eps):
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([515], 0, 0)
    g, p, m, v = values(np.random.default_rng(3), n, offs, numels)
    plan = B.Optim(table(B, offs, numels))
    d = [torch.from_numpy(a).cuda() for a in (g, p, m, v)]
    step = torch.tensor([4], device="cuda")
    plan.adamw(B.adamw(lr=1e-3, beta1=beta1, beta2=beta2, eps=eps, weight_decay=0.0), *d, step)
    new, tol = bounds(g, p, m, v, 5, 1e-3, 0.0, 1.0, beta1, beta2, eps)
    for a, want, e, what in zip(d[1:], new, tol, "pmv"):
        near(a.cpu().numpy()[:515], want[:515], e[:515], what)


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("max_norm", [1e-3, 1.0, 1e9])
def test_clipping(max_norm, coded):
    """Below the norm, above it, and far above: the step with gradients scaled by hand."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES["parts"])
    g, p, m, v = values(np.random.default_rng(5), n, offs, numels)
    plan = B.Optim(table(B, offs, numels))
    total = torch.zeros(len(numels) + 1, dtype=torch.float64, device="cuda")
    dg = torch.from_numpy(g).cuda()
    plan.norms(dg, total)
    c = O.clip(float(total[-1]), 0.5, max_norm)
    assert (c < 0.5) == (max_norm < 1e9)
    results = []
    for settings, sums in ((B.adamw(lr=1e-3, grad_scale=0.5, max_norm=max_norm), total), (B.adamw(lr=1e-3, grad_scale=c), None)):
        dp, step = torch.from_numpy(p).cuda(), torch.zeros(1, dtype=torch.int64, device="cuda")
        if coded:
            st = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
            st.append(torch.zeros(2 * plan.blocks, dtype=torch.uint8, device="cuda"))
            plan.adamw_coded(settings, dg, dp, *st, step, d_sumsq=sums)
        else:
            st = [torch.from_numpy(a).cuda() for a in (m, v)]
            plan.adamw(settings, dg, dp, *st, step, d_sumsq=sums)
        results.append([dp] + st)
    for a, b in zip(*results):
        assert torch.equal(a, b)                        # the same fp32 factor, up to one rounding of c in fp64


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_steps_with_bad_gradients_are_left_out(bad, coded):
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([700, 3000], 0, 0)
    rng = np.random.default_rng(6)
    g, p, m, v = values(rng, n, offs, numels)
    g[3000] = bad
    plan = B.Optim(table(B, offs, numels))
    dg, sums = torch.from_numpy(g).cuda(), torch.zeros(3, dtype=torch.float64, device="cuda")
    plan.norms(dg, sums)
    step = torch.tensor([7], device="cuda")
    copy = torch.full((n,), 2.0, dtype=torch.bfloat16, device="cuda")
    if coded:
        state = [torch.from_numpy(rng.integers(0, 256, n).astype(np.uint8)).cuda() for _ in range(2)]
        state.append(torch.from_numpy(rng.integers(90, 130, 2 * plan.blocks).astype(np.uint8)).cuda())
    else:
        state = [torch.from_numpy(a).cuda() for a in (m, v)]
    state = [torch.from_numpy(p).cuda()] + state
    old = [a.clone() for a in state + [copy]]
    f = plan.adamw_coded if coded else plan.adamw
    for max_norm in (0.0, 1.0):
        f(B.adamw(lr=1e-3, max_norm=max_norm), dg, *state, step, d_copy=copy, d_sumsq=sums)
        assert int(step) == 7
        for a, b in zip(old, state + [copy]):
            assert torch.equal(a, b)
    # without the sums nothing is left out, and what other blocks hold is right all the same
    f(B.adamw(lr=1e-3, weight_decay=0.0), dg, *state, step)
    assert int(step) == 8
    got = state[0].cpu().numpy()
    far = np.ones(n, bool)
    far[n - 3:] = False
    far[3000] = False
    assert np.isfinite(got[far]).all()
    if not coded:
        g[3000] = 0
        new, tol = bounds(g, p, m, v, 8, 1e-3, 0.0, 1.0)
        near(got[far], new[0][far], tol[0][far], "p")


# ------------------------------------------------------------------------------ 8-bit moments
def stored(codes, exps, octaves, signed):
    """Values of a layer's codes; one exponent a block."""
    x = np.repeat(exps.astype(np.int64), 128)[:codes.size]
    a = O.decode(codes & 127 if signed else codes, x, octaves)
    return np.where(codes > 127, -a, a) if signed else a


def check_coded(new, tol, codes_m, codes_v, exps, u):
    """Every code of a layer against what its 64-bit moment, give or take the fp32 step's error, rounds to."""
    for k, (octaves, codes, signed) in enumerate(((O.OCTAVES_M, codes_m, True), (O.OCTAVES_V, codes_v, False))):
        a, e = np.abs(new[1 + k]), tol[1 + k]
        got = stored(codes, exps[:, k], octaves, signed)
        for b in range(exps.shape[0]):
            c = slice(128 * b, min(128 * (b + 1), a.size))
            j = int(np.argmax(a[c]))
            top, off = a[c][j], e[c].max()
            x = int(exps[b, k])
            assert O.exponent(max(top - off, 0)) <= x <= O.exponent(top + off), (k, b, top, x)
            w = None if u is None else u[k][c]
            low, high = (O.rounded(np.maximum(z, 0), x, octaves, w) for z in (a[c] - e[c], a[c] + e[c]))
            if not signed:
                least = 2.0 ** (x - 127.0 - 14 - 4)
                low, high = np.where(a[c] > e[c], np.maximum(low, least), low), np.where(a[c] > 0, np.maximum(high, least), high)
            val = np.abs(got[c])
            assert ((low <= val) & (val <= high)).all(), (k, b, np.argmax((val < low) | (val > high)))
            sure = a[c] > e[c]
            assert (np.sign(got[c]) * np.sign(new[1 + k][c]) >= 0)[sure].all()


@pytest.mark.parametrize("name", sorted(TABLES))
@pytest.mark.parametrize("kind,copy,stochastic", [("f32", "none", False), ("f32", "none", True), ("bf16", "bf16", True),
                                                  ("bf16", "f16", False), ("f32", "f16", True), ("f32", "bf16", False),
                                                  ("bf16", "none", True), ("bf16", "none", False), ("f32", "bf16", True),
                                                  ("bf16", "f16", True), ("bf16", "bf16", False), ("f32", "f16", False),
                                                  ("f16", "none", True), ("f16", "f16", False), ("f16", "bf16", True),
                                                  ("f16", "none", False), ("f16", "f16", True), ("f16", "bf16", False)])
def test_adamw_coded(name, kind, copy, stochastic):
    """Three steps from zero moments: parameters, codes and exponents of each against the step in 64 bits from what the
    one before left."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES[name])
    rng = np.random.default_rng(8)
    _, p, _, _ = values(rng, n, offs, numels)
    lrs, ds = rng.uniform(0, 2, len(numels)).astype(np.float32), rng.integers(0, 2, len(numels)).astype(np.float32)
    plan = B.Optim(table(B, offs, numels), lrs, ds)
    seed = 0x123456789ABCDEF0
    s = B.adamw(lr=2e-3, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.1, grad_scale=1 / 3, stochastic=stochastic, seed=seed)
    dp, step = torch.from_numpy(p).cuda(), torch.tensor([2 ** 32 - 2], device="cuda")
    cm, cv = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    exps = np.zeros((plan.blocks, 2), np.uint8)
    inside = np.zeros(n, bool)
    for o, k in zip(offs, numels):
        inside[o:o + k] = True
    cm[~inside], cv[~inside] = 77, 78
    dm, dv, dx = (torch.from_numpy(a.reshape(-1).copy()).cuda() for a in (cm, cv, exps))
    dc = None if copy == "none" else torch.full((n,), 7.0, device="cuda").to(torch.bfloat16 if copy == "bf16" else torch.float16)
    for k in range(3):
        t = 2 ** 32 - 1 + k
        g, _, _, _ = values(rng, n, offs, numels)
        plan.adamw_coded(s, typed(torch, g, kind), dp, dm, dv, dx, step, d_copy=dc)
        gx = exact_grads(torch, g, kind)
        gp, gm, gv, gexp = (a.cpu().numpy() for a in (dp, dm, dv, dx))
        gexp = gexp.reshape(-1, 2)
        first = 0
        for l, (o, q) in enumerate(zip(offs, numels)):
            c, b = slice(o, o + q), slice(first, first + (q + 127) // 128)
            m_old = stored(cm[c], exps[b, 0], O.OCTAVES_M, True)
            v_old = stored(cv[c], exps[b, 1], O.OCTAVES_V, False)
            new, tol = bounds(gx[c], p[c], m_old, v_old, t, 2e-3 * float(lrs[l]), 0.1 * float(ds[l]), 1 / 3)
            near(gp[c], new[0], tol[0], ("p", k, l))
            check_coded(new, tol, gm[c], gv[c], gexp[b], O.halves(seed, t, l, q) if stochastic else None)
            first = b.stop
        assert (gm[~inside] == 77).all() and (gv[~inside] == 78).all() and np.array_equal(gp[~inside], p[~inside])
        p, cm, cv, exps = gp, gm, gv, gexp
        if dc is not None:
            want = rounded16(gp, copy)
            want[torch.from_numpy(~inside)] = 7.0
            assert torch.equal(dc.cpu(), want)
    assert int(step) == 2 ** 32 + 1


@pytest.mark.parametrize("stochastic", [False, True])
def test_coded_blocks_at_their_borders(stochastic):
    """Blocks of zeros, of one element that is not, at octave borders and where rounding carries, 40 octaves wide, of the
    smallest and the largest numbers; beta1 = 0 makes m the gradient itself."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    rng = np.random.default_rng(9)
    blocks = [np.zeros(128), np.r_[np.zeros(127), -3e-5], np.r_[1.0, np.full(127, 2.0 ** -12)],
              np.r_[31 / 16, 31.5 / 16 * 2.0 ** -np.arange(127.0) / 4], np.r_[np.nextafter(np.float32(31 / 16), np.float32(2)), np.ones(127)],
              np.nextafter(np.float32(2), np.float32(1)) * 2.0 ** -np.arange(128.0) / 2, 2.0 ** -rng.uniform(0, 40, 128),
              1e-38 * rng.random(128), 1e-44 * rng.integers(0, 5, 128), 1e18 * rng.standard_normal(128),
              rng.standard_normal(60) * 1e-3]
    g = np.concatenate(blocks).astype(np.float32)
    n = g.size
    plan = B.Optim(table(B, [0], [n]))
    s = B.adamw(lr=1e-3, beta1=0.0, beta2=0.5, eps=1e-6, weight_decay=0.0, stochastic=stochastic, seed=5)
    p = rng.standard_normal(n).astype(np.float32)
    d = [torch.from_numpy(g).cuda(), torch.from_numpy(p).cuda()]
    d += [torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, 2 * plan.blocks)]
    plan.adamw_coded(s, *d, torch.zeros(1, dtype=torch.int64, device="cuda"))
    z = np.zeros(n)
    new, tol = bounds(g, p, z, z, 1, 1e-3, 0.0, 1.0, 0.0, 0.5, 1e-6)
    near(d[1].cpu().numpy(), new[0], tol[0], "p")
    gm, gv, gx = (a.cpu().numpy() for a in d[2:])
    check_coded(new, tol, gm, gv, gx.reshape(-1, 2), O.halves(5, 1, 0, n) if stochastic else None)
    assert (gm[:128] == 0).all() and (gv[:128] == 0).all() and (gx[:2] == 0).all()
    assert (gv[(np.abs(g) > 1e-15)] > 0).all()


@pytest.mark.parametrize("stochastic", [False, True])
def test_codes_of_moments_known_exactly(stochastic):
    """With both betas 0, m' is the gradient and v' its square in fp32: every code and exponent has to be the definition's.  Ties
    and the numbers beside them, in every octave and below the lowest one, and magnitudes of every size."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    rng = np.random.default_rng(15)
    ties = np.concatenate([(np.arange(16) + 0.5) * 2.0 ** -10] + [(np.arange(16, 32) + 0.5) * 2.0 ** (e - 4) for e in range(-6, 0)])
    beside = [ties, np.nextafter(ties.astype(np.float32), np.float32(0)), np.nextafter(ties.astype(np.float32), np.float32(1)),
              ties * (1 + 2.0 ** -14), ties * (1 - 2.0 ** -14)]
    blocks = [np.r_[1.0, b, np.zeros(127 - b.size)] for b in beside]
    blocks += [2.0 ** rng.uniform(-24, 0, 128) * rng.choice([-1, 1], 128) for _ in range(400)]
    roots = rng.integers(1, 2048, (100, 128)) * 2.0 ** -rng.integers(11, 21, (100, 128))      # squares of 11 bits: exact, ties among them
    g = np.concatenate([np.concatenate(blocks), roots.reshape(-1)]).astype(np.float32)
    n = g.size
    plan = B.Optim(table(B, [0], [n]))
    d = [torch.from_numpy(g).cuda(), torch.zeros(n, device="cuda")]
    d += [torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, 2 * plan.blocks)]
    s = B.adamw(lr=1e-3, beta1=0.0, beta2=0.0, stochastic=stochastic, seed=6)
    plan.adamw_coded(s, *d, torch.zeros(1, dtype=torch.int64, device="cuda"))
    gm, gv, gx = (a.cpu().numpy() for a in d[2:])
    u = O.halves(6, 1, 0, n) if stochastic else (None, None)
    for k, (a, codes, octaves, signed) in enumerate(((g, gm, O.OCTAVES_M, True), (g * g, gv, O.OCTAVES_V, False))):
        got = stored(codes, gx.reshape(-1, 2)[:, k], octaves, signed)
        for b in range(plan.blocks):
            c = slice(128 * b, 128 * (b + 1))
            x = O.exponent(np.abs(a[c]))
            assert x == gx[2 * b + k]
            want = O.rounded(np.abs(a[c]), x, octaves, u[k] if u[k] is None else u[k][c])
            if not signed:
                want = np.where(a[c] > 0, np.maximum(want, 2.0 ** (x - 127.0 - 14 - 4)), want)
            assert np.array_equal(got[c], np.copysign(want, a[c]) if signed else want), (k, b)


def test_stochastic_rounding_keeps_the_expectation():
    """v that falls by a thousandth a step: rounded to the nearest it stays, stochastically it falls as in 64 bits.
    65536 elements; a step's rounding has a variance of at most (v / 16)^2 / 4, so 400 of them and a mean over the
    elements are within 6 * sqrt(400) / (2 * 16 * 256) = 1.5 % of the start's v."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    n = 65536
    plan = B.Optim(table(B, [0], [n]))
    g = torch.zeros(n, device="cuda")
    result = {}
    for stochastic in (False, True):
        st = [torch.zeros(k, dtype=torch.uint8, device="cuda") for k in (n, n, 2 * plan.blocks)]
        p, step = torch.zeros(n, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        plan.adamw_coded(B.adamw(lr=0.0, beta2=0.0, stochastic=stochastic), g + 1.0, p, *st, step)
        s = B.adamw(lr=0.0, beta2=0.999, stochastic=stochastic, seed=77)
        for _ in range(400):
            plan.adamw_coded(s, g, p, *st, step)
        out = [torch.zeros(n, device="cuda") for _ in range(2)]
        plan.decode(*st, *out)
        result[stochastic] = float(out[1].double().mean())
    assert result[False] == 1.0
    assert abs(result[True] - 0.999 ** 400) < 0.015


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["one", "short", "blocks", "parts", "large"])
def test_decode(name, kind):
    """Every code and exponent byte, at layers that start anywhere."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout(*TABLES[name])
    rng = np.random.default_rng(10)
    plan = B.Optim(table(B, offs, numels))
    cm, cv = (rng.integers(0, 256, n).astype(np.uint8) for _ in range(2))
    exps = rng.integers(0, 256, (plan.blocks, 2)).astype(np.uint8)
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    out = [torch.full((n,), 5.0, dtype=dt, device="cuda") for _ in range(2)]
    plan.decode(*(torch.from_numpy(a.reshape(-1)).cuda() for a in (cm, cv, exps)), *out)
    got = [a.double().cpu().numpy() for a in out]
    first, inside = 0, np.zeros(n, bool)
    for o, k in zip(offs, numels):
        c, b = slice(o, o + k), slice(first, first + (k + 127) // 128)
        first, inside[c] = b.stop, True
        for a, codes, x, octaves, signed in ((got[0], cm, 0, O.OCTAVES_M, True), (got[1], cv, 1, O.OCTAVES_V, False)):
            want = stored(codes[c], exps[b, x], octaves, signed)
            want = torch.from_numpy(want).float()                # 5 bits of mantissa; beyond fp32 infinite, below it rounded
            want = want.to(dt).double().numpy()
            assert np.array_equal(a[c], want), (name, o)
    assert all((a[~inside] == 5.0).all() for a in got)


# ------------------------------------------------------------------------------ long tables
@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("largest", [40_000_003, 140_000_003])
def test_a_long_table_is_its_layers_one_by_one(coded, largest):
    """Tables whose workgroups work out their own factors and tables beyond 65536 workgroups, which leave that to a kernel in
    front; layers of more than 64 parts: bit for bit what plans of one layer each give."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    numels = np.array([largest, 77, 2_500_001, 1])
    offs = np.cumsum(numels + 1) - numels
    n = int(offs[-1] + numels[-1]) + 2
    gen = torch.Generator(device="cuda").manual_seed(16)
    g = torch.randn(n, generator=gen, device="cuda") * 1e-3
    p = torch.randn(n, generator=gen, device="cuda")
    plan = B.Optim(table(B, offs, numels), [1.0, 0.5, 2.0, 1.0], [1.0, 0.0, 1.0, 0.5])
    s = B.adamw(lr=1e-3, max_norm=1.0, grad_scale=0.3, weight_decay=0.1)
    sums = torch.zeros(5, dtype=torch.float64, device="cuda")
    plan.norms(g, sums)
    want = [float((g[o:o + k].double() ** 2).sum()) for o, k in zip(offs.tolist(), numels.tolist())]
    got = sums.cpu().numpy()
    assert np.allclose(got[:4], want, rtol=1e-12, atol=0) and np.isclose(got[4], sum(want), rtol=1e-12, atol=0)
    kind = torch.uint8 if coded else torch.float32

    def fresh(blocks):
        st = [p.clone(), torch.zeros(n, dtype=kind, device="cuda"), torch.zeros(n, dtype=kind, device="cuda")]
        return st + ([torch.zeros(2 * blocks, dtype=torch.uint8, device="cuda")] if coded else [])

    whole, step = fresh(plan.blocks), torch.zeros(1, dtype=torch.int64, device="cuda")
    f = plan.adamw_coded if coded else plan.adamw
    for _ in range(2):
        f(s, g, *whole, step, d_sumsq=sums)
    assert int(step) == 2
    first = 0
    for l, (o, k) in enumerate(zip(offs.tolist(), numels.tolist())):
        one = B.Optim(table(B, [o], [k]), [[1.0, 0.5, 2.0, 1.0][l]], [[1.0, 0.0, 1.0, 0.5][l]])
        st, step = fresh(one.blocks), torch.zeros(1, dtype=torch.int64, device="cuda")
        f = one.adamw_coded if coded else one.adamw
        for _ in range(2):
            f(s, g, *st, step, d_sumsq=torch.stack((sums[l], sums[4])))
        for a, b in zip(whole[:3], st[:3]):
            assert torch.equal(a[o:o + k], b[o:o + k]), l
        if coded:
            assert torch.equal(whole[3][first:first + 2 * one.blocks], st[3])
            first += 2 * one.blocks
        assert int(step) == 2
    bad = g.clone()
    bad[-3] = float("inf")                              # the last layer's only element
    plan.norms(bad, sums)
    old = [a.clone() for a in whole]
    step = torch.tensor([5], device="cuda")
    f = plan.adamw_coded if coded else plan.adamw
    f(s, bad, *whole, step, d_sumsq=sums)
    assert int(step) == 5 and all(torch.equal(a, b) for a, b in zip(old, whole))


@pytest.mark.parametrize("layers", [64, 65, 4096, 4097, 20000])
def test_many_layers(layers):
    """Norms and a step of thousands of short layers, twice over one plan."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    rng = np.random.default_rng(layers)
    numels = rng.integers(1, 40, layers)
    numels[::997] = 20000
    offs = np.cumsum(numels) - numels
    n = int(numels.sum())
    g, p, m, v = values(rng, n, offs, numels)
    plan = B.Optim(table(B, offs, numels))
    d = [torch.from_numpy(a).cuda() for a in (g, p, m, v)]
    sums, step = torch.zeros(layers + 1, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    want = np.add.reduceat(g.astype(np.float64) ** 2, offs)
    for k in range(2):
        sums.fill_(-1.0)
        plan.norms(d[0], sums)
        got = sums.cpu().numpy()
        assert np.allclose(got[:-1], want, rtol=1e-12, atol=0) and np.isclose(got[-1], want.sum(), rtol=1e-12, atol=0)
        plan.adamw(B.adamw(lr=1e-3, weight_decay=0.0), *d, step, d_sumsq=sums)
        new, tol = bounds(g, p, m, v, k + 1, 1e-3, 0.0, 1.0)
        p, m, v = (a.cpu().numpy() for a in d[1:])
        for a, w, e, what in zip((p, m, v), new, tol, "pmv"):
            near(a, w, e, what)
    assert int(step) == 2


# ------------------------------------------------------------------------------ streams, graphs, far offsets, refusals
def test_far_offsets():
    """Layers beyond 2^32 elements into the buffers."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    far = 2 ** 32 + 5
    offs, numels = np.array([10, far]), np.array([300, 1003])
    n = far + 1003
    plan = B.Optim(table(B, offs, numels))
    rng = np.random.default_rng(11)
    g = rng.standard_normal(1303).astype(np.float32)
    p = rng.standard_normal(1303).astype(np.float32)
    where = (slice(10, 310), slice(far, far + 1003))
    part = (slice(0, 300), slice(300, 1303))

    def spread(a, dtype):
        d = torch.empty(n, dtype=dtype, device="cuda")
        for w, c in zip(where, part):
            d[w] = torch.from_numpy(a[c]).to(dtype).cuda()
        return d

    def small(a, dtype):
        return torch.from_numpy(a).to(dtype).cuda()

    near_plan = B.Optim(table(B, [0, 300], [300, 1003]))
    s = B.adamw(lr=1e-3, stochastic=True, seed=3)
    dg, zero = spread(g, torch.bfloat16), np.zeros(1303, np.float32)
    sums = torch.zeros(3, dtype=torch.float64, device="cuda")
    ref = torch.zeros_like(sums)
    plan.norms(dg, sums)
    near_plan.norms(small(g, torch.bfloat16), ref)
    assert torch.allclose(sums, ref, rtol=1e-14, atol=0)
    for coded in (True, False):
        dt = torch.uint8 if coded else torch.float32
        big = [spread(p, torch.float32), spread(zero, dt), spread(zero, dt)]
        few = [small(p, torch.float32), small(zero, dt), small(zero, dt)]
        for pl, grads, st in ((plan, dg, big), (near_plan, small(g, torch.bfloat16), few)):
            step = torch.zeros(1, dtype=torch.int64, device="cuda")
            if coded:
                pl.adamw_coded(s, grads, *st, torch.zeros(2 * pl.blocks, dtype=torch.uint8, device="cuda"), step)
            else:
                pl.adamw(s, grads, *st, step)
        for a, b in zip(big, few):
            for w, c in zip(where, part):
                assert torch.equal(a[w], b[c])
        del big


@pytest.mark.parametrize("coded", [False, True])
def test_captured_steps_replay_as_eager_ones(coded):
    """Norms, a clipped step and the moments' values in one graph, twice over the same plan: replays in turn with eager work
    and synchronisations between them, a schedule on the device, another gradient each time."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([5000, 129, 40000], 3, 1)
    plan = B.Optim(table(B, offs, numels))
    s = B.adamw(lr=1e-2, max_norm=0.5, grad_scale=0.5, stochastic=True, seed=1)
    rng = np.random.default_rng(12)
    p = rng.standard_normal(n).astype(np.float32)

    def state():
        dt = torch.uint8 if coded else torch.float32
        d = {"g": torch.zeros(n, device="cuda"), "p": torch.from_numpy(p).cuda(), "m": torch.zeros(n, dtype=dt, device="cuda"),
             "v": torch.zeros(n, dtype=dt, device="cuda"), "x": torch.zeros(2 * plan.blocks, dtype=torch.uint8, device="cuda"),
             "step": torch.zeros(1, dtype=torch.int64, device="cuda"), "lr": torch.ones(1, device="cuda"),
             "sums": torch.zeros(4, dtype=torch.float64, device="cuda"), "copy": torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
             "mo": torch.zeros(n, device="cuda"), "vo": torch.zeros(n, device="cuda")}
        return d

    def once(d):
        plan.norms(d["g"], d["sums"])
        if coded:
            plan.adamw_coded(s, d["g"], d["p"], d["m"], d["v"], d["x"], d["step"], d_copy=d["copy"], d_sumsq=d["sums"], d_lr=d["lr"])
            plan.decode(d["m"], d["v"], d["x"], d["mo"], d["vo"])
        else:
            plan.adamw(s, d["g"], d["p"], d["m"], d["v"], d["step"], d_copy=d["copy"], d_sumsq=d["sums"], d_lr=d["lr"])

    graphs, captured, eager = [], [state(), state()], [state(), state()]
    for d in captured:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            once(d)
        graphs.append(graph)
    for k in range(5):
        for w in range(2):
            g = torch.from_numpy((rng.standard_normal(n) * 10.0 ** (k - 2)).astype(np.float32)).cuda()
            if k == 3:
                g[700] = float("nan")
            for d in (captured[w], eager[w]):
                d["g"].copy_(g)
                d["lr"].fill_(1.0 / (k + 1))
            graphs[w].replay()
            once(eager[w])
            torch.cuda.synchronize()
            for key in ("p", "m", "v", "x", "step", "sums", "copy", "mo", "vo"):
                assert torch.equal(torch.nan_to_num(captured[w][key].double()), torch.nan_to_num(eager[w][key].double())), (k, w, key)
    assert int(eager[0]["step"]) == 4


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("max_norm", [0.7, 0.2])
def test_receive_is_the_sum_of_the_workers_and_a_step(coded, max_norm):
    """Three workers' payloads (quantization and Top-K), tensors that travel as they are, two steps; the driver against
    the images added up by hand and the step in 64 bits."""
    from paper_2210_17357_amd import binding as B
    from paper_2210_17357_amd.driver import AdamW
    torch = torch_cuda()
    numels = np.array([4096, 64, 3001, 7, 2500])
    offs = np.cumsum(numels) - numels
    n, workers = int(numels.sum()), 3
    sent = [0, 2, 4]                                    # matrices; the others travel as they are
    layers, ctab = table(B, offs[sent], numels[sent]), B.cand_table([(B.QUANT, 4.0), (B.TOPK, 0.05)])
    choice = np.array([0, 1, 0], np.int32)
    offsets = B.payload_layout(layers, ctab, choice)
    h = B.Handle(n, len(sent), 2)
    rng = np.random.default_rng(14)
    p = rng.standard_normal(n).astype(np.float32)
    decay = np.array([1, 0, 1, 0, 1], np.float32)
    s = B.adamw(lr=1e-2, beta1=B1, beta2=B2, eps=EPS, weight_decay=0.1, grad_scale=1 / workers, max_norm=max_norm)
    run = AdamW(table(B, offs, numels), torch.from_numpy(p).cuda(), s, decay_scale=decay, coded=coded,
                d_copy=torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
    efs = [torch.zeros(n, device="cuda") for _ in range(workers)]
    raw = np.ones(n, bool)
    for l in sent:
        raw[offs[l]:offs[l] + numels[l]] = False
    for t in (1, 2):
        payloads, summed = [], torch.zeros(n, device="cuda")
        for w in range(workers):
            g = torch.from_numpy((rng.standard_normal(n) * 0.01).astype(np.float32)).cuda()
            payloads.append(torch.zeros(int(offsets[-1]) + 16, dtype=torch.uint8, device="cuda"))
            h.compress(g, efs[w], layers, ctab, choice, payloads[w], offsets)
            summed += torch.where(torch.from_numpy(raw).cuda(), g, 0.0)
        image = torch.zeros(n, device="cuda")
        want_sum = summed.clone()
        for w in range(workers):
            h.decompress(payloads[w], offsets, layers, ctab, choice, image)
            want_sum += image
            image.zero_()
        m_old, v_old = (a.cpu().numpy() for a in run.moments())
        p_old = run.d_params.cpu().numpy()
        run.receive(h, payloads, offsets, layers, ctab, choice, summed)
        assert torch.equal(summed, want_sum) and int(run.d_step) == t
        x = summed.double().cpu().numpy()
        c = O.clip(float((x ** 2).sum()), 1 / workers, max_norm)      # the mean's norm is about 0.57
        assert (c < 1 / workers) == (max_norm == 0.2)
        got = run.d_params.cpu().numpy()
        for l, (o, k) in enumerate(zip(offs, numels)):
            cut = slice(o, o + k)
            new, tol = bounds(x[cut], p_old[cut], m_old[cut], v_old[cut], t, 1e-2, 0.1 * float(decay[l]), c)
            near(got[cut], new[0], tol[0], ("p", t, l))
            if not coded:
                near(run.d_m.cpu().numpy()[cut], new[1], tol[1], ("m", t, l))
                near(run.d_v.cpu().numpy()[cut], new[2], tol[2], ("v", t, l))
        assert torch.equal(run.d_copy, run.d_params.to(torch.bfloat16))


def test_the_largest_layer():
    """One layer of 2^31 - 1 elements: pieces of it, the last one among them, against plans of those pieces."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    n = 2 ** 31 - 1
    gen = torch.Generator(device="cuda").manual_seed(18)
    g = torch.empty(n, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    p = torch.ones(n, device="cuda")
    plan = B.Optim(table(B, [0], [n]))
    sums = torch.zeros(2, dtype=torch.float64, device="cuda")
    plan.norms(g, sums)
    want = sum(float(part.double().square().sum()) for part in g.split(1 << 28))
    assert np.allclose(sums.cpu().numpy(), want, rtol=1e-12, atol=0)
    s = B.adamw(lr=1e-2, max_norm=1e5)
    pieces = [(0, 5000), (2 ** 30 - 128, 4096), (n - n % 128 - 1280, 1280 + n % 128)]
    for coded in (False, True):
        kind = torch.uint8 if coded else torch.float32
        st = [p.clone(), torch.zeros(n, dtype=kind, device="cuda"), torch.zeros(n, dtype=kind, device="cuda")]
        st += [torch.zeros(2 * plan.blocks, dtype=torch.uint8, device="cuda")] if coded else []
        step = torch.zeros(1, dtype=torch.int64, device="cuda")
        (plan.adamw_coded if coded else plan.adamw)(s, g, *st, step, d_sumsq=sums)
        assert int(step) == 1
        for o, k in pieces:
            few = B.Optim(table(B, [0], [k]))
            part = [p[o:o + k].clone(), torch.zeros(k, dtype=kind, device="cuda"), torch.zeros(k, dtype=kind, device="cuda")]
            part += [torch.zeros(2 * few.blocks, dtype=torch.uint8, device="cuda")] if coded else []
            (few.adamw_coded if coded else few.adamw)(s, g[o:o + k].clone(), *part, torch.zeros(1, dtype=torch.int64, device="cuda"), d_sumsq=sums)
            # (a piece that ends inside a block of the layer has a block of its own there: whole blocks are compared)
            whole = k if not coded or o + k == n else k // 128 * 128
            for a, b in zip(st[:3], part[:3]):
                assert torch.equal(a[o:o + whole], b[:whole]), (coded, o)
            if coded:
                blocks = (whole + 127) // 128
                assert torch.equal(st[3][2 * (o // 128):2 * (o // 128) + 2 * blocks], part[3][:2 * blocks]), o
        del st


@pytest.mark.parametrize("coded", [False, True])
def test_layers_in_any_order_and_two_plans_at_once(coded):
    """A table that lists the layers from the last to the first, and two plans stepping their halves of the buffers on two
    streams at once: the same parameters and moments as one plan in order."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([70000, 129, 33333, 1, 4096, 50001], 1, 2)
    g, p, _, _ = values(np.random.default_rng(19), n, offs, numels)
    dg, kind = torch.from_numpy(g).cuda(), torch.uint8 if coded else torch.float32
    s = B.adamw(lr=1e-2)
    results = []
    for cuts in ([[0, 1, 2, 3, 4, 5]], [[5, 4, 3, 2, 1, 0]], [[0, 2, 4], [5, 3, 1]]):
        d = [torch.from_numpy(p).cuda(), torch.zeros(n, dtype=kind, device="cuda"), torch.zeros(n, dtype=kind, device="cuda")]
        plans = [B.Optim(table(B, offs[c], numels[c])) for c in cuts]
        streams = [torch.cuda.Stream() for _ in cuts]
        exps = [torch.zeros(2 * q.blocks, dtype=torch.uint8, device="cuda") for q in plans]
        steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in cuts]
        sums = [torch.zeros(q.L + 1, dtype=torch.float64, device="cuda") for q in plans]
        torch.cuda.synchronize()
        for _ in range(20):
            for q, stream, x, k, z in zip(plans, streams, exps, steps, sums):
                q.norms(dg, z, stream=stream.cuda_stream)
                if coded:
                    q.adamw_coded(s, dg, *d, x, k, d_sumsq=z, stream=stream.cuda_stream)
                else:
                    q.adamw(s, dg, *d, k, d_sumsq=z, stream=stream.cuda_stream)
        torch.cuda.synchronize()
        assert all(int(k) == 20 for k in steps)
        by_layer = {l: float(z[j]) for c, z in zip(cuts, sums) for j, l in enumerate(c)}
        results.append(d + [torch.tensor([by_layer[l] for l in range(6)], dtype=torch.float64)])
    for other in results[1:]:
        for a, b in zip(results[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("coded", [False, True])
def test_captured_steps_of_a_long_table(coded):
    """The same for a table beyond 65536 workgroups, against eager steps of another plan."""
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    n = 140_000_001 if coded else 70_000_001
    layers = table(B, [0], [n])
    plans = [B.Optim(layers), B.Optim(layers)]
    s = B.adamw(lr=1e-2, max_norm=0.5, stochastic=True, seed=1)
    kind = torch.uint8 if coded else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(17)
    g = torch.zeros(n, device="cuda")
    state = [{"p": torch.ones(n, device="cuda"), "m": torch.zeros(n, dtype=kind, device="cuda"), "v": torch.zeros(n, dtype=kind, device="cuda"),
              "x": torch.zeros(2 * plans[0].blocks, dtype=torch.uint8, device="cuda"), "step": torch.zeros(1, dtype=torch.int64, device="cuda"),
              "sums": torch.zeros(2, dtype=torch.float64, device="cuda")} for _ in plans]

    def once(plan, d):
        plan.norms(g, d["sums"])
        if coded:
            plan.adamw_coded(s, g, d["p"], d["m"], d["v"], d["x"], d["step"], d_sumsq=d["sums"])
        else:
            plan.adamw(s, g, d["p"], d["m"], d["v"], d["step"], d_sumsq=d["sums"])

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(plans[0], state[0])
    for k in range(4):
        g.normal_(generator=gen)
        if k == 2:
            g[n - 1] = float("inf")
        graph.replay()
        once(plans[1], state[1])
        torch.cuda.synchronize()
        for key in ("p", "m", "v", "x", "step", "sums"):
            assert torch.equal(state[0][key], state[1][key]), (k, key)
    assert int(state[0]["step"]) == 3


def test_on_another_stream():
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    offs, numels, n = layout([100000, 33], 0, 1)
    plan = B.Optim(table(B, offs, numels))
    g, p, m, v = values(np.random.default_rng(13), n, offs, numels)
    s = B.adamw(lr=1e-3, max_norm=1.0)
    results = []
    for stream in (None, torch.cuda.Stream()):
        d = [torch.from_numpy(a).cuda() for a in (g, p, m, v)]
        step, sums = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.float64, device="cuda")
        torch.cuda.synchronize()
        handle = None if stream is None else stream.cuda_stream
        plan.norms(d[0], sums, stream=handle)
        plan.adamw(s, *d, step, d_sumsq=sums, stream=handle)
        torch.cuda.synchronize()
        results.append(d + [step, sums])
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_refusals():
    from paper_2210_17357_amd import binding as B
    torch = torch_cuda()
    plan = B.Optim(table(B, [0, 600], [500, 100]))
    f32 = lambda n=700: torch.zeros(n, device="cuda")  # noqa: E731
    u8 = lambda n=700: torch.zeros(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    sums, step = torch.zeros(3, dtype=torch.float64, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    good = B.adamw(lr=1e-3)
    for bad in (dict(lr=-1.0), dict(lr=np.nan), dict(lr=np.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=np.nan), dict(beta2=1.0),
                dict(beta2=np.nan), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=np.nan), dict(eps=np.inf),
                dict(weight_decay=-0.1), dict(weight_decay=np.inf), dict(grad_scale=0.0), dict(grad_scale=-1.0), dict(grad_scale=np.inf),
                dict(grad_scale=np.nan), dict(max_norm=-1.0), dict(max_norm=np.nan), dict(max_norm=1.0)):
        s = B.adamw(**{"lr": 1e-3, **bad})
        with pytest.raises(B.LgrecoError) as e:         # (max_norm without the sums, too)
            plan.adamw(s, f32(), f32(), f32(), f32(), step)
        assert e.value.status == B.EINVAL
        with pytest.raises(B.LgrecoError):
            plan.adamw_coded(s, f32(), f32(), u8(), u8(), u8(10), step)
    for field in ("stochastic", "reserved"):
        s = B.adamw(lr=1e-3)
        setattr(s, field, 2)
        with pytest.raises(B.LgrecoError):
            plan.adamw(s, f32(), f32(), f32(), f32(), step)
    half = torch.zeros(700, dtype=torch.float16, device="cuda")
    with pytest.raises(B.LgrecoError):                  # an fp32 copy
        plan.adamw(good, f32(), f32(), f32(), f32(), step, d_copy=f32())
    with pytest.raises(B.LgrecoError):                  # values in fp16
        plan.decode(u8(), u8(), u8(10), half, half.clone())
    short, host, strided = f32(699), torch.zeros(700), f32(1400)[::2]
    for t in (short, host, strided, f32().double(), torch.zeros(700, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            plan.norms(t, sums)
        for place in range(4):
            d = [f32() for _ in range(4)]
            d[place] = t
            with pytest.raises(ValueError):
                plan.adamw(good, *d, step)
    with pytest.raises(ValueError):
        plan.norms(f32(), sums[:2])
    with pytest.raises(ValueError):
        plan.adamw(good, f32(), f32(), f32(), f32(), step.int())
    with pytest.raises(ValueError):
        plan.adamw_coded(good, f32(), f32(), u8(), u8(), u8(2 * plan.blocks - 1), step)
    with pytest.raises(ValueError):
        plan.decode(u8(), u8(), u8(10), f32(), torch.zeros(700, dtype=torch.bfloat16, device="cuda"))
    lib, st = B.lib(), torch.cuda.current_stream().cuda_stream
    g = f32()
    assert lib.lgreco_optim_norms(plan._o, g.data_ptr() + 2, 0, sums.data_ptr(), st) == B.EINVAL
    assert lib.lgreco_optim_norms(plan._o, None, 0, sums.data_ptr(), st) == B.EINVAL
    assert lib.lgreco_optim_norms(None, g.data_ptr(), 0, sums.data_ptr(), st) == B.EINVAL
    assert lib.lgreco_optim_norms(plan._o, g.data_ptr(), 5, sums.data_ptr(), st) == B.EINVAL
    torch.cuda.synchronize()
    assert int(step) == 0 and float(sums.abs().sum()) == 0
