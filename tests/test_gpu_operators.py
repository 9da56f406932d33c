"""GPU parity of the operators between an attention block's projections (position rotation, norm of query and key
heads, attention to another length) with their definitions in float64 on the CPU.

Tolerances are per entry and counted in roundings: u is the largest relative error of one rounding to the tensors' type
(finfo.eps / 2: bf16 2^-8, fp32 2^-24), E = 2^-24 that of an fp32 operation.  `bound` arrays come with every reference."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
BF16, F32 = "bf16", "f32"


def _t(dtype):
    import torch
    return torch.bfloat16 if dtype == BF16 else torch.float32


def _u(dtype):
    import torch
    return torch.finfo(_t(dtype)).eps / 2


def _randn(seed, *shape, dtype, scale=1.0):
    """float64 values that the type holds exactly."""
    import torch
    rng = np.random.Generator(np.random.PCG64(seed))
    return torch.from_numpy(rng.standard_normal(shape) * scale).to(_t(dtype)).double()


def _dev(x, dtype):
    return x.to(_t(dtype)).cuda()


def _close(got, want, bound, what):
    got = got.detach().double().cpu()
    assert got.shape == want.shape, what
    same = (got == want) | (got.isnan() & want.isnan())
    off = (got - want).abs()
    bad = ~(same | (off <= bound))
    assert not bad.any(), (what, int(bad.sum()), float((off / bound.clamp_min(1e-300))[bad].max()), bad.nonzero()[:4].tolist())


# ---------------------------------------------------------------------------------------------
# rotation, norm
# ---------------------------------------------------------------------------------------------


def _partners(rot, layout):
    import torch
    j = torch.arange(rot)
    if layout == "half":
        return j % (rot // 2), (j + rot // 2) % rot, j < rot // 2
    return j // 2, j ^ 1, j % 2 == 0


def _turn(x, pos, rot, layout, freqs, scale, sign=1.0):
    """(turned x, |a| + |b| per entry) in float64."""
    import torch
    y, mag = x.clone(), x.abs()
    if rot:
        pair, partner, first = _partners(rot, layout)
        ang = pos.double()[:, None] * torch.from_numpy(freqs)[pair]
        c, s = scale * ang.cos()[:, None], scale * sign * ang.sin()[:, None] * torch.where(first, -1.0, 1.0).double()
        part = x[..., :rot]
        y[..., :rot] = part * c + part[..., partner] * s
        mag = mag.clone()
        mag[..., :rot] = (part.abs() + part[..., partner].abs()) * abs(scale)
    return y, mag


def _freqs(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot) if rot else np.zeros(0)


def _plan(vf, rot, layout, scale=1.0, **kw):
    return vf.vf_rope_make(vf.VF_ROPE_HALF if layout == "half" else vf.VF_ROPE_INTERLEAVED, rot, scale=scale, **kw)


# cosine and sine: at most 4 ulp of sincospi, 1 of the argument, 1 of the scale; products and sum: 2
TURN = 8 * E

HEADS = [  # rows, heads, d_head, rot
    (1, 1, 64, 64), (1, 24, 64, 64), (7, 3, 128, 128), (33, 5, 128, 64), (130, 2, 80, 80), (65, 7, 80, 20), (19, 3, 96, 48),
    (5, 2, 40, 6), (9, 4, 37, 10), (3, 2, 2, 2), (4, 3, 512, 256), (2, 1, 511, 130), (1025, 2, 32, 32), (3, 70, 64, 32),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,heads,dh,rot", HEADS)
def test_rotation(rows, heads, dh, rot, dtype, layout):
    import torch
    import paper_2009_09523_amd as vf
    x = _randn(rows * dh + rot, rows, heads, dh, dtype=dtype)
    pos = torch.from_numpy(np.random.Generator(np.random.PCG64(rows)).integers(-5, 1 << 30, rows).astype(np.int32))
    plan = _plan(vf, rot, layout, scale=1.25)
    xd = _dev(x, dtype)
    for inverse in (False, True):
        y = torch.full_like(xd, 7.0)
        vf.vf_rope(xd, y, plan, positions=pos.cuda(), inverse=inverse)
        want, mag = _turn(x, pos, rot, layout, _freqs(rot), 1.25, -1.0 if inverse else 1.0)
        # the angle itself: position times turns is a float64 product, 2^-53 of up to 2^30 radians
        _close(y, want, mag * (TURN + 2.0 ** -22) + _u(dtype) * want.abs() * (dtype == BF16), f"inverse={inverse}")
        if rot < dh:
            assert torch.equal(y[..., rot:], xd[..., rot:])


@pytest.mark.parametrize("kind", ["plain", "linear", "parts"])
def test_stretched_frequencies(kind):
    """Far positions, where an fp32 product of position and frequency would have lost the angle."""
    import torch
    import paper_2009_09523_amd as vf
    rot, rows = 128, 64
    f = _freqs(rot, 500000.0)
    kw = {}
    if kind == "linear":
        f, kw = f / 8, dict(scaling=vf.VF_ROPE_LINEAR, factor=8.0)
    if kind == "parts":
        keep = np.clip((8192 * f / (2 * math.pi) - 1.0) / 3.0, 0, 1)
        assert 0 < keep.mean() < 1 and ((keep > 0) & (keep < 1)).any()
        f, kw = keep * f + (1 - keep) * f / 8, dict(scaling=vf.VF_ROPE_PARTS, factor=8.0, trained_len=8192, beta_fast=4.0, beta_slow=1.0)
    plan = _plan(vf, rot, "half", base=500000.0, **kw)
    x = _randn(3, rows, 2, rot, dtype=F32)
    y = torch.empty(rows, 2, rot, device="cuda")
    vf.vf_rope(_dev(x, F32), y, plan, first=1_000_000)
    want, mag = _turn(x, torch.arange(rows) + 1_000_000, rot, "half", f, 1.0)
    _close(y, want, mag * (TURN + 2.0 ** -30), kind)      # 2^-53 of 2^20 radians, a few times over


def test_positions_from_the_row():
    import torch
    import paper_2009_09523_amd as vf
    x = _randn(5, 50, 3, 64, dtype=BF16)
    plan = _plan(vf, 64, "half")
    xd = _dev(x, BF16)
    a, b = torch.empty_like(xd), torch.empty_like(xd)
    vf.vf_rope(xd, a, plan, first=17, seq_len=16)
    vf.vf_rope(xd, b, plan, positions=(17 + torch.arange(50) % 16).to(torch.int32).cuda())
    assert torch.equal(a, b)
    vf.vf_rope(xd, a, plan, first=3)
    vf.vf_rope(xd, b, plan, positions=(3 + torch.arange(50)).to(torch.int32).cuda())
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shift,pad", [(0, 0), (0, 8), (1, 3), (4, 4)])
def test_rotation_of_a_slice_in_place(shift, pad, dtype):
    """Heads inside wider rows, at addresses that 16-byte loads may and may not take; what lies beside them stays."""
    import torch
    import paper_2009_09523_amd as vf
    rows, heads, dh = 21, 4, 64
    wide = _dev(_randn(9, rows, heads * dh + 2 * pad + 8, dtype=dtype), dtype)
    before = wide.clone()
    view = wide[:, shift:shift + heads * dh].unflatten(1, (heads, dh))
    x = view.double().cpu()
    vf.vf_rope(view, view, _plan(vf, dh, "half"), first=4)
    want, mag = _turn(x, torch.arange(rows) + 4, dh, "half", _freqs(dh), 1.0)
    _close(view, want, mag * TURN + _u(dtype) * want.abs() * (dtype == BF16), "in place")
    assert torch.equal(wide[:, :shift], before[:, :shift]) and torch.equal(wide[:, shift + heads * dh:], before[:, shift + heads * dh:])


def test_rotation_back_is_the_transpose():
    """<R x, y> = <x, R^-1 y> up to roundings: the inverse is the backward pass."""
    import torch
    import paper_2009_09523_amd as vf
    x, y = _randn(1, 40, 3, 96, dtype=F32), _randn(2, 40, 3, 96, dtype=F32)
    plan = _plan(vf, 48, "interleaved", scale=0.75)
    a, b = torch.empty(40, 3, 96, device="cuda"), torch.empty(40, 3, 96, device="cuda")
    vf.vf_rope(_dev(x, F32), a, plan)
    vf.vf_rope(_dev(y, F32), b, plan, inverse=True)
    lhs, rhs = (a.double().cpu() * y).sum(), (x * b.double().cpu()).sum()
    assert abs(lhs - rhs) <= 2 * TURN * (2 * x.abs() * y.abs()).sum() + 2 * TURN * float(x.norm() * y.norm())


def _norm_ref(x, dy, q_heads, gq, gk, eps, pos, rot, layout, scale=1.0):
    """Forward and backward of the norm with rotation: values and, per entry, the sum of the magnitudes its roundings scale with."""
    import torch
    dh = x.shape[-1]
    f = _freqs(rot)
    r = 1 / ((x ** 2).mean(-1, keepdim=True) + eps).sqrt()
    gamma = torch.stack([gq if h < q_heads else gk for h in range(x.shape[1])])
    xhat = x * r
    y, ymag = _turn(xhat * gamma, pos, rot, layout, f, scale)
    out = {"y": (y, ymag)}
    if dy is not None:
        g, gmag = _turn(dy, pos, rot, layout, f, scale, -1.0)
        out["dgamma_q"] = (g * xhat)[:, :q_heads].sum((0, 1)), (gmag * xhat.abs())[:, :q_heads].sum((0, 1))
        out["dgamma_k"] = (g * xhat)[:, q_heads:].sum((0, 1)), (gmag * xhat.abs())[:, q_heads:].sum((0, 1))
        h, hmag = g * gamma, gmag * gamma.abs()
        out["dx"] = (r * (h - xhat * (h * xhat).mean(-1, keepdim=True)),
                     r * (hmag + xhat.abs() * (hmag * xhat.abs()).mean(-1, keepdim=True)))
    return out


NORMS = [  # rows, q heads, k heads, d_head, rot (0: the norm alone)
    (1, 12, 12, 64, 64), (1, 1, 0, 128, 128), (130, 4, 2, 128, 128), (257, 3, 3, 96, 96), (65, 0, 5, 80, 40), (33, 8, 1, 64, 0),
    (17, 2, 2, 37, 10), (9, 1, 2, 511, 130), (2100, 2, 1, 32, 32), (40, 33, 7, 40, 40),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,hq,hk,dh,rot", NORMS)
def test_norm_with_rotation(rows, hq, hk, dh, rot, dtype, layout):
    import torch
    import paper_2009_09523_amd as vf
    heads = hq + hk
    x, dy = _randn(rows + dh, rows, heads, dh, dtype=dtype), _randn(rows + dh + 1, rows, heads, dh, dtype=dtype, scale=0.1)
    gq, gk = 1 + 0.2 * _randn(1, dh, dtype=F32), 1 + 0.2 * _randn(2, dh, dtype=F32)
    gq, gk = gq.float().double(), gk.float().double()
    pos = torch.arange(rows) % 50 + 1000
    plan = _plan(vf, rot, layout, scale=1.1) if rot else None
    kw = dict(eps=1e-6, plan=plan, first=1000, seq_len=50)
    xd, dyd, gqd, gkd = _dev(x, dtype), _dev(dy, dtype), gq.float().cuda(), gk.float().cuda()
    y, dx = torch.full_like(xd, 7.0), torch.full_like(xd, 7.0)
    dq, dk = torch.full((dh,), 2.0, device="cuda"), torch.full((dh,), 3.0, device="cuda")
    ws = torch.empty(vf.vf_qk_norm_rope_workspace(rows, hq, hk, dh), dtype=torch.uint8, device="cuda")
    vf.vf_qk_norm_rope(xd, y, hq, gqd, gkd, **kw)
    vf.vf_qk_norm_rope_backward(xd, dyd, dx, hq, gqd, gkd, dq, dk, ws, alpha=0.5, accumulate=True, **kw)
    ref = _norm_ref(x, dy, hq, gq, gk, float(np.float32(1e-6)), pos, rot, layout, 1.1)
    # the mean square: a lane's 16 squares and up to 6 levels (scalar path: 8 and 6), half of it in rstd; sqrt, division, products
    norm = (0.5 * 24 + 8) * E
    u = _u(dtype) if dtype == BF16 else 0.0
    _close(y, ref["y"][0], ref["y"][1] * (norm + TURN) + u * ref["y"][0].abs(), "y")
    _close(dx, ref["dx"][0], ref["dx"][1] * (3 * norm + TURN + 32 * E) + u * ref["dx"][0].abs(), "dx")
    # a column's chain: the items of a thread (at most rows * heads / 4 units of a group, few here), 64 to 256 units, 2048 / 16
    # partials and 16 groups: under 512 additions
    for name, got, old in (("dgamma_q", dq, 2.0), ("dgamma_k", dk, 3.0)):
        want, mag = ref[name]
        _close(got, 0.5 * want + old, 0.5 * mag * (512 * E + norm + TURN) + E * (0.5 * want + old).abs(), name)


def test_norm_gradients_against_differences():
    """<dx, d> and <dgamma, d> against central differences of the definition in float64."""
    import torch
    import paper_2009_09523_amd as vf
    rows, hq, hk, dh = 12, 2, 1, 64
    x, dy = _randn(1, rows, 3, dh, dtype=F32), _randn(2, rows, 3, dh, dtype=F32)
    gq, gk = 1 + 0.2 * _randn(3, dh, dtype=F32), 1 + 0.2 * _randn(4, dh, dtype=F32)
    gq, gk = gq.float().double(), gk.float().double()
    d, dg = _randn(5, rows, 3, dh, dtype=F32), _randn(6, dh, dtype=F32)
    pos = torch.arange(rows)
    f = lambda a, g: (_norm_ref(a, None, hq, g, gk, 1e-5, pos, 64, "half")["y"][0] * dy).sum()  # noqa: E731
    h = 1e-5
    by_x = (f(x + h * d, gq) - f(x - h * d, gq)) / (2 * h)
    by_g = (f(x, gq + h * dg) - f(x, gq - h * dg)) / (2 * h)
    dx, dq, dk = torch.empty(rows, 3, dh, device="cuda"), torch.empty(dh, device="cuda"), torch.empty(dh, device="cuda")
    ws = torch.empty(vf.vf_qk_norm_rope_workspace(rows, hq, hk, dh), dtype=torch.uint8, device="cuda")
    vf.vf_qk_norm_rope_backward(_dev(x, F32), _dev(dy, F32), dx, hq, gq.float().cuda(), gk.float().cuda(), dq, dk, ws, eps=1e-5,
                                plan=_plan(vf, 64, "half"))
    got_x, got_g = (dx.double().cpu() * d).sum(), (dq.double().cpu() * dg).sum()
    # the difference's own error is of the order h^2 = 1e-10 and 1e-16 / h = 1e-11 of the sums; the kernel's under 100 roundings
    size_x, size_g = float((dx.double().cpu() * d).abs().sum()), float((dq.double().cpu() * dg).abs().sum())
    assert abs(got_x - by_x) <= (200 * E + 1e-8) * size_x * 4
    assert abs(got_g - by_g) <= (600 * E + 1e-8) * size_g * 4


def test_norm_without_weights_in_place_and_without_rows():
    import torch
    import paper_2009_09523_amd as vf
    x, dy = _randn(1, 30, 4, 64, dtype=BF16), _randn(2, 30, 4, 64, dtype=BF16)
    one = torch.ones(64, dtype=torch.float64)
    ref = _norm_ref(x, dy, 4, one, one, float(np.float32(1e-6)), torch.arange(30), 64, "half")
    plan = _plan(vf, 64, "half")
    y = _dev(x, BF16)
    vf.vf_qk_norm_rope(y, y, 4, plan=plan)
    _close(y, ref["y"][0], ref["y"][1] * 40 * E + 2.0 ** -8 * ref["y"][0].abs(), "y")
    for target in ("x", "dy"):
        xd, dyd = _dev(x, BF16), _dev(dy, BF16)
        dx = xd if target == "x" else dyd
        vf.vf_qk_norm_rope_backward(xd, dyd, dx, 4, plan=plan)
        _close(dx, ref["dx"][0], ref["dx"][1] * 100 * E + 2.0 ** -8 * ref["dx"][0].abs(), target)
    none = torch.empty(0, 4, 64, device="cuda")
    g, dg = torch.ones(64, device="cuda"), torch.full((64,), 5.0, device="cuda")
    ws = torch.empty(16, dtype=torch.uint8, device="cuda")
    vf.vf_qk_norm_rope(none, none, 4, g)
    vf.vf_rope(none, none, plan)
    vf.vf_qk_norm_rope_backward(none, none, none, 4, g, None, dg, None, ws, accumulate=True)
    assert (dg == 5).all()
    vf.vf_qk_norm_rope_backward(none, none, none, 4, g, None, dg, None, ws)
    assert (dg == 0).all()


def test_norm_of_zero_rows_and_large_values():
    """A head of zeros stays zero with finite gradients; values whose squares stay finite keep their direction."""
    import torch
    import paper_2009_09523_amd as vf
    x = torch.zeros(3, 2, 64, device="cuda")
    x[1] = 1e15
    y, dx, dy = torch.empty_like(x), torch.empty_like(x), torch.ones_like(x)
    vf.vf_qk_norm_rope(x, y, 2)
    vf.vf_qk_norm_rope_backward(x, dy, dx, 2)
    assert (y[0] == 0).all() and torch.allclose(y[1], torch.ones_like(y[1]), rtol=1e-5, atol=0)
    assert torch.allclose(dx[0], torch.full_like(dx[0], 1e3), rtol=1e-4)      # rstd = 1 / sqrt(eps)
    assert dx.isfinite().all()


# ---------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------


def _attn_ref(q, k, v, do, q_len, k_len, mask, scale, dtype):
    """Definition in float64 with its bounds.  Roundings of the kernels: the products q k in fp32 (dh additions of at most
    Z = max scale sum |q||k| each), p and dz rounded to the operands' type, o rounded before rowsum(dO o), results rounded."""
    import torch
    B, Tq, Hq, dh = q.shape
    Tk, Hk = k.shape[1], k.shape[2]
    G = Hq // Hk
    u = _u(dtype)
    up = u if dtype == BF16 else 0.0                     # operands p and dz
    out = {n: (torch.zeros(s, dtype=torch.float64), torch.zeros(s, dtype=torch.float64))
           for n, s in (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    lse, lse_bound = torch.full((B, Hq, Tq), -math.inf, dtype=torch.float64), torch.zeros(B, Hq, Tq, dtype=torch.float64)
    for b in range(B):
        n = Tq if q_len is None else min(max(int(q_len[b]), 0), Tq)
        vis = torch.arange(Tk) < (Tk if k_len is None else int(k_len[b]))
        if mask is not None:
            vis = vis & (mask[b] != 0)
        idx = vis.nonzero()[:, 0]
        if n == 0 or len(idx) == 0:
            continue
        for h in range(Hq):
            qq, kk, vv, dd = q[b, :n, h], k[b, idx, h // G], v[b, idx, h // G], do[b, :n, h]
            z = scale * qq @ kk.T
            Z = float((scale * qq.abs() @ kk.abs().T).max())
            rel = (2 * (dh + 4) * Z + 2 * len(idx) + 16) * E        # of p: its own z and the lse, exp2, the running sum
            L = torch.logsumexp(z, 1)
            p = torch.exp(z - L[:, None])
            o = p @ vv
            pv = p @ vv.abs()
            lse[b, h, :n], lse_bound[b, h, :n] = L, rel + 4 * E * L.abs()
            out["o"][0][b, :n, h], out["o"][1][b, :n, h] = o, pv * (up + rel + len(idx) * E) * 1.01 + u * o.abs()
            dp, dpa = dd @ vv.T, dd.abs() @ vv.abs().T
            delta, da = (dd * o).sum(1, keepdim=True), (dd.abs() * (o.abs())).sum(1, keepdim=True)
            ob = (dd.abs() * out["o"][1][b, :n, h]).sum(1, keepdim=True)
            dz = p * (dp - delta)
            dzb = p * ((dp - delta).abs() * (up + rel) + ob + (dpa + da) * (dh + 4) * E)
            g = scale * dz @ kk
            out["dq"][0][b, :n, h] = g
            out["dq"][1][b, :n, h] = scale * (dzb + dz.abs() * len(idx) * E) @ kk.abs() * 1.01 + u * g.abs()
            out["dk"][0][b, idx, h // G] += scale * dz.T @ qq
            out["dk"][1][b, idx, h // G] += scale * (dzb + dz.abs() * n * G * E).T @ qq.abs() * 1.01
            out["dv"][0][b, idx, h // G] += p.T @ dd
            out["dv"][1][b, idx, h // G] += p.T @ dd.abs() * (up + rel + n * G * E) * 1.01
    for name in ("dk", "dv"):
        out[name] = out[name][0], out[name][1] + u * out[name][0].abs()
    out["lse"] = lse, lse_bound
    return out


def _attend(q, k, v, do, dtype, q_len=None, k_len=None, mask=None, scale=None, lay=lambda t: t.contiguous(), stream=None):
    """Both passes on the device; q .. do float64 on the CPU."""
    import torch
    import paper_2009_09523_amd as vf
    qd, kd, vd, dd = (lay(_dev(t, dtype)) for t in (q, k, v, do))
    i32 = lambda t: None if t is None else torch.as_tensor(t, dtype=torch.int32).cuda()  # noqa: E731
    kw = dict(q_len=i32(q_len), k_len=i32(k_len), key_mask=None if mask is None else mask.to(torch.uint8).cuda(), scale=scale, stream=stream)
    o, lse = lay(torch.full_like(qd, 7.0)), torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device="cuda")
    dq, dk, dv = (lay(torch.full_like(t, 7.0)) for t in (qd, kd, vd))
    space = lambda b: torch.full((vf.vf_attention_workspace(qd, kd, vd, backward=b),), 255, dtype=torch.uint8, device="cuda")  # noqa: E731
    vf.vf_attention(qd, kd, vd, o, lse, workspace=space(False), **kw)
    vf.vf_attention_backward(qd, kd, vd, o, lse, dd, dq, dk, dv, workspace=space(True), **kw)
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _check_attn(got, ref):
    for name in ("lse", "o", "dv", "dq", "dk"):
        _close(got[name], *ref[name], name)


def _inputs(B, Tq, Tk, Hq, Hk, dh, dtype, seed=0):
    return (_randn(seed + 1, B, Tq, Hq, dh, dtype=dtype, scale=1.5), _randn(seed + 2, B, Tk, Hk, dh, dtype=dtype),
            _randn(seed + 3, B, Tk, Hk, dh, dtype=dtype), _randn(seed + 4, B, Tq, Hq, dh, dtype=dtype, scale=0.1))


SHAPES = [  # batch, q rows, k rows, q heads, kv heads, d_head
    (1, 1, 1, 1, 1, 64), (2, 1, 300, 2, 2, 64), (1, 1, 700, 8, 2, 128), (3, 5, 33, 2, 1, 32), (2, 33, 31, 3, 3, 40),
    (1, 128, 128, 2, 2, 64), (2, 129, 65, 2, 1, 128), (1, 200, 77, 4, 4, 80), (1, 63, 513, 3, 1, 96), (2, 7, 1, 4, 2, 8),
    (1, 300, 3, 5, 1, 120), (1, 257, 260, 6, 2, 64), (1, 1, 2500, 4, 1, 64), (1, 1030, 9, 2, 2, 64), (2, 4, 1111, 2, 2, 128),
    # many workgroups: rows, then keys, in tiles of 128 to a workgroup, every width
    (16, 260, 90, 8, 8, 64), (16, 260, 90, 8, 8, 96), (16, 260, 90, 8, 8, 128), (12, 90, 400, 8, 4, 64), (12, 90, 400, 8, 8, 80),
    (12, 90, 400, 8, 8, 104),
    # few: the streamed side in parts
    (1, 1, 20000, 1, 1, 64), (1, 2, 9000, 4, 2, 128), (1, 3000, 20, 2, 1, 128), (1, 40, 6000, 2, 2, 96), (1, 4000, 40, 2, 1, 96),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", SHAPES)
def test_attention(B, Tq, Tk, Hq, Hk, dh, dtype):
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    _check_attn(_attend(q, k, v, do, dtype), _attn_ref(q, k, v, do, None, None, None, dh ** -0.5, dtype))


# heads of 32 elements and less have a width of their own in fp32: whole tiles, wavefronts that share a tile, parts
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", [(16, 260, 90, 8, 8, 32), (12, 90, 400, 8, 4, 24), (1, 1, 20000, 1, 1, 32), (1, 3000, 20, 2, 1, 32),
                                              (2, 33, 31, 3, 3, 16), (1, 40, 6000, 2, 2, 32), (2, 700, 129, 6, 2, 32)])
def test_attention_of_short_heads(B, Tq, Tk, Hq, Hk, dh, dtype):
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    k_len = None if B == 1 else [Tk - 7 * b for b in range(B)]
    _check_attn(_attend(q, k, v, do, dtype, None, k_len), _attn_ref(q, k, v, do, None, k_len, None, dh ** -0.5, dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh,q_len,k_len", [
    (4, 70, 150, 2, 2, 64, [70, 1, 0, 33], [150, 64, 17, 0]),
    (3, 40, 90, 4, 2, 128, None, [1, 90, 65]),
    (3, 130, 40, 2, 1, 80, [129, 2, 130], None),
    (3, 1, 700, 2, 2, 64, None, [700, 0, 129]),
    (2, 9, 2000, 2, 1, 64, [9, 4], [3, 1999]),
    (2, 20, 30, 1, 1, 64, [-5, 99], [99, -5]),                # clamped into the tensors
])
def test_attention_over_padded_batches(B, Tq, Tk, Hq, Hk, dh, q_len, k_len, dtype):
    """What lies in the padding -- infinities and NaN here -- has no influence; padded rows come out as zeros."""
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    clean = _attn_ref(q, k, v, do, q_len, k_len, None, dh ** -0.5, dtype)
    for b in range(B):
        if q_len is not None:
            n = max(q_len[b], 0)
            q[b, n:], do[b, n:] = math.nan, math.inf
        if k_len is not None:
            n = max(k_len[b], 0)
            k[b, n:], v[b, n:] = math.inf, math.nan
    _check_attn(_attend(q, k, v, do, dtype, q_len, k_len), clean)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", [(4, 50, 211, 2, 2, 64), (3, 1, 333, 4, 2, 128), (4, 140, 64, 2, 1, 40), (3, 3, 1500, 2, 2, 64),
                                              (64, 1, 4200, 4, 4, 64)])
def test_attention_with_key_masks(B, Tq, Tk, Hq, Hk, dh, dtype):
    """Single keys masked out, one sample that sees nothing, one that sees its last key alone, with lengths on top."""
    import torch
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    mask = torch.from_numpy(np.random.Generator(np.random.PCG64(Tk)).random((B, Tk)) < 0.6)
    mask[0] = False
    mask[1] = False
    mask[1, -1] = True
    for k_len in (None, [Tk] * (B - 1) + [Tk // 2]):
        ref = _attn_ref(q, k, v, do, None, k_len, mask, dh ** -0.5, dtype)
        kk, vv = k.clone(), v.clone()
        kk[~mask], vv[~mask] = math.nan, -math.inf
        _check_attn(_attend(q, kk, vv, do, dtype, None, k_len, mask), ref)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_with_scores_far_apart(dtype):
    """One key outweighs all others by more than fp32's exponent range, first or last; scores of -1e30 and of equal size."""
    import torch
    q, k, v, do = _inputs(2, 40, 200, 1, 1, 64, dtype)
    q[:] = 1.0
    k[0] *= 0.01
    k[0, 3], k[0, 190] = 1000.0, 1008.0
    k[1] = -1e30
    k[1, 77] = -1e28
    q, k = (t.to(_t(dtype)).double() for t in (q, k))
    ref = _attn_ref(q, k, v, do, None, None, None, 0.125, dtype)
    got = _attend(q, k, v, do, dtype)
    for name in ("o", "dv"):                                  # one-hot rows: a key's value as it is, no rounding of p
        # the backward pass takes p from lse = 8064: lse stored, times log2 e, and scale times log2 e, one rounding each
        more = 3 * E * 8064 if name == "dv" else 0.0
        _close(got[name][0], ref[name][0][0], ref[name][0][0].abs() * (2 * _u(dtype) + more) + 1e-30, name)
        assert got[name].isfinite().all()
    assert torch.equal(got["o"][1, 0, 0].cpu(), _dev(v, dtype)[1, 77, 0].cpu())
    assert got["dq"].isfinite().all() and got["dk"].isfinite().all()


def test_nan_in_a_visible_place_is_not_hidden():
    import torch
    q, k, v, do = _inputs(1, 3, 70, 1, 1, 64, BF16)
    q[0, 1] = math.nan
    got = _attend(q, k, v, do, BF16)
    assert got["o"][0, 1].isnan().all() and got["o"][0, 0].isfinite().all() and got["o"][0, 2].isfinite().all()


# one workgroup of whole tiles, wavefronts that share a tile, the streamed side in parts; each pass in turn
NAN_SHAPES = [(1, 3, 70, 1, 1, 64), (16, 260, 90, 8, 8, 64), (16, 260, 90, 8, 8, 128), (2, 4, 9000, 4, 2, 64), (2, 3000, 20, 2, 1, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", NAN_SHAPES)
def test_nan_in_a_query_reaches_the_gradients_of_its_keys(B, Tq, Tk, Hq, Hk, dh, dtype):
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    q[0, 1, 0, 3] = math.nan                                  # every p of the row is NaN
    got = _attend(q, k, v, do, dtype)
    assert got["dq"][0, 1, 0].isnan().all() and got["dk"][0, :, 0].isnan().all() and got["dv"][0, :, 0].isnan().all()
    assert got["dq"][0, 0].isfinite().all() and got["dq"][0, 2].isfinite().all()
    for name in ("dk", "dv"):
        assert got[name][1:].isfinite().all() and got[name][:, :, 1:].isfinite().all(), name


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", NAN_SHAPES)
def test_padded_rows_are_zero_beside_keys_that_are_not_finite(B, Tq, Tk, Hq, Hk, dh, dtype):
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    k[0, 2], v[0, 5] = math.inf, math.nan
    got = _attend(q, k, v, do, dtype, q_len=[2] * B)
    for name in ("o", "dq"):
        assert (got[name][:, 2:] == 0).all() and got[name][0, :2].isnan().all(), name
        assert got[name][1:].isfinite().all(), name
    assert (got["lse"][:, :, 2:] == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_over_other_orders(dtype):
    """Heads before rows; heads inside wider rows; keys and values shared by the batch (stride 0)."""
    import torch
    q, k, v, do = _inputs(2, 50, 70, 4, 2, 64, dtype)
    ref = _attn_ref(q, k, v, do, None, None, None, 0.3, dtype)
    _check_attn(_attend(q, k, v, do, dtype, scale=0.3, lay=lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)), ref)

    def inside(t):
        w = torch.full((t.shape[0], t.shape[1], t.shape[2] + 1, t.shape[3] + 8), math.nan, dtype=t.dtype, device=t.device)
        w[:, :, :-1, 8:] = t
        return w[:, :, :-1, 8:]
    _check_attn(_attend(q, k, v, do, dtype, scale=0.3, lay=inside), ref)
    k[1], v[1] = k[0], v[0]
    ref = _attn_ref(q, k, v, do, None, None, None, 0.3, dtype)
    import paper_2009_09523_amd as vf
    qd, dd = _dev(q, dtype), _dev(do, dtype)
    kd, vd = (_dev(t[:1], dtype).expand(2, -1, -1, -1) for t in (k, v))
    got = {"o": torch.empty_like(qd), "lse": torch.empty(2, 4, 50, device="cuda"), "dq": torch.empty_like(qd),
           "dk": torch.empty(k.shape, dtype=qd.dtype, device="cuda"), "dv": torch.empty(k.shape, dtype=qd.dtype, device="cuda")}
    ws = torch.empty(max(1, vf.vf_attention_workspace(qd, kd, vd, backward=True)), dtype=torch.uint8, device="cuda")
    vf.vf_attention(qd, kd, vd, got["o"], got["lse"], scale=0.3, workspace=ws)
    vf.vf_attention_backward(qd, kd, vd, got["o"], got["lse"], dd, got["dq"], got["dk"], got["dv"], scale=0.3, workspace=ws)
    _check_attn(got, ref)


def test_attention_without_keys_rows_or_samples():
    import torch
    import paper_2009_09523_amd as vf
    for B, Tq, Tk in ((2, 5, 0), (2, 0, 5), (0, 5, 5)):
        q, k = torch.full((B, Tq, 2, 64), 3.0, device="cuda"), torch.full((B, Tk, 2, 64), 3.0, device="cuda")
        o, lse, dq, dk, dv = q.clone(), torch.zeros(B, 2, Tq, device="cuda"), q.clone(), k.clone(), k.clone()
        ws = torch.empty(max(1, vf.vf_attention_workspace(q, k, k, backward=True)), dtype=torch.uint8, device="cuda")
        vf.vf_attention(q, k, k, o, lse, workspace=ws)
        vf.vf_attention_backward(q, k, k, o, lse, q, dq, dk, dv, workspace=ws)
        for t in (o, dq, dk, dv):
            assert (t == 0).all()
        assert (lse == -math.inf).all()


def test_attention_gradients_against_differences():
    """Directional derivatives of sum(o do) by central differences of the definition in float64."""
    import torch
    q, k, v, do = _inputs(2, 20, 45, 4, 2, 64, F32)
    mask = torch.ones(2, 45)
    mask[1, 10:30] = 0
    got = _attend(q, k, v, do, F32, mask=mask)
    f = lambda a, b, c: (_attn_ref(a, b, c, do, None, None, mask, 0.125, F32)["o"][0] * do).sum()  # noqa: E731
    h = 1e-5
    for i, name in enumerate(("dq", "dk", "dv")):
        args = [q, k, v]
        d = _randn(50 + i, *args[i].shape, dtype=F32)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + h * d, args[i] - h * d
        by = (f(*up) - f(*down)) / (2 * h)
        g = got[name].double().cpu()
        # the kernel's part: under 2000 roundings of its entries; the difference's: 1e-16 / h and h^2 of the summed products
        assert abs((g * d).sum() - by) <= (2000 * E + 1e-8) * float((g * d).abs().sum()) * 4, name


def test_results_do_not_change_from_call_to_call():
    import torch
    q, k, v, do = _inputs(2, 3, 3000, 4, 2, 64, BF16)
    a = _attend(q, k, v, do, BF16)
    b = _attend(q, k, v, do, BF16)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_operators_on_another_stream_and_in_a_graph():
    """A block's operators together, as a node's pass uses them: projection, norm with rotation, attention, and back to the
    projection's gradient, on a side stream, then captured and replayed over new data between eager work."""
    import torch
    import paper_2009_09523_amd as vf
    B, T, Tk, H, dh, D = 2, 48, 70, 4, 64, 256
    g = torch.Generator(device="cuda").manual_seed(0)
    bf = torch.bfloat16
    W = (torch.randn(2 * H * dh, D, generator=g, device="cuda") / 16).to(bf)              # columns of q and of k
    gam = [1 + 0.1 * torch.randn(dh, generator=g, device="cuda") for _ in range(2)]
    plan = _plan(vf, dh, "half")
    x = torch.randn(B * T, D, generator=g, device="cuda").to(bf)
    enc, v = torch.randn(B, Tk, H, dh, generator=g, device="cuda").to(bf), torch.randn(B, Tk, H, dh, generator=g, device="cuda").to(bf)
    do = torch.randn(B, T, H, dh, generator=g, device="cuda").to(bf)
    k_len = torch.tensor([Tk, 31], dtype=torch.int32, device="cuda")
    qk32 = torch.empty(B * T, 2 * H * dh, device="cuda")
    raw = torch.empty(B * T, 2 * H, dh, device="cuda", dtype=bf)
    rot, draw, dqk = torch.empty_like(raw), torch.empty_like(raw), torch.zeros_like(raw)
    o, lse = torch.empty(B, T, H, dh, device="cuda", dtype=bf), torch.empty(B, H, T, device="cuda")
    denc, dv = torch.empty_like(enc), torch.empty_like(v)
    dg = [torch.empty(dh, device="cuda") for _ in range(2)]
    ws_n = torch.empty(vf.vf_qk_norm_rope_workspace(B * T, H, H, dh), dtype=torch.uint8, device="cuda")
    ws_a = torch.empty(max(1, vf.vf_attention_workspace(o, enc, v, True)), dtype=torch.uint8, device="cuda")

    def block(stream):
        vf.vf_gemm(x, W, qk32, B * T, 2 * H * dh, D, stream=stream)
        raw.copy_(qk32.view(raw.shape))
        vf.vf_qk_norm_rope(raw, rot, H, gam[0], gam[1], plan=plan, seq_len=T, stream=stream)
        q, dq = rot[:, :H].view(B, T, H, dh), dqk[:, :H].view(B, T, H, dh)
        vf.vf_attention(q, enc, v, o, lse, k_len=k_len, workspace=ws_a, stream=stream)
        vf.vf_attention_backward(q, enc, v, o, lse, do, dq, denc, dv, k_len=k_len, workspace=ws_a, stream=stream)
        vf.vf_qk_norm_rope_backward(raw, dqk, draw, H, gam[0], gam[1], dg[0], dg[1], ws_n, plan=plan, seq_len=T, stream=stream)

    outs = (rot, o, lse, denc, dv, draw, dg[0], dg[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(side)
    side.synchronize()
    eager = [t.clone() for t in outs]
    # against the definitions, step by step on what the device's own steps were given
    one = torch.arange(B * T) % T
    ref = _norm_ref(raw.double().cpu(), dqk.double().cpu(), H, gam[0].double().cpu(), gam[1].double().cpu(), float(np.float32(1e-6)), one, dh, "half")
    _close(rot, ref["y"][0], ref["y"][1] * 40 * E + 2.0 ** -8 * ref["y"][0].abs(), "rot")
    _close(draw, ref["dx"][0], ref["dx"][1] * 120 * E + 2.0 ** -8 * ref["dx"][0].abs(), "draw")
    ar = _attn_ref(rot[:, :H].view(B, T, H, dh).double().cpu(), enc.double().cpu(), v.double().cpu(), do.double().cpu(), None, k_len.cpu(), None, 0.125, BF16)
    _check_attn({"o": o, "lse": lse, "dq": dqk[:, :H].view(B, T, H, dh), "dk": denc, "dv": dv}, ar)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(torch.cuda.current_stream())
    for turn in range(3):
        x.copy_(torch.randn(B * T, D, generator=g, device="cuda").to(bf))
        k_len.copy_(torch.tensor([Tk - turn, 5 * turn], dtype=torch.int32))
        for t in outs:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in outs]
        block(None)
        torch.cuda.synchronize()
        for a, b in zip(replayed, outs):
            assert torch.equal(a, b), turn
    assert not torch.equal(eager[0], outs[0])


def test_heads_that_are_not_there_are_refused():
    import torch
    import paper_2009_09523_amd as vf
    x = torch.zeros(2, 3, 64, device="cuda")
    y = torch.empty_like(x)
    for heads in (-1, 4, 1 << 32):
        for call in (lambda: vf.vf_qk_norm_rope(x, y, heads), lambda: vf.vf_qk_norm_rope_backward(x, x, y, heads)):
            with pytest.raises(vf.VfError):
                call()


def test_two_calls_at_once_keep_apart():
    """Two streams, each with its own workspace, beside each other."""
    import torch
    import paper_2009_09523_amd as vf
    q, k, v, do = _inputs(2, 3, 2000, 4, 2, 64, BF16)
    want = _attend(q, k, v, do, BF16)
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st in s:
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            got.append(_attend(q, k, v, do, BF16, stream=st))
    torch.cuda.synchronize()
    for one in got:
        for n in want:
            assert torch.equal(one[n], want[n]), n


def test_offsets_beyond_32_bits():
    """Keys and values whose elements lie more than 2^32 bytes behind the first: rows far apart in one large buffer."""
    import torch
    import paper_2009_09523_amd as vf
    Tk, H, dh = 40, 1, 64
    row = 1 << 26                                               # 40 rows 128 MiB apart: 5 GiB
    big = torch.zeros(Tk * row, dtype=torch.bfloat16, device="cuda")
    kv = big.as_strided((1, Tk, 2, dh), (Tk * row, row, dh, 1))
    q, k, v, do = _inputs(1, 6, Tk, H, H, dh, BF16)
    kv[:, :, :1], kv[:, :, 1:] = _dev(k, BF16), _dev(v, BF16)
    kd, vd, qd, dd = kv[:, :, :1], kv[:, :, 1:], _dev(q, BF16), _dev(do, BF16)
    gr = torch.zeros(Tk * row, dtype=torch.bfloat16, device="cuda").as_strided((1, Tk, 2, dh), (Tk * row, row, dh, 1))
    got = {"o": torch.empty_like(qd), "lse": torch.empty(1, H, 6, device="cuda"), "dq": torch.empty_like(qd), "dk": gr[:, :, :1], "dv": gr[:, :, 1:]}
    ws = torch.empty(max(1, vf.vf_attention_workspace(qd, kd, vd, backward=True)), dtype=torch.uint8, device="cuda")
    vf.vf_attention(qd, kd, vd, got["o"], got["lse"], workspace=ws)
    vf.vf_attention_backward(qd, kd, vd, got["o"], got["lse"], dd, got["dq"], got["dk"], got["dv"], workspace=ws)
    _check_attn(got, _attn_ref(q, k, v, do, None, None, None, dh ** -0.5, BF16))
    y = torch.empty(Tk, 2, dh, device="cuda", dtype=torch.bfloat16)
    vf.vf_rope(kv[0], y, _plan(vf, dh, "half"), first=3)
    want, mag = _turn(torch.cat([k, v], 2)[0], torch.arange(Tk) + 3, dh, "half", _freqs(dh), 1.0)
    _close(y, want, mag * TURN + 2.0 ** -8 * want.abs(), "rope")


# wavefronts that share a tile's keys (four, two), one wavefront to a row, the keys in parts
FAR_SHAPES = [(1, 5, 200, 1, 1, 64), (32, 33, 257, 8, 8, 128), (16, 260, 90, 8, 8, 64), (2, 4, 9000, 4, 2, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", FAR_SHAPES)
def test_values_that_are_not_finite_show_however_small_their_weight(B, Tq, Tk, Hq, Hk, dh, dtype):
    """A visible key whose weight underflows to 0 beside another's: 0 times NaN or infinity is NaN, wherever the two keys lie."""
    import torch
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, dtype)
    q[0], G = 1.0, Hq // Hk
    k[0] *= 0.01
    for top in (3, Tk - 2):
        kk = k.clone()
        kk[0, top, 0] = 256.0 / dh ** 0.5                     # a score of 256 beside ones below 1: weights of exp(-255), below the range of fp32
        for bad, value in ((1, math.nan), (33, math.inf), (66, -math.inf), (Tk - 1, math.nan)):
            vv = v.clone()
            vv[0, bad, 0, 5] = value
            got = _attend(q, kk, vv, do, dtype)["o"]
            where = (top, bad)
            assert got[0, :, :G, 5].isnan().all(), where
            got[0, :, :G, 5] = 0
            assert got.isfinite().all(), where


@pytest.mark.parametrize("kw", [dict(first=1 << 64), dict(first=-(1 << 64)), dict(seq_len=(1 << 64) + 2), dict(seq_len=2 - (1 << 64))])
def test_positions_beyond_64_bits_are_refused(kw):
    """Cut to 64 bits they would be 0 and 2."""
    import torch
    import paper_2009_09523_amd as vf
    x = torch.zeros(2, 3, 64, device="cuda")
    plan = _plan(vf, 64, "half")
    for call in (lambda: vf.vf_rope(x, x, plan, **kw), lambda: vf.vf_qk_norm_rope(x, x, 1, plan=plan, **kw),
                 lambda: vf.vf_qk_norm_rope_backward(x, x, x, 1, plan=plan, **kw)):
        with pytest.raises(vf.VfError):
            call()


def test_attention_refuses_scales_and_empty_heads_on_the_device():
    import torch
    import paper_2009_09523_amd as vf
    q, ws = torch.zeros(1, 2, 1, 64, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    none, lse = torch.zeros(1, 2, 1, 0, device="cuda"), torch.zeros(1, 1, 2, device="cuda")
    for x, scale in ((q, 1e39), (q, 0.0), (q, math.nan), (none, None)):
        o, dq, dk, dv = (torch.empty_like(x) for _ in range(4))
        for call in (lambda: vf.vf_attention(x, x, x, o, scale=scale, workspace=ws),
                     lambda: vf.vf_attention_backward(x, x, x, x, lse, x, dq, dk, dv, scale=scale, workspace=ws)):
            with pytest.raises(vf.VfError):
                call()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh", [(2, 40, 300, 2, 2, 64), (8, 512, 4500, 8, 8, 64)])
def test_attention_without_a_workspace(B, Tq, Tk, Hq, Hk, dh, dtype):
    """One part, no mask: nothing is needed, and the backward pass does without the mask's bits."""
    import torch
    import paper_2009_09523_amd as vf
    g = torch.Generator(device="cuda").manual_seed(0)
    q, do = (torch.randn(B, Tq, Hq, dh, generator=g, device="cuda").to(_t(dtype)) for _ in range(2))
    k, v = (torch.randn(B, Tk, Hk, dh, generator=g, device="cuda").to(_t(dtype)) for _ in range(2))
    runs, most = [], vf.vf_attention_workspace(q, k, v, backward=True)
    bits = -(-B * -(-Tk // 64) * 8 // 16) * 16 if Tk > 4096 else 0
    for space in (0, most):
        o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(B, Hq, Tq, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        ws = torch.empty(space, dtype=torch.uint8, device="cuda") if space else None
        vf.vf_attention(q, k, v, o, lse, workspace=ws)
        vf.vf_attention_backward(q, k, v, o, lse, do, dq, dk, dv, workspace=torch.empty(space or most - bits, dtype=torch.uint8, device="cuda"))
        runs.append((o, lse, dq, dk, dv))
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    ones = torch.ones(B, Tk, dtype=torch.bool, device="cuda")
    if Tk > 4096:
        with pytest.raises(vf.VfError):
            vf.vf_attention(q, k, v, torch.empty_like(q), key_mask=ones)
    else:
        vf.vf_attention(q, k, v, o, lse, key_mask=ones)
        assert torch.equal(o, runs[0][0])


def _small_ints(g, lo, hi, dtype, *shape):
    import torch
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda").to(_t(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_largest_number_of_rows_to_a_problem(dtype):
    """65535 queries of 128 heads that share four keys, in whole numbers: scores of 0, weights of 1/4, values 0 to 3, o of 3/2, and sums of
    8388480 rows whose terms are of one sign."""
    import torch
    import paper_2009_09523_amd as vf
    T, H, dh = 65535, 128, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    q, do = _small_ints(g, 0, 1, dtype, 1, T, H, dh), _small_ints(g, 0, 2, dtype, 1, T, H, dh)
    k, v = torch.zeros(1, 4, 1, dh, device="cuda", dtype=_t(dtype)), torch.arange(4, device="cuda").to(_t(dtype))[None, :, None, None].expand(1, 4, 1, dh).contiguous()
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(1, H, T, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(vf.vf_attention_workspace(q, k, v, backward=True), dtype=torch.uint8, device="cuda")
    vf.vf_attention(q, k, v, o, lse, scale=0.5, workspace=ws)
    vf.vf_attention_backward(q, k, v, o, lse, do, dq, dk, dv, scale=0.5, workspace=ws)
    assert (o == 1.5).all() and (dq == 0).all()
    assert ((lse.double() - math.log(4)).abs() <= 8 * E).all()
    dd, qq = do.double().view(-1, dh), q.double().view(-1, dh)
    # dz = (key - 3/2) / 4 times the sum of dO, multiples of 1/8 up to 6
    dz = 0.25 * (torch.arange(4, device="cuda").double() - 1.5) * dd.sum(1, keepdim=True)
    # p = exp(0 - lse) and the exact rowsum leave 16 roundings, which bf16 operands (of up to 8 bits here) do not see; the rows go in
    # 64 parts, 16 (fp32: 2) to an instruction: additions one behind the other, and the rows of an instruction and the parts
    chain = 8388480 / 64 / (16 if dtype == BF16 else 2) + 128
    for got, want in ((dv, 0.25 * dd.sum(0).expand(4, dh)), (dk, 0.5 * dz.T @ qq)):
        _close(got[0, :, 0], want.cpu(), want.cpu().abs() * ((chain + 32) * E + _u(dtype)), "gradients")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_largest_number_of_keys(dtype):
    """One query and 8388480 keys of which a mask leaves the last 2^22: weights of 2^-22, whole values, sums below 2^24."""
    import torch
    import paper_2009_09523_amd as vf
    T, n, dh = 8388480, 1 << 22, 8
    g = torch.Generator(device="cuda").manual_seed(6)
    q, do = _small_ints(g, -1, 1, dtype, 1, 1, 1, dh), _small_ints(g, -2, 2, dtype, 1, 1, 1, dh)
    k, v = torch.zeros(1, T, 1, dh, device="cuda", dtype=_t(dtype)), _small_ints(g, -1, 2, dtype, 1, T, 1, dh)
    mask = torch.arange(T, device="cuda")[None] >= T - n
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(1, 1, 1, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(vf.vf_attention_workspace(q, k, v, backward=True), dtype=torch.uint8, device="cuda")
    vf.vf_attention(q, k, v, o, lse, key_mask=mask, workspace=ws)
    vf.vf_attention_backward(q, k, v, o, lse, do, dq, dk, dv, key_mask=mask, workspace=ws)
    want = (v[0, T - n:, 0].double().sum(0) / n).cpu()
    _close(o[0, 0, 0], want, want.abs() * (4 * E + _u(dtype)), "o")
    assert abs(float(lse) - 22 * math.log(2)) <= 4 * E * 22 and (dq == 0).all()
    assert (dv[0, :T - n] == 0).all() and (dk[0, :T - n] == 0).all() and dk.isfinite().all()
    # p from the stored logarithm: two roundings of 22 in the exponent, three in the logarithm and the exponential
    want = (do[0, 0].double() / n).cpu().expand(n, dh)
    _close(dv[0, T - n:, 0], want, want.abs() * (64 * E + _u(dtype)), "dv")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_largest_number_of_problems(dtype):
    """2^23 samples of one query and one key: every output is the value, and every score's gradient is 0."""
    import torch
    import paper_2009_09523_amd as vf
    B, dh = 1 << 23, 8
    g = torch.Generator(device="cuda").manual_seed(7)
    q, k, v, do = (_small_ints(g, -2, 2, dtype, B, 1, 1, dh) for _ in range(4))
    o, lse, dq, dk, dv = torch.empty_like(q), torch.empty(B, 1, 1, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    ws = torch.empty(vf.vf_attention_workspace(q, k, v, backward=True), dtype=torch.uint8, device="cuda")
    vf.vf_attention(q, k, v, o, lse, workspace=ws)
    vf.vf_attention_backward(q, k, v, o, lse, do, dq, dk, dv, workspace=ws)
    z = (q.double() * k.double()).sum(-1)[:, 0, 0] * dh ** -0.5
    assert ((lse.view(-1).double() - z).abs() <= 8 * E * (z.abs() + 1)).all()
    # scores of up to 12: p = exp(z - lse) is 1 within 64 roundings; o is p v / p, off by 4 roundings, so dp - rowsum(dO o), whose terms sum
    # up to 32, by 4 * 32, the exact rowsum by as much again, and dq and dk by 2 / sqrt(8) of that.  bf16 sees none of it
    f32 = dtype == F32
    assert ((o.double() - v.double()).abs() <= (4 * E if f32 else 0.0) * v.double().abs()).all()
    assert ((dv.double() - do.double()).abs() <= (64 * E if f32 else 0.0) * do.double().abs()).all()
    assert (dq.double().abs() <= (256 * E if f32 else 0.0)).all() and (dk.double().abs() <= (256 * E if f32 else 0.0)).all()


def test_largest_number_of_rows_of_the_rotation_and_norm():
    """2^31 - 1 rows of one short head: first and last rows and some between, rotation, norm, and the norm's gradient."""
    import torch
    import paper_2009_09523_amd as vf
    rows, dh, seq = (1 << 31) - 1, 2, 1000
    g = torch.Generator(device="cuda").manual_seed(8)
    piece = torch.randn(1 << 20, 1, dh, generator=g, device="cuda").to(torch.bfloat16)
    x = piece.repeat(2048, 1, 1)[:rows]
    some = torch.cat([torch.arange(300), torch.randint(0, rows, (2000,), generator=torch.Generator().manual_seed(9)), rows - 1 - torch.arange(300)])
    at = some.cuda()
    xs, dys = x[at].double().cpu(), x[at].double().cpu()
    pos, plan, one = some % seq + 5, _plan(vf, dh, "half"), torch.ones(dh, dtype=torch.float64)
    y = torch.empty_like(x)
    vf.vf_rope(x, y, plan, first=5, seq_len=seq)
    want, mag = _turn(xs, pos, dh, "half", _freqs(dh), 1.0)
    _close(y[at], want, mag * TURN + 2.0 ** -8 * want.abs(), "rotation")
    ref = _norm_ref(xs, dys, 1, one, one, float(np.float32(1e-6)), pos, dh, "half")
    vf.vf_qk_norm_rope(x, y, 1, plan=plan, first=5, seq_len=seq)
    _close(y[at], ref["y"][0], ref["y"][1] * 40 * E + 2.0 ** -8 * ref["y"][0].abs(), "norm")
    vf.vf_qk_norm_rope_backward(x, x, y, 1, plan=plan, first=5, seq_len=seq)
    _close(y[at], ref["dx"][0], ref["dx"][1] * 120 * E + 2.0 ** -8 * ref["dx"][0].abs(), "gradient")


def _exact_rowsum_ref(q, k, v, do, scale, o_dev):
    """dq and dk in float64 with bounds that leave no room for what rounding o puts into rowsum(dO o), and what they would be with it.

    The dq kernel starts from e = rowsum(dO (o' - o)) off; its dz = p (dp - rowsum) - p e sum up to rest = -e, which it takes out again.
    What stays: a rounding of dz - p e and (dq) of the p that -rest is spread by; the fp32 errors of dp, the rowsum and the sums."""
    import torch
    u, G = 2.0 ** -8, q.shape[2] // k.shape[2]
    dh = q.shape[3]
    dq, dqb, dqw = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(3))
    dk, dkb, dkw = (torch.zeros(k.shape, dtype=torch.float64) for _ in range(3))
    for b in range(q.shape[0]):
        for h in range(q.shape[2]):
            qq, kk, vv, dd = q[b, :, h], k[b, :, h // G], v[b, :, h // G], do[b, :, h]
            n = len(kk)
            z = scale * qq @ kk.T
            rel = (2 * (dh + 4) * float((scale * qq.abs() @ kk.abs().T).max()) + 2 * n + 16) * E         # of p, as in the reference above
            p = torch.softmax(z, 1)
            o = p @ vv
            e = (dd * (o_dev[b, :, h] - o)).sum(1, keepdim=True)
            dp, delta = dd @ vv.T, (dd * o).sum(1, keepdim=True)
            dz = p * (dp - delta)
            first = dz.abs() + p * e.abs()
            fp32 = (dd.abs() @ vv.abs().T + (dd.abs() * o.abs()).sum(1, keepdim=True)) * (dh + 4) * E
            rest = (p * fp32 + first * (rel + n * E)).sum(1, keepdim=True)                              # error of rest
            zq = first * (u + rel + n * E) + p * (fp32 + rest + e.abs() * (u + rel + n * E))
            zk = dz.abs() * (u + rel + len(qq) * G * E) + p * (fp32 + rest) * (1 + u)
            g = scale * dz @ kk
            dq[b, :, h], dqb[b, :, h], dqw[b, :, h] = g, scale * zq @ kk.abs() * 1.01 + u * g.abs(), g - scale * (p * e) @ kk
            dk[b, :, h // G] += scale * dz.T @ qq
            dkb[b, :, h // G] += scale * zk.T @ qq.abs() * 1.01
            dkw[b, :, h // G] += scale * (dz - p * e).T @ qq
    return (dq, dqb, dqw), (dk, dkb + u * dk.abs(), dkw)


# exact dq: four wavefronts to a block of rows (heads of 80, 128), two (128), one (64, 128; dk/dv in parts); dk alone: keys in parts
@pytest.mark.parametrize("B,Tq,Tk,Hq,Hk,dh,exact", [(1, 200, 77, 4, 4, 80, True), (4, 40, 300, 8, 4, 128, True), (32, 33, 257, 8, 8, 128, True),
                                                    (16, 260, 90, 8, 8, 64, True), (2, 9, 120, 4, 4, 128, True), (1, 1030, 9, 2, 2, 64, True),
                                                    (1, 40, 6000, 2, 2, 96, False), (2, 4, 9000, 4, 2, 64, False)])
def test_gradients_without_the_rounding_of_o(B, Tq, Tk, Hq, Hk, dh, exact):
    """Values far from 0, whose o is rounded by more than they differ, beside keys far from 0: left in the rowsum, that rounding is most of
    the error of dq and dk.  Rows of a head repeat, so that it does not cancel in dk."""
    q, k, v, do = _inputs(B, Tq, Tk, Hq, Hk, dh, BF16)
    q, do = (0.3 * q[:, :1]).expand(q.shape).contiguous(), do[:, :1].expand(do.shape).contiguous()
    q, k, v, do = (t.to(_t(BF16)).double() for t in (q, 8 + k, 64 + 2 * v, do))
    got = _attend(q, k, v, do, BF16)
    refs = _exact_rowsum_ref(q, k, v, do, dh ** -0.5, got["o"].double().cpu())
    for name, (want, bound, with_it) in zip(("dq", "dk"), refs):
        if name == "dq" and not exact:
            continue
        assert float(((with_it - want).abs() > bound).double().mean()) > 0.1, name       # such an error would not pass
        _close(got[name], want, bound, name)


def _inside(t, before, behind, between=0):
    """t's rows and heads inside wider rows of NaN: `before` and `behind` elements around a row, `between` behind every head."""
    import torch
    rows, heads, dh = t.shape
    wide = torch.full((rows, before + heads * (dh + between) + behind), math.nan, dtype=t.dtype, device=t.device)
    view = wide.as_strided((rows, heads, dh), (wide.stride(0), dh + between, 1), before)
    view.copy_(t)
    return wide, view


# what lies around a row and between its heads: 16-byte chunks everywhere, in x alone, nowhere (odd addresses; odd strides of heads)
PLACES = [((8, 24, 0), (0, 8, 8), (16, 0, 16)), ((8, 8, 0), (3, 5, 0), (0, 0, 0)), ((1, 2, 0), (2, 1, 0), (5, 6, 0)), ((0, 0, 1), (0, 3, 3), (7, 0, 5))]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rot,layout", [(64, "half"), (24, "interleaved"), (20, "half"), (0, "half")])
@pytest.mark.parametrize("places", PLACES)
def test_norm_of_heads_inside_wider_rows(places, rot, layout, dtype):
    """x, y (dx) and dy each with strides of its own; what lies around the outputs stays."""
    import torch
    import paper_2009_09523_amd as vf
    rows, hq, hk, dh = 37, 3, 2, 64
    x, dy = _randn(21, rows, hq + hk, dh, dtype=dtype), _randn(22, rows, hq + hk, dh, dtype=dtype, scale=0.1)
    gq, gk = (1 + 0.2 * _randn(s, dh, dtype=F32).float().double() for s in (23, 24))
    gq, gk = gq.float().double(), gk.float().double()
    xw, xv = _inside(_dev(x, dtype), *places[0])
    dw, dv = _inside(_dev(dy, dtype), *places[1])
    plan = _plan(vf, rot, layout) if rot else None
    ref = _norm_ref(x, dy, hq, gq, gk, float(np.float32(1e-6)), torch.arange(rows) + 9, rot, layout)
    norm, u = (0.5 * 24 + 8) * E, _u(dtype) if dtype == BF16 else 0.0            # as above
    kw = dict(plan=plan, first=9)
    yw, yv = _inside(torch.zeros_like(xv), *places[2])
    vf.vf_qk_norm_rope(xv, yv, hq, gq.float().cuda(), gk.float().cuda(), **kw)
    _close(yv, ref["y"][0], ref["y"][1] * (norm + TURN) + u * ref["y"][0].abs(), "y")
    dgq, dgk = torch.empty(dh, device="cuda"), torch.empty(dh, device="cuda")
    ws = torch.empty(vf.vf_qk_norm_rope_workspace(rows, hq, hk, dh), dtype=torch.uint8, device="cuda")
    gw, gv = _inside(torch.zeros_like(xv), *places[2])
    vf.vf_qk_norm_rope_backward(xv, dv, gv, hq, gq.float().cuda(), gk.float().cuda(), dgq, dgk, ws, **kw)
    _close(gv, ref["dx"][0], ref["dx"][1] * (3 * norm + TURN + 32 * E) + u * ref["dx"][0].abs(), "dx")
    for name, got in (("dgamma_q", dgq), ("dgamma_k", dgk)):
        want, mag = ref[name]
        _close(got, want, mag * (512 * E + norm + TURN), name)
    for wide, view in ((yw, yv), (gw, gv)):
        view.fill_(math.nan)
        assert wide.isnan().all()
    if rot:
        yw, yv = _inside(torch.zeros_like(xv), *places[2])
        vf.vf_rope(xv, yv, plan, first=9)
        want, mag = _turn(x, torch.arange(rows) + 9, rot, layout, _freqs(rot), 1.0)
        _close(yv, want, mag * TURN + u * want.abs(), "rotation")
        yv.fill_(math.nan)
        assert yw.isnan().all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_of_repeated_and_turned_round_tensors(dtype):
    """Heads ahead of rows in memory, and one row or head read for all (stride 0) of x and dy."""
    import torch
    import paper_2009_09523_amd as vf
    rows, hq, hk, dh = 29, 2, 3, 40
    gq, gk = torch.ones(dh, dtype=torch.float64), torch.full((dh,), 0.5, dtype=torch.float64)
    norm, u = (0.5 * 24 + 8) * E, _u(dtype) if dtype == BF16 else 0.0
    plan = _plan(vf, dh, "half")
    for kind in ("heads first", "one row", "one head"):
        x, dy = _randn(31, rows, hq + hk, dh, dtype=dtype), _randn(32, rows, hq + hk, dh, dtype=dtype, scale=0.1)
        if kind == "heads first":
            xd, dd = (_dev(t, dtype).transpose(0, 1).contiguous().transpose(0, 1) for t in (x, dy))
        else:
            one = (lambda t: t[:1]) if kind == "one row" else (lambda t: t[:, :1])
            xd, dd = (_dev(one(t), dtype).expand(rows, hq + hk, dh) for t in (x, dy))
            x, dy = (one(t).expand(rows, hq + hk, dh) for t in (x, dy))
        ref = _norm_ref(x, dy, hq, gq, gk, float(np.float32(1e-6)), torch.arange(rows), dh, "half")
        y, dx = (torch.empty(hq + hk, rows, dh, dtype=_t(dtype), device="cuda").transpose(0, 1) for _ in range(2))
        vf.vf_qk_norm_rope(xd, y, hq, None, gk.float().cuda(), plan=plan)
        vf.vf_qk_norm_rope_backward(xd, dd, dx, hq, None, gk.float().cuda(), plan=plan)
        _close(y, ref["y"][0], ref["y"][1] * (norm + TURN) + u * ref["y"][0].abs(), kind)
        _close(dx, ref["dx"][0], ref["dx"][1] * (3 * norm + TURN + 32 * E) + u * ref["dx"][0].abs(), kind)


@pytest.mark.parametrize("Tk", [70, 4500])
def test_truth_values_as_a_key_mask(Tk):
    """bool and uint8 masks are one; any value but 0 counts as visible."""
    import torch
    import paper_2009_09523_amd as vf
    q, k, v, do = (_dev(t, BF16) for t in _inputs(2, 5, Tk, 2, 2, 64, BF16))
    mask = torch.from_numpy(np.random.Generator(np.random.PCG64(3)).random((2, Tk)) < 0.5).cuda()
    ws = torch.empty(max(1, vf.vf_attention_workspace(q, k, v, backward=True)), dtype=torch.uint8, device="cuda")
    runs = []
    for m in (mask, mask.to(torch.uint8), mask.to(torch.uint8) * 0x40):
        out = [torch.empty_like(q), torch.empty(2, 2, 5, device="cuda"), torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
        vf.vf_attention(q, k, v, out[0], out[1], key_mask=m, workspace=ws)
        vf.vf_attention_backward(q, k, v, out[0], out[1], do, *out[2:], key_mask=m, workspace=ws)
        runs.append(out)
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
    assert (runs[0][3][~mask] == 0).all() and (runs[0][3][mask] != 0).any()
    for bad in (mask.t().contiguous().t(), mask[:, :-1], mask.int()):
        with pytest.raises(vf.VfError):
            vf.vf_attention(q, k, v, runs[0][0], key_mask=bad, workspace=ws)
