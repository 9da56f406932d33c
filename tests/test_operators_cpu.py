"""Host-side checks of the operators between an attention block's projections that need no GPU: the rotation's
frequencies, workspace sizes, and the refusal of malformed arguments before any device work."""
import ctypes as C
import math
import os
import re

import numpy as np
import pytest

import paper_2009_09523_amd as vf
from paper_2009_09523_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL = binding.VF_EINVAL
P = 1 << 20            # an aligned address that no accepted call would get as far as reading


@pytest.mark.parametrize("rot", [2, 20, 64, 128, 256])
def test_frequencies(rot):
    j = np.arange(rot // 2)
    f = 10000.0 ** (-2.0 * j / rot) / (2 * math.pi)
    plan = vf.vf_rope_make(vf.VF_ROPE_HALF, rot)
    np.testing.assert_allclose(np.array(plan.turns[:rot // 2]), f, rtol=1e-14)
    assert plan.rot_dim == rot and plan.scale == 1.0 and not any(plan.turns[rot // 2:])
    plan = vf.vf_rope_make(vf.VF_ROPE_INTERLEAVED, rot, scaling=vf.VF_ROPE_LINEAR, factor=4.0, scale=0.5)
    np.testing.assert_allclose(np.array(plan.turns[:rot // 2]), f / 4, rtol=1e-14)
    assert plan.layout == vf.VF_ROPE_INTERLEAVED and plan.scale == 0.5


def test_frequencies_by_parts():
    """Fast pairs keep their frequency, slow ones are divided, in between in proportion to the turns over the trained length."""
    rot, L, s = 128, 4096, 16.0
    plan = vf.vf_rope_make(vf.VF_ROPE_HALF, rot, scaling=vf.VF_ROPE_PARTS, factor=s, trained_len=L, beta_fast=32, beta_slow=1)
    f = 10000.0 ** (-2.0 * np.arange(64) / rot) / (2 * math.pi)
    r, got = L * f, np.array(plan.turns[:64])
    np.testing.assert_allclose(got[r >= 32], f[r >= 32], rtol=1e-14)
    np.testing.assert_allclose(got[r <= 1], f[r <= 1] / s, rtol=1e-14)
    mid = (r > 1) & (r < 32)
    keep = (r[mid] - 1) / 31
    assert mid.any()
    np.testing.assert_allclose(got[mid], keep * f[mid] + (1 - keep) * f[mid] / s, rtol=1e-13)


@pytest.mark.parametrize("kw", [dict(layout=2), dict(rot=0), dict(rot=3), dict(rot=258), dict(rot=-2), dict(base=1.0), dict(base=math.nan),
                                dict(base=math.inf), dict(scaling=3), dict(scaling=1, factor=0.0), dict(scaling=1, factor=-1.0),
                                dict(scaling=2, factor=2.0), dict(scaling=2, factor=2.0, trained_len=10, beta_fast=1.0, beta_slow=1.0),
                                dict(scaling=2, factor=math.inf, trained_len=10), dict(scale=math.nan)])
def test_plans_refused(kw):
    a = dict(layout=0, rot=64) | kw
    with pytest.raises(vf.VfError) as e:
        vf.vf_rope_make(a.pop("layout"), a.pop("rot"), **a)
    assert e.value.code == EINVAL


def _rope(**kw):
    a = dict(dtype=1, x=P, x_row=256, x_head=64, y=2 * P, y_row=256, y_head=64, rows=8, heads=4, dh=64, positions=None, first=0, seq_len=0,
             plan=vf.vf_rope_make(0, 64), inverse=0) | kw
    plan = a.pop("plan")
    plan = plan() if callable(plan) else plan
    v = list(a.values())
    return vf.lib().vf_rope(*v[:13], C.byref(plan) if plan is not None else None, v[13], None)


def _bad_plan(**kw):
    """A plan with fields set wrong, made when it is called for (nothing here loads the library at import)."""
    def make():
        p = vf.vf_rope_make(0, 64)
        for k, v in kw.items():
            setattr(p, k, v)
        return p
    return make


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(x=None), dict(y=None), dict(x=P + 1), dict(y=P + 1), dict(rows=-1), dict(rows=1 << 31),
                                dict(heads=-1), dict(heads=65536), dict(dh=62), dict(dh=513), dict(dh=0), dict(seq_len=-1), dict(plan=None),
                                dict(y_row=0), dict(y_head=0), dict(y_head=32), dict(y_row=255), dict(y_row=-256), dict(y=P, y_row=512),
                                dict(y=P, x_head=0), dict(plan=_bad_plan(layout=5)), dict(plan=_bad_plan(rot_dim=63)),
                                dict(plan=_bad_plan(rot_dim=0)), dict(plan=_bad_plan(rot_dim=258), dh=512, x_head=512, y_head=512, y_row=2048)])
def test_rotation_refused(kw):
    assert _rope(**kw) == EINVAL


def test_nothing_to_turn_is_a_no_op():
    assert _rope(rows=0, x=None, y=None) == 0 and _rope(heads=0) == 0


def _norm(backward=False, **kw):
    a = dict(dtype=1, x=P, x_row=512, x_head=64)
    if backward:
        a |= dict(dy=3 * P, dy_row=512, dy_head=64)
    a |= dict(y=2 * P, y_row=512, y_head=64, rows=8, hq=4, hk=4, dh=64, gq=None, gk=None, eps=1e-6, positions=None, first=0, seq_len=0,
              plan=vf.vf_rope_make(0, 64))
    if backward:
        a |= dict(dgq=None, dgk=None, alpha=1.0, accumulate=0, ws=None, ws_bytes=0)
    a |= kw
    plan = a["plan"]() if callable(a["plan"]) else a["plan"]
    a["plan"] = C.byref(plan) if plan is not None else None
    f = vf.lib().vf_qk_norm_rope_backward if backward else vf.lib().vf_qk_norm_rope
    return f(*a.values(), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [dict(dtype=7), dict(x=None), dict(y=None), dict(hq=-1), dict(hk=-1), dict(hq=65535, hk=1), dict(eps=-1.0),
                                dict(eps=math.nan), dict(dh=32), dict(y_head=0), dict(y=P, y_row=1024), dict(rows=-3), dict(seq_len=-2),
                                dict(plan=_bad_plan(rot_dim=66))])
def test_norm_refused(backward, kw):
    assert _norm(backward, **kw) == EINVAL


def test_norm_backward_refused():
    need = vf.vf_qk_norm_rope_workspace(8, 4, 4, 64)
    assert need > 0 and need % 4 == 0
    for kw in (dict(dy=None), dict(dy=P + 1), dict(dgq=P), dict(dgq=P, ws=P, ws_bytes=need - 1), dict(dgq=P, ws=P + 4, ws_bytes=need),
               dict(dgq=P, dgk=P, ws=P, ws_bytes=need), dict(y=3 * P, y_row=1024)):
        assert _norm(True, **kw) == EINVAL, kw
    for bad in ((-1, 1, 1, 64), (4, -1, 1, 64), (4, 1, 1, 0), (4, 1, 1, 513), (4, 65535, 1, 64), (1 << 31, 1, 1, 64)):
        with pytest.raises(vf.VfError):
            vf.vf_qk_norm_rope_workspace(*bad)


def _shape(**kw):
    a = dict(dtype=1, batch=2, q_rows=10, k_rows=20, q_heads=4, kv_heads=2, d_head=64, scale=0.125)
    lay = {n: kw.pop(n, None) for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv")}
    s = binding.VfAttnShape(*(a | kw).values())
    for n, l in lay.items():
        rows, heads = (s.q_rows, s.q_heads) if n in ("q", "o", "d_o", "dq") else (s.k_rows, s.kv_heads)
        setattr(s, n, binding.VfAttnLayout(*(l or (rows * heads * s.d_head, heads * s.d_head, s.d_head))))
    return s


def _forward(s, q=P, k=P, v=P, o=2 * P, lse=None, ws=P, bytes=1 << 40):
    return vf.lib().vf_attention(C.byref(s) if s is not None else None, q, k, v, None, None, None, o, lse, ws, bytes, None)


def _backward(s, q=P, k=P, v=P, o=P, lse=P, d_o=P, dq=2 * P, dk=3 * P, dv=4 * P, ws=P, bytes=1 << 40):
    return vf.lib().vf_attention_backward(C.byref(s) if s is not None else None, q, k, v, None, None, None, o, lse, d_o, dq, dk, dv, ws, bytes, None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(batch=-1), dict(q_rows=-1), dict(k_rows=-1), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=3),
                                dict(d_head=0), dict(d_head=4), dict(d_head=60), dict(d_head=136), dict(scale=0.0), dict(scale=-1.0),
                                dict(scale=math.nan), dict(scale=math.inf), dict(q_rows=1 << 30), dict(batch=1 << 23),
                                dict(q=(5120, 252, 64)), dict(k=(2560, 128, 4)), dict(v=(2561, 128, 64))])
def test_attention_shapes_refused(kw):
    s = _shape(**kw)
    assert _forward(s) == EINVAL and _backward(s) == EINVAL


def test_attention_refused():
    s = _shape()
    assert _forward(None) == EINVAL and _backward(None) == EINVAL and vf.lib().vf_attention_workspace(None, 0) == EINVAL
    for n in ("q", "k", "v", "o"):
        assert _forward(s, **{n: None}) == EINVAL and _forward(s, **{n: P + 8}) == EINVAL, n
    for n in ("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "ws"):
        assert _backward(s, **{n: None}) == EINVAL, n
    for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv", "ws"):
        assert _backward(s, **{n: P + 8}) == EINVAL, n
    assert _backward(s, bytes=vf.lib().vf_attention_workspace(C.byref(s), 1) - 1) == EINVAL
    # outputs whose entries coincide
    assert _forward(_shape(o=(0, 256, 64))) == EINVAL and _forward(_shape(o=(2560, 256, 32))) == EINVAL
    for n, l in (("dq", (2560, 0, 64)), ("dk", (0, 128, 64)), ("dv", (2560, 128, 0)), ("dk", (2560, 64, 64))):
        assert _backward(_shape(**{n: l})) == EINVAL, n


def test_attention_refuses_outputs_in_place():
    s = _shape()
    for n in ("q", "k", "v"):
        assert _forward(s, **{"q": 3 * P, "k": 4 * P, "v": 5 * P, n: 2 * P}) == EINVAL, n
    apart = dict(zip(("q", "k", "v", "o", "d_o", "dq", "dk", "dv"), range(P, 9 * P, P)))
    for out in ("dq", "dk", "dv"):
        for n in apart:
            if n != out:
                assert _backward(s, **(apart | {out: apart[n]})) == EINVAL, (out, n)


def test_sizes_beyond_32_bits_are_refused():
    with pytest.raises(vf.VfError):
        vf.vf_qk_norm_rope_workspace(4, (1 << 32) + 1, 1, 64)


def test_nothing_to_attend_is_a_no_op():
    assert _forward(_shape(batch=0), None, None, None, None, ws=None, bytes=0) == 0
    assert _forward(_shape(q_rows=0), None, P, P, None, ws=None, bytes=0) == 0
    assert _backward(_shape(batch=0), *[None] * 9, ws=None, bytes=0) == 0


def test_structures_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vf.h")).read(), flags=re.S)
    for name, cls in (("vf_rope_plan", binding.VfRopePlan), ("vf_attn_layout", binding.VfAttnLayout), ("vf_attn_shape", binding.VfAttnShape)):
        body = text[text.index("typedef struct %s {" % name):text.index("} %s;" % name)].split("{", 1)[1]
        names = [re.sub(r"\[.*\]", "", n.strip()) for d in body.split(";") if len(d.split(None, 1)) == 2 for n in d.split(None, 1)[1].split(",")]
        assert names == [f[0] for f in cls._fields_]
    assert binding._ATTN_SHAPE.size == C.sizeof(binding.VfAttnShape)
    packed = binding.VfAttnShape.from_buffer_copy(binding._ATTN_SHAPE.pack(*range(7), 0.5, *range(24)))
    assert packed.d_head == 6 and packed.scale == 0.5 and packed.q.batch == 0 and packed.d_o.row == 13 and packed.dv.head == 23


def test_binding_refuses_tensors_that_are_not_on_the_device():
    import torch
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a device")
    x = torch.zeros(4, 2, 64)
    q = torch.zeros(1, 4, 2, 64)
    for call in (lambda: vf.vf_rope(x, x, vf.vf_rope_make(0, 64)), lambda: vf.vf_qk_norm_rope(x, x, 1),
                 lambda: vf.vf_qk_norm_rope_backward(x, x, x, 1), lambda: vf.vf_attention(q, q, q, q),
                 lambda: vf.vf_attention_backward(q, q, q, q, torch.zeros(1, 2, 4), q, q, q, q)):
        with pytest.raises(vf.VfError) as e:
            call()
        assert e.value.code == EINVAL


@pytest.mark.parametrize("sizes", [((1 << 64) + 4, 1, 1, 64), (-(1 << 64) + 4, 1, 1, 64), (4, 1 - (1 << 32), 1, 64), (4, 1, 1 - (1 << 32), 64),
                                   (4, 1, 1, 64 - (1 << 32)), (4, 1, 1, 64 + (1 << 32))])
def test_workspaces_of_sizes_that_an_argument_does_not_hold_are_refused(sizes):
    """Each of them is (4, 1, 1, 64) once cut to its argument's width."""
    with pytest.raises(vf.VfError) as e:
        vf.vf_qk_norm_rope_workspace(*sizes)
    assert e.value.code == EINVAL


@pytest.mark.parametrize("kw", [dict(layout=1 << 32), dict(rot=64 + (1 << 32)), dict(rot=64 - (1 << 32)), dict(scaling=1 << 32),
                                dict(scaling=2, factor=2.0, trained_len=(1 << 64) + 9)])
def test_plans_of_numbers_that_an_argument_does_not_hold_are_refused(kw):
    a = dict(layout=0, rot=64) | kw
    with pytest.raises(vf.VfError) as e:
        vf.vf_rope_make(a.pop("layout"), a.pop("rot"), **a)
    assert e.value.code == EINVAL


@pytest.mark.parametrize("kw", [dict(scale=1e300), dict(scale=-1e39), dict(scale=math.inf), dict(scaling=1, factor=1e-320),
                                dict(scaling=2, factor=1e-320, trained_len=4096)])
def test_plans_that_come_out_infinite_are_refused(kw):
    with pytest.raises(vf.VfError) as e:
        vf.vf_rope_make(0, 64, **kw)
    assert e.value.code == EINVAL


@pytest.mark.parametrize("backward", [False, True])
def test_an_infinite_eps_is_refused(backward):
    """(Also what a number beyond fp32 becomes in the call: every head would come out as zeros.)"""
    assert _norm(backward, eps=math.inf) == EINVAL and _norm(backward, eps=1e39) == EINVAL


@pytest.mark.parametrize("first", [(1 << 52) + 1, -(1 << 52) - 1, (1 << 63) - 1])
def test_positions_that_float64_does_not_hold_are_refused(first):
    for call in (_rope, _norm, lambda **kw: _norm(True, **kw)):
        assert call(first=first) == EINVAL
    assert _rope(first=1 << 52, rows=0) == 0 and _norm(first=-(1 << 52), rows=0) == 0


def test_scales_and_heads_that_the_attention_call_cannot_take_are_its_own_errors():
    """No errors of the packing below: a scale beyond fp32, and the default scale of heads without elements."""
    import torch
    q = torch.zeros(1, 2, 1, 64)
    for scale in (1e39, -1.0, 0.0, math.nan, math.inf):
        with pytest.raises(vf.VfError) as e:
            binding._ATTN_SHAPE.pack(*binding._attn_sizes("vf_attention", 1, q, q, q, scale), *range(24))
        assert e.value.code == EINVAL
    none = torch.zeros(1, 2, 1, 0)
    s = binding.VfAttnShape.from_buffer_copy(binding._ATTN_SHAPE.pack(*binding._attn_sizes("vf_attention", 1, none, none, none, None), *range(24)))
    assert vf.lib().vf_attention_workspace(C.byref(s), 0) == EINVAL


def test_only_calls_that_use_a_workspace_need_one():
    """Bits of a long mask, and parts: the plainest forward call needs none."""
    need = lambda s, b: vf.lib().vf_attention_workspace(C.byref(s), b)  # noqa: E731
    short, long = _shape(batch=8, q_rows=512, k_rows=4096, q_heads=8, kv_heads=8), _shape(batch=8, q_rows=512, k_rows=4500, q_heads=8, kv_heads=8)
    rows = 8 * 8 * 512 * 4
    assert need(short, 0) == 0 and need(short, 1) == 2 * rows
    bits = -(-8 * 71 * 8 // 16) * 16
    assert need(long, 0) == bits and need(long, 1) == 2 * rows + bits

    def forward(mask, ws, size):
        return vf.lib().vf_attention(C.byref(long), P, P, P, None, None, mask, 2 * P, None, ws, size, None)
    assert forward(3 * P, None, 0) == EINVAL and forward(3 * P, 4 * P, bits - 1) == EINVAL
    assert _backward(long, bytes=2 * rows - 1) == EINVAL and _backward(long, ws=None, bytes=0) == EINVAL


@pytest.mark.parametrize("fits,beyond", [
    (dict(batch=1, q_heads=128, kv_heads=1, q_rows=65535), dict(q_rows=65536)),                   # rows of a problem: 8388480
    (dict(batch=1, q_heads=1, kv_heads=1, q_rows=8388480), dict(q_rows=8388481)),
    (dict(batch=1, q_heads=1, kv_heads=1, k_rows=8388480), dict(k_rows=8388481)),
    (dict(batch=1 << 23, q_heads=1, kv_heads=1, q_rows=1, k_rows=1), dict(batch=(1 << 23) + 1)),
    (dict(batch=1 << 20, q_heads=8, kv_heads=8, q_rows=1, k_rows=1), dict(batch=(1 << 20) + 1)),
    (dict(batch=1, q_heads=1024, kv_heads=1, q_rows=2047), dict(q_rows=2048)),                    # 1024^2 rows: 2^31
    (dict(batch=4096, q_heads=1, kv_heads=1, q_rows=1, k_rows=524287), dict(k_rows=524288)),
    (dict(batch=4096, q_heads=4, kv_heads=1, q_rows=131071, k_rows=1), dict(q_rows=131072)),
    (dict(batch=1, q_heads=1, kv_heads=1), dict(q_heads=(1 << 31) - 1, q_rows=(1 << 31) - 1)),    # products beyond 64 bits
])
def test_largest_attention_that_is_taken(fits, beyond):
    for backward in (0, 1):
        assert vf.lib().vf_attention_workspace(C.byref(_shape(**fits)), backward) >= 0
        assert vf.lib().vf_attention_workspace(C.byref(_shape(**(fits | beyond))), backward) == EINVAL
    assert _forward(_shape(**(fits | beyond))) == EINVAL and _backward(_shape(**(fits | beyond))) == EINVAL
