"""Host-side checks of the norm and rotation's C ABI: struct layouts, plans,
and every refusal of the calls.  Nothing here reaches a launch: the (fake)
device pointers are refused first."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2310_11960_amd as F

V = F.fma_view_t
FAKE = 1 << 20


def _desc(**kw):
    d = dict(dtype=F.FMA_BF16, heads=4, kv_heads=2, head_dim=64, rotary_dim=64, axes=1, side=0, interleaved=0,
             repeat_kv=0, eps=1e-6, base=10000.0)
    d.update(kw)
    x = F.fma_qk_desc_t(**d)
    x.struct_size = ctypes.sizeof(F.fma_qk_desc_t)
    return x


def _status(fn, *args):
    with pytest.raises(F.FmaError) as e:
        fn(*args)
    assert e.value.args[0].split(": ", 1)[1]
    return e.value.status


@pytest.mark.parametrize("name", ["fma_view_t", "fma_qk_desc_t"])
def test_struct_layouts_match_the_header(name, tmp_path):
    t = getattr(F, name)
    names = [f[0] for f in t._fields_]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "fma.h"\nint main(void){\n'
    src += 'printf("size %%zu\\n", sizeof(%s));\n' % name
    for n in names:
        src += 'printf("%s %%zu\\n", offsetof(%s, %s));\n' % (n, name, n)
    c, exe = str(tmp_path / "probe.c"), str(tmp_path / "probe")
    open(c, "w").write(src + "return 0;}\n")
    subprocess.run(["gcc", "-I", os.path.dirname(F.HEADER_PATH), c, "-o", exe], check=True)
    out = subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()
    got = dict(zip(out[0::2], map(int, out[1::2])))
    assert got["size"] == ctypes.sizeof(t)
    for n in names:
        assert got[n] == getattr(t, n).offset, n


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), F.FMA_ERR_ARG), (dict(heads=0), F.FMA_ERR_SHAPE), (dict(kv_heads=0), F.FMA_ERR_SHAPE),
    (dict(kv_heads=3), F.FMA_ERR_SHAPE), (dict(heads=1 << 15), F.FMA_ERR_SHAPE),
    (dict(head_dim=80), F.FMA_ERR_UNSUPPORTED), (dict(axes=3), F.FMA_ERR_ARG), (dict(axes=0), F.FMA_ERR_ARG),
    (dict(rotary_dim=-16), F.FMA_ERR_SHAPE), (dict(rotary_dim=80), F.FMA_ERR_SHAPE),
    (dict(rotary_dim=24), F.FMA_ERR_UNSUPPORTED), (dict(rotary_dim=48, axes=2), F.FMA_ERR_UNSUPPORTED),
    (dict(side=-1), F.FMA_ERR_SHAPE), (dict(interleaved=2), F.FMA_ERR_ARG), (dict(repeat_kv=-1), F.FMA_ERR_ARG),
    (dict(eps=-1.0), F.FMA_ERR_ARG), (dict(eps=float("nan")), F.FMA_ERR_ARG), (dict(base=0.0), F.FMA_ERR_ARG),
    (dict(base=float("inf")), F.FMA_ERR_ARG)])
def test_plan_refusals(change, status):
    assert _status(F.fma_qk_plan, _desc(**change)) == status


def test_plan_struct_size_rates_and_nulls():
    d = _desc()
    d.struct_size -= 4
    assert _status(F.fma_qk_plan, d) == F.FMA_ERR_ARG
    assert _status(F.fma_qk_plan, _desc(), [0.1] * 31 + [float("nan")]) == F.FMA_ERR_ARG
    F.fma_qk_destroy(F.fma_qk_plan(_desc(base=0.0), [0.1] * 32))      # the rates replace the base
    F.fma_qk_destroy(F.fma_qk_plan(_desc(base=0.0, rotary_dim=0)))
    F.fma_qk_destroy(None)
    assert F.library().fma_qk_plan(None, None, None) == F.FMA_ERR_NULL
    assert _status(F.QKNormRope, 4, None, 64, torch.float16) == F.FMA_ERR_ARG
    with pytest.raises(F.FmaError):
        F.QKNormRope(4, inv_freq=[1.0] * 31)


@pytest.fixture
def plan():
    p = F.fma_qk_plan(_desc())
    yield p
    F.fma_qk_destroy(p)


def _views(n=10, heads=(4, 2, 2), base=FAKE, gap=1 << 20):
    """Token-major inputs and head-major outputs of fake memory."""
    ins = [V(base + i * gap, n * h * 64, 64, h * 64) for i, h in enumerate(heads)]
    outs = [V(base + (i + 4) * gap, n * h * 64, n * 64, 64) for i, h in enumerate(heads)]
    return ins, outs


def _forward(p, ins, outs, B=2, n=10, gq=None, gk=None, pos=None):
    return _status(F.fma_qk_norm_rope, p, B, n, *ins, gq, gk, pos, *outs, 0)


def test_forward_refusals(plan):
    ins, outs = _views()
    assert _forward(None, ins, outs) == F.FMA_ERR_NULL
    assert _forward(plan, ins, outs, B=-1) == F.FMA_ERR_SHAPE
    assert _forward(plan, ins, outs, n=-1) == F.FMA_ERR_SHAPE
    assert _forward(plan, ins, outs, B=1 << 14, n=1 << 14) == F.FMA_ERR_SHAPE
    assert _forward(plan, [None, ins[1], ins[2]], outs) == F.FMA_ERR_NULL
    assert _forward(plan, [V(0, 1, 1, 1), ins[1], ins[2]], outs) == F.FMA_ERR_NULL
    assert _forward(plan, [ins[0], ins[1], None], outs) == F.FMA_ERR_NULL
    assert _forward(plan, ins, [outs[0], outs[1], None]) == F.FMA_ERR_NULL
    for i in range(3):
        for field, value, status in (("data", ins[i].data + 8, F.FMA_ERR_ALIGN),
                                     ("token_stride", ins[i].token_stride + 4, F.FMA_ERR_ALIGN),
                                     ("head_stride", -64, F.FMA_ERR_SHAPE),
                                     ("batch_stride", 1 << 61, F.FMA_ERR_SHAPE)):
            bad, _ = _views()
            setattr(bad[i], field, value)
            assert _forward(plan, bad, outs) == status, (i, field)
        for field, value in (("token_stride", 32), ("head_stride", 0), ("batch_stride", 64)):
            _, bad = _views()
            setattr(bad[i], field, value)
            assert _forward(plan, ins, bad) == F.FMA_ERR_ARG, (i, field)   # rows that share elements
    assert _forward(plan, ins, outs, gq=FAKE + 2) == F.FMA_ERR_ALIGN
    assert _forward(plan, ins, outs, gk=FAKE + 1) == F.FMA_ERR_ALIGN
    assert _forward(plan, ins, outs, pos=FAKE + 2) == F.FMA_ERR_ALIGN


def test_forward_overlaps(plan):
    ins, outs = _views()
    assert _forward(plan, ins, [ins[1], outs[1], outs[2]]) == F.FMA_ERR_ARG
    assert _forward(plan, ins, [V(ins[0].data + 128, 2560, 64, 256), outs[1], outs[2]]) == F.FMA_ERR_ARG
    assert _forward(plan, ins, [outs[0], outs[0], outs[2]]) == F.FMA_ERR_ARG
    assert _forward(plan, ins, [outs[0], outs[1], V(outs[1].data + 128, 1280, 640, 64)]) == F.FMA_ERR_ARG
    # heads of one packed row: neighbours do not share memory, shifted ones do
    row = 8 * 64
    packed = [V(FAKE + 2 * 64 * o, 10 * row, 64, row) for o in (0, 4, 6)]
    shifted = [packed[0], V(FAKE + 2 * 64 * 3, 10 * row, 64, row), packed[2]]
    assert _forward(plan, ins, shifted) == F.FMA_ERR_ARG
    # in place over shared heads that leave repeated
    p = F.fma_qk_plan(_desc(repeat_kv=1))
    assert _forward(p, packed, [packed[0], V(packed[1].data, 10 * row, 64, row), outs[2]]) == F.FMA_ERR_ARG
    F.fma_qk_destroy(p)


def test_maps_need_their_side():
    p = F.fma_qk_plan(_desc(axes=2))
    assert _forward(p, *_views()) == F.FMA_ERR_SHAPE
    F.fma_qk_destroy(p)


def test_empty_calls_need_nothing(plan):
    F.fma_qk_norm_rope(plan, 0, 5, None, None, None, None, None, None, None, None, None, 0)
    F.fma_qk_norm_rope(plan, 3, 0, None, None, None, None, None, None, None, None, None, 0)
    assert F.fma_qk_backward_workspace_size(plan, 0, 100) == 0
    F.fma_qk_norm_rope_backward(plan, 0, 5, *[None] * 13, None, 0, 0)


def test_backward_refusals(plan):
    B, n = 2, 10
    need = F.fma_qk_backward_workspace_size(plan, B, n)
    assert need > 0 and need % (2 * 64 * 4) == 0
    q, k = _views()[0][:2]
    grads = _views(base=FAKE + (8 << 20))[1]
    outs = _views(base=FAKE + (16 << 20))[0]
    ws = FAKE + (40 << 20)

    def call(q=q, k=k, gq=None, gk=None, pos=None, grads=grads, outs=outs, dgq=None, dgk=None, ws=ws, size=need, n=n):
        return _status(F.fma_qk_norm_rope_backward, plan, B, n, q, k, gq, gk, pos, *grads, *outs, dgq, dgk, ws, size, 0)

    assert call(size=need - 1) == F.FMA_ERR_WORKSPACE
    assert call(ws=None) == F.FMA_ERR_WORKSPACE
    assert call(ws=ws + 8) == F.FMA_ERR_ALIGN
    assert call(ws=outs[0].data) == F.FMA_ERR_ARG
    assert call(ws=q.data) == F.FMA_ERR_ARG
    assert call(q=None) == F.FMA_ERR_NULL
    assert call(grads=[grads[0], None, grads[2]]) == F.FMA_ERR_NULL
    assert call(grads=[grads[0], grads[1], None]) == F.FMA_ERR_NULL
    assert call(outs=[outs[0], outs[1], None]) == F.FMA_ERR_NULL
    assert call(outs=[outs[0], outs[0], outs[2]]) == F.FMA_ERR_ARG
    assert call(outs=[k, outs[1], outs[2]]) == F.FMA_ERR_ARG           # dq over k
    assert call(outs=[outs[0], outs[1], q]) == F.FMA_ERR_ARG           # dv over q
    assert call(outs=[V(outs[0].data, 2560, 64, 64), outs[1], outs[2]]) == F.FMA_ERR_ARG
    assert call(dgq=FAKE + 2) == F.FMA_ERR_ALIGN
    assert call(n=1 << 27) == F.FMA_ERR_SHAPE
    assert _status(F.fma_qk_backward_workspace_size, None, 1, 1) == F.FMA_ERR_NULL
    assert _status(F.fma_qk_backward_workspace_size, plan, 1, -1) == F.FMA_ERR_SHAPE


def test_object_refusals():
    """The object API's own checks (shapes, types, devices), on CPU tensors."""
    op = F.QKNormRope(heads=4, kv_heads=2)
    x = torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(F.FmaError) as e:
        op.forward(x, x[:, :, :2])
    assert e.value.status == F.FMA_ERR_ARG and "GPU" in str(e.value)
    with pytest.raises(F.FmaError) as e:
        op.forward(x[0], x[:, :, :2])
    assert e.value.status == F.FMA_ERR_SHAPE
    view = lambda t, shape, dtype=torch.bfloat16: F._view(t, "q", shape, F._TOKEN_MAJOR, dtype, -1)  # noqa: E731
    assert _status(view, x, (1, 3, 2, 64)) == F.FMA_ERR_SHAPE
    assert _status(view, x, (1, 3, 4, 64), torch.float32) == F.FMA_ERR_ARG
    assert _status(view, x.transpose(2, 3), (1, 3, 64, 4)) == F.FMA_ERR_SHAPE
    assert view(x, (1, 3, 4, 64)) == (x.data_ptr(), 768, 64, 256)
