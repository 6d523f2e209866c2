"""Rotary positions with several axes against the fp64 oracle. Tolerance: half a
step of the output's type, and in fp32 8 roundings of |a| + |b| (the angle's
remainder, sine and cosine to about two ulp, two products and a sum)."""
import numpy as np
import pytest

import oracle.block as ob
from gpu_util import torch
from test_gpu_layer_norm import half_step, make, np64

pytestmark = pytest.mark.gpu


def check(x, y, pos, sections, dtype, base=10000.0, **flags):
    X, Y = np64(x), np64(y)
    want = ob.rotary(X, pos.double().cpu().numpy(), sections, base, **flags)
    R = sum(sections)
    lo, hi = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if flags.get("interleaved") else (slice(0, R), slice(R, 2 * R))
    size = np.abs(X[..., lo]) + np.abs(X[..., hi])
    off = np.zeros_like(X)
    off[..., lo] = off[..., hi] = 8 * 2.0 ** -24 * size
    off += half_step(dtype) * (np.abs(want) + off)
    if dtype == "float16":
        off[..., :2 * R] += 2.0 ** -25  # half of fp16's smallest step
    off[..., 2 * R:] = 0
    assert Y.shape == X.shape
    bad = np.abs(Y - want) > off
    assert not bad.any(), (int(bad.sum()), float(np.abs(Y - want).max()))


def positions(N, A, kind, seed, B=None, far=0):
    t = torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    p = t.randint(0, 400, ((B, N, A) if B else (N, A)), generator=g, device="cuda") + far
    return {"int32": p.int(), "int64": p, "float32": p.float() / 4 if far < 1 << 20 else p.float()}[kind]


CASES = [  # B, Hq, Hk, N, d, sections
    (1, 1, 1, 1, 2, (1,)), (2, 3, 1, 37, 64, (8, 12, 12)), (1, 2, 2, 130, 72, (18, 18)), (1, 4, 2, 9, 80, (17, 17)),
    (2, 2, 2, 33, 96, (5, 0, 11)), (1, 2, 1, 50, 35, (3, 4)), (3, 1, 1, 7, 160, (80,)), (1, 1, 1, 300, 256, (128,)),
    (1, 2, 2, 5, 8, (1, 1, 1)), (1, 2, 2, 64, 40, (9,)), (1, 2, 2, 3, 300, (1, 2, 3, 4, 5, 6, 7, 8))]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16", "float32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_shapes(case, interleaved, dtype):
    import paper_2405_15780_amd as va

    B, Hq, Hk, N, d, sections = case
    print(f"case rotary {case} {dtype} interleaved={interleaved}", flush=True)
    q, k = make((B, Hq, N, d), dtype, 1), make((B, Hk, N, d), dtype, 2)
    pos = positions(N, len(sections), "int64", 3)
    for joint in (False, True):
        for inverse in (False, True):
            flags = dict(interleaved=interleaved, joint=joint, inverse=inverse)
            q1, k1 = va.rotary_fwd(q, k, pos, sections, **flags)
            check(q, q1, pos, sections, dtype, **flags)
            check(k, k1, pos, sections, dtype, **flags)


@pytest.mark.parametrize("kind", ["int32", "int64", "float32"])
@pytest.mark.parametrize("far", [0, 1 << 20, (1 << 24) - 500])
def test_positions(kind, far):
    import paper_2405_15780_amd as va

    t = torch()
    q = make((2, 2, 40, 64), "float32", 4)
    sections = (16, 10)
    for B in (None, 2):
        pos = positions(40, 2, kind, 5, B, far)
        check(q, va.rotary_fwd(q, None, pos, sections), pos, sections, "float32")
    # axes first in memory, and one row shared by all tokens
    pos = positions(40, 2, kind, 6, 2, far).permute(2, 0, 1).contiguous().permute(1, 2, 0)
    check(q, va.rotary_fwd(q, None, pos, sections), pos, sections, "float32")
    pos = positions(1, 2, kind, 7, None, far).expand(40, 2)
    check(q, va.rotary_fwd(q, None, pos, sections), pos, sections, "float32")
    if kind == "int64":
        pos = t.full((40, 2), 10 ** 9, device="cuda")
        check(q, va.rotary_fwd(q, None, pos, sections, base=500.0), pos, sections, "float32", base=500.0)
        check(q, va.rotary_fwd(q, None, -pos, sections), -pos, sections, "float32")


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_layouts_in_place_and_views(dtype):
    import paper_2405_15780_amd as va

    t = torch()
    pos, sections = positions(21, 2, "int64", 8), (16, 13)
    qkv = make((2, 21, 3, 4, 64), dtype, 9)  # a fused projection's output
    q, k = (qkv[:, :, i].transpose(1, 2) for i in (0, 1))
    q1, k1 = va.rotary_fwd(q, k, pos, sections)
    check(q, q1, pos, sections, dtype)
    check(k, k1, pos, sections, dtype)
    before = qkv.clone()
    got = va.rotary_fwd(q, k, pos, sections, out=(q, k))
    assert got[0].data_ptr() == q.data_ptr() and t.equal(q, q1) and t.equal(k, k1)
    assert t.equal(qkv[:, :, 2], before[:, :, 2])
    # rows that start anywhere, and an output of another layout
    x = make((2, 3, 21, 71), dtype, 10)[..., 3:68]
    out = t.empty((21, 3, 2, 65), dtype=x.dtype, device="cuda").permute(2, 1, 0, 3)
    va.rotary_fwd(x, None, pos, sections, out=out)
    check(x, out, pos, sections, dtype)
    # queries that share one head's memory
    x = make((2, 1, 21, 64), dtype, 11).expand(2, 5, 21, 64)
    check(x, va.rotary_fwd(x, None, pos, sections), pos, sections, dtype)


def test_many_tokens_take_groups_of_heads():
    """Enough work for several heads per thread: the same bits as head by head."""
    import paper_2405_15780_amd as va

    t = torch()
    q, k = make((1, 19, 40000, 64), "bfloat16", 12, layout=[0, 2, 1, 3]), make((1, 3, 40000, 64), "bfloat16", 13)
    pos = positions(40000, 3, "int32", 14)
    q1, k1 = va.rotary_fwd(q, k, pos, (8, 12, 12))
    for h in (0, 15, 16, 18):
        a = slice(0, 300)
        one = va.rotary_fwd(q[:, h:h + 1, a], None, pos[a], (8, 12, 12))
        assert t.equal(q1[:, h:h + 1, a], one)
        check(q[:, h:h + 1, a], one, pos[a], (8, 12, 12), "bfloat16")
    check(k[:, :, -50:], k1[:, :, -50:], pos[-50:], (8, 12, 12), "bfloat16")


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(interleaved):
    import paper_2405_15780_amd as va

    t = torch()
    pos, sections = positions(17, 3, "int64", 15), (4, 5, 6)
    leaves = [make((2, h, 17, 40), "float32", 16 + h).requires_grad_() for h in (3, 2)]
    q1, k1 = va.rotary(*leaves, pos, sections, interleaved=interleaved)
    gs = [make(tuple(x.shape), "float32", 20).requires_grad_() for x in (q1, k1)]
    grads = t.autograd.grad((q1, k1), leaves, gs, create_graph=True)
    for g, dx in zip(gs, grads):
        check(g, dx, pos, sections, "float32", interleaved=interleaved, inverse=True)
    # the gradient's gradient turns forward again
    v = make((2, 3, 17, 40), "float32", 21)
    back = t.autograd.grad(grads[0], gs[0], v)[0]
    check(v, back, pos, sections, "float32", interleaved=interleaved)
    # one operand, a gradient shared by heads
    x = make((2, 3, 17, 40), "float32", 22).requires_grad_()
    va.rotary(x, None, pos, sections).sum().backward()
    check(t.ones_like(x), x.grad, pos, sections, "float32", inverse=True)


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    q, k = make((1, 2, 5, 16), "bfloat16", 30), make((1, 1, 5, 16), "bfloat16", 31)
    pos = positions(5, 2, "int64", 32)
    ok = (4, 4)
    va.rotary_fwd(q, k, pos, ok)
    for bad in (q.double(), q[0], q.cpu(), q.transpose(2, 3)):
        with pytest.raises(TypeError):
            va.rotary_fwd(bad, None, pos, ok)
    with pytest.raises(TypeError):
        va.rotary_fwd(q, k.float(), pos, ok)
    with pytest.raises(ValueError):
        va.rotary_fwd(q, k[:, :, :4], pos, ok)
    for p in (pos[:4], pos.double(), pos.cpu(), pos[:, :1]):
        with pytest.raises(TypeError):
            va.rotary_fwd(q, k, p, ok)
    for s in ((5, 4), (0, 0), (-1, 2)):
        with pytest.raises(va.VitattnError):
            va.rotary_fwd(q, k, pos, s)
    for base in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(va.VitattnError):
            va.rotary_fwd(q, k, pos, ok, base=base)
    with pytest.raises(va.VitattnError):
        va.rotary_fwd(make((1, 1, 5, 300), "bfloat16", 1), None, pos, (129, 0))
    with pytest.raises(va.VitattnError):  # an output over part of the input
        buf = make((1, 3, 5, 16), "bfloat16", 33)
        va.rotary_fwd(buf[:, :2], None, pos, ok, out=buf[:, 1:])
    with pytest.raises(va.VitattnError):  # heads of the output share memory
        va.rotary_fwd(q, None, pos, ok, out=t.empty((1, 1, 5, 16), dtype=q.dtype, device="cuda").expand(1, 2, 5, 16))
    with pytest.raises(TypeError):
        va.rotary_fwd(q, None, pos, ok, out=t.empty((1, 2, 5, 8), dtype=q.dtype, device="cuda"))


def test_sections_are_whole_numbers_in_range():
    import paper_2405_15780_amd as va

    t = torch()
    q, pos = make((1, 2, 5, 16), "bfloat16", 34), positions(5, 2, "int64", 35)
    want = va.rotary_fwd(q, None, pos, (5, 3))
    for same in ([5, 3], (n for n in (5, 3)), np.array([5, 3]), t.tensor([5, 3]), (5.0, 3.0)):
        assert t.equal(va.rotary_fwd(q, None, pos, same), want)
    with pytest.raises(ValueError):
        va.rotary_fwd(q, None, pos, (5.5, 2.5))
    for bad in ((2 ** 32 + 5, 3), (2 ** 31, 0)):
        with pytest.raises(va.VitattnError):
            va.rotary_fwd(q, None, pos, bad)


@pytest.mark.parametrize("need", ["q", "k", "qk"])
def test_gradient_of_one_operand(need):
    import paper_2405_15780_amd as va

    t = torch()
    pos, sections = positions(17, 2, "int64", 36), (8, 7)
    q, k = make((2, 3, 17, 40), "float32", 37), make((2, 2, 17, 40), "float32", 38)
    leaves = [x.detach().requires_grad_(n in need) for x, n in ((q, "q"), (k, "k"))]
    gs = [make(tuple(x.shape), "float32", 39) for x in leaves]
    out = va.rotary(*leaves, pos, sections)
    t.autograd.backward(out, gs)
    for x, g, n in zip(leaves, gs, "qk"):
        assert x.grad is None if n not in need else t.equal(x.grad, va.rotary_fwd(g, None, pos, sections, inverse=True))


def test_sliding_windows():
    import paper_2405_15780_amd as va

    t = torch()
    long = make((2, 3, 40), "bfloat16", 40)
    q, k = long.unfold(2, 32, 1), long[:, :2].unfold(2, 32, 1)  # [2, 3, 9, 32], rows one element apart
    pos = positions(9, 2, "int64", 41)
    q1, k1 = va.rotary_fwd(q, k, pos, (8, 8))
    check(q, q1, pos, (8, 8), "bfloat16")
    want = va.rotary_fwd(q.contiguous(), k.contiguous(), pos, (8, 8))
    assert t.equal(q1, want[0]) and t.equal(k1, want[1])
