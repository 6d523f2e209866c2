"""The rms norm with the residual's addition and dropout, forward, backward and in 8
bits, against the fp64 oracle, element by element: half a step of a type for each
rounding, and the fp32 sums of a lane (up to 64 values) with a tree over the lanes."""
import numpy as np
import pytest

import oracle.sparse as os_
from gpu_util import torch
from test_gpu_layer_norm import close, half_step, make, np64

pytestmark = pytest.mark.gpu

EPS = 1e-5
F = 2.0 ** -24
N_SUM = 96  # fp32 additions in a row's sum, rounded up
TYPES = [("bfloat16", "bfloat16"), ("bfloat16", "float32"), ("float16", "float16"), ("float16", "float32"), ("float32", "float32")]


def tiny(dtype):
    return 2.0 ** -24 if dtype == "float16" else 1e-37  # fp16's smallest step


def step_of(x, dtype):
    return half_step(dtype) * np.abs(x) + tiny(dtype)


def case(shape, dtype, rtype, seed, weight=True, residual=True, layout=None):
    x, res, dy, dh = (make(shape, t, seed + i, 0.2, 1.0, layout) for i, t in enumerate((dtype, rtype, dtype, rtype)))
    w = make(shape[-1:], dtype, seed + 9, 1.0, 0.3) if weight else None
    return x, w, res if residual else None, dy, dh


def check(x, w, res, dy, dh, p=0.0, rng=None, eps=EPS):
    import paper_2405_15780_amd as va

    t = torch()
    y, h, rstd = va.rms_norm_fwd(x, w, res, eps, p, rng)
    dx, dres, dw = va.rms_norm_bwd(h, w, rstd, dy, dh, p, rng)
    t.cuda.synchronize()
    dtype, rtype = str(x.dtype)[6:], str(h.dtype)[6:]
    X, DY = np64(x), np64(dy)
    state = rng.tolist() if isinstance(rng, t.Tensor) else rng
    m = 1.0
    if p:
        keep, up = os_.kept(X.shape, p, *state)
        m = keep * up
    if res is None:
        assert h is x
    else:
        H = np64(res) + m * X
        off = 3 * F * (np.abs(H) + np.abs(m * X))  # (the factor, the sum)
        close(h, H, off + half_step(rtype) * (np.abs(H) + off) + tiny(rtype), "h")
    # the rest from h as it is stored
    H, W = np64(h), None if w is None else np64(w)
    Y, R = os_.rms_norm(H, W, eps)
    rel = F * (N_SUM + 8)
    close(y, Y, rel * np.abs(Y) + half_step(dtype) * np.abs(Y) * (1 + rel) + tiny(dtype), "y")
    close(rstd, R, rel * R, "rstd")
    DH, DW = os_.rms_norm_backward(H, W, eps, DY)
    g, n = np.abs(DY if W is None else DY * W), np.abs(H * R[..., None])
    grad = DH + (0.0 if dh is None else np64(dh))
    off = rel * (R[..., None] * (g + n * (g * n).mean(-1, keepdims=True)) + np.abs(grad) + np.abs(grad - DH))
    close(dres, grad, off + half_step(rtype) * (np.abs(grad) + off) + tiny(rtype), "dres")
    close(dx, m * grad, m * off + half_step(dtype) * (np.abs(m * grad) * (1 + 2 * F) + m * off) + 2 * F * np.abs(m * grad) + tiny(dtype), "dx")
    if w is not None:
        rows = X.size // X.shape[-1]
        off = (rel + F * (rows // 256 + 1100)) * (np.abs(DY) * n).sum(tuple(range(X.ndim - 1)))
        close(dw, DW, off + half_step(str(w.dtype)[6:]) * (np.abs(DW) + off) + 1e-7, "dw")
    return y, h, dx, dres, dw


@pytest.mark.parametrize("dtype,rtype", TYPES)
@pytest.mark.parametrize("D", [1, 2, 3, 4, 5, 7, 8, 9, 31, 64, 72, 127, 257, 511, 513, 768, 1025, 1537, 2048, 4099, 8192])
def test_widths(dtype, rtype, D):
    print(f"case rms D={D} {dtype} {rtype}", flush=True)
    check(*case((3, 7, D), dtype, rtype, D))
    check(*case((37, D), dtype, rtype, D + 1), p=0.3, rng=(D, 2 ** 33 + 5))


@pytest.mark.parametrize("D", [12000, 16383, 16384])
def test_widest(D):
    print(f"case rms D={D}", flush=True)
    check(*case((5, D), "bfloat16", "bfloat16", D), p=0.5, rng=(1, 2))
    check(*case((5, D), "float16", "float32", D))


@pytest.mark.parametrize("rows", [1, 2, 63, 64, 65, 1000, 4099])
@pytest.mark.parametrize("D", [72, 1024, 1537])
def test_rows(rows, D):
    print(f"case rms rows={rows} D={D}", flush=True)
    check(*case((rows, D), "bfloat16", "bfloat16", rows), p=0.1, rng=(rows, 0))


@pytest.mark.parametrize("layout", [[1, 0, 2, 3], [0, 2, 1, 3], [2, 1, 0, 3]])
def test_other_orders(layout):
    """Rows in another order than their indexes: the mask and the statistics go by the indexes."""
    import paper_2405_15780_amd as va

    t = torch()
    shape = (3, 5, 11, 40)
    a = case(shape, "bfloat16", "bfloat16", 3, layout=layout)
    got = check(*a, p=0.4, rng=(7, 8))
    dense = [None if x is None else x.contiguous() for x in a]
    want = check(*dense, p=0.4, rng=(7, 8))
    assert all(t.equal(x, y) for x, y in zip(got, want))
    # a residual in an order of its own, rows with a pitch, more than four dims
    x, w, res, dy, dh = dense
    wide = t.zeros((3, 5, 11, 47), dtype=x.dtype, device="cuda")[..., 3:43]
    wide.copy_(x)
    other = check(wide, w, a[2], dy, a[4], p=0.4, rng=(7, 8))
    assert all(t.equal(x, y) for x, y in zip(other, want))
    five = [None if v is None or v is w else v.reshape(3, 5, 1, 11, 40) for v in (x, w, res, dy, dh)]
    five[1] = w
    y, h, _ = va.rms_norm_fwd(five[0], w, five[2], EPS, 0.4, (7, 8))
    assert t.equal(y.view(shape), want[0]) and t.equal(h.view(shape), want[1])


def test_without_weight_or_residual():
    check(*case((9, 130), "bfloat16", "bfloat16", 1, weight=False))
    check(*case((9, 130), "float32", "float32", 2, residual=False))
    x, w, _, dy, _ = case((9, 130), "float16", "float16", 3, residual=False)
    check(x, w, None, dy, None)
    x, w, res, dy, _ = case((9, 130), "bfloat16", "bfloat16", 4)
    check(x, w.float(), res, dy, None, p=0.2, rng=(3, 4))


def test_parts_are_those_of_the_whole():
    """A row's bits do not depend on the call; unwanted gradients are None; in place."""
    import paper_2405_15780_amd as va

    t = torch()
    x, w, res, dy, dh = case((64, 1024), "bfloat16", "bfloat16", 5)
    y, h, rstd = va.rms_norm_fwd(x, w, res, EPS, 0.25, (9, 1))
    one = va.rms_norm_fwd(x[:1], w, res[:1], EPS, 0.25, (9, 1))
    assert all(t.equal(a[:1], b) for a, b in zip((y, h, rstd), one))
    dx, dres, dw = va.rms_norm_bwd(h, w, rstd, dy, dh, 0.25, (9, 1))
    for i in range(3):
        want = [False] * 3
        want[i] = True
        part = va.rms_norm_bwd(h, w, rstd, dy, dh, 0.25, (9, 1), *want)
        assert all((b is None) != want[k] for k, b in enumerate(part)) and t.equal(part[i], (dx, dres, dw)[i])
    a = va.rms_norm_bwd(h, w, rstd, dy, dh)
    assert a[0] is a[1]
    x2, r2 = x.clone(), res.clone()
    va.rms_norm_fwd(x2, w, r2, EPS, 0.25, (9, 1), out=(x2, r2))
    assert t.equal(x2, y) and t.equal(r2, h)
    assert va.rms_norm_fwd(x, w, res, stats=False)[2] is None


def test_values_at_the_ends():
    """Zeros, huge and tiny rows, NaN and infinities in dropped places and in kept ones."""
    import paper_2405_15780_amd as va

    t = torch()
    x = t.zeros(4, 64, device="cuda", dtype=t.bfloat16)
    res = t.zeros(4, 64, device="cuda", dtype=t.bfloat16)
    x[1], x[2, 5] = 1e-30, 3e4
    y, h, rstd = va.rms_norm_fwd(x, None, res, 1e-6)
    assert (y[0] == 0).all() and t.isfinite(y).all() and abs(rstd[0].item() - 1e3) < 1e-2
    keep = t.from_numpy(os_.kept((4, 64), 0.5, 1, 2)[0]).cuda()
    x = t.where(keep, t.ones_like(x), t.full_like(x, float("nan")))
    y, h, _ = va.rms_norm_fwd(x, None, res, 1e-6, 0.5, (1, 2))
    assert t.isfinite(y).all() and t.equal(h, t.where(keep, 2.0, 0.0).to(h.dtype))
    x[2, int(keep[2].nonzero()[0])] = float("inf")
    y, h, _ = va.rms_norm_fwd(x, None, res, 1e-6, 0.5, (1, 2))
    assert t.isfinite(y[[0, 1, 3]]).all() and not t.isfinite(y[2]).all()
    y8, scale, _ = va.rms_norm_fp8(x.nan_to_num(0, 0, 0), None, res)
    assert t.isfinite(y8.float()).all()
    z, s, _ = va.rms_norm_fp8(t.zeros_like(x), None, res)
    assert (z.float() == 0).all() and (s == 2.0 ** -126).all()


@pytest.mark.parametrize("dtype,rtype", TYPES)
@pytest.mark.parametrize("D", [1, 8, 33, 72, 128, 200, 768, 1537, 2048, 5000])
@pytest.mark.parametrize("group", [None, 32, 64, 128])
def test_eight_bits(dtype, rtype, D, group):
    import paper_2405_15780_amd as va

    t = torch()
    print(f"case fp8 D={D} {dtype} {rtype} group={group}", flush=True)
    x, w, res, _, _ = case((23, D), dtype, rtype, D)
    y, scale, h = va.rms_norm_fp8(x, w, res, EPS, group)
    plain, h2, _ = va.rms_norm_fwd(x, w, res, EPS)
    assert y.dtype == t.float8_e4m3fn and t.equal(h, h2)
    Y, _ = os_.rms_norm(np64(h), np64(w), EPS)
    G = group or D
    n = -(-D // G)
    top = np.abs(np.pad(Y, ((0, 0), (0, n * G - D)))).reshape(23, n, G).max(-1)
    want = np.maximum(top / 448, 2.0 ** -126)
    rel = F * (N_SUM + 12)
    close(scale, want if group else want[:, 0], rel * (want if group else want[:, 0]), "scale")
    v = Y / np.repeat(want, G, 1)[:, :D]
    off = 2.0 ** -4 * np.abs(v) + 2.0 ** -10 + 2 * rel * np.abs(v) * (1 + 2.0 ** -4)  # half a step, of the least too
    close(y.float(), v, off, "y")
    assert np.abs(np64(y.float())).max() <= 448


@pytest.mark.parametrize("D,group", [(64, None), (256, 32), (1024, 64), (2048, 128), (2048, None), (8192, 128), (8192, None)])
@pytest.mark.parametrize("dtype,rtype", TYPES)
def test_eight_bits_round_once(dtype, rtype, D, group):
    """Rows of +-1, whose norm is 1, so that |y| is the weight: values on and beside the middle between two bytes go
    where y / scale is, to the even one in the middle (y, scale and their products with a middle are exact in fp64)."""
    import paper_2405_15780_amd as va

    t = torch()
    print(f"case fp8 once D={D} group={group} {dtype} {rtype}", flush=True)
    values = np.arange(127, dtype=np.uint8)  # magnitudes 0 .. 448 by their bytes
    values = t.from_numpy(values).view(t.float8_e4m3fn).double().numpy()
    middles = (values[1:] + values[:-1]) / 2
    rng = np.random.default_rng(D)
    G = group or D
    w = np.zeros(D, dtype=np.float32)
    for g in range(D // G):
        # the largest of the group: any, powers of two (ties that are met), scales at and near the least one
        top = np.float32([rng.uniform(0.5, 2) * 10.0 ** rng.integers(-30, 30), 448 * 2.0 ** rng.integers(-60, 60),
                          448 * 2.0 ** -126 * rng.uniform(0.3, 8)][g % 3])
        s = np.maximum(top / np.float32(448), np.float32(2.0 ** -126))
        x = (rng.choice(middles, G) * float(s)).astype(np.float32)
        for _ in range(3):  # up to three steps beside the nearest
            x = np.where(rng.random(G) < 0.3, np.nextafter(x, rng.choice(np.float32([0, np.inf]), G)), x)
        w[g * G:(g + 1) * G] = np.minimum(x, top)
        w[g * G + rng.integers(G)] = top
    sign = t.from_numpy(rng.choice([-1.0, 1.0], (5, D))).cuda()
    x, res = t.zeros((5, D), dtype=getattr(t, dtype), device="cuda"), sign.to(getattr(t, rtype))
    assert (va.rms_norm_fwd(x, None, res, 0.0)[2] == 1).all()
    y, scale, _ = va.rms_norm_fp8(x, t.from_numpy(w).cuda(), res, 0.0, group)
    want = np.maximum(w.reshape(-1, G).max(1) / np.float32(448), np.float32(2.0 ** -126))
    assert np.array_equal(scale.cpu().numpy().reshape(5, -1), np.tile(want, (5, 1)))
    edge = middles * want.astype(np.float64).repeat(G)[:, None]
    above, met = (w[:, None] > edge).sum(1), (w[:, None] == edge).any(1)
    byte = above + (met & (above % 2 == 1))
    got = y.view(t.uint8).cpu().numpy()
    assert np.array_equal(got & 127, np.tile(byte, (5, 1))), int(((got & 127) != byte).sum())
    assert np.array_equal(got >> 7, (sign < 0).cpu().numpy().astype(np.uint8))


def test_eight_bits_of_other_layouts():
    import paper_2405_15780_amd as va

    t = torch()
    a = case((2, 3, 17, 96), "bfloat16", "float32", 8, layout=[0, 2, 1, 3])
    y, s, h = va.rms_norm_fp8(a[0], a[1], a[2], group=64)
    y2, s2, h2 = va.rms_norm_fp8(a[0].contiguous(), a[1], a[2].contiguous(), group=64)
    assert t.equal(y.float(), y2.float()) and t.equal(s, s2) and t.equal(h, h2) and s.shape == (2, 3, 17, 2)
    y3, s3, h3 = va.rms_norm_fp8(a[0], a[1])
    assert h3 is a[0] and s3.shape == (2, 3, 17)


def test_autograd():
    """Gradients through the function against torch's in fp64, for y alone, h alone and both."""
    import paper_2405_15780_amd as va

    t = torch()
    x, w, res, dy, dh = case((6, 5, 48), "float32", "float32", 6)
    keep, up = os_.kept((6, 5, 48), 0.3, 5, 6)
    m = t.from_numpy(keep * up).cuda()
    for use in ("y", "h", "both"):
        ours = [v.detach().clone().requires_grad_() for v in (x, w, res)]
        refs = [v.detach().double().requires_grad_() for v in (x, w, res)]
        y, h = va.rms_norm(*ours, eps=EPS, p=0.3, rng=(5, 6))
        H = refs[2] + m * refs[0]
        Y = H * (H.square().mean(-1, keepdim=True) + EPS).rsqrt() * refs[1]
        loss, ref = 0.0, 0.0
        if use != "h":
            loss, ref = loss + (y * dy).sum(), ref + (Y * dy).sum()
        if use != "y":
            loss, ref = loss + (h * dh).sum(), ref + (H * dh).sum()
        loss.backward()
        ref.backward()
        for a, b in zip(ours, refs):
            want = t.zeros_like(b) if b.grad is None else b.grad
            assert (a.grad.double() - want).abs().max() <= 2e-5 * want.abs().max() + 1e-12, use
    y = va.rms_norm(x.requires_grad_(), w)
    y.sum().backward()
    assert x.grad is not None
    with t.no_grad():
        assert not va.rms_norm(x, w, res)[0].requires_grad


def test_a_state_on_the_device():
    """The same mask as from numbers; a change between forward and backward is found."""
    import paper_2405_15780_amd as va

    t = torch()
    x, w, res, dy, dh = case((31, 200), "bfloat16", "bfloat16", 7)
    state = t.tensor([-5, 2 ** 62 + 1], device="cuda")
    a, b = check(x, w, res, dy, dh, 0.2, state), check(x, w, res, dy, dh, 0.2, (-5, 2 ** 62 + 1))
    assert all(t.equal(u, v) for u, v in zip(a, b))
    y, h = va.rms_norm(x.requires_grad_(), w, res, p=0.2, rng=state)
    state += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (y.float().sum() + h.float().sum()).backward()


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    x, w, res, dy, dh = case((6, 64), "bfloat16", "bfloat16", 8)
    bad = [(TypeError, lambda: va.rms_norm_fwd(x, w[:-1], res)), (TypeError, lambda: va.rms_norm_fwd(x, w.half(), res)),
           (TypeError, lambda: va.rms_norm_fwd(x, w, res.half())), (TypeError, lambda: va.rms_norm_fwd(x, w, res[:3])),
           (TypeError, lambda: va.rms_norm_fwd(x.t(), None)), (TypeError, lambda: va.rms_norm_fwd(x.double(), None)),
           (ValueError, lambda: va.rms_norm_fwd(x, w, res, p=0.1)), (va.VitattnError, lambda: va.rms_norm_fwd(x, w, p=0.1, rng=(1, 2))),
           (TypeError, lambda: va.rms_norm_fwd(x, w, res, p=0.1, rng=t.zeros(2, device="cuda"))),
           (TypeError, lambda: va.rms_norm_fwd(x, w, res, p=0.1, rng=t.zeros(2, dtype=t.int64))),
           (ValueError, lambda: va.rms_norm_fwd(x[:0], w, res[:0])), (ValueError, lambda: va.rms_norm_fp8(x, w, res, group=16)),
           (va.VitattnError, lambda: va.rms_norm_fwd(t.zeros(2, 16385, device="cuda", dtype=t.bfloat16))),
           (va.VitattnError, lambda: va.rms_norm_fwd(x, w, res, out=(x, x))),
           (va.VitattnError, lambda: va.rms_norm_fwd(x, w, res, out=(res, x))),
           (TypeError, lambda: va.rms_norm_fwd(t._neg_view(x.float()))), (TypeError, lambda: va.rms_norm_bwd(x, w, dy, dy)),
           (TypeError, lambda: va.rms_norm_bwd(x, w, t.zeros(6, device="cuda"), dy.half()))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("not refused", i)
    leaf = x.clone().requires_grad_() * 1.0
    with pytest.raises(ValueError):
        va.rms_norm_fwd(x, w, res, out=(leaf, res))
