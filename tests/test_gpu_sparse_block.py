"""Rms norm with the residual's addition, dropout, the choice of blocks and the attention
over them together, as a block runs them: gradients against fp64, captured graphs whose
masks advance, two streams at once, tensors past 2^31 elements, poisoned LDS, outputs
among other operands and what autograd knows of them."""
import numpy as np
import pytest

import oracle.sparse as os_
from gpu_util import torch
from test_gpu_block import block_params
from test_gpu_layer_norm import make
from test_gpu_sparse import choose, inputs, run

pytestmark = pytest.mark.gpu

EPS, P, BLOCK, QB, TOPK = 1e-5, 0.25, 64, 16, 2


def block(va, p, x, carry, H, d, rng, lens=None, chosen=None):
    """x is added to the stream `carry`, normed and attended over; 4 query heads share 2 of keys."""
    B, N, W = x.shape
    y, h = va.rms_norm(x, p["w"], carry, eps=EPS, p=P, rng=rng)
    q = (y @ p["wq"]).view(B, N, 2 * H, d).transpose(1, 2)
    k, v = ((y @ p[n][:, :H * d]).view(B, N, H, d).transpose(1, 2) for n in ("wk", "wv"))
    if chosen is None:
        chosen = va.block_select(q.detach(), va.block_means(k.detach(), BLOCK, lens), TOPK, QB)
    o = va.block_attention(q, k, v, chosen, BLOCK, QB, key_lens=lens)
    o = o.transpose(1, 2).reshape(B, N, 2 * H * d) @ p["wo"]
    return va.dropout(o, P, (rng[0], rng[1] + 1) if isinstance(rng, tuple) else rng, h), chosen


def block64(p, x, carry, H, d, rng, chosen, lens=None):
    import torch as t

    B, N, W = x.shape

    def m(off):
        keep, up = os_.kept((B, N, W), P, rng[0], rng[1] + off)
        return t.from_numpy(keep * up)

    h = carry + m(0) * x
    y = h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * p["w"]
    q = (y @ p["wq"]).view(B, N, 2 * H, d).transpose(1, 2)
    k, v = ((y @ p[n][:, :H * d]).view(B, N, H, d).transpose(1, 2).repeat_interleave(2, 1) for n in ("wk", "wv"))
    mask = t.from_numpy(os_.allowed(chosen.cpu().numpy(), N, N, BLOCK, QB, lens))
    s = (q @ k.transpose(-1, -2) / d ** 0.5).masked_fill(~mask, -1e300)
    o = (s.softmax(-1) * mask) @ v
    return h + m(1) * (o.transpose(1, 2).reshape(B, N, 2 * H * d) @ p["wo"])


@pytest.mark.parametrize("lens", [None, (200, 90)])
def test_block_and_its_gradients(lens):
    """Against fp64 from the same bf16 values and the same choice. Each of a path's tensors
    is rounded to bf16, at most half a step (2^-8) of every element: h, y, q or k, P or dS,
    o, the product, the sum; and as many on the way back. Norm against norm they add to at
    most 16 * 2^-8 of the result."""
    import paper_2405_15780_amd as va

    t = torch()
    B, N, W, H, d = 2, 200, 128, 2, 32
    p = block_params(t, W, H, d, 1, t.bfloat16)
    p = {n: p[n] for n in ("w", "wq", "wk", "wv", "wo")}
    x, carry = make((B, N, W), "bfloat16", 2).requires_grad_(), make((B, N, W), "bfloat16", 3).requires_grad_()
    g = make((B, N, W), "bfloat16", 4, mean=0.0)
    key_lens = None if lens is None else t.tensor(lens, dtype=t.int32, device="cuda")
    y, chosen = block(va, p, x, carry, H, d, (5, 6), key_lens)
    y.backward(g)
    p64 = {n: a.detach().double().cpu().requires_grad_() for n, a in p.items()}
    x64, c64 = (a.detach().double().cpu().requires_grad_() for a in (x, carry))
    y64 = block64(p64, x64, c64, H, d, (5, 6), chosen, lens)
    y64.backward(g.double().cpu())
    for name, a, b in [("y", y, y64), ("x", x.grad, x64.grad), ("carry", carry.grad, c64.grad)] + [(n, p[n].grad, p64[n].grad) for n in p]:
        a, b = a.detach().double().cpu(), b.detach()
        off = float((a - b).norm() / b.norm())
        print("block", name, off, flush=True)
        assert off <= 16 * 2.0 ** -8, (name, off)


def step(va, q, k, v, do, x, res, w, dy, dh, state, lens):
    """Every kernel of the operators, by their explicit entry points."""
    y, h, rstd = va.rms_norm_fwd(x, w, res, EPS, P, state)
    grads = va.rms_norm_bwd(h, w, rstd, dy, dh, P, state)
    y8, s8, _ = va.rms_norm_fp8(x, w, res, EPS, 64)
    z = va.dropout_fwd(x, P, state, res)
    out = [y, h, rstd, *grads, y8.view(torch().uint8), s8, z]
    for q_block in (1, 64):
        m = va.block_means(k, BLOCK, lens)
        chosen = va.block_select(q, m, 3, q_block)
        o, o32, lse = va.block_fwd(q, k, v, chosen, BLOCK, q_block, key_lens=lens)
        out += [*m, chosen, o, o32, lse, *va.block_bwd(q, k, v, chosen, o32, lse, do, BLOCK, q_block, key_lens=lens)]
        one = va.block_select(q[:, :, :1], m, 3)
        out.append(va.block_fwd(q[:, :, :1], k, v, one, BLOCK, key_lens=lens)[0])
    return out


def step_inputs(t, N, seed):
    q, k, v, do = inputs(2, 4, 2, N, N, 64, seed=seed)
    x, res, dy, dh = (make((3 * N, 200), "bfloat16", seed + i) for i in range(5, 9))
    lens = t.tensor([N, N // 3], dtype=t.int32, device="cuda")
    return [q, k, v, do, x, res, make((200,), "float32", seed + 9), dy, dh, t.tensor([seed, 7], device="cuda"), lens]


@pytest.mark.parametrize("N", [130, 520])
def test_captured_step_replays_match_eager(N):
    import paper_2405_15780_amd as va

    t = torch()
    a = step_inputs(t, N, 10)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        step(va, *a)
    t.cuda.current_stream().wait_stream(side)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        out = step(va, *a)
    for seed in (10, 40, 70):
        for x, y in zip(a, step_inputs(t, N, seed)):
            x.copy_(y)
        ref = step(va, *a)
        t.cuda.synchronize()
        graph.replay()
        step(va, *a)
        t.cuda.synchronize()
        assert all(t.equal(x, y) for x, y in zip(out, ref)), seed


def test_two_streams_at_once():
    import paper_2405_15780_amd as va

    t = torch()
    a, b = step_inputs(t, 700, 20), step_inputs(t, 640, 50)
    want = [step(va, *a), step(va, *b)]
    t.cuda.synchronize()
    streams = [t.cuda.Stream(), t.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, x in zip(streams, (a, b)):
            with t.cuda.stream(s):
                got.append(step(va, *x))
        t.cuda.synchronize()
        assert all(t.equal(x, y) for g, w in zip(got, want) for x, y in zip(g, w))


def test_captured_block_with_its_gradients():
    """Forward and gradients through the autograd functions, captured; the state on the device advances between replays."""
    import paper_2405_15780_amd as va

    t = torch()
    B, N, W, H, d = 2, 150, 128, 2, 32
    p = block_params(t, W, H, d, 5, t.bfloat16)
    p = {n: p[n] for n in ("w", "wq", "wk", "wv", "wo")}
    x, carry = (make((B, N, W), "bfloat16", i).requires_grad_() for i in (6, 7))
    g, state = make((B, N, W), "bfloat16", 8), t.tensor([9, 1], device="cuda")

    def go():
        y, chosen = block(va, p, x, carry, H, d, state)
        return (y.detach(), chosen, *t.autograd.grad(y, [x, carry, *p.values()], g))

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        go()
    t.cuda.current_stream().wait_stream(side)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        out = go()
    for seed in (6, 20, 30):
        with t.no_grad():
            x.copy_(make((B, N, W), "bfloat16", seed))
            g.copy_(make((B, N, W), "bfloat16", seed + 1))
        state += 1
        ref = go()
        t.cuda.synchronize()
        graph.replay()
        go()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(out, ref)), seed


@pytest.mark.parametrize("d,q_block,Nq", [(64, 1, 130), (64, 128, 700), (72, 1, 700), (72, 64, 40), (80, 3, 300), (96, 64, 300), (128, 1, 300),
                                          (128, 128, 400), (160, 1, 130), (160, 64, 400)])
def test_poisoned_lds_changes_no_output(d, q_block, Nq):
    import paper_2405_15780_amd as va
    import paper_2405_15780_amd.binding as b
    from paper_2405_15780_amd._build import LDS_POISON_LIB_PATH

    t = torch()
    print(f"case sparse LDS poison d={d} q_block={q_block} Nq={Nq}", flush=True)
    q, k, v, do = inputs(1, 4, 2, Nq, 1100, d, 60)
    blocks = choose(1, 4, -(-Nq // q_block), 18, 4, 61)
    rows = [[make((50, D), "bfloat16", 62 + i) for i in range(4)] for D in (33, 72, 768, 5000, 16000)]
    normal, res = b.library(), []
    try:
        for lib in (normal, b.open_library(LDS_POISON_LIB_PATH)):
            b._lib = lib
            r = run(q, k, v, blocks, do, 64, q_block)
            m = va.block_means(k, 64)
            out = [r[n] for n in sorted(r)] + [*m] + [va.block_select(q, m, n, q_block) for n in (1, 5, 100)]
            for x, c, dy, dh in rows:
                y, h, rstd = va.rms_norm_fwd(x, x[0], c, EPS, P, (1, 2))
                out += [y, h, rstd, *va.rms_norm_bwd(h, x[0], rstd, dy, dh, P, (1, 2)), va.dropout_fwd(x, P, (3, 4), c)]
                for group in (None, 32, 128):
                    y8, s8, _ = va.rms_norm_fp8(x, x[0], c, EPS, group)
                    out += [y8.view(t.uint8), s8]
            t.cuda.synchronize()
            res.append(out)
    finally:
        b._lib = normal
    for n, (x, y) in enumerate(zip(*res)):
        assert t.equal(x, y), n


def test_offsets_past_32_bits():
    """Operands of over 2^31 elements: their far ends against calls on those alone."""
    import paper_2405_15780_amd as va

    t = torch()
    x = t.empty((140_000, 16_384), dtype=t.bfloat16, device="cuda").normal_()  # 2.3e9 elements
    y, h, rstd = va.rms_norm_fwd(x, None, x)
    dx, _, _ = va.rms_norm_bwd(h, None, rstd, y, x)
    tail = slice(139_997, None)
    want = va.rms_norm_fwd(x[tail], None, x[tail])
    assert all(t.equal(a[tail], b) for a, b in zip((y, h, rstd), want))
    assert t.equal(dx[tail], va.rms_norm_bwd(want[1], None, want[2], want[0], x[tail])[0])
    y8, s8, _ = va.rms_norm_fp8(x, group=128)
    w8 = va.rms_norm_fp8(x[tail], group=128)
    assert t.equal(y8[tail].view(t.uint8), w8[0].view(t.uint8)) and t.equal(s8[tail], w8[1])
    del x, y, h, dx, rstd, want, y8, s8, w8
    k = t.empty((1, 128, 150_000, 128), dtype=t.bfloat16, device="cuda").normal_()  # 2.5e9
    v = t.empty_like(k).normal_()
    q, do = (t.randn((1, 256, 300, 128), device="cuda").bfloat16() for _ in range(2))
    m = va.block_means(k, 128)
    last = va.block_means(k[:, -1:], 128)
    assert t.equal(m[0][:, -1:], last[0]) and t.equal(m[1][:, -1:], last[1])
    for q_block in (1, 128):
        blocks = va.block_select(q, m, 4, q_block)
        tail = va.block_select(q[:, -2:], last, 4, q_block)
        assert t.equal(blocks[:, -2:], tail)
        o, o32, lse = va.block_fwd(q, k, v, blocks, 128, q_block)
        dq, dk, dv = va.block_bwd(q, k, v, blocks, o32, lse, do, 128, q_block)
        one = run(q[:, -2:], k[:, -1:], v[:, -1:], tail, do[:, -2:], 128, q_block)
        for n, a in zip(("o", "o32", "lse", "dq"), (o, o32, lse, dq)):
            assert t.equal(a[:, -2:], one[n]), n
        assert t.equal(dk[:, -1:], one["dk"]) and t.equal(dv[:, -1:], one["dv"])
        del dk, dv, dq
    del k, v
    t.cuda.empty_cache()


def test_outputs_among_other_operands():
    """Outputs interleaved with other operands in one tensor share no memory with them; those that do are refused."""
    import paper_2405_15780_amd as va

    t = torch()
    buf = make((40, 3, 64), "bfloat16", 1)
    x, res, out = (buf[:, i] for i in range(3))
    want = va.rms_norm_fwd(x.contiguous(), None, res.contiguous())
    h = t.empty_like(want[1])
    va.rms_norm_fwd(x, None, res, out=(out, h))
    assert t.equal(out, want[0]) and t.equal(h, want[1])
    drop = va.dropout_fwd(x.contiguous(), P, (1, 2), res.contiguous())
    assert t.equal(va.dropout_fwd(x, P, (1, 2), res, out=out), drop)
    wide = buf.view(40, 192)
    for call in (lambda: va.dropout_fwd(x, P, (1, 2), out=wide[:, 8:72]), lambda: va.rms_norm_fwd(x, None, res, out=(wide[:, 8:72], h)),
                 lambda: va.rms_norm_fwd(x, None, res, out=(out, wide[:, 120:184]))):
        with pytest.raises(va.VitattnError):
            call()
    q, k, v, _ = inputs(1, 1, 1, 100, 100, 64, 2)
    blocks = choose(1, 1, 100, 2, 1, 3)
    both = t.zeros((1, 1, 100, 128), dtype=q.dtype, device="cuda")
    both[..., :64] = q
    o = va.block_fwd(q, k, v, blocks, 64)[0]
    assert t.equal(va.block_fwd(both[..., :64], k, v, blocks, 64, out=both[..., 64:])[0], o)
    with pytest.raises(va.VitattnError):
        va.block_fwd(both[..., :64], k, v, blocks, 64, out=both[..., 32:96])


def test_outputs_written_in_place_are_known_to_autograd():
    import paper_2405_15780_amd as va

    t = torch()
    x = make((6, 64), "float32", 1)
    for write in (lambda y: va.dropout_fwd(x, P, (1, 2), out=y), lambda y: va.rms_norm_fwd(x, out=y)):
        w = t.ones(6, 64, device="cuda", requires_grad=True)
        y = x.clone()
        z = (w * y).sum()  # keeps y for w's gradient
        write(y)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.backward()


def test_other_types_of_rng_and_refused_devices():
    import paper_2405_15780_amd as va

    t = torch()
    x = make((6, 64), "float32", 1)
    a = va.dropout_fwd(x, P, (2 ** 64 - 3, 5))
    assert t.equal(a, va.dropout_fwd(x, P, t.tensor([-3, 5], device="cuda")))
    for call in (lambda: va.dropout_fwd(x.cpu(), P, (1, 2)), lambda: va.rms_norm_fwd(x.cpu()), lambda: va.rms_norm_fwd(x, x[0].cpu()),
                 lambda: va.block_means(make((1, 1, 64, 64), "bfloat16", 1).cpu(), 64)):
        with pytest.raises((TypeError, ValueError)):
            call()


def test_lazily_negated_operands_are_refused():
    """Their memory holds the opposite values. (Gradients are resolved by the autograd functions.)"""
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, do = inputs(1, 2, 2, 20, 70, 64, 5)
    x, w = make((20, 32), "float32", 6), make((32,), "float32", 7)
    blocks, n = choose(1, 2, 20, 2, 1, 8), t._neg_view
    m = va.block_means(k, 64)
    o, o32, lse = va.block_fwd(q, k, v, blocks, 64)
    y, h, rstd = va.rms_norm_fwd(x, w, x)
    calls = [lambda: va.rms_norm_fwd(n(x)), lambda: va.rms_norm_fwd(x, n(w)), lambda: va.rms_norm(x, w, n(x)), lambda: va.rms_norm_fp8(n(x)),
             lambda: va.rms_norm_bwd(n(h), w, rstd, x), lambda: va.rms_norm_bwd(h, w, rstd, n(x)), lambda: va.rms_norm_bwd(h, w, rstd, x, n(x)),
             lambda: va.dropout(n(x), P, (1, 2)), lambda: va.dropout_fwd(x, P, (1, 2), n(x)), lambda: va.dropout_fwd(x, P, (1, 2), out=n(x)),
             lambda: va.block_means(n(k), 64), lambda: va.block_select(n(q), m, 1), lambda: va.block_select(q, (m[0], n(m[1])), 1),
             lambda: va.block_attention(n(q), k, v, blocks, 64), lambda: va.block_attention(q, n(k), v, blocks, 64),
             lambda: va.block_fwd(q, k, n(v), blocks, 64), lambda: va.block_bwd(q, k, v, blocks, o32, lse, n(do), 64),
             lambda: va.block_bwd(q, k, v, blocks, n(o32), lse, do, 64), lambda: va.block_bwd(q, k, v, blocks, o32, n(lse), do, 64),
             lambda: va.block_fwd(q, k, v, n(blocks), 64), lambda: va.dropout_fwd(x, P, n(t.tensor([1, 2], device="cuda"))),
             lambda: va.block_fwd(q, k, v, blocks, 64, key_lens=n(t.tensor([7], dtype=t.int32, device="cuda"))),
             lambda: va.rms_norm_bwd(h, w, n(rstd), x)]
    for i, call in enumerate(calls):
        with pytest.raises(TypeError, match="resolve_neg"):
            call()
            print("not refused", i)
    a = [z.clone().requires_grad_() for z in (q, k, v)]
    got = t.autograd.grad(va.block_attention(*a, blocks, 64), a, n(do))
    want = t.autograd.grad(va.block_attention(*a, blocks, 64), a, -do)
    assert all(t.equal(b, c) for b, c in zip(got, want))
    z = x.clone().requires_grad_()
    for f in (lambda: va.rms_norm(z, w), lambda: va.dropout(z, P, (1, 2))):
        assert t.equal(t.autograd.grad(f(), z, n(x))[0], t.autograd.grad(f(), z, -x)[0])
