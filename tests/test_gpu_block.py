"""Layer norm, rotary positions and differential attention together, as a block
runs them: gradients against fp64, the explicit entry points, captured graphs,
two streams at once, tensors past 2^31 elements, poisoned LDS, and every
workgroup form of the differential attention."""
import numpy as np
import pytest

from gpu_util import torch
from test_gpu_diff import inputs, run
from test_gpu_layer_norm import make

pytestmark = pytest.mark.gpu

EPS, SECTIONS = 1e-5, (4, 6, 6)


def block_params(t, W, H, d, seed, dtype):
    """Weights of one block of width W: norm, q, k, v, o projections, per-head norm, lam."""
    g = t.Generator(device="cuda").manual_seed(seed)

    def rand(*s, scale=1.0, shift=0.0):
        return (t.randn(s, generator=g, device="cuda") * scale + shift).to(dtype).requires_grad_()

    return {"w": rand(W, scale=0.2, shift=1.0), "b": rand(W, scale=0.1), "wq": rand(W, 2 * H * d, scale=W ** -0.5),
            "wk": rand(W, 2 * H * d, scale=W ** -0.5), "wv": rand(W, 2 * H * d, scale=W ** -0.5),
            "wo": rand(2 * H * d, W, scale=W ** -0.5), "hw": rand(2 * d, scale=0.2, shift=1.0),
            "lam": rand(H, scale=0.2, shift=0.5)}


def block(va, p, x, pos, H, d, lens=None):
    B, N, W = x.shape
    y = va.layer_norm(x, p["w"], p["b"], eps=EPS)
    q, k = ((y @ p[n]).view(B, N, 2 * H, d).transpose(1, 2) for n in ("wq", "wk"))
    v = (y @ p["wv"]).view(B, N, H, 2 * d).transpose(1, 2)
    q, k = va.rotary(q, k, pos, SECTIONS)
    o = va.diff_attention(q, k, v, p["lam"], key_lens=lens)
    o = va.layer_norm(o, p["hw"], eps=EPS)  # each head's output
    return x + o.transpose(1, 2).reshape(B, N, H * 2 * d) @ p["wo"]


def block64(p, x, pos, H, d, lens=None):
    """The same in fp64 torch operations on the CPU."""
    import torch as t

    B, N, W = x.shape
    y = t.nn.functional.layer_norm(x, (W,), p["w"], p["b"], EPS)
    q, k = ((y @ p[n]).view(B, N, 2 * H, d).transpose(1, 2) for n in ("wq", "wk"))
    v = (y @ p["wv"]).view(B, N, H, 2 * d).transpose(1, 2)
    f = t.cat([10000.0 ** (-t.arange(n, dtype=t.float64) / n) for n in SECTIONS])
    axis = t.repeat_interleave(t.arange(len(SECTIONS)), t.tensor(SECTIONS))
    a = pos.double()[:, axis] * f
    R = len(f)

    def turn(z):
        u, w = z[..., :R], z[..., R:2 * R]
        return t.cat((u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin(), z[..., 2 * R:]), -1)

    q, k = turn(q), turn(k)
    s = q @ k.transpose(-1, -2) / d ** 0.5
    if lens is not None:
        s = s.masked_fill((t.arange(N) >= lens.view(-1, 1)).view(B, 1, 1, N), -t.inf)
    pr = s.softmax(-1)
    o = pr[:, 0::2] @ v - p["lam"].view(1, -1, 1, 1) * (pr[:, 1::2] @ v)
    o = t.nn.functional.layer_norm(o, (2 * d,), p["hw"], None, EPS)
    return x + o.transpose(1, 2).reshape(B, N, H * 2 * d) @ p["wo"]


def positions(t, N):
    n = t.arange(N, device="cuda")
    return t.stack((n // 16, n // 4 % 4, n % 4), 1)


@pytest.mark.parametrize("lens", [None, (70, 33)])
def test_block_and_its_gradients(lens):
    """Against fp64 from the same bf16 values. Each of a path's tensors is rounded
    to bf16, at most half a step (2^-8) of every element: y, q or k, its turned
    form, P or dS, o, the normed o, the product, the sum; and as many on the way
    back. Norm against norm they add to at most 16 * 2^-8 of the result."""
    import paper_2405_15780_amd as va

    t = torch()
    B, N, W, H, d = 2, 70, 128, 2, 32
    p = block_params(t, W, H, d, 1, t.bfloat16)
    x = make((B, N, W), "bfloat16", 2).requires_grad_()
    g = make((B, N, W), "bfloat16", 3, mean=0.0)
    pos = positions(t, N)
    key_lens = None if lens is None else t.tensor(lens, dtype=t.int32, device="cuda")
    y = block(va, p, x, pos, H, d, key_lens)
    y.backward(g)
    p64 = {n: a.detach().double().cpu().requires_grad_() for n, a in p.items()}
    x64 = x.detach().double().cpu().requires_grad_()
    y64 = block64(p64, x64, pos.cpu(), H, d, None if lens is None else t.tensor(lens))
    y64.backward(g.double().cpu())
    for name, a, b in [("y", y, y64), ("x", x.grad, x64.grad)] + [(n, p[n].grad, p64[n].grad) for n in p]:
        a, b = a.detach().double().cpu(), b.detach()
        off = float((a - b).norm() / b.norm())
        print("block", name, off, flush=True)
        assert off <= 16 * 2.0 ** -8, (name, off)


def step(va, q, k, v, lam, x, w, dy, do, pos, lens):
    """Every kernel of the three operators, by their explicit entry points."""
    y, mean, rstd = va.layer_norm_fwd(x, w, None, eps=EPS)
    dx, dw, db = va.layer_norm_bwd(x, w, mean, rstd, dy)
    qr, kr = va.rotary_fwd(q, k, pos, SECTIONS)
    o, o2, lse = va.diff_fwd(qr, kr, v, lam, key_lens=lens)
    dq, dk, dv, dlam = va.diff_bwd(qr, kr, v, lam, o, o2, lse, do, key_lens=lens)
    dq, dk = va.rotary_fwd(dq, dk, pos, SECTIONS, inverse=True)
    one = va.diff_fwd(qr[:, :, :1], kr, v, lam)[0]  # split keys where there are enough
    return y, dx, dw, db, o, o2, lse, dq, dk, dv, dlam, one


def step_inputs(t, N, seed):
    q, k, v, lam, do = inputs(2, 2, N, N, 32, 64, seed=seed)
    x, dy = make((3 * N, 200), "bfloat16", seed + 5), make((3 * N, 200), "bfloat16", seed + 6)
    w = make((200,), "float32", seed + 7)
    lens = t.tensor([N, N // 3], dtype=t.int32, device="cuda")
    return [q, k, v, lam, x, w, dy, do, positions(t, N), lens]


@pytest.mark.parametrize("N", [90, 1500])
def test_captured_step_replays_match_eager(N):
    import paper_2405_15780_amd as va

    t = torch()
    static = step_inputs(t, N, 11)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        step(va, *static)
    t.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):  # two graphs of the same calls, replayed in turn
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            out = step(va, *static)
        graphs.append((g, out))
    for rep, seed in enumerate((11, 30, 50)):
        for a, b in zip(static, step_inputs(t, N, seed)):
            a.copy_(b)
        ref = step(va, *static)
        t.cuda.synchronize()
        for g, out in graphs:
            g.replay()
            step(va, *step_inputs(t, N, 70 + rep))  # other eager work beside it
            t.cuda.synchronize()
            for n, (a, b) in enumerate(zip(out, ref)):
                assert t.equal(a, b), (rep, n)


def test_two_streams_at_once():
    import paper_2405_15780_amd as va

    t = torch()
    args = [step_inputs(t, 400, s) for s in (3, 4)]
    refs = [step(va, *a) for a in args]
    t.cuda.synchronize()
    streams = [t.cuda.Stream() for _ in args]
    for s in streams:
        s.wait_stream(t.cuda.current_stream())
    for _ in range(3):
        outs = []
        for s, a in zip(streams, args):
            with t.cuda.stream(s):
                outs.append(step(va, *a))
        t.cuda.synchronize()
        for out, ref in zip(outs, refs):
            assert all(t.equal(a, b) for a, b in zip(out, ref))


# d, e, heads, N: two whole rounds of wide dK/dV and forward workgroups, one round and a
# rest in narrow ones, and full grids of the tiles that take narrow ones only
FORMS = [(64, 128, 16, 4096), (64, 128, 9, 4096), (72, 144, 16, 4096), (80, 160, 9, 4001), (64, 64, 16, 4096), (64, 64, 9, 4000),
         (32, 64, 24, 2048)]


@pytest.mark.parametrize("d,e,H,N", FORMS)
def test_workgroup_forms_give_the_same_bits(d, e, H, N):
    t = torch()
    print(f"case diff forms d={d} e={e} H={H} N={N}", flush=True)
    q, k, v, lam, do = inputs(1, H, N, N, d, e, seed=40 + d + H)
    whole = run(q, k, v, lam, do)
    for h in (0, H - 1):  # single heads take narrow workgroups throughout
        two, one = slice(2 * h, 2 * h + 2), slice(h, h + 1)
        part = run(q[:, two], k[:, two], v[:, one], lam[one], do[:, one])
        for n in ("o", "dv"):
            assert t.equal(part[n], whole[n][:, one]), n
        for n in ("o2", "lse", "dq", "dk"):
            assert t.equal(part[n], whole[n][:, two]), n
        assert t.equal(part["dlam"], whole["dlam"][one])


@pytest.mark.parametrize("case", FORMS[1:2] + [(80, 160, 9, 4001), (64, 64, 2, 333), (32, 64, 2, 333), (64, 128, 2, 333), (72, 144, 2, 333)])
def test_poisoned_lds_changes_no_output(case):
    import paper_2405_15780_amd as va
    import paper_2405_15780_amd.binding as b
    from paper_2405_15780_amd._build import LDS_POISON_LIB_PATH

    t = torch()
    d, e, H, N = case
    print(f"case block LDS poison {case}", flush=True)
    q, k, v, lam, do = inputs(1, H, N, N, d, e, seed=60)
    norms = [(make((50, D), "bfloat16", 61), make((50, D), "bfloat16", 62)) for D in (72, 768, 5000, 20000)]
    normal, res = b.library(), []
    try:
        for lib in (normal, b.open_library(LDS_POISON_LIB_PATH)):
            b._lib = lib
            r = run(q, k, v, lam, do)
            out = [r[n] for n in sorted(r)] + [va.diff_fwd(q[:, :, :3], k, v, lam)[0]]
            out.append(va.diff_fwd(q[:, :, :3], k.repeat(1, 1, 5, 1), v.repeat(1, 1, 5, 1), lam)[0])
            for x, dy in norms:
                y, mean, rstd = va.layer_norm_fwd(x)
                out += [y, mean, rstd, *va.layer_norm_bwd(x, x[0], mean, rstd, dy)]
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
    y, mean, rstd = va.layer_norm_fwd(x)
    dx, _, _ = va.layer_norm_bwd(x, None, mean, rstd, y)
    tail = slice(139_997, None)
    want = va.layer_norm_fwd(x[tail])
    assert all(t.equal(a[tail], b) for a, b in zip((y, mean, rstd), want))
    assert t.equal(dx[tail], va.layer_norm_bwd(x[tail], None, want[1], want[2], want[0])[0])
    del x, y, dx, mean, rstd, want
    q = t.empty((1, 2, 9_000_000, 128), dtype=t.bfloat16, device="cuda").normal_()  # 2.3e9
    pos = t.arange(9_000_000, device="cuda").view(-1, 1)
    r = va.rotary_fwd(q, None, pos, (64,))
    tail = slice(8_999_990, None)
    assert t.equal(r[:, 1:, tail], va.rotary_fwd(q[:, 1:, tail].contiguous(), None, pos[tail], (64,)))
    del q, r
    k = t.empty((1, 256, 150_000, 64), dtype=t.bfloat16, device="cuda").normal_()  # 2.5e9
    v = t.empty((1, 128, 150_000, 128), dtype=t.bfloat16, device="cuda").normal_()
    q, lam = t.randn((1, 256, 3, 64), device="cuda").bfloat16(), t.rand(128, device="cuda")
    o, o2, lse = va.diff_fwd(q, k, v, lam)
    last = va.diff_fwd(q[:, -2:], k[:, -2:], v[:, -1:], lam[-1:])
    assert t.equal(o[:, -1:], last[0]) and t.equal(o2[:, -2:], last[1]) and t.equal(lse[:, -2:], last[2])
    do = t.randn((1, 128, 3, 128), device="cuda").bfloat16()
    dq, dk, dv, dlam = va.diff_bwd(q, k, v, lam, o, o2, lse, do)
    part = va.diff_bwd(q[:, -2:], k[:, -2:], v[:, -1:], lam[-1:], *last, do[:, -1:])
    for a, b, n in zip((dq, dk, dv, dlam.view(1, -1)), (*part[:3], part[3].view(1, -1)), (2, 2, 1, 1)):
        assert t.equal(a[:, -n:], b)




def test_outputs_among_other_operands():
    """Outputs interleaved with other operands in one tensor share no memory with them; those that do are refused."""
    import paper_2405_15780_amd as va

    t = torch()
    B, H, N, d, e = 2, 2, 70, 32, 64
    q, k, v, lam, _ = inputs(B, H, N, N, d, e, seed=90, layout=[0, 2, 1, 3])
    want = va.diff_fwd(q, k, v, lam)[0]
    buf = t.full((B, N, 2 * H * d + H * e + 8), 7.0, dtype=t.bfloat16, device="cuda")
    qi = buf[..., :2 * H * d].view(B, N, 2 * H, d).transpose(1, 2)
    oi = buf[..., 2 * H * d:-8].view(B, N, H, e).transpose(1, 2)
    qi.copy_(q)
    va.diff_fwd(qi, k, v, lam, out=oi)
    assert t.equal(oi, want) and t.equal(qi, q) and (buf[..., -8:] == 7).all()
    shifted = buf[..., 2 * H * d - 8:-16].view(B, N, H, e).transpose(1, 2)  # from q's last columns on
    for inputs_, out in (((qi, k, v), shifted), ((q, k, v), v)):
        with pytest.raises(va.VitattnError):
            va.diff_fwd(*inputs_, lam, out=out)
    # rotary: outputs interleaved in a new tensor, and operands in place that share a head
    pos, both = positions(t, N), t.empty((B, N, 5, d), dtype=t.bfloat16, device="cuda")
    q1, k1 = va.rotary_fwd(q[:, :3], k[:, :2], pos, SECTIONS)
    va.rotary_fwd(q[:, :3], k[:, :2], pos, SECTIONS, out=(both[:, :, :3].transpose(1, 2), both[:, :, 3:].transpose(1, 2)))
    assert t.equal(both[:, :, :3].transpose(1, 2), q1) and t.equal(both[:, :, 3:].transpose(1, 2), k1)
    x = both.transpose(1, 2)
    before = both.clone()
    for a, c in ((x, x[:, 1:]), (x[:, :3], x[:, 2:]), (x, x)):
        with pytest.raises(va.VitattnError):
            va.rotary_fwd(a, c, pos, SECTIONS, out=(a, c))
    with pytest.raises(va.VitattnError):
        va.rotary_fwd(q[:, :3], k[:, :3], pos, SECTIONS, out=(x[:, :3], x[:, 2:]))
    assert t.equal(both, before)


def test_outputs_written_in_place_are_known_to_autograd():
    """out= is refused where it requires a gradient, and a tensor that was saved before it was written is not read as if
    it had not been."""
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, _ = inputs(1, 2, 20, 20, 32, 64, seed=91)
    pos = positions(t, 20)
    writes = {"norm": (q, lambda x: va.layer_norm_fwd(x, out=x)), "rotary": (q, lambda x: va.rotary_fwd(x, None, pos, SECTIONS, out=x)),
              "rotary k": (k, lambda x: va.rotary_fwd(q, x, pos, SECTIONS, out=(q.clone(), x))),
              "diff": (v, lambda x: va.diff_fwd(q, k, v, lam, out=x))}
    for n, (like, write) in writes.items():
        leaf = like.clone().requires_grad_()
        x = leaf * 1.0
        y = x * x  # saves x
        before = x.detach().clone()
        with pytest.raises(ValueError):
            write(x)
        assert t.equal(x.detach(), before), n
        with t.no_grad():
            write(x)
        assert not t.equal(x.detach(), before), n
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
        # a leaf that is not in a graph, and one whose value autograd has no use for
        x = leaf * 1.0
        write(x.detach())
        x.sum().backward()
        assert t.equal(leaf.grad, t.ones_like(leaf)), n


def test_lazily_negated_operands_are_refused():
    """Their memory holds the opposite values. (Gradients are resolved by the autograd functions.)"""
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, do = inputs(1, 2, 20, 20, 32, 64, seed=92)
    x, w = make((20, 32), "float32", 93), make((32,), "float32", 94)
    pos = t.complex(t.zeros(20, 3, device="cuda"), positions(t, 20).float()).conj().imag
    assert pos.is_neg()
    n = t._neg_view
    o, o2, lse = va.diff_fwd(q, k, v, lam)
    y, mean, rstd = va.layer_norm_fwd(x, w)
    calls = [lambda: va.layer_norm_fwd(n(x)), lambda: va.layer_norm(x, n(w)), lambda: va.layer_norm_fwd(x, w, n(w)),
             lambda: va.layer_norm_fwd(x, out=n(x)), lambda: va.layer_norm_bwd(n(x), w, mean, rstd, x),
             lambda: va.layer_norm_bwd(x, w, mean, rstd, n(x)), lambda: va.rotary(n(q), k, pos.resolve_neg(), SECTIONS),
             lambda: va.rotary(q, n(k), pos.resolve_neg(), SECTIONS), lambda: va.rotary(q, k, pos, SECTIONS),
             lambda: va.diff_attention(n(q), k, v, lam), lambda: va.diff_attention(q, n(k), v, lam),
             lambda: va.diff_attention(q, k, n(v), lam), lambda: va.diff_fwd(q, k, v, n(lam)),
             lambda: va.diff_bwd(q, k, v, lam, o, o2, lse, n(do))]
    for i, call in enumerate(calls):
        with pytest.raises(TypeError, match="resolve_neg"):
            call()
            print("not refused", i)
    turned = va.rotary(q, k, pos.resolve_neg(), SECTIONS)
    assert all(t.equal(a, b) for a, b in zip(turned, va.rotary(q, k, -positions(t, 20), SECTIONS)))


def test_captured_block_with_its_gradients():
    """Forward and gradients of the block through the autograd functions, captured and replayed on new inputs."""
    import paper_2405_15780_amd as va

    t = torch()
    B, N, W, H, d = 2, 70, 128, 2, 32
    p = block_params(t, W, H, d, 5, t.bfloat16)
    x = make((B, N, W), "bfloat16", 6).requires_grad_()
    g, pos, lens = make((B, N, W), "bfloat16", 7), positions(t, N), t.tensor([70, 41], dtype=t.int32, device="cuda")

    def go():
        y = block(va, p, x, pos, H, d, lens)
        return (y.detach(), *t.autograd.grad(y, [x, *p.values()], g))

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
        ref = go()
        t.cuda.synchronize()
        graph.replay()
        go()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for a, b in zip(out, ref)), seed
