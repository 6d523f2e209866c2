"""Differential attention, forward and backward, against the fp64 oracle with
its bounds, element by element (half a step of bf16 for each rounding of P, dS
and the outputs)."""
import numpy as np
import pytest

import oracle.block as ob
from gpu_util import torch
from test_gpu_layer_norm import make, np64

pytestmark = pytest.mark.gpu


def inputs(B, H, Nq, Nk, d, e, seed=0, layout=None, sigma=1.0, lam_type="bfloat16"):
    t = torch()
    g = t.Generator(device="cuda").manual_seed(seed + 77)
    q, k = (make((B, 2 * H, n, d), "bfloat16", seed + i, 0.0, sigma, layout) for i, n in ((1, Nq), (2, Nk)))
    v, do = (make((B, H, n, e), "bfloat16", seed + i, 0.2, 1.0, layout) for i, n in ((3, Nk), (4, Nq)))
    lam = (t.rand(H, generator=g, device="cuda") - 0.3).to(getattr(t, lam_type))
    return q, k, v, lam, do


def close(got, want, off, name):
    got = np64(got)
    assert got.shape == want.shape, name
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), name
    got, want, off = got[fine], want[fine], off[fine] + 1e-30
    bad = ~(np.abs(got - want) <= off)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(np.abs(got - want) / off)))


def run(q, k, v, lam, do, scale=None, lens=None):
    import paper_2405_15780_amd as va

    t = torch()
    key_lens = None if lens is None else t.tensor(lens, dtype=t.int32, device="cuda")
    o, o2, lse = va.diff_fwd(q, k, v, lam, scale, key_lens)
    r = {"o": o, "o2": o2, "lse": lse}
    if do is not None:
        r.update(zip(("dq", "dk", "dv", "dlam"), va.diff_bwd(q, k, v, lam, o, o2, lse, do, scale, key_lens)))
    t.cuda.synchronize()
    return r


def check(q, k, v, lam, do, scale=None, lens=None):
    got = run(q, k, v, lam, do, scale, lens)
    s = float(np.float32(1 / np.sqrt(q.shape[3]) if scale is None else scale))
    want = ob.diff_attention(np64(q), np64(k), np64(v), np64(lam), s, lens, None if do is None else np64(do))
    if do is not None and lam.dtype == torch().float32:
        want["dlam_off"] += 2.0 ** -22 * np.abs(want["dlam"])
    for n in got:
        close(got[n], want[n], want[n + "_off"], n)
    return got


SHAPES = [(32, 64), (8, 8), (16, 24), (40, 80), (64, 64), (64, 128), (56, 104), (72, 144), (80, 160), (8, 160), (80, 8), (48, 136)]


@pytest.mark.parametrize("d,e", SHAPES)
@pytest.mark.parametrize("Nq,Nk", [(1, 1), (5, 70), (130, 33), (257, 200)])
def test_shapes(d, e, Nq, Nk):
    print(f"case diff Nq={Nq} Nk={Nk} d={d} e={e}", flush=True)
    check(*inputs(2, 2, Nq, Nk, d, e, seed=d + e + Nq))


@pytest.mark.parametrize("d,e", [(32, 64), (64, 64), (64, 128), (72, 144)])
@pytest.mark.parametrize("N", [31, 32, 63, 64, 65, 127, 128, 129, 160, 191, 256, 384, 513, 1025])
def test_lengths_around_tiles(d, e, N):
    print(f"case diff N={N} d={d} e={e}", flush=True)
    check(*inputs(1, 1, N, N, d, e, seed=N))


@pytest.mark.parametrize("d,e", [(32, 64), (64, 64), (64, 128), (80, 160)])
@pytest.mark.parametrize("Nq,Nk", [(1, 1024), (1, 5000), (3, 1023), (33, 3111), (64, 2048), (65, 2048), (65, 8192), (200, 9001), (256, 8192),
                                   (257, 8192)])
def test_few_queries_over_many_keys(d, e, Nq, Nk):
    print(f"case diff few queries Nq={Nq} Nk={Nk} d={d} e={e}", flush=True)
    check(*inputs(2, 1, Nq, Nk, d, e, seed=Nk + Nq))


@pytest.mark.parametrize("d,e", [(32, 64), (64, 128)])
@pytest.mark.parametrize("Nq,Nk", [(1, 1090), (2, 16385), (1, 20000), (16, 17409), (17, 20000), (32, 33500), (33, 17000), (5, 66001)])
def test_joins_of_few_and_many_splits(d, e, Nq, Nk):
    """3 to 128 splits of 512 keys and more, the last one short; one wave per map joins them, or eight."""
    print(f"case diff joins Nq={Nq} Nk={Nk} d={d} e={e}", flush=True)
    check(*inputs(1, 2, Nq, Nk, d, e, seed=Nk + Nq), None, [Nk])


@pytest.mark.parametrize("d,e", [(32, 64), (64, 64), (64, 128), (72, 144)])
def test_split_keys_of_many_heads_are_those_of_one(d, e):
    """The same bits whatever form the grid takes: 1,024 workgroups against 128."""
    import paper_2405_15780_amd as va

    print(f"case diff split forms d={d} e={e}", flush=True)
    q, k, v, lam, _ = inputs(1, 8, 2, 65536, d, e, seed=d + e)
    o, o2, lse = va.diff_fwd(q, k, v, lam)
    for h in (0, 5, 7):
        m = slice(2 * h, 2 * h + 2)
        one = va.diff_fwd(q[:, m], k[:, m], v[:, h:h + 1], lam[h:h + 1])
        for got, ref in zip((o[:, h:h + 1], o2[:, m], lse[:, m]), one):
            assert torch().equal(got, ref)


@pytest.mark.parametrize("lens", [[300, 0, 1], [64, 65, 299], [0, 0, 0], [128, 300, 31]])
@pytest.mark.parametrize("d,e", [(32, 64), (64, 128), (72, 144)])
def test_key_lens(lens, d, e):
    """Samples with fewer keys, one key or none; the keys behind hold NaN and are not read."""
    print(f"case diff lens={lens} d={d} e={e}", flush=True)
    q, k, v, lam, do = inputs(3, 2, 70, 300, d, e, seed=5)
    clean = [x.clone() for x in (k, v)]
    for b, n in enumerate(lens):
        k[b, :, n:] = float("nan")
        v[b, :, n:] = float("inf")
    got = run(q, k, v, lam, do, None, lens)
    ref = check(q, *clean, lam, do, None, lens)
    for n in got:
        assert torch().equal(got[n], ref[n]), n
    for b, n in enumerate(lens):
        assert not got["dk"][b, :, n:].any() and not got["dv"][b, :, n:].any()


@pytest.mark.parametrize("lens", [[5000, 0], [513, 512], [1, 4096]])
def test_key_lens_with_split_keys(lens):
    q, k, v, lam, do = inputs(2, 2, 2, 5000, 64, 128, seed=6)
    check(q, k, v, lam, do, None, lens)


def test_key_lens_out_of_range_are_brought_into_it():
    t = torch()
    x = inputs(2, 1, 40, 50, 32, 64, seed=7)
    got, ref = run(*x, lens=[-3, 51 + 10 ** 6]), run(*x, lens=[0, 50])
    for n in got:
        assert t.equal(got[n], ref[n]), n


@pytest.mark.parametrize("layout", [[0, 2, 1, 3], [2, 0, 1, 3], [1, 2, 0, 3]])
def test_layouts(layout):
    """Any order of batch, heads and rows gives the dense layout's bits."""
    t = torch()
    for d, e in ((64, 128), (72, 144)):
        x = inputs(2, 3, 150, 90, d, e, seed=8, layout=layout)
        got = run(*x)
        ref = check(*(a.contiguous() for a in x))
        for n in got:
            assert t.equal(got[n], ref[n]), n


def test_slices_of_a_fused_projection():
    t = torch()
    B, N, H, d = 2, 77, 2, 32
    qkv = make((B, N, 3, 2 * H * d), "bfloat16", 9)
    q, k = (qkv[:, :, i].view(B, N, 2 * H, d).transpose(1, 2) for i in (0, 1))
    v = qkv[:, :, 2].view(B, N, H, 2 * d).transpose(1, 2)
    lam = t.tensor([0.2, 0.9], device="cuda")
    do = make((B, H, N, 2 * d), "bfloat16", 10)
    got = check(q, k, v, lam, do)
    assert got["o"].transpose(1, 2).is_contiguous()  # in q's order: the next projection reads it as it is


@pytest.mark.parametrize("lam_type", ["bfloat16", "float32"])
def test_lam(lam_type):
    t = torch()
    q, k, v, lam, do = inputs(2, 3, 40, 50, 32, 64, seed=11, lam_type=lam_type)
    check(q, k, v, lam, do)
    zero = t.zeros_like(lam)
    got = check(q, k, v, zero, do)
    assert not got["dk"][:, 1::2].any() and not got["dq"][:, 1::2].any()


@pytest.mark.parametrize("sigma", [0.01, 4.0, 8.0])
def test_flat_and_peaked_rows(sigma):
    check(*inputs(1, 2, 130, 200, 64, 128, seed=12, sigma=sigma))


def test_all_scores_far_below_zero():
    """Every key opposes every query: exp of a padding key's zero score would overflow."""
    t = torch()
    q, k, v, lam, do = inputs(1, 1, 40, 45, 64, 128, seed=13)
    u = t.randn(64, device="cuda").sign()
    q[:], k[:] = (6 * u).bfloat16(), (-6 * u).bfloat16()
    q += make(tuple(q.shape), "bfloat16", 14, 0.0, 0.05)
    got = check(q, k, v, lam, do)
    assert all(x.isfinite().all() for x in got.values()) and got["lse"].max() < -200


def test_first_tile_of_infinite_scores():
    """Keys whose score is -inf weigh nothing, also where a whole first tile is such."""
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, _ = inputs(1, 1, 40, 300, 64, 128, seed=25)
    q = q.abs() + 0.1
    k[:, :, :100, 0] = -float("inf")
    o, o2, lse = va.diff_fwd(q, k, v, lam)
    ref = va.diff_fwd(q, k[:, :, 100:].contiguous(), v[:, :, 100:].contiguous(), lam)
    for a, b, off in zip((o, o2, lse), ref, (2 ** -6, 2 ** -6, 1e-5)):  # other tiles, so other roundings of P
        assert a.isfinite().all() and ((a.float() - b.float()).abs() <= off * (1 + b.float().abs())).all()


@pytest.mark.parametrize("maps", ["both", "second"])
@pytest.mark.parametrize("d,e", [(32, 64), (64, 64), (64, 128), (72, 144)])
@pytest.mark.parametrize("Nq,Nk", [(40, 300), (300, 300), (3, 5000), (40, 2000), (100, 9000)])
def test_rows_whose_scores_are_all_infinite(Nq, Nk, d, e, maps):
    """A query that scores -inf against every key (a product past fp32's range) is one without keys, whether the
    keys are split or not: zeros, an LSE of -inf and no part in any gradient. The others do not see it."""
    print(f"case diff all -inf Nq={Nq} Nk={Nk} d={d} e={e} {maps}", flush=True)
    t = torch()
    q, k, v, lam, do = inputs(1, 2, Nq, Nk, d, e, seed=26)
    q[..., 0], k[..., 0] = 0, -2.0 ** 70
    bad, good = [0, 2, Nq - 1], [i for i in range(Nq) if i not in (0, 2, Nq - 1)]
    do0 = do.clone()
    do0[:, :, bad] = 0
    ref = run(q, k, v, lam, do0)
    m = slice(0 if maps == "both" else 1, None, 1 if maps == "both" else 2)
    q[:, m, bad, 0] = 2.0 ** 70
    got = run(q, k, v, lam, do)
    for n in ("o", "o2", "lse", "dq"):
        assert t.equal(got[n][:, :, good], ref[n][:, :, good]), n
    for n in ("o2", "dq"):
        assert not got[n][:, m, bad].any(), n
    assert (got["lse"][:, m, bad] == -float("inf")).all()
    if maps == "both":
        assert not got["o"][:, :, bad].any()
        for n in ("dk", "dv", "dlam"):
            assert t.equal(got[n], ref[n]), n
    else:
        assert t.equal(got["o"][:, :, bad], got["o2"][:, 0::2, bad].bfloat16())
        assert t.equal(got["dk"][:, 1::2], ref["dk"][:, 1::2]) and t.equal(got["dlam"], ref["dlam"])
        assert all(got[n].isfinite().all() for n in ("dq", "dk", "dv"))


@pytest.mark.parametrize("d,e", [(32, 64), (64, 64), (64, 128), (72, 144)])
@pytest.mark.parametrize("Nq", [130, 3])
def test_keys_that_every_query_scores_low(Nq, d, e):
    """A key's gradient is a sum over its column of P. Where that is small throughout (2^-20 to 2^-86), each row of
    dK and dV still has the accuracy of the others, relative to its own size: the bounds below are P's multiples."""
    print(f"case diff low keys Nq={Nq} d={d} e={e}", flush=True)
    q, k, v, lam, do = inputs(1, 2, Nq, 200, d, e, seed=27)
    q[..., 0] = 4.0
    for j in range(16):
        k[:, :, 7 * j, 0] = -(14 + 3 * j) * d ** 0.5 / 4
    got = check(q, k, v, lam, do)
    assert got["dk"][:, :, :112:7].any(-1).all() and got["dv"][:, :, :112:7].any(-1).all()


def test_broadcast_heads_and_batches():
    t = torch()
    q, k, v, lam, do = inputs(2, 3, 60, 80, 32, 64, seed=15)
    k1, v1 = k[:, :1].expand(2, 6, 80, 32), v[:1].expand(2, 3, 80, 64)
    import paper_2405_15780_amd as va

    o, o2, lse = va.diff_fwd(q, k1, v1, lam)
    ref = va.diff_fwd(q, k1.contiguous(), v1.contiguous(), lam)
    assert all(t.equal(a, b) for a, b in zip((o, o2, lse), ref))
    # autograd adds the shared operands' gradients
    leaves = [x.detach().requires_grad_() for x in (q, k[:, :1], v[:1], lam)]
    va.diff_attention(leaves[0], leaves[1].expand(2, 6, 80, 32), leaves[2].expand(2, 3, 80, 64), leaves[3]).backward(do)
    dq, dk, dv, dlam = va.diff_bwd(q, k1.contiguous(), v1.contiguous(), lam, *ref, do)
    assert t.equal(leaves[0].grad, dq) and t.equal(leaves[3].grad, dlam)
    # the sums over heads and samples are torch's, in bf16
    for got, parts, dim in ((leaves[1].grad, dk, 1), (leaves[2].grad, dv, 0)):
        want = parts.double().sum(dim, keepdim=True)
        off = (parts.shape[dim] * 2.0 ** -8) * parts.double().abs().sum(dim, keepdim=True)
        assert ((got.double() - want).abs() <= off).all()


def test_a_head_does_not_depend_on_the_call():
    t = torch()
    for Nq, Nk in ((300, 300), (2, 3000)):
        q, k, v, lam, do = inputs(3, 4, Nq, Nk, 64, 128, seed=16)
        whole = run(q, k, v, lam, do)
        for b, h in ((0, 0), (2, 3)):
            two, one = slice(2 * h, 2 * h + 2), slice(h, h + 1)
            part = run(q[b:b + 1, two], k[b:b + 1, two], v[b:b + 1, one], lam[one], do[b:b + 1, one])
            for n in ("o", "dv"):
                assert t.equal(part[n], whole[n][b:b + 1, one]), n
            for n in ("o2", "lse", "dq", "dk"):
                assert t.equal(part[n], whole[n][b:b + 1, two]), n
        again = run(q, k, v, lam, do)
        assert all(t.equal(again[n], whole[n]) for n in whole)


def test_longer_sequences_fill_the_chip():
    """Sampled rows of a call with many workgroups per CU, against the oracle's rows."""
    B, H, N, d, e = 1, 4, 6000, 64, 128
    q, k, v, lam, do = inputs(B, H, N, N, d, e, seed=17)
    got = run(q, k, v, lam, do)
    rows = np.array([0, 31, 2999, 5887, 5999])
    for h in (0, 3):
        Q, K, V = np64(q[0, 2 * h:2 * h + 2]), np64(k[0, 2 * h:2 * h + 2]), np64(v[0, h])
        want = ob.diff_attention(Q[None][:, :, rows], K[None], V[None, None], np64(lam[h:h + 1]), 0.125,
                                 dout=np64(do[0, h])[None, None][:, :, rows])
        for n, x in (("o", got["o"][:, h:h + 1]), ("o2", got["o2"][:, 2 * h:2 * h + 2]), ("lse", got["lse"][:, 2 * h:2 * h + 2]),
                     ("dq", got["dq"][:, 2 * h:2 * h + 2])):
            close(x[:, :, rows], want[n], want[n + "_off"], n)
    want = ob.diff_attention(np64(q[:, 2:4]), np64(k[:, 2:4]), np64(v[:, 1:2]), np64(lam[1:2]), 0.125, dout=np64(do[:, 1:2]))
    for n, x in (("dk", got["dk"][:, 2:4]), ("dv", got["dv"][:, 1:2]), ("dlam", got["dlam"][1:2])):
        close(x, want[n], want[n + "_off"], n)


@pytest.mark.parametrize("form", ["dense", "bnhd", "shared rows", "odd pitch", "offset", "column major", "negated", "sum"])
def test_autograd_gradient_layouts(form):
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, _ = inputs(2, 2, 33, 40, 32, 64, seed=18)
    shape = (2, 2, 33, 64)
    base = make(shape, "bfloat16", 19)
    do = {"dense": base, "bnhd": make(shape, "bfloat16", 19, layout=[0, 2, 1, 3]),
          "shared rows": base[:, :, :1].expand(shape), "odd pitch": make((2, 2, 33, 67), "bfloat16", 20)[..., :64],
          "offset": make((2 * 2 * 33 * 64 + 1,), "bfloat16", 21)[1:].view(shape),
          "column major": base.reshape(2, 2, 64, 33).transpose(2, 3), "negated": t._neg_view(base),
          "sum": t.ones((), device="cuda", dtype=t.bfloat16).expand(shape)}[form]
    leaves = [x.detach().requires_grad_() for x in (q, k, v, lam)]
    va.diff_attention(*leaves).backward(do)
    want = run(q, k, v, lam, do.resolve_neg().clone(memory_format=t.contiguous_format))
    for x, n in zip(leaves, ("dq", "dk", "dv", "dlam")):
        assert t.equal(x.grad, want[n]), n


def test_one_lam_for_all_heads_and_inference():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, _, do = inputs(1, 3, 20, 30, 32, 64, seed=22)
    lam = t.tensor(0.4, device="cuda", requires_grad=True)
    o = va.diff_attention(q, k, v, lam)
    ref = run(q, k, v, t.full((3,), 0.4, device="cuda"), do)
    assert t.equal(o, ref["o"])
    o.backward(do)
    assert lam.grad.shape == () and np.isclose(float(lam.grad), float(ref["dlam"].double().sum()), rtol=1e-5)
    with t.no_grad():
        assert t.equal(va.diff_attention(q, k, v, lam), ref["o"])


def test_out_workspaces_and_rows_around():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, do = inputs(1, 2, 3, 2000, 64, 128, seed=23)
    ref = run(q, k, v, lam, do)
    big = t.full((1, 4, 9, 128), 7.0, dtype=t.bfloat16, device="cuda")
    need = va.library().vitattn_diff_fwd_workspace_bytes(1, 2, 3, 2000, 64, 128)
    assert need > 0
    ws = t.full((need // 4 + 64,), float("nan"), device="cuda")
    va.diff_fwd(q, k, v, lam, out=big[:, 1:3, 2:5], save=False, workspace=ws)
    assert t.equal(big[:, 1:3, 2:5], ref["o"])
    big[:, 1:3, 2:5] = 7.0
    assert (big == 7.0).all() and ws[need // 4:].isnan().all()
    with pytest.raises(va.VitattnError):
        va.diff_fwd(q, k, v, lam, workspace=ws[:need // 4 - 1].clone())


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, do = inputs(2, 2, 10, 12, 32, 64, seed=24)
    for bad in ((q.float(), k, v, lam), (q, k.cpu(), v, lam), (q, k, v[0], lam), (q, k, v, lam.half()), (q, k, v, lam[:1]),
                (q.transpose(2, 3), k, v, lam)):
        with pytest.raises(TypeError):
            va.diff_fwd(*bad)
    for bad in ((q[:, :3], k, v, lam), (q, k[:, :, :, :24], v, lam), (q, k[:, :, :11], v, lam), (q[:1], k, v, lam)):
        with pytest.raises(ValueError):
            va.diff_fwd(*bad)
    for lens in (t.tensor([1, 2], device="cuda"), t.tensor([1], dtype=t.int32, device="cuda"), t.tensor([1, 2], dtype=t.int32)):
        with pytest.raises(TypeError):
            va.diff_fwd(q, k, v, lam, key_lens=lens)
    for s in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(va.VitattnError):
            va.diff_fwd(q, k, v, lam, s)
    for d, e in ((12, 64), (88, 64), (32, 168), (32, 60)):
        a = inputs(1, 1, 4, 4, d, e)
        with pytest.raises(va.VitattnError):
            va.diff_fwd(*a[:4])
    o, o2, lse = va.diff_fwd(q, k, v, lam)
    for bad in ((o.float(), o2, lse, do), (o, o2[:, :2], lse, do), (o, o2.bfloat16(), lse, do), (o, o2, lse[:, :2], do), (o, o2, lse, do[:, :1])):
        with pytest.raises(TypeError):
            va.diff_bwd(q, k, v, lam, *bad)
    with pytest.raises(va.VitattnError):
        va.diff_bwd(q, k, v, lam, o, o2, lse, do, workspace=t.empty(8, device="cuda"))
    with pytest.raises(TypeError):
        va.diff_attention(q, k, v, 0.5)
    with pytest.raises(va.VitattnError):  # rows that are not 16-byte aligned
        va.diff_fwd(make((2, 4, 10, 36), "bfloat16", 1)[..., :32], k, v, lam)


def test_backward_without_the_rounded_output():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, lam, do = inputs(1, 2, 33, 40, 32, 64, seed=28)
    ref = run(q, k, v, lam, do)
    for got, n in zip(va.diff_bwd(q, k, v, lam, None, ref["o2"], ref["lse"], do), ("dq", "dk", "dv", "dlam")):
        assert t.equal(got, ref[n]), n
    leaves = [x.detach().requires_grad_() for x in (q, k, v, lam)]
    o = va.diff_attention(*leaves)
    o.mul_(2.0)  # the backward has no use for it
    o.backward(do)
    want = run(q, k, v, lam, 2 * do)
    for x, n in zip(leaves, ("dq", "dk", "dv", "dlam")):
        assert t.equal(x.grad, want[n]), n


@pytest.mark.parametrize("Nq,Nk", [(1, 65537), (2, 131073), (128, 131073)])
def test_one_key_past_whole_splits(Nq, Nk):
    print(f"case diff Nq={Nq} Nk={Nk} past whole splits", flush=True)
    check(*inputs(1, 1, Nq, Nk, 32, 64, seed=Nq))
