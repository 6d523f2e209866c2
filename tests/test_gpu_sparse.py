"""Attention over chosen key blocks, forward and backward, against the fp64 oracle with
its bounds, element by element (half a step of bf16 for each rounding of P, dS and the
outputs)."""
import numpy as np
import pytest

import oracle.sparse as os_
from gpu_util import torch
from test_gpu_diff import close
from test_gpu_layer_norm import make, np64

pytestmark = pytest.mark.gpu


def inputs(B, H, Hk, Nq, Nk, d, seed=0, layout=None, sigma=1.0):
    q, do = (make((B, H, Nq, d), "bfloat16", seed + i, 0.0, sigma, layout) for i in (1, 4))
    k, v = (make((B, Hk, Nk, d), "bfloat16", seed + i, m, sigma, layout) for i, m in ((2, 0.0), (3, 0.2)))
    return q, k, v, do


def choose(B, H, groups, nb, topk, seed, least=-1):
    """Random numbers of blocks, some given twice, some standing for none."""
    t = torch()
    g = t.Generator(device="cuda").manual_seed(seed)
    return t.randint(least, nb, (B, H, groups, topk), generator=g, device="cuda", dtype=t.int32)


def run(q, k, v, blocks, do, block, q_block, scale=None, lens=None):
    import paper_2405_15780_amd as va

    t = torch()
    key_lens = None if lens is None else t.tensor(lens, dtype=t.int32, device="cuda")
    o, o32, lse = va.block_fwd(q, k, v, blocks, block, q_block, scale, key_lens)
    r = {"o": o, "o32": o32, "lse": lse}
    if do is not None:
        r.update(zip(("dq", "dk", "dv"), va.block_bwd(q, k, v, blocks, o32, lse, do, block, q_block, scale, key_lens)))
    t.cuda.synchronize()
    return r


def check(q, k, v, blocks, do, block, q_block, scale=None, lens=None):
    got = run(q, k, v, blocks, do, block, q_block, scale, lens)
    s = float(np.float32(1 / np.sqrt(q.shape[3]) if scale is None else scale))
    mask = os_.allowed(blocks.cpu().numpy(), q.shape[2], k.shape[2], block, q_block, lens)
    want = os_.block_attention(np64(q), np64(k), np64(v), mask, s, None if do is None else np64(do))
    for n in got:
        close(got[n], want[n], want[n + "_off"], n)
    return got


@pytest.mark.parametrize("d", [8, 24, 64, 72, 80, 88, 96, 104, 128, 160])
@pytest.mark.parametrize("block,q_block", [(64, 128), (128, 64), (64, 1), (128, 7)])
def test_head_dims(d, block, q_block):
    """Every tile width with one group per tile (of 64 and 128) and with rows that choose apart, 64 and 128 keys."""
    print(f"case sparse d={d} block={block} q_block={q_block}", flush=True)
    B, H, Hk, Nq, Nk = 2, 2, 1, 199, 421
    q, k, v, do = inputs(B, H, Hk, Nq, Nk, d, d)
    check(q, k, v, choose(B, H, -(-Nq // q_block), -(-Nk // block), 3, d), do, block, q_block)


@pytest.mark.parametrize("Nq", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 193, 257, 320, 513])
@pytest.mark.parametrize("q_block", [1, 5, 64, 96, 128])
def test_queries_around_tiles(Nq, q_block):
    print(f"case sparse Nq={Nq} q_block={q_block}", flush=True)
    q, k, v, do = inputs(1, 2, 2, Nq, 500, 64, Nq)
    check(q, k, v, choose(1, 2, -(-Nq // q_block), 8, 4, Nq + q_block), do, 64, q_block)


@pytest.mark.parametrize("Nk", [1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
@pytest.mark.parametrize("block", [64, 128, 192])
def test_keys_around_blocks(Nk, block):
    print(f"case sparse Nk={Nk} block={block}", flush=True)
    for q_block in (64, 1):
        q, k, v, do = inputs(2, 1, 1, 70, Nk, 64, Nk)
        check(q, k, v, choose(2, 1, -(-70 // q_block), -(-Nk // block), 2, Nk), do, block, q_block)


@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 1), (6, 2), (8, 8)])
@pytest.mark.parametrize("q_block", [1, 64])
def test_grouped_heads(H, Hk, q_block):
    print(f"case sparse H={H} Hk={Hk} q_block={q_block}", flush=True)
    q, k, v, do = inputs(2, H, Hk, 150, 300, 72, H)
    check(q, k, v, choose(2, H, -(-150 // q_block), 5, 2, H), do, 64, q_block)


@pytest.mark.parametrize("Nq", [1, 3, 17, 64, 65, 200, 256, 257])
@pytest.mark.parametrize("d,topk", [(64, 40), (128, 33), (160, 9), (72, 1)])
def test_few_queries_over_many_blocks(Nq, d, topk):
    """2 to 32 splits and their join, some of them empty."""
    print(f"case sparse few queries Nq={Nq} d={d} topk={topk}", flush=True)
    q, k, v, do = inputs(1, 2, 2, Nq, 3000, d, Nq)
    for q_block in (1, 128):
        check(q, k, v, choose(1, 2, -(-Nq // q_block), 24, topk, Nq, -20), do, 128, q_block)


@pytest.mark.parametrize("lens", [[300, 0, 1], [64, 65, 299], [0, 0, 0], [128, 300, 31]])
@pytest.mark.parametrize("q_block", [1, 64, 128])
def test_key_lens(lens, q_block):
    """Samples with fewer keys, one key or none; the keys behind hold NaN and are not read."""
    print(f"case sparse lens={lens} q_block={q_block}", flush=True)
    q, k, v, do = inputs(3, 2, 2, 140, 300, 72, 5)
    blocks = choose(3, 2, -(-140 // q_block), 5, 3, 6)
    want = check(q, k, v, blocks, do, 64, q_block, None, lens)
    for b, n in enumerate(lens):
        k[b, :, n:] = float("nan")
        v[b, :, n:] = float("inf")
    got = run(q, k, v, blocks, do, 64, q_block, None, lens)
    assert all(torch().equal(got[n], want[n]) for n in got)


@pytest.mark.parametrize("q_block", [1, 4, 64, 128])
def test_choices_of_every_kind(q_block):
    """Nothing chosen, all of it, one block by every query, twice the same, numbers past the last and below the first."""
    t = torch()
    Nq, Nk, nb = 300, 640, 10
    q, k, v, do = inputs(1, 1, 1, Nq, Nk, 64, q_block)
    groups = -(-Nq // q_block)
    none = t.full((1, 1, groups, 3), -1, dtype=t.int32, device="cuda")
    r = check(q, k, v, none, do, 64, q_block)
    assert not r["o"].any() and (r["lse"] == -np.inf).all() and not any(r[n].any() for n in ("dq", "dk", "dv"))
    some = none.clone()
    some[:, :, ::3, 1] = 4
    check(q, k, v, some, do, 64, q_block)
    whole = t.arange(nb, dtype=t.int32, device="cuda").expand(1, 1, groups, nb).contiguous()
    full = check(q, k, v, whole, do, 64, q_block)
    back = whole.flip(-1).contiguous()
    twice = t.cat([back, whole], -1)
    odd = t.cat([t.full_like(whole, nb), back, t.full_like(whole, -2 ** 31), t.full_like(whole, 2 ** 31 - 1)], -1)
    for blocks in (back, twice, odd):
        got = run(q, k, v, blocks, do, 64, q_block)
        assert all(t.equal(got[n], full[n]) for n in got)
    import paper_2405_15780_amd as va

    dense, lse = va.fwd(q, k, v)
    close(full["o32"], np64(dense), 2.0 ** -7 * np.abs(np64(v)).max() + 0 * np64(dense), "dense o")
    close(full["lse"], np64(lse), 1e-5 + 0 * np64(lse), "dense lse")


@pytest.mark.parametrize("q_block", [1, 64])
def test_a_block_that_all_queries_choose(q_block):
    """More query tiles than an item's run: shares of fp32 that are added."""
    t = torch()
    Nq = 9000
    q, k, v, do = inputs(1, 1, 1, Nq, 130, 64, 11)
    blocks = choose(1, 1, -(-Nq // q_block), 3, 2, 12)
    blocks[..., 0] = 1
    check(q, k, v, blocks, do, 64, q_block)
    q, k, v, do = inputs(1, 4, 2, 3000, 130, 128, 13)
    blocks = t.zeros((1, 4, -(-3000 // q_block), 1), dtype=t.int32, device="cuda")
    check(q, k, v, blocks, do, 128, q_block)


@pytest.mark.parametrize("q_block", [1, 48, 63])
def test_longer_sequences_that_choose_apart(q_block):
    """Several words of the map, heads that share keys, samples of other lengths, tiles that hold two groups and more."""
    q, k, v, do = inputs(2, 4, 2, 4300, 640, 72, 24)
    check(q, k, v, choose(2, 4, -(-4300 // q_block), 10, 3, 25), do, 64, q_block, None, [640, 200])


def test_rows_past_65536():
    """Gathered rows are numbered within 65,536: steps that end there, of two heads that share keys."""
    q, k, v, do = inputs(1, 2, 1, 140_001, 128, 8, 28)
    check(q, k, v, choose(1, 2, 140_001, 3, 1, 29), do, 64, 1)


def test_more_blocks_in_a_tile_than_are_listed():
    """A tile whose rows chose more than 128 blocks, of several heads, forward and backward."""
    q, k, v, do = inputs(1, 2, 1, 200, 64 * 200, 64, 26)
    check(q, k, v, choose(1, 2, 200, 200, 64, 27, 0), do, 64, 1)


def test_longer_lists_than_fit():
    """A tile's rows that chose more blocks together than are listed at a time."""
    q, k, v, do = inputs(1, 1, 1, 70, 64 * 300, 8, 14)
    check(q, k, v, choose(1, 1, 70, 300, 20, 15, 0), do, 64, 1)
    check(q, k, v, choose(1, 1, 1, 300, 1024, 16, 0), do, 64, 128)


@pytest.mark.parametrize("q_block", [1, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq", [150, 400])
def test_what_a_row_did_not_choose_does_not_reach_it(q_block, d, Nq):
    """Keys, values, queries and gradients that are not finite, in blocks and rows that others chose;
    of few queries, whose blocks are split, and of more."""
    t = torch()
    Nk = 512
    q, k, v, do = inputs(1, 2, 1, Nq, Nk, d, 17)
    groups = -(-Nq // q_block)
    blocks = choose(1, 2, groups, 7, 3, 18, 0)  # not the last block
    bad = blocks.clone()
    hit = t.zeros(groups, dtype=t.bool, device="cuda")
    hit[2], hit[groups - 1] = True, True
    bad[:, 0, hit, 1] = 7  # of head 0, two groups' choice
    kb, vb = k.clone(), v.clone()
    kb[:, :, 450], vb[:, :, 460], vb[:, :, 470] = float("nan"), float("inf"), float("nan")
    qb, gb = q.clone(), do.clone()
    qb[0, 1, 5], gb[0, 1, 7], gb[0, 1, 8] = float("nan"), float("inf"), float("nan")
    want = run(q, k, v, bad, do, 64, q_block)
    got = run(qb, kb, vb, bad, gb, 64, q_block)
    rows = hit.repeat_interleave(q_block)[:Nq]
    fine = ~rows
    for n in ("o", "o32", "lse", "dq"):
        a, b = got[n][0, 0, fine], want[n][0, 0, fine]
        assert t.equal(a, b), n
        assert not t.isfinite(got[n][0, 0, rows].float()).all(), n
    others = t.ones(Nq, dtype=t.bool, device="cuda")
    others[[5, 7, 8]] = False
    for n in ("o", "o32", "lse", "dq"):
        assert t.equal(got[n][0, 1, others], want[n][0, 1, others]), n
    # keys that neither the bad rows' groups nor the bad keys' rows chose
    touched = t.zeros(8, dtype=t.bool, device="cuda")
    for r in (5, 7, 8):
        touched[blocks[0, 1, r // q_block].long()] = True
    touched[bad[0, 0, hit].flatten().long()] = True
    keys = ~touched.repeat_interleave(64)
    for n in ("dk", "dv"):
        assert t.equal(got[n][0, 0, keys], want[n][0, 0, keys]), n


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Nq,block", [(2, 256), (5, 256), (64, 64), (65, 64), (256, 64)])
def test_rows_that_chose_nothing_of_a_split(Nq, block, d):
    """Few queries of one block each, split over workgroups: where a value is not finite the rows that share a tile are
    gone over again, one after the other, most of them without a block in the split."""
    print(f"case sparse redone rows Nq={Nq} block={block} d={d}", flush=True)
    t = torch()
    nb = 20
    q, k, v, _ = inputs(2, 8, 8, Nq, nb * block, d, 23)
    blocks = ((7 * t.arange(Nq, device="cuda", dtype=t.int32) + 3) % nb).expand(2, 8, Nq).unsqueeze(-1).contiguous()
    want = run(q, k, v, blocks, None, block, 1)
    vb = v.clone()
    for j in (3, 11):
        vb[:, :, j * block + 5] = float("inf")
    hit = (blocks[0, 0, :, 0] == 3) | (blocks[0, 0, :, 0] == 11)
    assert hit.any() and not hit.all()
    for _ in range(4):
        got = run(q, k, vb, blocks, None, block, 1)
        for n in ("o", "o32"):
            assert t.equal(got[n][:, :, ~hit], want[n][:, :, ~hit]), n
            assert (got[n][:, :, hit] == float("inf")).all(), n
        assert t.equal(got["lse"], want["lse"])


@pytest.mark.parametrize("q_block", [1, 64])
def test_large_and_masked_scores(q_block):
    """Scores of several hundred, and rows whose scores are all -inf."""
    t = torch()
    q, k, v, do = inputs(1, 1, 1, 130, 300, 64, 20, sigma=6.0)
    blocks = choose(1, 1, -(-130 // q_block), 5, 3, 21, 0)
    check(q, k, v, blocks, do, 64, q_block)
    k[0, 0, :, 0], q[..., 0] = -float("inf"), 1.0
    r = run(q, k, v, blocks, None, 64, q_block)
    assert not r["o"].any() and (r["lse"] == -np.inf).all()
    assert t.isfinite(r["o32"]).all()


@pytest.mark.parametrize("Nq", [32, 64, 130, 257])
@pytest.mark.parametrize("q_block", [1, 64])
def test_rows_whose_scores_overflow_have_no_gradients(q_block, Nq):
    """Finite operands whose scores are all -inf: of every row (steps of the key side in fours and not), and of every
    other group, whose keys have the gradients of the groups between."""
    t = torch()
    print(f"case sparse overflow q_block={q_block} Nq={Nq}", flush=True)
    q, k, v, do = inputs(1, 2, 1, Nq, 300, 64, 33)
    groups = -(-Nq // q_block)
    blocks = choose(1, 2, groups, 5, 3, 34, 0)
    k[..., 0], q[..., 0] = -3e38, 3e38
    r = run(q, k, v, blocks, do, 64, q_block)
    assert (r["lse"] == -np.inf).all() and not any(r[n].any() for n in ("o", "o32", "dq", "dk", "dv"))
    none = t.arange(Nq, device="cuda") // q_block % 2 == 0
    q[:, :, ~none, 0] = 0.0
    got = run(q, k, v, blocks, do, 64, q_block)
    mask = os_.allowed(blocks.cpu().numpy(), Nq, 300, 64, q_block)
    mask[:, :, none.cpu().numpy()] = False
    want = os_.block_attention(np64(q), np64(k), np64(v), mask, 0.125, np64(do))
    for n in ("o", "o32", "lse", "dk", "dv"):
        close(got[n], want[n], want[n + "_off"], n)
    close(got["dq"][..., 1:], want["dq"][..., 1:], want["dq_off"][..., 1:], "dq")  # (column 0 meets the -3e38)
    assert not got["dq"][:, :, none].any()


@pytest.mark.parametrize("q_block", [1, 64])
@pytest.mark.parametrize("Nq", [64, 150])
def test_an_infinite_key_that_no_row_can_see(q_block, Nq):
    """A key whose scores are -inf by an infinite element: outputs, and the gradients of the other keys and of rows that
    did not choose its block, are those without it."""
    t = torch()
    print(f"case sparse infinite key q_block={q_block} Nq={Nq}", flush=True)
    q, k, v, do = inputs(1, 2, 1, Nq, 300, 64, 35)
    blocks = choose(1, 2, -(-Nq // q_block), 5, 3, 36, 0)
    blocks[:, 0, 0] = t.tensor([1, 3, 1], device="cuda")
    q[..., 0], k[..., 100, 0] = 1.0, -float("inf")
    got = run(q, k, v, blocks, do, 64, q_block)
    mask = os_.allowed(blocks.cpu().numpy(), Nq, 300, 64, q_block)
    met = mask[..., 100].copy()
    assert met.any()
    mask[..., 100] = False
    other = np.arange(300) != 100
    kk = k.clone()
    kk[..., 100, 0] = 0.0
    want = os_.block_attention(np64(q), np64(kk), np64(v), mask, 0.125, np64(do))
    for n in ("o", "o32", "lse"):
        close(got[n], want[n], want[n + "_off"], n)
    for n in ("dk", "dv"):
        close(got[n][:, :, other], want[n][:, :, other], want[n + "_off"][:, :, other], n)
    at = t.from_numpy(~met).cuda()
    close(got["dq"][at], want["dq"][~met], want["dq_off"][~met], "dq")


@pytest.mark.parametrize("q_block", [1, 64, 128])
def test_layouts(q_block):
    """Sequence-major operands, a fused tensor's views, rows with a pitch; outputs in place of a buffer's part."""
    import paper_2405_15780_amd as va

    t = torch()
    B, H, N, d = 2, 3, 200, 64
    x = make((B, N, 4, H, d), "bfloat16", 30)
    q, k, v, do = (x[:, :, i].transpose(1, 2) for i in range(4))
    blocks = choose(B, H, -(-N // q_block), 4, 2, 31)
    got = check(q, k, v, blocks, do, 64, q_block)
    dense = run(*(y.contiguous() for y in (q, k, v)), blocks, do.contiguous(), 64, q_block)
    assert all(t.equal(got[n], dense[n]) for n in got)
    buf = t.full((B, N, H * d + 8), 7.0, dtype=t.bfloat16, device="cuda")
    out = buf[..., :-8].view(B, N, H, d).transpose(1, 2)
    va.block_fwd(q, k, v, blocks, 64, q_block, out=out)
    assert t.equal(out, got["o"]) and (buf[..., -8:] == 7).all()
    with pytest.raises(va.VitattnError):
        va.block_fwd(q, k, v, blocks, 64, q_block, out=v)


@pytest.mark.parametrize("q_block", [1, 64, 128])
def test_heads_are_those_of_one(q_block):
    """A head's bits do not depend on the call it is part of, and are the same every time."""
    t = torch()
    q, k, v, do = inputs(2, 8, 4, 700, 1500, 64, 40)
    blocks = choose(2, 8, -(-700 // q_block), 24, 6, 41)
    whole = run(q, k, v, blocks, do, 64, q_block)
    again = run(q, k, v, blocks, do, 64, q_block)
    assert all(t.equal(whole[n], again[n]) for n in whole)
    for b, g in ((0, 0), (1, 3)):
        h, hk = slice(2 * g, 2 * g + 2), slice(g, g + 1)
        s = slice(b, b + 1)
        one = run(q[s, h], k[s, hk], v[s, hk], blocks[s, h].contiguous(), do[s, h], 64, q_block)
        for n in whole:
            assert t.equal(whole[n][s, hk if n in ("dk", "dv") else h], one[n]), n


def test_autograd_and_scale():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, do = inputs(1, 4, 2, 100, 300, 64, 50)
    blocks = choose(1, 4, 2, 5, 2, 51)
    a = run(q, k, v, blocks, do, 64, 64, 0.3)
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    o = va.block_attention(*leaves, blocks, 64, 64, 0.3)
    assert t.equal(o, a["o"])
    o.backward(do)
    assert all(t.equal(x.grad, a[n]) for x, n in zip(leaves, ("dq", "dk", "dv")))
    # gradients that are expanded, negated lazily or in another order
    for g in (t.ones((), dtype=t.bfloat16, device="cuda").expand(o.shape), do.transpose(1, 2).contiguous().transpose(1, 2),
              make((1, 4, 64, 100), "bfloat16", 52).transpose(2, 3)):
        grads = t.autograd.grad(va.block_attention(*leaves, blocks, 64, 64, 0.3), leaves, g)
        want = run(q, k, v, blocks, g.contiguous(), 64, 64, 0.3)
        assert all(t.equal(x, want[n]) for x, n in zip(grads, ("dq", "dk", "dv")))
    with t.no_grad():
        assert t.equal(va.block_attention(q, k, v, blocks, 64, 64, 0.3), a["o"])


def test_gradients_against_differences():
    """dq, dk and dv along random directions against differences of the outputs (of steps that bf16 holds)."""
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, do = inputs(1, 2, 1, 130, 260, 64, 60)
    for q_block in (1, 64):
        blocks = choose(1, 2, -(-130 // q_block), 5, 3, 61, 0)
        r = run(q, k, v, blocks, do, 64, q_block)
        ops = {"dq": q, "dk": k, "dv": v}
        for n in ops:
            step = make(ops[n].shape, "bfloat16", 62).float().sign() * 2.0 ** -4
            ends = [{m: (x.float() + s * step).bfloat16() if m == n else x for m, x in ops.items()} for s in (1, -1)]
            real = (ends[0][n].double() - ends[1][n].double())
            f = [(va.block_fwd(e["dq"], e["dk"], e["dv"], blocks, 64, q_block)[1].double() * do.double()).sum().item() for e in ends]
            want = (r[n].double() * real).sum().item()
            # O is 2^-8 off in P, which differences do not share: sums of 2 x 130 x 64 such terms; and cubic terms
            noise = 2 * 2.0 ** -8 * float((do.double().abs() * r["o32"].double().abs().clamp_min(0.2)).square().sum().sqrt())
            assert abs(f[0] - f[1] - want) <= 4 * noise + 0.05 * abs(want), (n, q_block, f[0] - f[1], want, noise)


def test_streams_graphs_and_shared_workspaces():
    """On another stream than the current default, captured with its gradients and replayed on new inputs; one workspace
    for two graphs that run in turn."""
    import paper_2405_15780_amd as va

    t = torch()
    B, H, N, d = 1, 2, 300, 64
    q, k, v, do = inputs(B, H, H, N, N, d, 70)
    blocks = {qb: choose(B, H, -(-N // qb), 5, 3, 71) for qb in (1, 64)}
    lib = va.library()
    ws = t.empty(max(lib.vitattn_block_bwd_workspace_bytes(B, H, H, N, N, d, 64, qb, 3) for qb in (1, 64)) // 4, device="cuda")

    def go(qb):
        o, o32, lse = va.block_fwd(q, k, v, blocks[qb], 64, qb)
        return (o, lse, *va.block_bwd(q, k, v, blocks[qb], o32, lse, do, 64, qb, workspace=ws))

    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        first = [go(qb) for qb in (1, 64)]
    t.cuda.current_stream().wait_stream(side)
    assert all(t.equal(a, b) for qb, f in zip((1, 64), first) for a, b in zip(f, go(qb)))
    graphs, outs = [], []
    for qb in (1, 64):
        graphs.append(t.cuda.CUDAGraph())
        with t.cuda.graph(graphs[-1]):
            outs.append(go(qb))
    for seed in (80, 90, 100):
        for x, y in zip((q, k, v, do), inputs(B, H, H, N, N, d, seed)):
            x.copy_(y)
        for qb in blocks:
            blocks[qb].copy_(choose(B, H, -(-N // qb), 5, 3, seed))
        ref = [go(qb) for qb in (1, 64)]
        t.cuda.synchronize()
        for g in graphs:
            g.replay()
        t.cuda.synchronize()
        assert all(t.equal(a, b) for o, r in zip(outs, ref) for a, b in zip(o, r)), seed


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    q, k, v, do = inputs(2, 4, 2, 100, 300, 64, 50)
    blocks = choose(2, 4, 100, 5, 2, 51)
    o, o32, lse = va.block_fwd(q, k, v, blocks, 64)
    bad = [(TypeError, lambda: va.block_fwd(q.half(), k, v, blocks, 64)), (TypeError, lambda: va.block_fwd(q, k, v.float(), blocks, 64)),
           (ValueError, lambda: va.block_fwd(q, k[:, :, :200], v, blocks, 64)), (ValueError, lambda: va.block_fwd(q[:, :3], k, v, blocks, 64)),
           (TypeError, lambda: va.block_fwd(q, k, v, blocks.long(), 64)), (TypeError, lambda: va.block_fwd(q, k, v, blocks[:, :, :50], 64)),
           (TypeError, lambda: va.block_fwd(q, k, v, blocks.cpu(), 64)), (TypeError, lambda: va.block_fwd(q, k, v, blocks, 64, 2)),
           (TypeError, lambda: va.block_fwd(q, k, v, blocks.transpose(1, 2).contiguous().transpose(1, 2), 64)),
           (va.VitattnError, lambda: va.block_fwd(q, k, v, blocks, 96)), (ValueError, lambda: va.block_fwd(q, k, v, blocks, 64, 0)),
           (ValueError, lambda: va.block_fwd(q, k, v, blocks, 0)), (va.VitattnError, lambda: va.block_fwd(q, k, v, blocks, 64, scale=-1.0)),
           (TypeError, lambda: va.block_fwd(q, k, v, blocks, 64, key_lens=t.tensor([1, 2], device="cuda"))),
           (TypeError, lambda: va.block_bwd(q, k, v, blocks, o32.bfloat16(), lse, do, 64)),
           (TypeError, lambda: va.block_bwd(q, k, v, blocks, o32, lse[:1], do, 64)),
           (va.VitattnError, lambda: va.block_bwd(q, k, v, blocks, o32, lse, do, 64, workspace=t.empty(64, device="cuda"))),
           (va.VitattnError, lambda: va.block_fwd(q[..., :60].contiguous(), k[..., :60].contiguous(), v[..., :60].contiguous(), blocks, 64))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("not refused", i)
    leaf = o.clone().requires_grad_() * 1.0
    with pytest.raises(ValueError):
        va.block_fwd(q, k, v, blocks, 64, out=leaf)
