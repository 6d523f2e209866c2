"""The means in 8 bits and the choice of blocks: the oracle's very numbers."""
import numpy as np
import pytest

import oracle.sparse as os_
from gpu_util import torch
from test_gpu_layer_norm import make, np64

pytestmark = pytest.mark.gpu


def check(q, k, block, q_block, topk, lens=None):
    import paper_2405_15780_amd as va

    t = torch()
    key_lens = None if lens is None else t.tensor(lens, dtype=t.int32, device="cuda")
    m, scale = va.block_means(k, block, key_lens)
    M, S = os_.block_means(np64(k), block, lens)
    d = k.shape[3]
    assert np.array_equal(np64(m)[..., :d], M) and not m[..., d:].any() and np.array_equal(scale.cpu().numpy(), S)
    got = va.block_select(q, (m, scale), topk, q_block).cpu().numpy()
    want = os_.block_select(np64(q), (M, S), topk, q_block)
    assert np.array_equal(got, want), int((got != want).sum())
    return got


@pytest.mark.parametrize("d", [8, 40, 64, 72, 128, 136, 160])
@pytest.mark.parametrize("q_block", [1, 3, 64, 100])
def test_head_dims(d, q_block):
    print(f"case select d={d} q_block={q_block}", flush=True)
    q, k = make((2, 4, 130, d), "bfloat16", d, 0.1), make((2, 2, 700, d), "bfloat16", d + 1, 0.1)
    check(q, k, 64, q_block, 5, [700, 450])


@pytest.mark.parametrize("Nq", [1, 2, 15, 16, 17, 33])
@pytest.mark.parametrize("nb", [1, 2, 63, 64, 65, 256, 257, 512, 513, 1024, 1025, 2048])
def test_numbers_of_blocks(Nq, nb):
    print(f"case select Nq={Nq} nb={nb}", flush=True)
    q, k = make((1, 1, Nq, 32), "bfloat16", nb, 0.1), make((1, 1, nb * 64 - 5, 32), "bfloat16", nb + 1, 0.1)
    check(q, k, 64, 1, min(7, nb + 2))


@pytest.mark.parametrize("nb", [2049, 3841, 3842, 5000, 16384])
@pytest.mark.parametrize("topk", [1, 40, 256])
def test_more_blocks_than_fit_at_once(nb, topk):
    print(f"case select nb={nb} topk={topk}", flush=True)
    q, k = make((1, 1, 3, 8), "bfloat16", nb, 0.1), make((1, 1, nb * 64, 8), "bfloat16", topk, 0.1)
    check(q, k, 64, 1, topk)


@pytest.mark.parametrize("topk", [1, 2, 16, 17, 63, 64, 65, 100, 256])
def test_numbers_that_are_chosen(topk):
    print(f"case select topk={topk}", flush=True)
    q, k = make((1, 2, 20, 64), "bfloat16", topk, 0.1), make((1, 2, 300 * 64, 64), "bfloat16", topk + 1, 0.1)
    check(q, k, 64, 1, topk)
    check(q, k[:, :, :50 * 64], 64, 1, topk)  # fewer than are asked for, from 64 on


@pytest.mark.parametrize("block", [64, 128, 192, 1024])
def test_block_sizes(block):
    check(make((1, 2, 40, 64), "bfloat16", 1, 0.1), make((1, 2, 5003, 64), "bfloat16", 2, 0.1), block, 8, 3)


def test_ties_go_to_the_lowest():
    """Equal scores, few or all of them, within a lane's and across; none at all."""
    t = torch()
    q = make((1, 1, 5, 64), "bfloat16", 1)
    one = make((1, 1, 64, 64), "bfloat16", 2)
    for nb in (3, 64, 65, 300, 3000):
        same = one.repeat(1, 1, nb, 1)
        got = check(q, same, 64, 1, 2)
        assert (got == np.arange(2)).all()
        check(q, same, 64, 1, min(nb, 200))
        two = t.cat([same, 2 * one, same, 2 * one], 2)
        check(q, two, 64, 1, 3)
    got = check(t.zeros_like(q), make((1, 1, 900, 64), "bfloat16", 3), 64, 1, 4)
    assert (got == np.arange(4)).all()


def test_the_smallest_keys():
    """One key of 1,024 of bf16's least value: the scale is fp32's least, 2^-149 (2^-143 / 127 is above
    half of it), and not 0, so that blocks below zero come behind those of zeros."""
    t = torch()
    q = t.ones((1, 1, 3, 64), dtype=t.bfloat16, device="cuda")
    k = t.zeros((1, 1, 8 * 1024, 64), dtype=t.bfloat16, device="cuda")
    for j in (0, 3, 4):
        k[0, 0, 1024 * j, 5] = -2.0 ** -133
    assert (k != 0).sum() == 3
    got = check(q, k, 1024, 1, 5)
    assert (got == [1, 2, 5, 6, 7]).all()


@pytest.mark.parametrize("lens", [[0, 1, 700], [64, 65, 63], [0, 0, 0]])
def test_key_lens(lens):
    """Samples with few keys or none; the keys behind are not read."""
    t = torch()
    q, k = make((3, 2, 20, 64), "bfloat16", 1, 0.1), make((3, 2, 700, 64), "bfloat16", 2, 0.1)
    want = check(q, k, 64, 4, 3, lens)
    for b, n in enumerate(lens):
        k[b, :, n:] = float("nan")
    import paper_2405_15780_amd as va

    key_lens = t.tensor(lens, dtype=t.int32, device="cuda")
    got = va.block_select(q, va.block_means(k, 64, key_lens), 3, 4).cpu().numpy()
    assert np.array_equal(got, want)
    big = t.tensor([2000, -7, 700], dtype=t.int32, device="cuda")  # brought into 0 .. Nk
    k = make((3, 2, 700, 64), "bfloat16", 2, 0.1)
    m, s = va.block_means(k, 64, big)
    M, S = va.block_means(k, 64, t.tensor([700, 0, 700], dtype=t.int32, device="cuda"))
    assert t.equal(m, M) and t.equal(s, S) and (s[1] == -1).all()


def test_values_that_are_not_finite_count_as_zero():
    t = torch()
    q, k = make((1, 1, 10, 64), "bfloat16", 1, 0.1), make((1, 1, 640, 64), "bfloat16", 2, 0.1)
    k[0, 0, 70, 3], k[0, 0, 200, 5], q[0, 0, 2, 9], q[0, 0, 3, 1] = float("inf"), float("nan"), float("nan"), -float("inf")
    with np.errstate(invalid="ignore"):
        check(q, k, 64, 1, 3)
        check(q, k, 64, 4, 3)
    assert t.isfinite(q[0, 0, 0]).all()


def test_layouts_and_streams():
    import paper_2405_15780_amd as va

    t = torch()
    q, k = (make((2, 4, n, 64), "bfloat16", n, 0.1, layout=[0, 2, 1, 3]) for n in (130, 1300))
    want = check(q, k, 64, 16, 4)
    check(q, k[:, :1], 64, 16, 4)  # keys that all heads share
    wide = t.zeros((2, 4, 1300, 80), dtype=k.dtype, device="cuda")[..., 8:72]
    wide.copy_(k)
    assert np.array_equal(check(q, wide, 64, 16, 4), want)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        got = va.block_select(q, va.block_means(k, 64), 4, 16)
    side.synchronize()
    assert np.array_equal(got.cpu().numpy(), want)
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        out = va.block_select(q, va.block_means(k, 64), 4, 16)
    for seed in (1, 2, 3):
        q.copy_(make((2, 4, 130, 64), "bfloat16", seed, 0.1))
        k.copy_(make((2, 4, 1300, 64), "bfloat16", seed + 5, 0.1))
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, va.block_select(q, va.block_means(k, 64), 4, 16))


def test_refusals():
    import paper_2405_15780_amd as va

    t = torch()
    q, k = make((2, 4, 40, 64), "bfloat16", 1), make((2, 2, 300, 64), "bfloat16", 2)
    m = va.block_means(k, 64)
    bad = [(TypeError, lambda: va.block_means(k.half(), 64)), (TypeError, lambda: va.block_means(k[0], 64)),
           (va.VitattnError, lambda: va.block_means(k, 100)), (ValueError, lambda: va.block_means(k, 0)),
           (TypeError, lambda: va.block_means(k, 64, t.tensor([1, 2], device="cuda"))),
           (TypeError, lambda: va.block_select(q, (m[0].float(), m[1]), 2)), (TypeError, lambda: va.block_select(q, (m[0], m[1].half()), 2)),
           (TypeError, lambda: va.block_select(q[:1], m, 2)), (TypeError, lambda: va.block_select(make((2, 4, 40, 72), "bfloat16", 1), m, 2)),
           (ValueError, lambda: va.block_select(q[:, :3], m, 2)), (ValueError, lambda: va.block_select(q, m, 0)),
           (ValueError, lambda: va.block_select(q, m, 2, 0)), (va.VitattnError, lambda: va.block_select(q, m, 257)),
           (TypeError, lambda: va.block_select(q, m, 2.5))]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            print("not refused", i)
