"""Cases of the operators that a block with sparse attention runs: root-mean-square norm with the residual's addition
(and an output in 8 bits), dropout from a counter-based generator, the choice of key blocks by a cheap score, and the
attention over the chosen blocks, each as a ViT block over a long sequence uses it.

A case is a dict of plain values. `kind` says which entry points it goes through:

  rms_fp8       rms_norm_fp8                      inference: the norm before an 8-bit product, with the residual's addition
  rms_train     rms_norm_fwd, rms_norm_bwd        the two halves of a training step, dropout on the added branch
  dropout       dropout_fwd                       y = [residual +] dropout(x), and dx from dy with the same mask
  select        block_means, block_select         the chosen blocks of each group of queries, from q and k
  select_kept   block_select                      the same over means that a server keeps
  sparse_fwd    block_attention                   inference, down to one query over a long key set
  sparse_train  block_fwd, block_bwd              the two halves of a training step

With `own` false, run() computes the same in elementary torch operations.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # a served model's last token before its 8-bit head: launch and latency
        _rms("rms_token_fp8", "rms_fp8", 1, 1, 768, "bf16", "bf16", group=0),
        # a long sequence's tokens before an 8-bit projection, a scale for each 128 columns
        _rms("rms_block_fp8", "rms_fp8", 2, 16384, 2048, "bf16", "bf16", group=128),
        # one training block of width 1,024 over 8,192 tokens of 4 images, a tenth of the branch dropped
        _rms("rms_block_train", "rms_train", 4, 8192, 1024, "bf16", "bf16", p=0.1),
        # an odd crop of an odd width beside an fp32 residual stream
        _rms("rms_odd_train", "rms_train", 3, 2731, 1537, "fp16", "fp32", p=0.25),
        # the hidden layer of an MLP in training, forward and backward
        _drop("dropout_mlp", 4, 1, 8192, 4096, "bf16", "none", 0.1),
        # heads of 72, sequence-major as the projection leaves them, added to a residual, an odd length
        _drop("dropout_heads", 1, 16, 20001, 72, "fp32", "fp32", 0.5, layout="bnhd"),
        # every query of a 32K sequence chooses 16 of 512 blocks of 64 keys
        _sel("select_rows_32k", "select", 1, 8, 8, 32768, 32768, 64, 64, 1, 16),
        # one query of a served clip over the means that it keeps
        _sel("select_token_128k", "select_kept", 1, 8, 8, 1, 131072, 128, 128, 1, 32),
        # one query of 8 heads reads 32 of 1,024 blocks
        _sparse("sparse_token_128k", "sparse_fwd", 1, 8, 8, 1, 131072, 128, 128, 1, 32),
        # inference over a clip of 368x512 patches, tiles of 128 neighbours share their choice
        _sparse("sparse_clip_188k", "sparse_fwd", 1, 4, 4, 188416, 188416, 64, 128, 128, 16),
        # a training shard of a 32K sequence, tiles of 64
        _sparse("sparse_shard_32k_train", "sparse_train", 1, 8, 8, 32768, 32768, 64, 64, 64, 32),
        # heads of 72, two to a key head, each query its own blocks, sequence-major, odd length, the second sample padded
        _sparse("sparse_rows_8k_train", "sparse_train", 2, 4, 2, 8003, 8003, 72, 64, 1, 8, layout="bnhd", padded=True),
    ]


def _rms(name, kind, B, N, D, dtype, res, p=0.0, group=0):
    """res: the residual's type; group: columns that share a scale (0: a row's)."""
    return dict(name=name, kind=kind, B=B, N=N, D=D, dtype=dtype, res=res, p=p, group=group)


def _drop(name, B, H, N, D, dtype, res, p, layout="bhnd"):
    return dict(name=name, kind="dropout", B=B, H=H, N=N, D=D, dtype=dtype, res=res, p=p, layout=layout)


def _sel(name, kind, B, H, Hk, Nq, Nk, d, block, q_block, topk, layout="bhnd", padded=False):
    """q_block neighbouring queries choose topk blocks of `block` keys together."""
    return dict(name=name, kind=kind, B=B, H=H, Hk=Hk, Nq=Nq, Nk=Nk, d=d, block=block, q_block=q_block, topk=topk,
                layout=layout, padded=padded)


_sparse = _sel


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rms_fp8", "rms_train", "rms_train", "dropout", "dropout", "select", "select_kept", "sparse_fwd",
                       "sparse_fwd", "sparse_train", "sparse_train"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if kind.startswith("rms"):
        D = rng.choice([768, 1024, 2048, 4096, _log_int(rng, 64, 8200), _log_int(rng, 64, 8200)])
        c = _rms("", kind, rng.choice([1, 1, 2, 4]), _log_int(rng, 1, 32768), D, dtype, rng.choice([dtype, dtype, "fp32"]))
        if kind == "rms_train":
            c["p"] = rng.choice([0.0, 0.1, 0.1, 0.3])
        else:
            c["group"] = rng.choice([0, 128, 128, 64])
        while c["B"] * c["N"] * c["D"] > 32768 * 2048:
            c["N"] = c["N"] // 2 + 1
    elif kind == "dropout":
        D = rng.choice([72, 128, 1024, 4096, _log_int(rng, 33, 16400), _log_int(rng, 33, 16400)])
        c = _drop("", rng.choice([1, 1, 2, 4]), rng.choice([1, 1, 8, 16]), _log_int(rng, 1, 40000), D, dtype,
                  rng.choice(["none", dtype, "fp32"]), rng.choice([0.05, 0.1, 0.5]), rng.choice(["bhnd", "bnhd"]))
        while c["B"] * c["H"] * c["N"] * c["D"] > 16384 * 4096:
            c["N"] = c["N"] // 2 + 1
    else:
        H, Hk = rng.choice([(4, 4), (8, 8), (6, 6), (8, 2), (4, 1), (12, 4)])
        d, block = rng.choice([64, 64, 128, 72, 80, 160, 32]), rng.choice([64, 128, 128, 256])
        Nk = _log_int(rng, 512, 131072)
        q_block = rng.choice([64, 128, 128, 256, 1, 16])
        topk = rng.choice([4, 8, 16, 32, rng.randint(1, 40)])
        if kind == "select_kept" or kind == "sparse_fwd" and rng.random() < 0.4:
            Nq, q_block = rng.choice([1, 1, 2, rng.randint(3, 64)]), 1
        else:
            Nq = Nk
        c = _sel("", kind, rng.choice([1, 1, 2]), H, Hk, Nq, Nk, d, block, q_block, topk, rng.choice(["bhnd", "bnhd"]),
                 rng.random() < 0.3)
        while _more_than_listed(c):
            c["Nk"] = c["Nk"] * 3 // 4
            if Nq == Nk:
                c["Nq"] = c["Nk"]
    del c["name"]
    return c


def _more_than_listed(c):
    """Whether a case of the sparse attention or its choice costs more than the largest listed one of its kind."""
    B, H, Hk, Nq, Nk, d, block, qb, topk = (c[x] for x in ("B", "H", "Hk", "Nq", "Nk", "d", "block", "q_block", "topk"))
    if B * Hk * Nk * d > 8 * 131072 * 128:
        return True
    if c["kind"].startswith("select"):
        return B * H * (Nq / qb) * (Nk / block) > 8 * 32768 * 512
    if Nq > 64 and qb < 64 and B * H * Nq * Nk > 2 * 4 * 8003 ** 2:  # the plain form has every score
        return True
    return B * H * Nq * topk * block * d * (14 if c["kind"] == "sparse_train" else 4) > 4 * 188416 * 2048 * 64 * 4


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _rows(g, B, H, N, D, dtype, layout="bhnd"):
    """Normal values [B, H, N, D]."""
    x = torch.randn((B, N, H, D) if layout == "bnhd" else (B, H, N, D), generator=g, device="cuda").to(dtype)
    return x.transpose(1, 2) if layout == "bnhd" else x


def _patches(g, B, H, N, d, layout, at):
    """Queries or keys [B, H, N, d] of patches: neighbours (64 in a row, centres `at`) are alike, which is what makes
    a block's mean tell of its keys."""
    x = torch.randn((B, H, N, d), generator=g, device="cuda")
    n = torch.arange(N, device="cuda") * at.shape[2] // N
    x = (0.8 * x + 0.9 * at[:, :, n]).to(torch.bfloat16)
    return x.transpose(1, 2).contiguous().transpose(1, 2) if layout == "bnhd" else x


def _rng_state(g):
    """(seed, offset) of the generator that dropout counts in, as a training loop holds it."""
    s = torch.randint(0, 1 << 62, (2,), generator=g, device="cuda", dtype=torch.int64).tolist()
    return s[0], s[1]


def prepare(case, seed):
    g = _gen(seed)
    kind, B, N = case["kind"], case["B"], case.get("N")
    s = {"case": case}
    if kind.startswith("rms"):
        t, r, D = TYPES[case["dtype"]], TYPES[case["res"]], case["D"]
        s["x"] = _rows(g, B, 1, N, D, t).squeeze(1)
        s["residual"] = (2 * torch.randn((B, N, D), generator=g, device="cuda")).to(r)
        s["w"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(torch.float32 if t == torch.float16 else t)
        s["rng"] = _rng_state(g)
        if kind == "rms_train":
            s["dy"] = _rows(g, B, 1, N, D, t).squeeze(1)
            s["dh"] = torch.randn((B, N, D), generator=g, device="cuda").to(r)
    elif kind == "dropout":
        t, H, D = TYPES[case["dtype"]], case["H"], case["D"]
        s["x"], s["dy"] = _rows(g, B, H, N, D, t, case["layout"]), _rows(g, B, H, N, D, t, case["layout"])
        s["residual"] = None if case["res"] == "none" else _rows(g, B, H, N, D, TYPES[case["res"]], case["layout"])
        s["rng"] = _rng_state(g)
    else:
        H, Hk, Nq, Nk, d = (case[x] for x in ("H", "Hk", "Nq", "Nk", "d"))
        centres = torch.randn((B, 1, (Nk + 63) // 64, d), generator=g, device="cuda")
        turn = torch.randn((1, Hk, 1, d), generator=g, device="cuda")
        at = centres * turn
        s["k"] = _patches(g, B, Hk, Nk, d, case["layout"], at)
        if Nq != Nk:  # a few queries, each near some place of the keys
            at = at[:, :, torch.randint(0, at.shape[2], (Nq,), generator=g, device="cuda")]
        s["q"] = _patches(g, B, H, Nq, d, case["layout"], at.repeat_interleave(H // Hk, 1))
        s["lens"] = None
        if case["padded"]:  # the first sample is whole
            lens = torch.randint(max(1, Nk // 2), Nk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            lens[0] = Nk
            s["lens"] = lens
        if kind == "select_kept" or kind.startswith("sparse"):
            means = _plain_means(s["k"], case["block"], s["lens"])
            if kind == "select_kept":
                s["means"] = means
                del s["k"]
            else:
                s["blocks"] = _plain_select(s["q"], means, case["topk"], case["q_block"])
        if kind.startswith("sparse"):
            s["v"] = _rows(g, B, Hk, Nk, d, torch.bfloat16, case["layout"])
        if kind == "sparse_train":
            s["dout"] = _rows(g, B, H, Nq, d, torch.bfloat16, case["layout"])
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2405_15780_amd as va

    c = s["case"]
    kind = c["kind"]
    if kind == "rms_fp8":
        y, scale, h = va.rms_norm_fp8(s["x"], s["w"], s["residual"], eps=EPS, group=c["group"] or None)
        return {"y": y, "scale": scale, "h": h}
    if kind == "rms_train":
        y, h, rstd = va.rms_norm_fwd(s["x"], s["w"], s["residual"], eps=EPS, p=c["p"], rng=s["rng"])
        dx, dres, dw = va.rms_norm_bwd(h, s["w"], rstd, s["dy"], s["dh"], p=c["p"], rng=s["rng"])
        return {"y": y, "h": h, "dx": dx, "dres": dres, "dw": dw}
    if kind == "dropout":
        return {"y": va.dropout_fwd(s["x"], c["p"], s["rng"], residual=s["residual"]),
                "dx": va.dropout_fwd(s["dy"], c["p"], s["rng"])}
    if kind == "select":
        means = va.block_means(s["k"], c["block"], key_lens=s["lens"])
        return va.block_select(s["q"], means, c["topk"], q_block=c["q_block"])
    if kind == "select_kept":
        return va.block_select(s["q"], s["means"], c["topk"], q_block=c["q_block"])
    how = dict(block=c["block"], q_block=c["q_block"], key_lens=s["lens"])
    if kind == "sparse_fwd":
        return va.block_attention(s["q"], s["k"], s["v"], s["blocks"], **how)
    o, o32, lse = va.block_fwd(s["q"], s["k"], s["v"], s["blocks"], **how)
    dq, dk, dv = va.block_bwd(s["q"], s["k"], s["v"], s["blocks"], o32, lse, s["dout"], **how)
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind.startswith("rms"):
        return _plain_rms(s)
    if kind == "dropout":
        keep, up = _plain_mask(s["rng"], c["p"], s["x"].shape), _up(c["p"])
        y = torch.where(keep, s["x"].float() * up, 0.0)
        if s["residual"] is not None:
            y = s["residual"].float() + y
        out = s["x"] if s["residual"] is None else s["residual"]
        return {"y": y.to(out.dtype), "dx": torch.where(keep, s["dy"].float() * up, 0.0).to(s["dy"].dtype)}
    if kind == "select":
        return _plain_select(s["q"], _plain_means(s["k"], c["block"], s["lens"]), c["topk"], c["q_block"])
    if kind == "select_kept":
        return _plain_select(s["q"], s["means"], c["topk"], c["q_block"])
    if c["q_block"] >= 32 or c["Nq"] <= 64:
        return _plain_gathered(s)
    return _plain_masked(s)


# dropout: element c of row r (rows in order) is kept if its 16 bits are at least round(65536 p). They are half c % 8 of
# the four words that the Philox 4x32 generator of ten rounds gives for the counter (c / 8, r, offset) and the key `seed`.


def _threshold(p):
    return round(p * 65536)


def _up(p):
    return 65536 / (65536 - _threshold(p)) if _threshold(p) < 65536 else 0.0


def _philox(words, key):
    low = 0xffffffff
    for _ in range(10):
        a, b = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57
        words = [((b >> 32) & low) ^ words[1] ^ key[0], b & low, ((a >> 32) & low) ^ words[3] ^ key[1], a & low]
        key = [(key[0] + 0x9E3779B9) & low, (key[1] + 0xBB67AE85) & low]
    return words


def _plain_mask(rng, p, shape):
    seed, offset = rng
    D, rows = shape[-1], math.prod(shape[:-1])
    low = 0xffffffff
    c = torch.arange((D + 7) // 8, device="cuda").expand(rows, -1)
    r = torch.arange(rows, device="cuda").unsqueeze(1).expand_as(c)
    words = [c, r, torch.full_like(c, offset & low), torch.full_like(c, (offset >> 32) & low)]
    words = torch.stack(_philox(words, [seed & low, (seed >> 32) & low]), -1)
    halves = torch.stack((words & 0xffff, words >> 16), -1).flatten(1)[:, :D]
    return (halves >= _threshold(p)).view(shape)


def _plain_rms(s):
    c = s["case"]
    x, r, w = s["x"].float(), s["residual"].float(), s["w"].float()
    keep = _plain_mask(s["rng"], c["p"], x.shape) if c["p"] else None
    if keep is not None:
        x = torch.where(keep, x * _up(c["p"]), 0.0)
    h = (r + x).to(s["residual"].dtype)
    n = h.float()
    rstd = torch.rsqrt((n * n).mean(-1, keepdim=True) + EPS)
    n = n * rstd
    y = n * w
    if c["kind"] == "rms_fp8":
        N, D, G = c["N"], c["D"], c["group"] or c["D"]
        y = torch.nn.functional.pad(y, (0, -D % G)).unflatten(-1, (-1, G))
        scale = (y.abs().amax(-1) / 448.0).clamp_min(2.0 ** -126)
        y = (y / scale.unsqueeze(-1)).flatten(-2)[..., :D].to(torch.float8_e4m3fn)
        return {"y": y, "scale": scale if c["group"] else scale.squeeze(-1), "h": h}
    dy = s["dy"].float()
    g = dy * w
    dh = rstd * (g - n * (g * n).mean(-1, keepdim=True)) + s["dh"].float()
    dx = dh if keep is None else torch.where(keep, dh * _up(c["p"]), 0.0)
    dw = (dy * n).sum((0, 1), dtype=torch.float64)
    return {"y": y.to(s["x"].dtype), "h": h, "dx": dx.to(s["x"].dtype), "dres": dh.to(s["residual"].dtype),
            "dw": dw.to(s["w"].dtype)}


# the cheap score: the product of the queries' and the keys' means in 8 bits, each with a scale of its own


def _plain_eighths(mean):
    """Means (fp64) as whole numbers of -127 .. 127 and the largest magnitude."""
    mean = torch.nan_to_num(mean, nan=0.0, posinf=0.0, neginf=0.0)
    top = mean.abs().amax(-1)
    return torch.round(mean * torch.where(top > 0, 127.0 / top, 0.0).unsqueeze(-1)), top


def _plain_means(k, block, lens):
    """Each block's mean key: int8 [B, Hk, blocks, d up to a multiple of 64], and its scale, fp32, -1 of a block without keys."""
    B, Hk, Nk, d = k.shape
    nb = (Nk + block - 1) // block
    first = torch.arange(nb, device=k.device) * block
    end = torch.full((B, 1), Nk, device=k.device) if lens is None else lens.clamp(0, Nk).view(B, 1)
    count = (end - first).clamp(0, block).view(B, 1, nb)
    real = torch.arange(block, device=k.device) < count.unsqueeze(-1)
    x = torch.nn.functional.pad(k, (0, 0, 0, nb * block - Nk)).view(B, Hk, nb, block, d)
    total = torch.where(real.unsqueeze(-1), x.double(), 0.0).sum(3)
    m, top = _plain_eighths(total / count.clamp_min(1).unsqueeze(-1))
    scale = torch.where(count > 0, (top / 127.0).float(), -1.0)
    return torch.nn.functional.pad(m, (0, -d % 64)).to(torch.int8), scale


def _plain_select(q, means, topk, q_block):
    """The topk blocks of highest score in ascending order, then -1; ties go to the lowest."""
    m, scale = means
    B, H, Nq, d = q.shape
    Hk, nb = m.shape[1:3]
    groups = (Nq + q_block - 1) // q_block
    count = (Nq - torch.arange(groups, device=q.device) * q_block).clamp_max(q_block)
    x = torch.nn.functional.pad(q.double(), (0, 0, 0, groups * q_block - Nq)).view(B, H, groups, q_block, d)
    x, _ = _plain_eighths(x.sum(3) / count.unsqueeze(-1))
    # whole numbers below 2^24: exact in fp32
    score = torch.matmul(x.float().view(B, Hk, -1, d), m[..., :d].float().transpose(-1, -2).contiguous())
    score = torch.where(scale.unsqueeze(2) < 0, -math.inf, score * scale.unsqueeze(2)).view(B, H, groups, nb)
    n = min(topk, nb)
    top, at = torch.sort(score, dim=-1, descending=True, stable=True)
    at = torch.where(top[..., :n] == -math.inf, nb, at[..., :n]).sort(-1)[0]
    at = torch.nn.functional.pad(at, (0, topk - n), value=nb)
    return torch.where(at == nb, -1, at).to(torch.int32)


def _plain_softmax(x):
    """softmax over the last dim; rows of -inf alone are zero."""
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    return x.div_(torch.where(total == 0, 1.0, total))


def _plain_gathered(s):
    """Each group's queries over the keys of its blocks, gathered."""
    c = s["case"]
    q, k, v, blocks = s["q"], s["k"], s["v"], s["blocks"]
    B, H, Nq, d = q.shape
    Hk, Nk, block, qb = k.shape[1], k.shape[2], c["block"], c["q_block"]
    groups, topk = blocks.shape[2:]
    scale = 1.0 / math.sqrt(d)
    end = torch.full((B,), Nk, device=q.device) if s["lens"] is None else s["lens"].clamp(0, Nk)
    keys = (blocks.long().unsqueeze(-1) * block + torch.arange(block, device=q.device)).flatten(-2)  # [B, H, groups, keys]
    real = (blocks.repeat_interleave(block, -1) >= 0) & (keys < end.view(B, 1, 1, 1))
    head = torch.arange(B * Hk, device=q.device).view(B, Hk).repeat_interleave(H // Hk, 1)
    rows = torch.where(real, keys, 0) + head.view(B, H, 1, 1) * Nk
    n = B * H * groups
    k_ = k.reshape(-1, d)[rows.view(-1)].float().view(n, -1, d)
    v_ = v.reshape(-1, d)[rows.view(-1)].float().view(n, -1, d)

    def grouped(x):
        return torch.nn.functional.pad(x.float(), (0, 0, 0, groups * qb - Nq)).view(n, qb, d)

    def whole(x):
        return x.view(B, H, groups * qb, d)[:, :, :Nq].to(torch.bfloat16)

    q_ = grouped(q)
    x = torch.bmm(q_, k_.transpose(1, 2)).mul_(scale).masked_fill_(~real.view(n, 1, -1), -math.inf)
    p = _plain_softmax(x)
    o = torch.bmm(p, v_)
    if "dout" not in s:
        return whole(o)
    do = grouped(s["dout"])
    dv = torch.bmm(p.transpose(1, 2), do)
    dp = torch.bmm(do, v_.transpose(1, 2))
    ds = dp.sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.bmm(ds, k_), torch.bmm(ds.transpose(1, 2), q_)

    def summed(x):
        """Back to [B, Hk, Nk, d], a key's shares added."""
        x = torch.where(real.view(n, -1, 1), x, 0.0)
        return torch.zeros((B * Hk * Nk, d), device=q.device).index_add_(0, rows.view(-1), x.view(-1, d)) \
            .view(B, Hk, Nk, d).to(torch.bfloat16)

    return {"o": whole(o), "dq": whole(dq), "dk": summed(dk), "dv": summed(dv)}


def _plain_masked(s):
    """Every score, those of blocks that a query did not choose masked."""
    c = s["case"]
    q, k, v, blocks = s["q"], s["k"], s["v"], s["blocks"]
    B, H, Nq, d = q.shape
    Hk, Nk, block = k.shape[1], k.shape[2], c["block"]
    G, nb, scale = H // Hk, (Nk + block - 1) // block, 1.0 / math.sqrt(d)
    chosen = torch.zeros((B, H, blocks.shape[2], nb + 1), dtype=torch.bool, device=q.device)
    chosen.scatter_(3, torch.where(blocks < 0, nb, blocks).long(), True)
    mask = chosen[..., :nb].repeat_interleave(block, 3)[..., :Nk].repeat_interleave(c["q_block"], 2)[:, :, :Nq]
    if s["lens"] is not None:
        mask = mask & (torch.arange(Nk, device=q.device) < s["lens"].view(B, 1, 1, 1))
    q_, k_, v_ = q.float(), k.float().repeat_interleave(G, 1), v.float().repeat_interleave(G, 1)
    p = _plain_softmax(torch.matmul(q_, k_.transpose(-1, -2)).mul_(scale).masked_fill_(~mask, -math.inf))
    o = torch.matmul(p, v_)
    t = torch.bfloat16
    if "dout" not in s:
        return o.to(t)
    do = s["dout"].float()
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = torch.matmul(do, v_.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = torch.matmul(ds, k_), torch.matmul(ds.transpose(-1, -2), q_)
    dk, dv = (x.view(B, Hk, G, Nk, d).sum(2) for x in (dk, dv))
    return {"o": o.to(t), "dq": dq.to(t), "dk": dk.to(t), "dv": dv.to(t)}


# ------------------------------------------------------------------ what a pass cannot do without


def _bytes(name):
    return {"bf16": 2, "fp16": 2, "fp32": 4, "none": 0}[name]


def work(case):
    kind, B = case["kind"], case["B"]
    if kind.startswith("rms"):
        n, w, r = B * case["N"] * case["D"], _bytes(case["dtype"]), _bytes(case["res"])
        wb = case["D"] * (2 if case["dtype"] == "bf16" else 4)
        if kind == "rms_fp8":  # x and residual in, h, y and the scales out
            return {"bytes": n * (w + 2 * r + 1) + 4 * n // (case["group"] or case["D"]) + wb, "flops": 8 * n}
        # forward x, residual, h, y; backward dy, dh, dx, dres
        return {"bytes": n * 4 * (w + r) + 2 * wb, "flops": 20 * n}
    if kind == "dropout":
        n, w, r = B * case["H"] * case["N"] * case["D"], _bytes(case["dtype"]), _bytes(case["res"])
        return {"bytes": n * (3 * w + (2 * r if r else w)), "flops": 4 * n}
    H, Hk, Nq, Nk, d, block, qb, topk = (case[x] for x in ("H", "Hk", "Nq", "Nk", "d", "block", "q_block", "topk"))
    groups, nb = -(-Nq // qb), -(-Nk // block)
    chosen = min(topk, nb)
    out = B * H * groups * topk * 4
    if kind == "select_kept":
        return {"bytes": 2 * B * H * Nq * d + B * Hk * nb * (d + 4) + out, "flops": 2 * B * H * groups * nb * d}
    if kind == "select":
        return {"bytes": 2 * B * d * (H * Nq + Hk * Nk) + out, "flops": 2 * B * H * groups * nb * d}
    pairs = B * H * Nq * min(chosen * block, Nk)
    q, k = B * H * Nq * d, B * Hk * Nk * d
    if kind == "sparse_fwd":  # K and V: at most those that are chosen
        k = min(k, B * H * groups * min(chosen * block, Nk) * d)
        return {"bytes": 2 * (2 * q + 2 * k) + out, "flops": 4 * pairs * d}
    return {"bytes": 2 * (4 * q + 4 * k) + out, "flops": 14 * pairs * d}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("rms"):
        return _exact_rms(s)
    if kind == "dropout":
        kept = _exact_kept(s["rng"], case["p"], s["x"].shape)
        y = s["x"].double() * kept
        return {"y": y if s["residual"] is None else y + s["residual"].double(), "dx": s["dy"].double() * kept}
    if kind.startswith("select"):
        return _exact_select(s)
    return _exact_sparse(s)


def _exact_kept(rng, p, shape):
    """What each element is multiplied with: 0 or 1/(1 - p), by the generator's definition in 16-bit limbs."""
    seed, offset = rng
    D, rows, mask = shape[-1], math.prod(shape[:-1]), 0xffffffff
    n = (D + 7) // 8

    def product(x, m):
        """High and low 32 bits of x m."""
        a, b = x >> 16, x & 0xffff
        hi, lo = m >> 16, m & 0xffff
        mid = (b * lo >> 16) + (a * lo & 0xffff) + (b * hi & 0xffff)
        return a * hi + (a * lo >> 16) + (b * hi >> 16) + (mid >> 16), (b * lo & 0xffff) | ((mid & 0xffff) << 16)

    i = torch.arange(rows * n, device="cuda")
    c0, c1 = i % n, i // n
    c2, c3 = torch.full_like(i, offset & mask), torch.full_like(i, offset >> 32 & mask)
    for turn in range(10):
        k0, k1 = ((seed & mask) + turn * 0x9E3779B9) & mask, ((seed >> 32 & mask) + turn * 0xBB67AE85) & mask
        (h0, l0), (h1, l1) = product(c0, 0xD2511F53), product(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
    bits = torch.empty((rows, n, 8), dtype=torch.int64, device="cuda")
    for w, c in enumerate((c0, c1, c2, c3)):
        bits[..., 2 * w], bits[..., 2 * w + 1] = (c & 0xffff).view(rows, n), (c >> 16).view(rows, n)
    t = round(p * 65536)
    return (bits.view(rows, 8 * n)[:, :D] >= t).double().mul_(65536 / (65536 - t)).view(shape)


def _exact_rms(s):
    c = s["case"]
    x, w = s["x"].double(), s["w"].double()
    kept = _exact_kept(s["rng"], c["p"], x.shape) if c["p"] else 1.0
    h = s["residual"].double() + x * kept
    z = h.to(s["residual"].dtype).double()  # what is stored is what is normalised
    D = c["D"]
    norm = (z.square().sum(-1, keepdim=True) / D + EPS).sqrt()
    y = z / norm * w
    if c["kind"] == "rms_fp8":
        G = c["group"] or D
        scale = torch.stack([part.abs().amax(-1) for part in y.split(G, -1)], -1).div(448).clamp_min(2.0 ** -126)
        y = y / scale.repeat_interleave(G, -1)[..., :D]
        return {"y": y, "scale": scale if c["group"] else scale[..., 0], "h": h}
    dy = s["dy"].double()
    g = dy * w
    dh = g / norm - z * (g * z).sum(-1, keepdim=True) / (D * norm ** 3) + s["dh"].double()
    return {"y": y, "h": h, "dx": dh * kept, "dres": dh, "dw": (dy * z / norm).flatten(0, 1).sum(0)}


def _exact_select(s):
    c = s["case"]
    q, qb, topk, block = s["q"].double(), c["q_block"], c["topk"], c["block"]
    B, H, Nq, d = q.shape
    nb, per = -(-c["Nk"] // block), H // c["Hk"]
    out = torch.full((B, H, -(-Nq // qb), topk), -1, dtype=torch.int32, device=q.device)

    def whole(x):
        """Rows in 8 bits, and each row's largest magnitude."""
        top = x.abs().amax(1, keepdim=True)
        return (x * (127 / top).nan_to_num(0, 0, 0)).round(), top.squeeze(1)

    def means(x, n):
        return torch.stack([part.mean(0) for part in x.split(n)]) if n > 1 else x

    for b in range(B):
        for h in range(H):
            n = c["Nk"] if s["lens"] is None else int(s["lens"][b])
            if "means" in s:
                m, scale = s["means"][0][b, h // per, :, :d].double(), s["means"][1][b, h // per]
                m, scale = m[scale >= 0], scale[scale >= 0]
            else:
                m, top = whole(means(s["k"][b, h // per, :n].double(), block))
                scale = (top / 127).float()
            x, _ = whole(means(q[b, h], qb))
            score = (x @ m.T * scale.double()).float()  # (a score is an fp32 number)
            k = min(topk, m.shape[0])
            order = torch.argsort(score, dim=1, descending=True, stable=True)[:, :k].sort(1)[0]
            out[b, h, :, :k] = order.int()
    return out


def _exact_sparse(s):
    c = s["case"]
    B, H, Hk, Nq, Nk, d, block, qb = (c[x] for x in ("B", "H", "Hk", "Nq", "Nk", "d", "block", "q_block"))
    train = c["kind"] == "sparse_train"
    dev = s["q"].device
    new = lambda h, n: torch.zeros((B, h, n, d), dtype=torch.float64, device=dev)  # noqa: E731
    r = {"o": new(H, Nq), "dq": new(H, Nq), "dk": new(Hk, Nk), "dv": new(Hk, Nk)}
    few = qb < 32 and Nq > 64  # a group of queries at a time, or blocks of rows against all keys
    step = qb if not few else 1024
    blocks = s["blocks"].cpu()
    for b in range(B):
        n = Nk if s["lens"] is None else int(s["lens"][b])
        for h in range(H):
            hk = h // (H // Hk)
            k, v = s["k"][b, hk].double(), s["v"][b, hk].double()
            for i in range(0, Nq, step):
                at = slice(i, min(Nq, i + step))
                q = s["q"][b, h, at].double()
                if few:
                    rows = torch.arange(i, min(Nq, i + step), device=dev) // qb
                    mine = s["blocks"][b, h, rows]
                    keys = torch.arange(n, device=dev)
                    hit = torch.zeros((len(rows), Nk // block + 2), dtype=torch.bool, device=dev)
                    hit[torch.arange(len(rows), device=dev).unsqueeze(1), mine.long()] = True  # (-1: the last column)
                    mask = hit[:, keys // block]
                else:
                    ids = blocks[b, h, i // qb]
                    keys = (ids[ids >= 0].long().unsqueeze(1) * block + torch.arange(block)).flatten()
                    keys = keys[keys < n].to(dev)
                    mask = None
                if not len(keys):
                    continue
                kk, vv = k[keys], v[keys]
                x = q @ kk.T / math.sqrt(d)
                if mask is not None:
                    x = x.masked_fill(~mask, -math.inf)
                p = torch.softmax(x, -1).nan_to_num(0.0)
                r["o"][b, h, at] = p @ vv
                if not train:
                    continue
                do = s["dout"][b, h, at].double()
                ds = do @ vv.T
                ds = p * (ds - (p * ds).sum(-1, keepdim=True)) / math.sqrt(d)
                r["dq"][b, h, at] = ds @ kk
                r["dk"][b, hk].index_add_(0, keys, ds.T @ q)
                r["dv"][b, hk].index_add_(0, keys, p.T @ do)
    return r if train else r["o"]
