"""Cases of the operators around the attention: layer norm, rotary positions with several axes, and differential
attention, each as a ViT block uses it, timed and checked one by one.

A case is a dict of plain values. `kind` says which entry points it goes through:

  norm_fwd     layer_norm_fwd                       inference
  norm_train   layer_norm_fwd, layer_norm_bwd       the two halves of a training step
  rotary       rotary_fwd on q and k                forward
  rotary_grad  rotary_fwd(inverse=True) on dq, dk   backward
  diff_fwd     diff_attention                       inference, down to one query over a long key set
  diff_train   diff_fwd, diff_bwd                   the two halves of a training step

With `own` false, run() computes the same in elementary torch operations.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # the class token's row alone, as a served model's last norm sees it: launch and latency
        _norm("norm_token", "norm_fwd", 1, 1, 1, 768, "bf16"),
        # one block of a model of width 1,024 over 8,192 tokens of 4 images: an ordinary training norm
        _norm("norm_block_train", "norm_train", 4, 1, 8192, 1024, "bf16"),
        # per-head norm of the queries of 16 heads of 72, sequence-major as the projection leaves them, odd length
        _norm("norm_heads_train", "norm_train", 1, 16, 20001, 72, "bf16", layout="bnhd"),
        # a wide fp32 stem whose width is no multiple of a vector, few rows
        _norm("norm_wide_fp32_train", "norm_train", 2, 1, 1531, 5001, "fp32"),
        # time, height and width of a clip of 368x512 patches, q and k of 16 heads as the projection leaves them
        _rotary("rotary_188k", "rotary", 1, 16, 16, 188416, 64, "8,12,12", "bf16", layout="bnhd"),
        # a served frame's one new token
        _rotary("rotary_token", "rotary", 1, 8, 8, 1, 128, "16,24,24", "bf16", far=1000000),
        # gradient of a 2-axis rotation in fp32, adjacent pairs, a part of each row left as it is, odd length
        _rotary("rotary_fp32_grad", "rotary_grad", 2, 12, 4, 5003, 80, "17,17", "fp32", interleaved=True),
        # one class-token query over a small image's patches: launch and latency
        _diff("diff_token_197", "diff_fwd", 1, 8, 1, 197, 32, 64),
        # one query of 8 heads over a long clip's keys: the bytes of K and V
        _diff("diff_token_128k", "diff_fwd", 1, 8, 1, 131072, 64, 128),
        # a whole batch of small images in a training step
        _diff("diff_vit_1k_train", "diff_train", 8, 8, 1024, 1024, 32, 64),
        # heads of 72, sequence-major, an odd crop, the second image padded
        _diff("diff_crop_5k_d72_train", "diff_train", 2, 4, 5003, 5003, 72, 144, layout="bnhd", padded=True),
        # four heads of a long sequence: the matrix cores
        _diff("diff_shard_32k_train", "diff_train", 1, 4, 32768, 32768, 64, 128),
    ]


def _norm(name, kind, B, H, N, D, dtype, layout="bhnd"):
    return dict(name=name, kind=kind, B=B, H=H, N=N, D=D, dtype=dtype, layout=layout)


def _rotary(name, kind, B, H, Hk, N, d, sections, dtype, layout="bhnd", interleaved=False, far=0):
    """sections: pairs of columns per axis; far: positions start there."""
    return dict(name=name, kind=kind, B=B, H=H, Hk=Hk, N=N, d=d, sections=sections, dtype=dtype, layout=layout,
                interleaved=interleaved, far=far)


def _diff(name, kind, B, H, Nq, Nk, d, e, layout="bhnd", padded=False):
    """d columns of q and k, e of v; padded: the samples after the first hold fewer keys."""
    return dict(name=name, kind=kind, B=B, H=H, Nq=Nq, Nk=Nk, d=d, e=e, layout=layout, padded=padded)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_train", "norm_train", "rotary", "rotary_grad", "diff_fwd", "diff_fwd",
                       "diff_train", "diff_train"])
    if kind.startswith("norm"):
        c = _norm("", kind, rng.choice([1, 1, 2, 4]), rng.choice([1, 1, 2, 8, 16]), _log_int(rng, 1, 40000),
                  rng.choice([64, 72, 128, 160, _log_int(rng, 33, 8200), _log_int(rng, 33, 8200)]),
                  rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice(["bhnd", "bnhd"]))
        while c["B"] * c["H"] * c["N"] * c["D"] > 32768 * 1024:
            c["N"] = c["N"] // 2 + 1
    elif kind.startswith("rotary"):
        d = rng.choice([32, 64, 72, 80, 128, 160])
        axes = rng.choice([1, 2, 2, 3, 3])
        s = [rng.randint(1, d // 2 // axes) for _ in range(axes)] if rng.random() < 0.4 else [d // 2 // axes] * axes
        c = _rotary("", kind, rng.choice([1, 1, 2, 4]), rng.choice([4, 8, 12, 16]), rng.choice([2, 4, 8, 16]),
                    _log_int(rng, 1, 188416), d, ",".join(str(x) for x in s), rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                    rng.choice(["bhnd", "bnhd"]), rng.random() < 0.4, rng.choice([0, 0, 1000000]))
        while c["B"] * (c["H"] + c["Hk"]) * c["N"] * c["d"] * (2 if c["dtype"] == "fp32" else 1) > 32 * 188416 * 64:
            c["N"] = c["N"] // 2 + 1
    else:
        d, e = rng.choice([(32, 64), (64, 128), (64, 128), (72, 144), (80, 160), (40, 80), (64, 64)])
        Nk = _log_int(rng, 16, 131072)
        Nq = Nk if kind == "diff_train" else rng.choice([1, 1, rng.randint(2, 64), Nk])
        if kind == "diff_train" and rng.random() < 0.25:
            Nq = max(1, Nk // rng.randint(2, 9))
        c = _diff("", kind, rng.choice([1, 1, 2, 4]), rng.choice([4, 6, 8, 12]), Nq, Nk, d, e,
                  rng.choice(["bhnd", "bnhd"]), rng.random() < 0.3)
        while c["B"] * c["H"] * c["Nq"] * c["Nk"] * max(2 * d + e, 256) > 4 * 32768 ** 2 * 256 \
                or c["B"] * c["H"] * c["Nk"] * (2 * d + e) > 8 * 131072 * 256:
            c["Nk"] = c["Nk"] // 2 + 1
            c["Nq"] = min(c["Nq"], c["Nk"])
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _rows(g, B, H, N, D, dtype, layout, mean=None):
    """Activations [B, H, N, D]: normal values, about a mean of each column's own if one is given."""
    x = torch.randn((B, N, H, D) if layout == "bnhd" else (B, H, N, D), generator=g, device="cuda")
    if mean is not None:
        x += mean
    x = x.to(dtype)
    return x.transpose(1, 2) if layout == "bnhd" else x


def prepare(case, seed):
    g = _gen(seed)
    kind, B, H = case["kind"], case["B"], case["H"]
    s = {"case": case}
    if kind.startswith("norm"):
        t, N, D = TYPES[case["dtype"]], case["N"], case["D"]
        wt = torch.float32 if t == torch.float16 else t  # mixed precision keeps fp32 weights beside fp16
        s["x"] = _rows(g, B, H, N, D, t, case["layout"], 0.5 * torch.randn(D, generator=g, device="cuda"))
        s["w"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(wt)
        s["b"] = (0.1 * torch.randn(D, generator=g, device="cuda")).to(wt)
        if kind == "norm_train":
            s["dy"] = _rows(g, B, H, N, D, t, case["layout"], 0.2 * torch.randn(D, generator=g, device="cuda"))
    elif kind.startswith("rotary"):
        t, N, d = TYPES[case["dtype"]], case["N"], case["d"]
        s["sections"] = tuple(int(x) for x in case["sections"].split(","))
        s["q"] = _rows(g, B, H, N, d, t, case["layout"])
        s["k"] = _rows(g, B, case["Hk"], N, d, t, case["layout"])
        s["pos"] = _positions(g, N, len(s["sections"]), case["far"])
    else:
        Nq, Nk, d, e = case["Nq"], case["Nk"], case["d"], case["e"]
        s["q"] = _rows(g, B, 2 * H, Nq, d, torch.bfloat16, case["layout"])
        s["k"] = _rows(g, B, 2 * H, Nk, d, torch.bfloat16, case["layout"])
        # values share a mean, and the gradient has a part along it (a loss that grows with the output), so that
        # lam's gradient is a signal and not the sum of independent noise
        mean = torch.randn(e, generator=g, device="cuda")
        s["v"] = _rows(g, B, H, Nk, e, torch.bfloat16, case["layout"], 0.5 * mean)
        s["lam"] = (0.2 + 0.6 * torch.rand(H, generator=g, device="cuda")).to(torch.bfloat16)
        s["lens"] = None
        if case["padded"]:  # the first sample is whole
            lens = torch.randint(max(1, Nk // 2), Nk + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            lens[0] = Nk
            s["lens"] = lens
        if kind == "diff_train":
            s["dout"] = _rows(g, B, H, Nq, e, torch.bfloat16, case["layout"], 0.3 * mean)
    return s


def _positions(g, N, axes, far):
    """Patch coordinates [N, axes] of a grid as near to a cube as N allows, the first axis from `far` on."""
    side = max(1, math.ceil(N ** (1.0 / axes) - 1e-9))
    n = torch.arange(N, device="cuda")
    cols = []
    for a in range(axes):
        cols.append(n % side if a < axes - 1 else n)
        n = n // side
    pos = torch.stack(cols[::-1], 1)
    pos[:, 0] += far + torch.randint(0, 64, (1,), generator=g, device="cuda")
    return pos


# ------------------------------------------------------------------ one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2405_15780_amd as va

    c = s["case"]
    kind = c["kind"]
    if kind == "norm_fwd":
        return va.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
    if kind == "norm_train":
        y, mean, rstd = va.layer_norm_fwd(s["x"], s["w"], s["b"], eps=EPS)
        dx, dw, db = va.layer_norm_bwd(s["x"], s["w"], mean, rstd, s["dy"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if kind.startswith("rotary"):
        q, k = va.rotary_fwd(s["q"], s["k"], s["pos"], s["sections"], interleaved=c["interleaved"],
                             inverse=kind == "rotary_grad")
        return {"q": q, "k": k}
    if kind == "diff_fwd":
        return va.diff_attention(s["q"], s["k"], s["v"], s["lam"], key_lens=s["lens"])
    o, o2, lse = va.diff_fwd(s["q"], s["k"], s["v"], s["lam"], key_lens=s["lens"])
    dq, dk, dv, dlam = va.diff_bwd(s["q"], s["k"], s["v"], s["lam"], o, o2, lse, s["dout"], key_lens=s["lens"])
    return {"o": o, "dq": dq, "dk": dk, "dv": dv, "dlam": dlam}


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("norm"):
        return _plain_norm(s)
    if kind.startswith("rotary"):
        return _plain_rotary(s)
    return _plain_diff(s)


def _plain_norm(s):
    t = s["x"].dtype
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    mean = x.mean(-1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    h = x * rstd
    y = (h * w + b).to(t)
    if "dy" not in s:
        return y
    dy = s["dy"].float()
    gw = dy * w
    dx = rstd * (gw - gw.mean(-1, keepdim=True) - h * (gw * h).mean(-1, keepdim=True))
    dw = (dy * h).sum((0, 1, 2), dtype=torch.float64)
    db = dy.sum((0, 1, 2), dtype=torch.float64)
    return {"y": y, "dx": dx.to(t), "dw": dw.to(s["w"].dtype), "db": db.to(s["b"].dtype)}


def _plain_rotary(s):
    c = s["case"]
    sections = s["sections"]
    dev = s["q"].device
    freq = torch.cat([torch.arange(n, device=dev, dtype=torch.float64).div(-n).mul(math.log(10000.0)).exp()
                      for n in sections])
    axis = torch.repeat_interleave(torch.arange(len(sections), device=dev), torch.tensor(sections, device=dev))
    angle = s["pos"].double()[:, axis] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    if c["kind"] == "rotary_grad":
        sin = -sin
    return {"q": _rotate(s["q"], cos, sin, c["interleaved"]), "k": _rotate(s["k"], cos, sin, c["interleaved"])}


def _rotate(x, cos, sin, interleaved):
    R = cos.shape[-1]
    out = x.clone()
    first, second = (slice(0, 2 * R, 2), slice(1, 2 * R, 2)) if interleaved else (slice(0, R), slice(R, 2 * R))
    a, b = x[..., first].float(), x[..., second].float()
    out[..., first] = (a * cos - b * sin).to(x.dtype)
    out[..., second] = (b * cos + a * sin).to(x.dtype)
    return out


def _plain_softmax(q, k, scale, keep):
    """softmax(scale q k^T) over the kept keys; rows without any are zero."""
    x = torch.matmul(q, k.transpose(-1, -2)).mul_(scale)
    if keep is not None:
        x.masked_fill_(~keep, -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    return x.div_(torch.where(total == 0, 1.0, total))


def _plain_diff(s):
    c = s["case"]
    t, scale = s["q"].dtype, 1.0 / math.sqrt(c["d"])
    q1, q2 = s["q"][:, 0::2].float(), s["q"][:, 1::2].float()
    k1, k2 = s["k"][:, 0::2].float(), s["k"][:, 1::2].float()
    v, lam = s["v"].float(), s["lam"].float().view(1, -1, 1, 1)
    keep = None
    if s["lens"] is not None:
        keep = (torch.arange(c["Nk"], device=v.device) < s["lens"].view(-1, 1)).view(-1, 1, 1, c["Nk"])
    p1, p2 = _plain_softmax(q1, k1, scale, keep), _plain_softmax(q2, k2, scale, keep)
    o1, o2 = torch.matmul(p1, v), torch.matmul(p2, v)
    o = (o1 - lam * o2).to(t)
    if "dout" not in s:
        return o
    do = s["dout"].float()
    d1, d2 = (do * o1).sum(-1, keepdim=True), (do * o2).sum(-1, keepdim=True)
    dlam = d2.sum((0, 2, 3), dtype=torch.float64).neg()
    dp = torch.matmul(do, v.transpose(-1, -2))
    dv = torch.matmul(p1.transpose(-1, -2), do) - lam * torch.matmul(p2.transpose(-1, -2), do)
    ds1 = p1.mul_(dp - d1).mul_(scale)
    ds2 = p2.mul_(dp.sub_(d2)).mul_(-scale * lam)
    dq = torch.stack((torch.matmul(ds1, k1), torch.matmul(ds2, k2)), 2).flatten(1, 2)
    dk = torch.stack((torch.matmul(ds1.transpose(-1, -2), q1), torch.matmul(ds2.transpose(-1, -2), q2)), 2).flatten(1, 2)
    return {"o": o, "dq": dq.to(t), "dk": dk.to(t), "dv": dv.to(t), "dlam": dlam.to(t)}


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    kind, B, H = case["kind"], case["B"], case["H"]
    if kind.startswith("norm"):
        n, w = B * H * case["N"] * case["D"], 4 if case["dtype"] == "fp32" else 2
        weights = case["D"] * (2 if case["dtype"] == "bf16" else 4)  # of one of w, b, dw, db
        if kind == "norm_fwd":
            return {"bytes": n * w * 2 + 2 * weights, "flops": 8 * n}
        return {"bytes": n * w * 4 + 4 * weights, "flops": 20 * n}
    if kind.startswith("rotary"):
        w, axes = 4 if case["dtype"] == "fp32" else 2, case["sections"].count(",") + 1
        n = B * (H + case["Hk"]) * case["N"] * case["d"]
        return {"bytes": 2 * n * w + case["N"] * axes * 8, "flops": 3 * n}
    Nq, Nk, d, e = case["Nq"], case["Nk"], case["d"], case["e"]
    q, k, v, o = B * 2 * H * Nq * d, B * 2 * H * Nk * d, B * H * Nk * e, B * H * Nq * e
    keys = H * Nq * Nk * (1 + (B - 1) * (0.75 if case["padded"] else 1.0))  # padded samples hold 3/4 on average
    fwd = keys * 4 * (d + e)
    if kind == "diff_fwd":
        return {"bytes": 2 * (q + k + v + o), "flops": fwd}
    # the backward's products once each: two scores, dP, dV, two dK, two dQ
    return {"bytes": 2 * (2 * (q + k + v) + 2 * o), "flops": fwd + keys * (12 * d + 4 * e)}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        return _exact_norm(s)
    if kind.startswith("rotary"):
        return _exact_rotary(s)
    return _exact_diff(s)


def _exact_norm(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    sd = (var + EPS).sqrt()
    hat = (x - mean) / sd
    y = torch.addcmul(b, hat, w)
    if "dy" not in s:
        return y
    dy = s["dy"].double()
    D = x.shape[-1]
    g = dy * w
    dx = (D * g - g.sum(-1, keepdim=True) - hat * (g * hat).sum(-1, keepdim=True)) / (D * sd)
    return {"y": y, "dx": dx, "dw": (dy * hat).flatten(0, 2).sum(0), "db": dy.flatten(0, 2).sum(0)}


def _exact_rotary(s):
    c = s["case"]
    R = sum(s["sections"])
    sign = -1.0 if c["kind"] == "rotary_grad" else 1.0
    out = {}
    for name in ("q", "k"):
        y = s[name].double()
        p = 0
        for a, n in enumerate(s["sections"]):
            for i in range(n):
                angle = sign * s["pos"][:, a].double() * 10000.0 ** (-i / n)
                lo, hi = (2 * p, 2 * p + 1) if c["interleaved"] else (p, p + R)
                z = torch.complex(y[..., lo], y[..., hi]) * torch.polar(torch.ones_like(angle), angle)
                y[..., lo], y[..., hi] = z.real, z.imag
                p += 1
        out[name] = y
    return out


def _exact_diff(s):
    c = s["case"]
    B, H, Nq, Nk, d, e = (c[x] for x in ("B", "H", "Nq", "Nk", "d", "e"))
    train = c["kind"] == "diff_train"
    if B * H * Nq * Nk * (d + e) * (7 if train else 2) > 1e14:
        return None
    dev = s["q"].device
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=dev)  # noqa: E731
    r = {"o": new(B, H, Nq, e), "dq": new(B, 2 * H, Nq, d), "dk": new(B, 2 * H, Nk, d), "dv": new(B, H, Nk, e),
         "dlam": new(H)}
    step = max(1, (1 << 28) // Nk)
    for b in range(B):
        n = Nk if s["lens"] is None else int(s["lens"][b])
        if n == 0:
            continue
        for h in range(H):
            lam, v = s["lam"][h].double(), s["v"][b, h, :n].double()
            k = [s["k"][b, 2 * h + m, :n].double() for m in (0, 1)]
            for i in range(0, Nq, step):
                at = slice(i, min(Nq, i + step))
                q = [s["q"][b, 2 * h + m, at].double() for m in (0, 1)]
                p = [torch.softmax(q[m] @ k[m].T / math.sqrt(d), -1) for m in (0, 1)]
                r["o"][b, h, at] = (p[0] - lam * p[1]) @ v
                if not train:
                    continue
                do = s["dout"][b, h, at].double()
                dp = do @ v.T
                r["dv"][b, h, :n] += (p[0] - lam * p[1]).T @ do
                for m, f in ((0, 1.0), (1, -lam)):
                    row = (p[m] * dp).sum(-1, keepdim=True)
                    if m:
                        r["dlam"][h] -= row.sum()
                    p[m] *= (dp - row) * (f / math.sqrt(d))
                    r["dq"][b, 2 * h + m, at] = p[m] @ k[m]
                    r["dk"][b, 2 * h + m, :n] += p[m].T @ q[m]
    return r if train else r["o"]
