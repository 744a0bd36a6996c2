"""The dense side of a layer over nodes of several types, as cases that can be timed and compared: layer normalisation, the
projection with a weight matrix for each node type, and checkpoints of activations in 8 bits that the backward pass reads.

Sizes follow the workloads of the benchmark (2,000 nodes of 64 columns; 1 and 2.45 million of 256; 170,000 with 47 classes)
and ragged ones between them.  A case is a dict of plain values:

  kind    norm_forward         x -> y = gamma xhat + beta, mean, rstd
          norm_backward        x, mean, rstd, gy -> gx, dgamma, dbeta
          norm_checkpoint      x -> y, rstd and the checkpoint of xhat (returned as the values that it stands for)
          norm_backward_ckpt   checkpoint of xhat, rstd, gy -> gx, dgamma, dbeta
          checkpoint           x -> checkpoint -> the values that it stands for
          typed_forward        z = h W[type], rows sorted by type
          typed_backward       dh = dz W[type]^T and dW[type] = h^T dz over the type's rows
          weight_ckpt          dW[type] = (gamma v + beta)^T dz from the checkpoint of v
  n       rows (nodes)
  c       columns of a normalised or checkpointed array; d_in, d_out, types: of a projection
  dtype   f32 | bf16: storage of the node arrays

A checkpoint holds, for every 32 consecutive columns of a row (the last of a row may be fewer), int8 codes and one byte s:
the values are code * 2^(s - 127), 0 for s = 0 and NaN for s = 255.  With E = floor(log2(max |x|)) over the block,
s = max(E - 6, -126) + 127 and code = x / 2^(s - 127) rounded to the nearest whole number (ties to even) within -127..127;
a block of zeros has s = 0, a block that holds anything infinite or NaN has s = 255.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # Normalisation of a small graph's hidden features at inference: the smallest call, launch and host time.
        dict(name="norm-forward-tiny-bf16", kind="norm_forward", n=2_000, c=64, dtype="bf16"),
        # The same of a products-sized graph in single precision.
        dict(name="norm-forward-medium-f32", kind="norm_forward", n=2_450_000, c=256, dtype="f32"),
        # Its backward pass over a million nodes in bf16: one training step's hidden layer.
        dict(name="norm-backward-dense-bf16", kind="norm_backward", n=1_000_000, c=256, dtype="bf16"),
        # Backward of a normalisation over class scores: rows of 47 columns, no whole number of 16-byte words.
        dict(name="norm-backward-classes-f32", kind="norm_backward", n=170_000, c=47, dtype="f32"),
        # Projection of a small graph with four node types: latency.
        dict(name="typed-forward-tiny-bf16", kind="typed_forward", n=2_000, d_in=64, d_out=64, types=4, dtype="bf16"),
        # Projection of a products-sized graph with eight node types of very different sizes.
        dict(name="typed-forward-medium-bf16", kind="typed_forward", n=2_450_000, d_in=256, d_out=256, types=8, dtype="bf16"),
        # Both gradients of the projection over a million nodes.
        dict(name="typed-backward-dense-bf16", kind="typed_backward", n=1_000_000, d_in=256, d_out=256, types=8, dtype="bf16"),
        # Both gradients with 64 types, a third of them empty, and widths that fill no tile.
        dict(name="typed-backward-ragged-bf16", kind="typed_backward", n=300_003, d_in=136, d_out=72, types=64, dtype="bf16"),
        # Packing an aggregate and reading it back, rows whose last block is short.
        dict(name="checkpoint-ragged-f32", kind="checkpoint", n=500_000, c=100, dtype="f32"),
        # Normalisation that leaves the checkpoint of its normalised rows for the backward pass.
        dict(name="norm-checkpoint-medium-bf16", kind="norm_checkpoint", n=2_450_000, c=256, dtype="bf16"),
        # The normalisation's backward pass from that checkpoint.
        dict(name="norm-backward-ckpt-dense-bf16", kind="norm_backward_ckpt", n=1_000_000, c=256, dtype="bf16"),
        # The projection's weight gradients from that checkpoint.
        dict(name="weight-ckpt-dense-bf16", kind="weight_ckpt", n=1_000_000, d_in=256, d_out=256, types=8, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above: rows log-uniform from some hundreds to 2.45 million; any number of columns for the
    normalisation and the checkpoints, multiples of eight (16-byte rows) for the projections."""
    kind = rng.choice(["norm_forward", "norm_backward", "norm_checkpoint", "norm_backward_ckpt", "checkpoint", "typed_forward",
                       "typed_backward", "weight_ckpt"])
    if kind in ("typed_forward", "typed_backward", "weight_ckpt"):
        d_in, d_out = 8 * _log_int(rng, 2, 64), 8 * _log_int(rng, 2, 64)
        most = min(2_450_000, int(6e10 / (d_in * d_out)), int(2.5e8 / max(d_in, d_out)))
        return dict(kind=kind, n=_log_int(rng, 300, most), d_in=d_in, d_out=d_out, types=_log_int(rng, 1, 64), dtype="bf16")
    c = 8 * _log_int(rng, 1, 128) if rng.random() < 0.6 else _log_int(rng, 3, 1000)
    n = _log_int(rng, 300, min(2_450_000, int(2.5e8 / c)))
    return dict(kind=kind, n=n, c=c, dtype=rng.choice(["f32", "bf16"]))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _scale_value(s):
    """2^(s - 127) of the bytes s as float32, from the bits of the exponent: 0 for s = 0, infinity for s = 255."""
    return (s.to(torch.int32) << 23).view(torch.float32)


def _pack(x):
    """float32 [n, c] -> (codes int8 [n, c], scales uint8 [n, blocks]).  Every step is exact: the scales are powers of two."""
    n, c = x.shape
    blocks = (c + BLOCK - 1) // BLOCK
    v = torch.zeros(n, blocks * BLOCK, dtype=torch.float32, device=x.device)
    v[:, :c] = x
    v = v.view(n, blocks, BLOCK)
    top = v.abs().amax(dim=2)
    exponent = (top.view(torch.int32) >> 23) & 255        # floor(log2(top)) + 127; 255 where top is infinite or NaN
    s = (exponent - 6).clamp(min=1)
    s = torch.where(top == 0, 0, s)
    s = torch.where(exponent == 255, 255, s)
    inverse = ((254 - s) << 23).view(torch.float32)       # 2^(127 - s)
    inverse = torch.where((s == 0) | (s == 255), 0.0, inverse)
    codes = torch.where((s == 255).unsqueeze(2), 0.0, v * inverse.unsqueeze(2)).round().clamp(-127, 127)
    return codes.to(torch.int8).view(n, blocks * BLOCK)[:, :c].contiguous(), s.to(torch.uint8)


def _unpack(codes, scales):
    """The values that a checkpoint stands for, float32 [n, c]."""
    n, c = codes.shape
    return codes.float() * _scale_value(scales).repeat_interleave(BLOCK, dim=1)[:, :c]


def _normalised(x):
    """xhat and rstd of float rows (in the type of x)."""
    d = x - x.mean(dim=1, keepdim=True)
    rstd = 1.0 / ((d * d).mean(dim=1, keepdim=True) + EPS).sqrt()
    return d * rstd, rstd


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    kind, n, dt = case["kind"], case["n"], DTYPES[case["dtype"]]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        x = torch.randn(*shape, generator=gen, device=dev, dtype=dtype)
        return x if scale == 1.0 else x.mul_(scale)

    def features(c):
        """What an aggregation leaves: columns of different means and spreads, rows of different sizes."""
        x = normal(n, c)
        x.mul_(torch.exp(normal(c, scale=0.5))).add_(normal(c, scale=0.5)).mul_(torch.exp(normal(n, 1, scale=0.7)))
        return x

    s = dict(case=case)
    if "types" in case:
        t = case["types"]
        share = torch.exp(normal(t, scale=1.5))
        if t >= 3:                                        # some types have no node in this graph
            share = torch.where(torch.rand(t, generator=gen, device=dev) < 0.33, 0.0, share)
            share[int(seed) % t] = 1.0
        ends = (torch.cumsum(share.double(), 0) / share.double().sum() * n).round().long()
        s["offsets"] = torch.cat([ends.new_zeros(1), ends])
        host = s["offsets"].tolist()
        s["rows"] = [slice(a, b) for a, b in zip(host, host[1:])]
    if kind.startswith("typed"):
        s["h"] = features(case["d_in"]).to(dt)
        s["W"] = normal(case["types"], case["d_in"], case["d_out"], scale=case["d_in"] ** -0.5).to(dt)
        if kind == "typed_backward":
            s["gz"] = normal(n, case["d_out"], dtype=dt)
        return s
    c = case["d_in"] if kind == "weight_ckpt" else case["c"]
    if kind != "checkpoint":
        s.update(gamma=normal(c, scale=0.2).add_(1.0), beta=normal(c, scale=0.3))
    x = features(c)
    if kind in ("norm_backward_ckpt", "weight_ckpt"):
        xhat, rstd = _normalised(x)
        s["codes"], s["scales"] = _pack(xhat)
        if kind == "weight_ckpt":
            s["gz"] = normal(n, case["d_out"], dtype=dt)
        else:
            s.update(rstd=rstd.view(n), gy=normal(n, c, dtype=dt))
        return s
    s["x"] = x.to(dt)
    if kind == "norm_backward":
        x = s["x"].float()
        s["mean"], s["rstd"] = x.mean(dim=1), _normalised(x)[1].view(n)
        s["gy"] = normal(n, c, dtype=dt)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def _norm_gradients(xhat, rstd, gamma, gy):
    g = gy * gamma
    gx = rstd.unsqueeze(1) * (g - g.mean(dim=1, keepdim=True) - xhat * (g * xhat).mean(dim=1, keepdim=True))
    return gx, (gy * xhat).sum(dim=0), gy.sum(dim=0)


def _typed_weight(h, gz, rows):
    return torch.stack([h[r].float().t() @ gz[r].float() for r in rows])


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "norm_forward":
        x = s["x"].float()
        xhat, rstd = _normalised(x)
        return dict(y=(xhat * s["gamma"] + s["beta"]).to(dt), mean=x.mean(dim=1), rstd=rstd.view(-1))
    if kind == "norm_backward":
        rstd = s["rstd"]
        xhat = (s["x"].float() - s["mean"].unsqueeze(1)) * rstd.unsqueeze(1)
        gx, dgamma, dbeta = _norm_gradients(xhat, rstd, s["gamma"], s["gy"].float())
        return dict(gx=gx.to(dt), dgamma=dgamma, dbeta=dbeta)
    if kind == "norm_checkpoint":
        xhat, rstd = _normalised(s["x"].float())
        return dict(y=(xhat * s["gamma"] + s["beta"]).to(dt), rstd=rstd.view(-1), xhat=_unpack(*_pack(xhat)).to(torch.bfloat16))
    if kind == "norm_backward_ckpt":
        gx, dgamma, dbeta = _norm_gradients(_unpack(s["codes"], s["scales"]), s["rstd"], s["gamma"], s["gy"].float())
        return dict(gx=gx.to(dt), dgamma=dgamma, dbeta=dbeta)
    if kind == "checkpoint":
        return _unpack(*_pack(s["x"].float())).to(dt)
    if kind == "typed_forward":
        return torch.cat([s["h"][r].float() @ w for r, w in zip(s["rows"], s["W"].float())]).to(dt)
    if kind == "typed_backward":
        dh = torch.cat([s["gz"][r].float() @ w.t() for r, w in zip(s["rows"], s["W"].float())]).to(dt)
        return dict(dh=dh, dW=_typed_weight(s["h"], s["gz"], s["rows"]))
    if kind == "weight_ckpt":
        return _typed_weight(_unpack(s["codes"], s["scales"]) * s["gamma"] + s["beta"], s["gz"], s["rows"])
    raise ValueError(kind)


def _run_own(s):
    from paper_2111_06483_b200 import api
    case = s["case"]
    kind, dt = case["kind"], DTYPES[case["dtype"]]
    if kind == "norm_forward":
        y, (mean, rstd) = api.ln_forward(s["x"], EPS, s["gamma"], s["beta"])
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "norm_backward":
        gx, dgamma, dbeta = api.ln_backward(s["x"], s["gy"], (s["mean"], s["rstd"]), s["gamma"])
        return dict(gx=gx, dgamma=dgamma, dbeta=dbeta)
    if kind == "norm_checkpoint":
        y, (ckpt, rstd) = api.ln_forward(s["x"], EPS, s["gamma"], s["beta"], checkpoint=True)
        return dict(y=y, rstd=rstd, xhat=api.ckpt8_unpack(ckpt, torch.bfloat16))
    if kind == "norm_backward_ckpt":
        gx, dgamma, dbeta = api.ln_backward(None, s["gy"], (api.Checkpoint8(s["codes"], s["scales"]), s["rstd"]), s["gamma"])
        return dict(gx=gx, dgamma=dgamma, dbeta=dbeta)
    if kind == "checkpoint":
        return api.ckpt8_unpack(api.ckpt8_pack(s["x"]), dt)
    if kind == "typed_forward":
        return api.typed_linear_forward(s["h"], s["W"], s["offsets"])
    if kind == "typed_backward":
        dh, dW = api.typed_linear_backward(s["h"], s["W"], s["offsets"], s["gz"])
        return dict(dh=dh, dW=dW)
    if kind == "weight_ckpt":
        return api.typed_linear_backward_weight(api.Checkpoint8(s["codes"], s["scales"]), s["offsets"], s["gz"], s["gamma"], s["beta"])
    raise ValueError(kind)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    """Bytes: every input read once, every output written once.  Operations: the multiplications and additions of the formulas."""
    kind, n = case["kind"], case["n"]
    b = 2 if case["dtype"] == "bf16" else 4
    if "types" in case:
        d, f, t = case["d_in"], case["d_out"], case["types"]
        product, weights = 2 * n * d * f, t * d * f
        if kind == "typed_forward":
            return {"bytes": n * (d + f) * b + weights * b + 8 * t, "flops": product}
        if kind == "typed_backward":
            return {"bytes": n * (2 * d + f) * b + weights * (b + 4) + 8 * t, "flops": 2 * product}
        packed = n * d + n * ((d + BLOCK - 1) // BLOCK)
        return {"bytes": packed + n * f * b + weights * 4 + 8 * t, "flops": product + 2 * n * d}
    c = case["c"]
    array, packed = n * c * b, n * c + n * ((c + BLOCK - 1) // BLOCK)
    if kind == "norm_forward":
        return {"bytes": 2 * array + 8 * n + 8 * c, "flops": 8 * n * c}
    if kind == "norm_backward":
        return {"bytes": 3 * array + 8 * n + 12 * c, "flops": 14 * n * c}
    if kind == "norm_checkpoint":      # the values that the checkpoint stands for are read back: its bytes twice, and 2 bytes a value
        return {"bytes": 2 * array + 2 * packed + 2 * n * c + 4 * n + 8 * c, "flops": 11 * n * c}
    if kind == "norm_backward_ckpt":
        return {"bytes": 2 * array + packed + 4 * n + 12 * c, "flops": 13 * n * c}
    if kind == "checkpoint":
        return {"bytes": 2 * array + 2 * packed, "flops": 4 * n * c}
    raise ValueError(kind)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

_POWERS = [0.0] + [2.0 ** (s - 127) for s in range(1, 255)] + [math.nan]


def _exact_checkpoint(x):
    """What the checkpoint of the 64-bit rows x stands for, block by block from the definition."""
    out = torch.empty_like(x)
    powers = torch.tensor(_POWERS, dtype=torch.float64, device=x.device)
    for at in range(0, x.shape[1], BLOCK):
        v = x[:, at:at + BLOCK]
        top = v.abs().max(dim=1, keepdim=True).values
        fine = torch.isfinite(top)
        floor_log2 = torch.frexp(torch.where(fine & (top > 0), top, 1.0)).exponent - 1
        s = torch.clamp(floor_log2 - 6, min=-126) + 127
        unit = powers[s.long()]
        held = torch.clamp(torch.round(torch.where(fine, v, 0.0) / unit), -127, 127) * unit
        out[:, at:at + BLOCK] = torch.where(fine, held, math.nan)
    return out


def _exact_values(s):
    codes, scales = s["codes"].double(), s["scales"].long()
    powers = torch.tensor(_POWERS, dtype=torch.float64, device=codes.device)
    column_block = torch.arange(codes.shape[1], device=codes.device) // BLOCK
    return codes.mul_(powers[scales][:, column_block])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    f64 = torch.float64
    if kind in ("norm_forward", "norm_checkpoint"):
        x = s["x"].to(f64)
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPS).rsqrt()
        xhat = x.sub_(mean[:, None]).mul_(rstd[:, None])
        y = xhat * s["gamma"].to(f64) + s["beta"].to(f64)
        if kind == "norm_forward":
            return dict(y=y, mean=mean, rstd=rstd)
        return dict(y=y, rstd=rstd, xhat=_exact_checkpoint(xhat))
    if kind in ("norm_backward", "norm_backward_ckpt"):
        rstd = s["rstd"].to(f64)[:, None]
        xhat = _exact_values(s) if kind == "norm_backward_ckpt" else (s["x"].to(f64) - s["mean"].to(f64)[:, None]) * rstd
        gy, gamma, c = s["gy"].to(f64), s["gamma"].to(f64), case["c"]
        # gx = rstd (g - <g, 1>/c - xhat <g, xhat>/c) with g = gamma gy
        along = torch.einsum("nc,nc,c->n", gy, xhat, gamma)[:, None] / c
        level = (gy @ gamma)[:, None] / c
        dgamma, dbeta = torch.einsum("nc,nc->c", gy, xhat), gy.sum(0)
        gx = gy.mul_(gamma).sub_(level).sub_(xhat.mul_(along)).mul_(rstd)
        return dict(gx=gx, dgamma=dgamma, dbeta=dbeta)
    if kind == "checkpoint":
        return _exact_checkpoint(s["x"].to(f64))
    if kind == "weight_ckpt":
        h = _exact_values(s).mul_(s["gamma"].to(f64)).add_(s["beta"].to(f64))
        gz = s["gz"].to(f64)
        return torch.stack([torch.einsum("nd,nf->df", h[r], gz[r]) for r in s["rows"]])
    W = s["W"].to(f64)
    if kind == "typed_forward":
        z = torch.empty(case["n"], case["d_out"], dtype=f64, device=W.device)
        for t, r in enumerate(s["rows"]):
            z[r] = torch.einsum("nd,df->nf", s["h"][r].to(f64), W[t])
        return z
    if kind == "typed_backward":
        dh = torch.empty(case["n"], case["d_in"], dtype=f64, device=W.device)
        dW = torch.empty(W.shape, dtype=f64, device=W.device)
        for t, r in enumerate(s["rows"]):
            gz = s["gz"][r].to(f64)
            dh[r] = torch.einsum("nf,df->nd", gz, W[t])
            dW[t] = torch.einsum("nd,nf->df", s["h"][r].to(f64), gz)
        return dict(dh=dh, dW=dW)
    raise ValueError(kind)
