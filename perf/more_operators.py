"""Operators around the residual stream of a language model and its sampling, for k worker replicas, as cases that can be
timed and compared.

Four kinds of case, each over the workers in one call:
  embed    rows of a table [k][vocab][n] for tokens, times a scale; what = "lookup", or "grad": the gradient of the table, fp32,
           every row of it, from that of the rows.  table: its type; blank: share of tokens that are padding (-1)
  norm     root-mean-square norm of h = residual + dropout(x), [k][rows][n].  what = "forward": h, the norm, 1/rms;
           "serve": the norm in 8 bits (e4m3, a power-of-two scale per block of 128) and the product with weights kept so;
           "train": the same with the transposed form too, and the product that gives the weights' gradient;
           "grad": backward pass with the gradient that arrives through the residual stream, and the sum for the weight.
           p: dropped share (0: no dropout); pad: columns by which a row of the buffers is longer than n
  dropout  residual + dropout(x), or its backward pass (residual = False)
  adjust   logits [k][rows][vocab] with penalties for tokens of the request so far (history of up to `length` tokens, prompt and
           answer), a bias for each token (bias = True) and a grammar's mask, a bit a token (mask = True)

The mask of a dropout is a function of seed, worker, step, row and column alone.  dtype is the type of activations or logits.
"""
from __future__ import annotations

import math
import random

import torch

own = False                    # True: run() makes the framework's calls; False: the plain form

DEVICE = "cuda:0"
EPS = 1e-6                     # of the norm's mean square
SCALE = 64.0                   # of the embedding
F32, BF16 = torch.float32, torch.bfloat16
GAMMA = 0x9E3779B97F4A7C15     # SplitMix64
MUL1, MUL2 = 0xBF58476D1CE4E5B9, 0x94D049BB133111EB
ALL64 = (1 << 64) - 1


# ---- cases -----------------------------------------------------------------------------------------------------------

def _case(name, kind, k, dtype, **more):
    c = {"name": name} if name else {}
    c.update(kind=kind, k=k, dtype=dtype)
    c.update(more)
    return c


def _norm(name, what, k, dtype, rows, n, n_out=0, p=0.0, pad=0):
    return _case(name, "norm", k, dtype, what=what, rows=rows, n=n, n_out=n_out, p=p, pad=pad)


def listed():
    return [
        # the next token of a served model: one row of the table, nothing but latency
        _case("embed_token", "embed", 1, "bf16", what="lookup", table="bf16", rows=1, vocab=32000, n=4096, blank=0.0),
        # a training batch of 8 workers whose parameters are fp32
        _case("embed_batch", "embed", 8, "bf16", what="lookup", table="f32", rows=1024, vocab=32000, n=4096, blank=0.0),
        # a small table's gradient in fp32, padded answers, no size a multiple of anything
        _case("embed_grad_ragged", "embed", 3, "f32", what="grad", table="f32", rows=333, vocab=5003, n=1001, blank=0.2),
        # the gradient of four workers' whole tables: common tokens come hundreds of times, most rows are zeros
        _case("embed_grad_wide", "embed", 4, "bf16", what="grad", table="f32", rows=4096, vocab=32000, n=4096, blank=0.0),
        # one token through a norm and the layer behind it, whose weights are in 8 bits
        _norm("norm_serve", "serve", 1, "bf16", 1, 4096, n_out=4096),
        # the widest configuration's minibatches, 16 workers of 512 rows: bound by memory
        _norm("norm_forward", "forward", 16, "bf16", 512, 4096),
        # a training step's norm with dropout in front and a narrow projection behind it, both in 8 bits
        _norm("norm_train", "train", 8, "bf16", 1024, 4096, n_out=256, p=0.1),
        # backward pass in fp32 with dropout and an odd width inside wider buffers
        _norm("norm_grad_ragged", "grad", 3, "f32", 2731, 5003, p=0.1, pad=13),
        # a small model's hidden layer in fp32, odd rows
        _case("dropout_small", "dropout", 4, "f32", rows=37, n=513, p=0.5, residual=False, pad=1),
        # a training batch's residual stream
        _case("dropout_wide", "dropout", 8, "bf16", rows=4096, n=4096, p=0.1, residual=True, pad=0),
        # four requests in the middle of their answers
        _case("adjust_few", "adjust", 1, "bf16", rows=4, vocab=32000, length=300, bias=False, mask=False, pad=0),
        # a rollout of 512 requests over a large vocabulary, all features on
        _case("adjust_rollout", "adjust", 8, "bf16", rows=64, vocab=131072, length=2048, bias=True, mask=True, pad=0),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "norm", "norm", "dropout", "adjust"])
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 3, 16])
    if kind == "embed":
        k, n = _spread(rng, 1, 8), _spread(rng, 8, 8192)
        vocab = _spread(rng, 16, max(16, min(131072, (1 << 29) // (k * n))))
        rows = _spread(rng, 1, max(1, min(16384, (1 << 26) // (k * n))))
        return _case("", kind, k, dtype, what=rng.choice(["lookup", "grad", "grad"]), table=rng.choice(["f32", "bf16"]), rows=rows,
                     vocab=vocab, n=n, blank=rng.choice([0.0, 0.0, 0.3]))
    if kind == "norm":
        what = rng.choice(["forward", "serve", "train", "grad"])
        dtype = "bf16" if what in ("serve", "train") else dtype        # (8 bits behind fp32 would save nobody anything)
        k, n = _spread(rng, 1, 16), _spread(rng, 16, 16384)
        rows = _spread(rng, 1, max(1, min(8192, (1 << 25) // (k * n))))
        n_out = _spread(rng, 16, max(16, min(512, (1 << 33) // (k * rows * n)))) if what in ("serve", "train") else 0
        return _norm("", what, k, dtype, rows, n, n_out=n_out, p=0.0 if what == "serve" else rng.choice([0.0, 0.1, 0.3]), pad=pad)
    if kind == "dropout":
        k, n = _spread(rng, 1, 16), _spread(rng, 3, 16384)
        rows = _spread(rng, 1, max(1, min(16384, (1 << 26) // (k * n))))
        return _case("", kind, k, dtype, rows=rows, n=n, p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.5, pad=pad)
    k, vocab = _spread(rng, 1, 8), _spread(rng, 33, 131072)
    rows = _spread(rng, 1, max(1, min(256, (1 << 26) // (k * vocab))))
    return _case("", kind, k, dtype, rows=rows, vocab=vocab, length=_spread(rng, 1, 8192), bias=rng.random() < 0.5, mask=rng.random() < 0.5,
                 pad=pad)


def _expected_distinct(rows, vocab):
    """Of the tokens that _tokens draws, how many different ones there are on average."""
    v = torch.arange(1, vocab + 1, dtype=torch.float64)
    share = torch.log1p(1.0 / v) / math.log(vocab + 1)
    return float((1.0 - (1.0 - share) ** rows).sum())


def _eight_bytes(rows, n):
    return rows * ((n + 127) // 128 * 128 + (n + 127) // 128)


def work(case):
    k, rows, e = case["k"], case["rows"], 2 if case["dtype"] == "bf16" else 4
    m = k * rows
    if case["kind"] == "embed":
        n, vocab = case["n"], case["vocab"]
        used = int(rows * (1.0 - case["blank"]))
        if case["what"] == "lookup":
            distinct = _expected_distinct(used, vocab)
            return {"bytes": int(k * distinct * n * (2 if case["table"] == "bf16" else 4) + m * n * e + 4 * m), "flops": m * n}
        return {"bytes": k * used * n * e + 4 * m + 4 * k * vocab * n, "flops": 2 * m * n}
    if case["kind"] == "norm":
        n, o, cells = case["n"], case["n_out"], m * case["n"]
        if case["what"] == "forward":
            return {"bytes": 4 * e * cells + 4 * m + 4 * k * n, "flops": 6 * cells}
        if case["what"] == "serve":
            return {"bytes": 3 * e * cells + k * _eight_bytes(o, n) + e * m * o + 4 * k * n, "flops": 6 * cells + 2 * cells * o}
        if case["what"] == "train":
            return {"bytes": 3 * e * cells + 4 * m + 4 * k * n + k * (_eight_bytes(o, n) + _eight_bytes(o, rows)) + e * m * o + e * k * o * n,
                    "flops": 8 * cells + 4 * cells * o}
        return {"bytes": (4 + (case["p"] > 0)) * e * cells + 4 * m + 8 * k * n, "flops": 10 * cells}
    if case["kind"] == "dropout":
        cells = m * case["n"]
        return {"bytes": (3 if case["residual"] else 2) * e * cells, "flops": 3 * cells}
    cells = m * case["vocab"]
    return {"bytes": 2 * e * cells + 4 * m * (case["length"] + 5) + (4 * case["vocab"] if case["bias"] else 0) + (cells // 8 if case["mask"] else 0),
            "flops": 3 * cells}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _type(name):
    return BF16 if name == "bf16" else F32


def _padded(shape, pad, dtype, g, scale=1.0, shift=0.0):
    """Normal numbers in a [..., n] view of rows that are `pad` longer."""
    full = torch.randn(*shape[:-1], shape[-1] + pad, generator=g, device=DEVICE, dtype=dtype)
    if scale != 1.0 or shift != 0.0:
        full.mul_(scale).add_(shift)
    return full[..., : shape[-1]]


def _tokens(shape, vocab, g):
    """Tokens as they come in text, low ones more often: uniform in the logarithm."""
    u = torch.rand(*shape, generator=g, device=DEVICE, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp_(0, vocab - 1).to(torch.int32)


def _inputs(case, seed):
    """What the seed alone decides."""
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    k, rows, dt = case["k"], case["rows"], _type(case["dtype"])
    s = dict(case)
    s["seed"], s["step"] = seed * 2654435761 % (1 << 63), seed % 1000          # of the dropout
    if case["kind"] == "embed":
        vocab, n = case["vocab"], case["n"]
        s["token"] = _tokens((k, rows), vocab, g)
        if case["blank"]:                                                       # the ends of short answers
            s["token"][:, rows - int(rows * case["blank"]):] = -1
        if case["what"] == "lookup":
            s["weight"] = torch.randn(k, vocab, n, generator=g, device=DEVICE, dtype=_type(case["table"])).mul_(0.02)
        else:
            s["dy"] = torch.randn(k, rows, n, generator=g, device=DEVICE, dtype=dt).mul_(1e-3)
    elif case["kind"] == "norm":
        n, o = case["n"], case["n_out"]
        shape = (k, rows, n)
        s["gamma"] = torch.randn(k, n, generator=g, device=DEVICE).mul_(0.2).add_(1.0)
        if case["what"] == "grad":
            s["h"] = _padded(shape, case["pad"], dt, g, 2.0)
            s["dy"] = _padded(shape, case["pad"], dt, g, 0.01)
            s["dh"] = _padded(shape, case["pad"], dt, g, 0.01)
            s["rstd"] = (s["h"].float().square().mean(-1) + EPS).rsqrt()
        else:
            s["x"] = _padded(shape, case["pad"], dt, g)
            s["residual"] = _padded(shape, case["pad"], dt, g, 2.0)
            if o:
                s["w"] = torch.randn(k, o, n, generator=g, device=DEVICE).div_(math.sqrt(n)).to(dt)
            if case["what"] == "train":
                s["dz"] = torch.randn(k, rows, o, generator=g, device=DEVICE, dtype=dt).mul_(1e-3)
    elif case["kind"] == "dropout":
        s["x"] = _padded((k, rows, case["n"]), case["pad"], dt, g)
        s["stream"] = _padded((k, rows, case["n"]), case["pad"], dt, g, 2.0) if case["residual"] else None
    else:
        vocab, length = case["vocab"], case["length"]

        def uniform(lo, hi):
            return torch.rand(k, rows, generator=g, device=DEVICE).mul_(hi - lo).add_(lo)
        s["logits"] = _padded((k, rows, vocab), case["pad"], dt, g, 3.0)
        s["history"] = _tokens((k, rows, length), vocab, g)
        s["filled"] = uniform(0, length + 1).to(torch.int32).clamp_(0, length)  # tokens so far
        s["answer"] = (s["filled"] * uniform(0, 1)).to(torch.int32)             # where the prompt ends
        s["repetition"], s["presence"], s["frequency"] = uniform(1.0, 1.3), uniform(0.0, 1.0), uniform(0.0, 0.5)
        s["bias"] = torch.randn(vocab, generator=g, device=DEVICE).expand(k, rows, vocab) if case["bias"] else None
        s["mask"] = None
        if case["mask"]:                                                        # free text, a few words, and everything in between
            words = (vocab + 31) // 32
            bits = torch.randint(-(1 << 31), 1 << 31, (2, k, rows, words), generator=g, device=DEVICE).to(torch.int32)
            kind = torch.randint(0, 3, (k, rows, 1), generator=g, device=DEVICE)
            s["mask"] = torch.where(kind == 0, -1, torch.where(kind == 1, bits[0], bits[0] & bits[1] & (bits[0] << 7) & (bits[1] >> 5)))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if "w" in s:                                   # weights, and what the layer behind sends back, are in 8 bits already
        if own:
            from paper_2409_09242_amd import operators as OPS
            s["w"] = OPS.fp8_quantize(s["w"], square=True)
            if "dz" in s:
                s["dz"] = OPS.fp8_quantize(s["dz"], transposed=True)[1]
        else:
            s["w"] = _fp8_values(s["w"], square=True)
            if "dz" in s:
                s["dz"] = _fp8_values(s["dz"].transpose(1, 2))
    return s


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2409_09242_amd import operators as OPS
    if s["kind"] == "embed":
        if s["what"] == "lookup":
            return {"y": OPS.embedding(s["token"], s["weight"], SCALE, dtype=_type(s["dtype"]))}
        return {"grad": OPS.embedding_grad(s["dy"], s["token"], s["vocab"], SCALE)}
    if s["kind"] == "norm":
        drop = {"p": s["p"], "seed": s["seed"], "step": s["step"]}
        if s["what"] == "grad":
            dh, dx, dgamma = OPS.rms_norm_grad(s["dy"], s["h"], s["gamma"], s["rstd"], dh=s["dh"], **drop)
            return {"dh": dh, "dx": dx, "dgamma": dgamma}
        if s["what"] == "forward":
            y, h, rstd = OPS.rms_norm(s["x"], s["gamma"], EPS, residual=s["residual"], **drop)
            return {"y": y, "h": h, "rstd": rstd}
        dt = s["x"].dtype
        if s["what"] == "serve":
            y, h, _ = OPS.rms_norm_fp8(s["x"], s["gamma"], EPS, residual=s["residual"], stats=False)
            return {"h": h, "z": OPS.fp8_matmul(y, s["w"], dtype=dt)}
        (y, yt), h, rstd = OPS.rms_norm_fp8(s["x"], s["gamma"], EPS, residual=s["residual"], transposed=True, **drop)
        return {"h": h, "rstd": rstd, "z": OPS.fp8_matmul(y, s["w"], dtype=dt), "dw": OPS.fp8_matmul(s["dz"], yt, dtype=dt)}
    if s["kind"] == "dropout":
        return {"y": OPS.dropout(s["x"], s["p"], s["seed"], s["step"], residual=s["stream"])}
    return {"z": OPS.adjust_logits(s["logits"], s["history"], s["filled"], s["answer"], s["repetition"], s["presence"], s["frequency"],
                                   s["bias"], s["mask"])}


def _signed(v):
    """A 64-bit pattern as torch holds it."""
    v &= ALL64
    return v - (1 << 64) if v >> 63 else v


def _mixed(x):
    """SplitMix64's output function of a Python number."""
    x &= ALL64
    x = (x ^ (x >> 30)) * MUL1 & ALL64
    x = (x ^ (x >> 27)) * MUL2 & ALL64
    return x ^ (x >> 31)


def _shifted(x, by):
    """A logical shift to the right of a tensor of 64-bit patterns."""
    return (x >> by) & ((1 << (64 - by)) - 1)


def _kept(s, k, rows, n):
    """(what survives the dropout, the factor of it): four neighbours of a row share a number, 16 bits each."""
    groups = (n + 3) // 4
    x = torch.arange(1, rows * groups + 1, device=DEVICE) * _signed(GAMMA)
    keys = [_mixed(_mixed(s["seed"] + GAMMA * (w + 1)) + GAMMA * (s["step"] + 1)) for w in range(k)]
    x = x[None] + torch.tensor([_signed(v) for v in keys], device=DEVICE)[:, None]
    x = (x ^ _shifted(x, 30)) * _signed(MUL1)
    x = (x ^ _shifted(x, 27)) * _signed(MUL2)
    x = x ^ _shifted(x, 31)
    bits = torch.stack([(x >> (16 * q)) & 0xFFFF for q in range(4)], -1)
    limit = round((1.0 - s["p"]) * 65536)
    return (bits < limit).view(k, rows, 4 * groups)[..., :n], 65536.0 / limit


def _fp8_values(x, square=False):
    """The numbers that x stands for in e4m3 with a power-of-two scale per block of 128 of the last axis (per square of
    128 x 128 of the last two): the least power that brings the block's largest magnitude to at most 448, and ties to even."""
    k, r, c = x.shape
    high = 128 if square else 1
    rp, cp = -(-r // high) * high, -(-c // 128) * 128
    v = torch.zeros(k, rp, cp, device=x.device, dtype=torch.float64 if x.dtype == torch.float64 else F32)
    v[:, :r, :c] = x
    v = v.view(k, rp // high, high, cp // 128, 128)
    part, power = torch.frexp(v.abs().amax((2, 4), keepdim=True))      # part in [0.5, 1); 448 = 0.875 2^9
    power = torch.where(part > 0, power - 9 + (part > 0.875), 0).clamp(min=-126)
    up, down = (((127 + sign * power).to(torch.int32) << 23).view(F32) for sign in (1, -1))
    v = v * down
    if v.dtype == torch.float64:                   # to fp32 towards zero with the last bit set where something is lost: no tie arises
        near = v.float()
        bits = near.view(torch.int32) - (near.double().abs() > v.abs()).int()
        v = torch.where(near.double() == v, bits, bits | 1).view(F32)
    v = v.to(torch.float8_e4m3fn).float() * up
    return v.reshape(k, rp, cp)[:, :r, :c].contiguous()


def _times_transposed(a, b):
    return torch.matmul(a, b.transpose(1, 2).contiguous())


def _run_plain(s):
    dt = _type(s["dtype"])
    k, rows = s["k"], s["rows"]
    if s["kind"] == "embed":
        token = s["token"].long()
        if s["what"] == "lookup":
            flat = (token.clamp(min=0) + torch.arange(k, device=DEVICE)[:, None] * s["vocab"]).view(-1)
            y = s["weight"].view(k * s["vocab"], s["n"])[flat].view(k, rows, s["n"]).float() * SCALE
            return {"y": (y * (token >= 0)[..., None]).to(dt)}
        grad = torch.zeros(k * (s["vocab"] + 1), s["n"], device=DEVICE)         # a row more for what is no token
        flat = (torch.where(token < 0, s["vocab"], token) + torch.arange(k, device=DEVICE)[:, None] * (s["vocab"] + 1)).view(-1)
        grad.index_add_(0, flat, s["dy"].view(k * rows, s["n"]).float() * SCALE)
        return {"grad": grad.view(k, s["vocab"] + 1, s["n"])[:, :-1]}
    if s["kind"] == "norm":
        return _plain_norm(s, dt)
    if s["kind"] == "dropout":
        keep, factor = _kept(s, k, rows, s["n"])
        y = torch.where(keep, s["x"].float() * factor, 0.0)
        return {"y": (y + s["stream"].float() if s["residual"] else y).to(dt)}
    z, vocab = s["logits"].float(), s["vocab"]
    place = torch.arange(s["length"], device=DEVICE)
    used = place < s["filled"][..., None]
    answered = used & (place >= s["answer"][..., None])
    token = s["history"].long()
    seen = torch.zeros(k, rows, vocab, device=DEVICE).scatter_add_(2, token, used.float()) > 0
    count = torch.zeros(k, rows, vocab, device=DEVICE).scatter_add_(2, token, answered.float())
    r = s["repetition"][..., None]
    z = torch.where(seen, torch.where(z > 0, z / r, z * r), z)
    z = z - (s["frequency"][..., None] * count + s["presence"][..., None] * (count > 0))
    if s["bias"] is not None:
        z = z + s["bias"]
    if s["mask"] is not None:
        bits = (s["mask"][..., None] >> torch.arange(32, device=DEVICE, dtype=torch.int32)) & 1
        z = torch.where(bits.view(k, rows, -1)[..., :vocab] > 0, z, -math.inf)
    return {"z": z.to(dt)}


def _plain_norm(s, dt):
    k, rows, n = s["k"], s["rows"], s["n"]
    gamma = s["gamma"][:, None, :]
    keep, factor = _kept(s, k, rows, n) if s["p"] else (None, 1.0)
    if s["what"] == "grad":
        rstd = s["rstd"][..., None]
        hat, dy = s["h"].float() * rstd, s["dy"].float()
        a = dy * gamma
        dh = rstd * (a - hat * (a * hat).mean(-1, keepdim=True)) + s["dh"].float()
        dx = torch.where(keep, dh * factor, 0.0) if s["p"] else dh
        return {"dh": dh.to(dt), "dx": dx.to(dt), "dgamma": (dy * hat).sum(1)}
    x = s["x"].float()
    if s["p"]:
        x = torch.where(keep, x * factor, 0.0)
    h = (x + s["residual"].float()).to(dt)         # the norm is that of h as it is handed on
    v = h.float() if s["what"] == "forward" else h.double()            # (64 bits in front of e4m3: values next to a border)
    rstd = (v.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y = v * rstd * gamma
    if s["what"] == "forward":
        return {"y": y.to(dt), "h": h, "rstd": rstd[..., 0]}
    rstd = rstd.float()
    z = _times_transposed(_fp8_values(y), s["w"]).to(dt)
    if s["what"] == "serve":
        return {"h": h, "z": z}
    return {"h": h, "rstd": rstd[..., 0], "z": z, "dw": _times_transposed(s["dz"], _fp8_values(y.transpose(1, 2))).to(dt)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact(case, seed):
    definition = {"embed": _exact_embed, "norm": _exact_norm, "dropout": _exact_dropout, "adjust": _exact_adjust}[case["kind"]]
    return definition(case, _inputs(case, seed))


def _exact_embed(case, s):
    out = []
    for w in range(case["k"]):
        token = s["token"][w].long()
        there = torch.nonzero(token >= 0)[:, 0]
        if case["what"] == "lookup":
            y = torch.zeros(case["rows"], case["n"], dtype=torch.float64, device=DEVICE)
            y[there] = s["weight"][w].index_select(0, token[there]).double() * SCALE
        else:
            y = torch.zeros(case["vocab"], case["n"], dtype=torch.float64, device=DEVICE)
            y.index_put_((token[there],), s["dy"][w][there].double() * SCALE, accumulate=True)
        out.append(y)
    return {"y" if case["what"] == "lookup" else "grad": torch.stack(out)}


def _rotated_product(x, factor):
    """x times factor in 64 bits from 32-bit halves, all in int64 without a carry lost."""
    lo, hi = x & 0xFFFFFFFF, (x >> 32) & 0xFFFFFFFF
    f_lo, f_hi = factor & 0xFFFFFFFF, factor >> 32
    low = (lo & 0xFFFF) * f_lo + ((((lo >> 16) * f_lo) & 0xFFFFFFFFFFFF) << 16)
    return low + ((lo * f_hi + hi * f_lo) << 32)


def _exact_factor(case, s, w):
    """What the dropout multiplies every element of worker w by."""
    rows, n, p = case["rows"], case["n"], case["p"]
    state = s["seed"]
    for index in (w, s["step"]):                   # the key is the index-th number of a stream, twice
        state = (state + GAMMA * (index + 1)) % (1 << 64)
        for by, f in ((30, MUL1), (27, MUL2), (31, 1)):
            state = ((state ^ (state >> by)) * f) % (1 << 64)
    column = torch.arange(n, device=DEVICE)
    groups = (n + 3) // 4
    parts = []
    for r0 in range(0, rows, 1024):
        row = torch.arange(r0, min(rows, r0 + 1024), device=DEVICE)
        number = row[:, None] * groups + torch.arange(groups, device=DEVICE)[None, :] + 1
        v = _rotated_product(number, GAMMA) + (state - (1 << 64) if state >= 1 << 63 else state)
        for by, f in ((30, MUL1), (27, MUL2), (31, 1)):
            v = v ^ torch.bitwise_and(torch.bitwise_right_shift(v, by), 2 ** (64 - by) - 1)
            v = v if f == 1 else _rotated_product(v, f)
        sixteen = torch.bitwise_right_shift(v[:, column // 4], 16 * (column % 4)) % 65536
        parts.append(sixteen)
    limit = math.floor((1.0 - p) * 65536 + 0.5)
    return (torch.cat(parts) < limit).double() * (65536.0 / limit)


def _exact_e4m3(x, square=False):
    """The definition of _fp8_values by comparisons and by rounding to multiples of the last place."""
    x = x.double()
    k, r, c = x.shape
    high = 128 if square else 1
    full = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % high))
    tiles = full.reshape(k, full.shape[1] // high, high, full.shape[2] // 128, 128)
    top = tiles.abs().amax(4, keepdim=True).amax(2, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 448.0) / 448.0))
    e = torch.where(top > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where(top <= 448.0 * torch.exp2(e - 1), e - 1, e)
    unit = torch.exp2(torch.where(top > 0, e, 0.0).clamp(min=-126))
    v = tiles / unit
    place = torch.exp2(torch.clamp(torch.frexp(v.abs())[1] - 1, min=-6).double() - 3)          # three bits behind the leading one
    return (torch.round(v / place) * place * unit).reshape(full.shape)[:, :r, :c]


def _exact_norm(case, s):
    parts = [_exact_norm_worker(case, s, w) for w in range(case["k"])]
    return {name: torch.stack([p[name] for p in parts]) for name in parts[0]}


def _exact_norm_worker(case, s, w):
    n, dt = case["n"], _type(case["dtype"])
    gamma = s["gamma"][w].double()
    factor = _exact_factor(case, s, w) if case["p"] else torch.ones((), dtype=torch.float64, device=DEVICE)
    if case["what"] == "grad":
        r = s["rstd"][w].double().unsqueeze(1)
        hat, dy = s["h"][w].double() * r, s["dy"][w].double()
        along = (dy * gamma * hat).sum(1, keepdim=True) / n
        dh = (dy * gamma - along * hat) * r + s["dh"][w].double()
        return {"dh": dh, "dx": dh * factor, "dgamma": torch.einsum("rj,rj->j", dy, hat)}
    h = (s["residual"][w].double() + factor * s["x"][w].double()).to(dt)
    r = 1.0 / torch.sqrt((h.double() ** 2).sum(1) / n + EPS)
    y = gamma * (h.double() * r.unsqueeze(1))
    if case["what"] == "forward":
        return {"y": y, "h": h.double(), "rstd": r}
    z = _exact_e4m3(y[None])[0] @ _exact_e4m3(s["w"][w][None], square=True)[0].T.contiguous()
    if case["what"] == "serve":
        return {"h": h.double(), "z": z}
    dw = _exact_e4m3(s["dz"][w].T[None])[0] @ _exact_e4m3(y.T[None])[0].T.contiguous()
    return {"h": h.double(), "rstd": r, "z": z, "dw": dw}


def _exact_dropout(case, s):
    out = []
    for w in range(case["k"]):
        y = s["x"][w].double() * _exact_factor(case, s, w)
        out.append(y + s["stream"][w].double() if case["residual"] else y)
    return {"y": torch.stack(out)}


def _exact_adjust(case, s):
    k, rows, vocab = case["k"], case["rows"], case["vocab"]
    out = torch.empty(k, rows, vocab, dtype=torch.float64, device=DEVICE)
    filled, answer = s["filled"].tolist(), s["answer"].tolist()
    for w in range(k):
        for r in range(rows):
            z = s["logits"][w, r].double()
            said = s["history"][w, r, : filled[w][r]].long()
            rep, pre, freq = (float(s[name][w, r]) for name in ("repetition", "presence", "frequency"))
            old = torch.unique(said)
            z[old] = torch.where(z[old] > 0, z[old] / rep, z[old] * rep)
            new, times = torch.unique(said[answer[w][r]:], return_counts=True)
            z[new] -= pre + freq * times.double()
            if case["bias"]:
                z = z + s["bias"][w, r].double()
            if case["mask"]:
                j = torch.arange(vocab, device=DEVICE)
                word = s["mask"][w, r].long()[j // 32] & 0xFFFFFFFF
                z[(word >> (j % 32)) % 2 == 0] = -math.inf
            out[w, r] = z
    return {"z": out}
