"""The language-model operators of this library, as cases that can be timed and compared.

Three operators, which one training step of a recurrent language model runs together and whose
gradients the compression step then takes: the gated linear recurrence (forward, forward and
backward, and its single-token form), dropout whose mask is drawn again from a counter instead of
being stored (with the residual sum), and softmax cross-entropy over a vocabulary with its gradient.
Where ``own`` is false they are computed in elementary torch operations.

Sizes are those of this repository's language-model-sized workload (22,000 embedding rows of 1,500
columns), generic ones, and odd ones in between.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
IGNORE = -100
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
MASK64 = (1 << 64) - 1


def listed():
    def rec(name, mode, B, T, C, dtype, **more):
        return dict(name=name, op="recurrence", mode=mode, B=B, T=T, C=C, dtype=dtype,
                    **{**dict(gate=True, h0=True, ragged=False, packed=False), **more})

    def drop(name, mode, rows, cols, dtype, p, residual):
        return dict(name=name, op="dropout", mode=mode, rows=rows, cols=cols, dtype=dtype, p=p, residual=residual)

    def xent(name, mode, N, V, dtype, **more):
        return dict(name=name, op="xent", mode=mode, N=N, V=V, dtype=dtype, **{**dict(padded=False, ignored=0.05), **more})

    return [
        # serving: one token of one sequence; launch and latency decide
        rec("recurrence-token", "forward", 1, 1, 1_500, "f32"),
        # serving: one token of each of many sequences
        rec("recurrence-tokens", "forward", 256, 1, 1_500, "bf16", packed=True),
        # reading a few prompts of unlike lengths, one of them empty, before the first token
        rec("recurrence-prompts", "forward", 5, 1_037, 1_500, "f16", ragged=True, packed=True),
        # an ordinary training step of one worker
        rec("recurrence-train", "train", 32, 512, 1_500, "bf16", ragged=True, packed=True, h0=False),
        # one long document: few channels, all parallelism along time
        rec("recurrence-long", "train", 1, 65_536, 1_024, "bf16", packed=True),
        # the largest: a large batch of long sequences
        rec("recurrence-large", "train", 16, 4_096, 2_048, "bf16", packed=True, h0=False),
        # a small batch's activations in full precision
        drop("dropout-small", "forward", 20 * 35, 1_500, "f32", 0.5, False),
        # an ordinary training step of one worker: the residual branch, forward and backward
        drop("dropout-train", "train", 32 * 512, 1_500, "bf16", 0.1, True),
        # the largest
        drop("dropout-large", "train", 65_536, 2_048, "bf16", 0.2, True),
        # evaluation of a few tokens: the loss alone
        xent("xent-eval", "forward", 35, 22_000, "f32", ignored=0.0),
        # an ordinary training step: the loss and the logits' gradient
        xent("xent-train", "train", 4_096, 22_000, "bf16"),
        # the largest: an odd number of rows of an odd, large vocabulary
        xent("xent-large", "train", 8_191, 131_071, "bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def other(n, step):  # 3,072 is no size of this library's workloads: the next smaller one
        return n - step if n == 3_072 else n

    def size(lo, hi, step):  # odd sizes, multiples of a power of two and of 100
        n = log(lo, hi)
        step = rng.choice([1, 1, step, step, 100 if n >= 100 else 1])
        return other(max(step, n - n % step), step)

    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    op = rng.choice(["recurrence", "recurrence", "dropout", "xent"])
    if op == "recurrence":
        kind = rng.choice(["tokens", "prompts", "train", "train"])
        C = size(64, 4_096, 64)
        most = (1 << 26) // (2 if dtype == "f32" else 1)
        if kind == "tokens":
            T, B = 1, log(1, 1_024)
        else:
            T = size(2, 65_536 if kind == "train" else 16_384, 16)
            B = log(1, max(1, min(64, most // (T * C))))
        while B * T * C > most:
            T = T // 2 + 1
        return dict(op=op, mode="train" if kind == "train" else "forward", B=other(B, 1), T=other(T, 1), C=C, dtype=dtype,
                    gate=rng.random() < 0.8, h0=rng.random() < 0.5, ragged=T > 1 and rng.random() < 0.4,
                    packed=rng.random() < 0.6)
    if op == "dropout":
        cols = size(64, 8_192, 64)
        most = (1 << 27) // (2 if dtype == "f32" else 1)
        rows = log(1, min(65_536, most // cols))
        return dict(op=op, mode=rng.choice(["forward", "train"]), rows=other(rows, 1), cols=cols, dtype=dtype,
                    p=rng.choice([0.1, 0.2, 0.5, 0.65]), residual=rng.random() < 0.5)
    V = size(256, 200_000, 64)
    most = (1 << 29) // (2 if dtype == "f32" else 1)
    return dict(op=op, mode=rng.choice(["forward", "train", "train"]), N=other(log(1, min(16_384, most // V)), 1), V=V,
                dtype=dtype, padded=rng.random() < 0.3, ignored=rng.choice([0.0, 0.05, 0.3]))


def _lengths(case):
    """Tokens of each sequence: all of T, or for a ragged batch between half of T and T and, from three
    sequences on, none at all in one of them."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    n = [max(1, T - int(T * 0.5 * ((b * 0.6180339887) % 1.0))) for b in range(B)]
    if B >= 3:
        n[B // 2] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1_000_003 + 29)
    dt = DTYPES[case["dtype"]]

    def randn(*shape, scale=1.0, shift=0.0):
        return torch.randn(shape, generator=gen, device=DEV).mul_(scale).add_(shift).to(dt)

    s = dict(case)
    if case["op"] == "recurrence":
        B, T, C = case["B"], case["T"], case["C"]
        n = 3 if case["gate"] else 2
        if case["packed"]:  # slices of one projection of the layer's input
            proj = torch.empty((B, T, n * C), dtype=dt, device=DEV)
            parts = [proj[:, :, j * C:(j + 1) * C] for j in range(n)]
        else:
            parts = [torch.empty((B, T, C), dtype=dt, device=DEV) for _ in range(n)]
        parts[0].copy_(randn(B, T, C))
        parts[1].copy_(randn(B, T, C, scale=1.5, shift=2.0))  # forget gates remember: biased upwards
        if case["gate"]:
            parts[2].copy_(randn(B, T, C))
        s["x"], s["f"], s["o"] = parts[0], parts[1], parts[2] if case["gate"] else None
        s["h0"] = torch.randn((B, C), generator=gen, device=DEV) if case["h0"] else None
        order = torch.randperm(B, generator=gen, device=DEV)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)[order].contiguous() \
            if case["ragged"] else None
        if case["mode"] == "train":
            s["gy"] = randn(B, T, C, scale=0.02)
            s["gh"] = torch.randn((B, C), generator=gen, device=DEV).mul_(0.02) if case["h0"] else None
    elif case["op"] == "dropout":
        rows, cols = case["rows"], case["cols"]
        s["x"] = randn(rows, cols)
        s["r"] = randn(rows, cols) if case["residual"] else None
        s["seed"], s["site"] = int(seed) * 7_919 + 3, 5  # the program's seed, and which dropout of it this is
        s["step"] = torch.tensor([int(seed) % 1_000 + 1], dtype=torch.int64, device=DEV)
        if case["mode"] == "train":
            s["gy"] = randn(rows, cols, scale=0.02)
    else:
        N, V = case["N"], case["V"]
        z = torch.empty((N, -(-V // 64) * 64 if case["padded"] else V), dtype=dt, device=DEV)
        for at in range(0, N, 1_024):
            z[at:at + 1_024] = randn(min(1_024, N - at), z.shape[1], scale=3.0)
        z = z[:, :V]
        # frequent words first, their logits raised as a trained model has them
        t = (torch.rand(N, generator=gen, device=DEV).pow(3) * V).long().clamp_(max=V - 1)
        z[torch.arange(N, device=DEV), t] += 6.0
        t[torch.rand(N, generator=gen, device=DEV) < case["ignored"]] = IGNORE
        s["logits"], s["targets"] = z, t
    return s


def run(s):
    if own:
        return _call(s)
    return {"recurrence": _plain_recurrence, "dropout": _plain_dropout, "xent": _plain_xent}[s["op"]](s)


# ---- the framework's operators


def _call(s):
    from paper_2108_06004_amd import lm

    if s["op"] == "recurrence":
        train = s["mode"] == "train"
        y, h, saved = lm.recurrence_forward(s["x"], s["f"], s["o"], h0=s["h0"], lengths=s["lengths"], save=train)
        if not train:
            return {"y": y, "h": h}
        dx, df, do, dh0 = lm.recurrence_backward(s["gy"], s["x"], s["f"], s["o"], saved, lengths=s["lengths"],
                                                 gh=s["gh"])
        return {"y": y, "h": h, "dx": dx, "df": df, "do": do, "dh0": dh0}
    if s["op"] == "dropout":
        y = lm.dropout_forward(s["x"], s["p"], s["seed"], site=s["site"], step=s["step"], residual=s["r"])
        if s["mode"] == "forward":
            return {"y": y}
        return {"y": y, "dx": lm.dropout_backward(s["gy"], s["p"], s["seed"], site=s["site"], step=s["step"])}
    mean, rows, grad = lm.cross_entropy_forward(s["logits"], s["targets"], ignore_index=IGNORE,
                                                grad=s["mode"] == "train")
    return {"mean": mean, "rows": rows, "grad": grad}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, h before the first step zero, by doubling."""
    T, n = a.shape[1], 1
    while n < T:
        b = torch.cat([b[:, :n], b[:, n:] + a[:, n:] * b[:, :-n]], 1)
        a = torch.cat([a[:, :n], a[:, n:] * a[:, :-n]], 1)
        n *= 2
    return b


def _plain_recurrence(s):
    x, dt = s["x"].float(), s["x"].dtype
    B, T, C = x.shape
    a, rest = torch.sigmoid(s["f"].float()), torch.sigmoid(-s["f"].float())
    g = torch.sigmoid(s["o"].float()) if s["o"] is not None else None
    valid = None
    if s["lengths"] is not None:  # beyond its length a sequence keeps its state
        valid = (torch.arange(T, device=x.device)[None, :] < s["lengths"][:, None])[:, :, None]
        a, rest = torch.where(valid, a, 1.0), torch.where(valid, rest, 0.0)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros((B, C), device=x.device)
    b = rest * x
    b[:, 0] += a[:, 0] * h0
    h = _scan(a, b)
    y = h if g is None else g * h
    if valid is not None:
        y = torch.where(valid, y, 0.0)
    out = {"y": y.to(dt), "h": h[:, -1].clone()}
    if s["mode"] != "train":
        return out
    gy = s["gy"].float()
    if valid is not None:
        gy = torch.where(valid, gy, 0.0)
    q = gy if g is None else gy * g
    if s["gh"] is not None:
        q = torch.cat([q[:, :-1], (q[:, -1] + s["gh"])[:, None]], 1)
    # the gradient of each state, from the last step to the first
    later = torch.cat([torch.ones_like(a[:, :1]), a[:, 1:].flip(1)], 1)
    d = _scan(later, q.flip(1)).flip(1)
    before = torch.cat([h0[:, None], h[:, :-1]], 1)
    out["dx"] = (rest * d).to(dt)
    out["df"] = (d * (before - x) * a * rest).to(dt)
    out["do"] = None if g is None else (gy * h * g * torch.sigmoid(-s["o"].float())).to(dt)
    out["dh0"] = a[:, 0] * d[:, 0]
    return out


def _signed(v):
    v &= MASK64
    return v - (1 << 64) if v >> 63 else v


def _shift(z, n):
    return (z >> n) & ((1 << (64 - n)) - 1)


def _mix(z):
    """SplitMix64's output function on a tensor of 64-bit words."""
    z = (z ^ _shift(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shift(z, 27)) * _signed(0x94D049BB133111EB)
    return z ^ _shift(z, 31)


def _plain_mask(s, n):
    """(element kept, its factor) of n elements: element i has bits 16 (i mod 4) on of word i / 4."""
    word = lambda v: torch.full((1,), _signed(v), dtype=torch.int64, device=DEV)  # noqa: E731
    key = _mix(_mix(_mix(word(s["seed"])) ^ s["step"]) ^ word(s["site"]))
    w = _mix(key + torch.arange(1, -(-n // 4) + 1, device=DEV) * _signed(0x9E3779B97F4A7C15))
    u = torch.stack([_shift(w, j) & 0xFFFF if j else w & 0xFFFF for j in (0, 16, 32, 48)], 1).reshape(-1)[:n]
    t = int(s["p"] * 65536 + 0.5)
    return u >= t, 65536 / (65536 - t) if t < 65536 else 0.0


def _plain_dropout(s):
    x, dt = s["x"].float(), s["x"].dtype
    keep, factor = _plain_mask(s, x.numel())
    keep = keep.view(x.shape)
    y = torch.where(keep, x * factor, 0.0)
    if s["r"] is not None:
        y = s["r"].float() + y
    out = {"y": y.to(dt)}
    if s["mode"] == "train":
        out["dx"] = torch.where(keep, s["gy"].float() * factor, 0.0).to(dt)
    return out


def _plain_xent(s):
    z, t = s["logits"].float(), s["targets"]
    live = t != IGNORE
    at = torch.where(live, t, 0)[:, None]
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    rows = torch.where(live, torch.log(total)[:, 0] - (z.gather(1, at) - top)[:, 0], 0.0)
    share = 1.0 / live.sum().clamp(min=1)
    out = {"mean": rows.sum() * share, "rows": rows, "grad": None}
    if s["mode"] == "train":
        g = e / total
        g.scatter_add_(1, at, torch.full_like(top, -1.0))
        out["grad"] = torch.where(live[:, None], g * share, 0.0).to(s["logits"].dtype)
    return out


# ---- what a pass cannot do without


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "recurrence":
        B, T, C = case["B"], case["T"], case["C"]
        read = sum(_lengths(case)) * C * e  # one array of the tokens that are there
        n = 3 if case["gate"] else 2
        state = 4 * B * C
        b = n * read + B * T * C * e + (2 if case["h0"] else 1) * state
        flops = (14 if case["gate"] else 8) * B * T * C
        if case["mode"] == "train":
            b += read + n * B * T * C * e + (2 if case["h0"] else 1) * state
            flops *= 3
        return {"bytes": b, "flops": flops}
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        arrays = (3 if case["residual"] else 2) + (2 if case["mode"] == "train" else 0)
        return {"bytes": arrays * n * e, "flops": 4 * n}
    N, V = case["N"], case["V"]
    return {"bytes": (2 if case["mode"] == "train" else 1) * N * V * e + 12 * N,
            "flops": (6 if case["mode"] == "train" else 3) * N * V}


# ---- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"recurrence": _exact_recurrence, "dropout": _exact_dropout, "xent": _exact_xent}[case["op"]](s)


def _exact_recurrence(s):
    """Step by step along time, then back."""
    x, f = s["x"], s["f"]
    B, T, C = x.shape
    if T > 20_000 and s["mode"] == "train" and B * C > 4_096:
        return None
    f64 = dict(dtype=torch.float64, device=x.device)
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device=x.device)
    h = s["h0"].double() if s["h0"] is not None else torch.zeros((B, C), **f64)
    one = torch.ones((B, C), **f64)
    train = s["mode"] == "train"
    out = {"y": torch.empty((B, T, C), **f64)}
    hs = torch.empty((T, B, C), **f64) if train else None
    for t in range(T):
        if train:
            hs[t] = h
        on = (t < n)[:, None]
        k = 1 / (1 + torch.exp(-f[:, t].double()))
        h = torch.where(on, k * h + x[:, t].double() / (1 + torch.exp(f[:, t].double())), h)
        gate = 1 / (1 + torch.exp(-s["o"][:, t].double())) if s["o"] is not None else one
        out["y"][:, t] = torch.where(on, gate * h, 0 * one)
    out["h"] = h
    if not train:
        return out
    out["dx"], out["df"] = torch.empty((B, T, C), **f64), torch.empty((B, T, C), **f64)
    out["do"] = torch.empty((B, T, C), **f64) if s["o"] is not None else None
    carry = s["gh"].double() if s["gh"] is not None else torch.zeros((B, C), **f64)
    for t in reversed(range(T)):
        on = (t < n)[:, None]
        ft, xt, gt = f[:, t].double(), x[:, t].double(), s["gy"][:, t].double()
        k, left = 1 / (1 + torch.exp(-ft)), 1 / (1 + torch.exp(ft))
        now = k * hs[t] + left * xt
        gate = one
        if s["o"] is not None:
            ot = s["o"][:, t].double()
            gate = 1 / (1 + torch.exp(-ot))
            out["do"][:, t] = torch.where(on, gt * now * gate / (1 + torch.exp(ot)), 0 * one)
        d = carry + gt * gate
        out["dx"][:, t] = torch.where(on, d * left, 0 * one)
        out["df"][:, t] = torch.where(on, d * (hs[t] - xt) * k * left, 0 * one)
        carry = torch.where(on, k * d, carry)
    out["dh0"] = carry
    return out


def _exact_dropout(s):
    """The generator in unsigned 64-bit words on the host."""
    n = s["x"].numel()

    def mix(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        key = mix(np.array([s["seed"]], np.uint64))
        key = mix(key ^ np.array([int(s["step"])], np.uint64))
        key = mix(key ^ np.array([s["site"]], np.uint64))
        words = mix(key + np.arange(1, (n + 3) // 4 + 1, dtype=np.uint64) * np.uint64(0x9E3779B97F4A7C15))
    draws = words.astype("<u8").view("<u2")[:n]
    dropped = math.floor(s["p"] * 65536 + 0.5)
    keep = torch.from_numpy(draws >= dropped).to(DEV).view(s["x"].shape)
    keep = keep.double() * (65536.0 / (65536.0 - dropped))
    y = s["x"].double() * keep
    if s["r"] is not None:
        y = y + s["r"].double()
    return {"y": y, "dx": s["gy"].double() * keep} if s["mode"] == "train" else {"y": y}


def _exact_xent(s):
    z, t = s["logits"], s["targets"]
    N, V = z.shape
    rows = torch.zeros(N, dtype=torch.float64, device=z.device)
    count = max(1, int((t != IGNORE).sum()))
    train = s["mode"] == "train"
    grad = torch.zeros((N, V), dtype=torch.float64, device=z.device) if train else None
    for at in range(0, N, 512):
        part, tt = z[at:at + 512].double(), t[at:at + 512]
        lse = torch.logsumexp(part, 1)
        live = (tt != IGNORE).nonzero()[:, 0]
        rows[at + live] = lse[live] - part[live, tt[live]]
        if train:
            p = torch.exp(part[live] - lse[live, None]) / count
            p[torch.arange(live.numel(), device=z.device), tt[live]] -= 1.0 / count
            grad[at + live] = p
    return {"mean": rows.sum() / count, "rows": rows, "grad": grad}
