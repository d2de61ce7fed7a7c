"""The language-model operators step by step in 64 bits on the CPU, with bounds on the error of a
32-bit evaluation, for the GPU tests.

Bounds. u = 2^-24. A gate evaluated in fp32 (exponential, reciprocal, product) is within
(|z| + 8) u of itself, relatively; with |z| <= 12 in the tests that is 20 u, which K = 24 covers together
with the two or three roundings of a step. A quantity r_t = a_t r_(t-1) + b_t whose terms are
each off by K u of themselves is off by at most E_t = a_t E_(t-1) + K u R_t, R the same recurrence over
absolute values; a scan that splits time and joins the parts by products of gates obeys the same
bound, since the product of n gates off by K u each is off by n K u, and the recurrence counts every one of the n.
"""
import numpy as np
import torch

U = 2.0 ** -24
K = 24.0
# rounding to nearest with p significant bits is off by at most 2^-p of the value: 24, 8 and 11 bits
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def stored(bound, value, dtype):
    """The bound of a value that is rounded to dtype on its store (and to fp32 before it)."""
    return 1.01 * bound + (HALF_ULP[dtype] + 4 * U) * value.abs() + TINY[dtype]


def recurrence(x, f, o, h0, lengths, gy=None, gh=None):
    """{name: (value, error bound of a 32-bit evaluation)} in float64, on the CPU. The inputs are read
    as they are stored; what padding holds is not used."""
    d = lambda t: t.detach().cpu().double() if t is not None else None  # noqa: E731
    x, f, o, h0, gy, gh = map(d, (x, f, o, h0, gy, gh))
    B, T, C = x.shape
    n = lengths.cpu().long().clamp(0, T) if lengths is not None else torch.full((B,), T)
    on = torch.arange(T)[None, :, None] < n[:, None, None]
    zero = torch.zeros(())
    x, f = torch.where(on, x, zero), torch.where(on, f, zero)
    a, rest = torch.where(on, 1 / (1 + torch.exp(-f)), 1 + zero), torch.where(on, 1 / (1 + torch.exp(f)), zero)
    if o is not None:
        o = torch.where(on, o, zero)
        g, shut = 1 / (1 + torch.exp(-o)), 1 / (1 + torch.exp(o))
    else:
        g, shut = torch.ones_like(x), torch.zeros_like(x)
    h = h0 if h0 is not None else torch.zeros((B, C), dtype=torch.float64)
    size, err = h.abs(), torch.zeros_like(h)
    before, hs, errs_before, errs, sizes = [], [], [], [], []
    for t in range(T):
        before.append(h)
        errs_before.append(err)
        h = a[:, t] * h + rest[:, t] * x[:, t]
        size = a[:, t] * size + rest[:, t] * x[:, t].abs()
        err = a[:, t] * err + torch.where(on[:, t], K * U * size, zero)
        hs.append(h)
        errs.append(err)
        sizes.append(size)
    out = {"h_last": (h, err)}
    stack = lambda v: torch.stack(v, 1) if v else torch.zeros((B, 0, C), dtype=torch.float64)  # noqa: E731
    H, EH, P, EP, SH = stack(hs), stack(errs), stack(before), stack(errs_before), stack(sizes)
    out["y"] = (torch.where(on, g * H, zero), torch.where(on, g * (EH + K * U * SH), zero))
    if gy is None:
        return out
    gy = torch.where(on, gy, zero)
    q = gy * g
    c = gh if gh is not None else torch.zeros((B, C), dtype=torch.float64)
    size, err = c.abs(), torch.zeros_like(c)
    s, es, ss = [None] * T, [None] * T, [None] * T
    for t in reversed(range(T)):
        s[t] = q[:, t] + c
        ss[t] = q[:, t].abs() + size
        es[t] = err + torch.where(on[:, t], K * U * ss[t], zero)
        c, size, err = a[:, t] * s[t], a[:, t] * ss[t], a[:, t] * es[t]
    S, ES, SS = stack(s), stack(es), stack(ss)
    out["dh0"] = (c, err + 2 * U * size)
    out["dx"] = (torch.where(on, rest * S, zero), torch.where(on, rest * (ES + K * U * SS), zero))
    w = a * rest
    out["df"] = (torch.where(on, S * (P - x) * w, zero),
                 torch.where(on, w * (ES * (P - x).abs() + SS * EP + 2 * K * U * SS * (P.abs() + x.abs())), zero))
    if o is not None:
        w = gy.abs() * g * shut
        out["do"] = (torch.where(on, gy * H * g * shut, zero), torch.where(on, w * (EH + 2 * K * U * SH), zero))
    return out


M64 = (1 << 64) - 1


def draws(n, seed, site, step):
    """The 16-bit draws of n elements, by Python integers and NumPy's unsigned words."""
    def mix(z):
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
        return z ^ (z >> 31)

    key = mix(mix(mix(seed & M64) ^ (step & M64)) ^ (site & M64))
    with np.errstate(over="ignore"):
        z = np.uint64(key) + (np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z = z ^ (z >> np.uint64(31))
    return z.astype("<u8").view("<u2")[:n]


def dropout(x, p, seed, site=0, step=0, residual=None):
    """The result itself, bit for bit: fp32 product and sum, one rounding to x's type."""
    below = int(np.floor(p * 65536 + 0.5))
    keep = torch.from_numpy(draws(x.numel(), seed, site, step) >= below).view(x.shape)
    factor = np.float32(65536.0 / (65536.0 - below)) if below < 65536 else np.float32(0)
    y = torch.where(keep, x.cpu().float() * float(factor), torch.zeros(()))
    if residual is not None:
        y = residual.cpu().float() + y
    return y.to(x.dtype)


def cross_entropy(z, t, ignore=-100):
    """losses, mean, gradient of the mean, and the bounds of each. A probability in fp32 is off by (2 |z - top| + 8) u
    of itself and by the sum's error, which is at most u for each addition that one term goes through: V / 64
    of a lane and 64 more."""
    z, t = z.detach().cpu().double(), t.cpu()
    N, V = z.shape
    live = t != ignore
    at = torch.where(live, t, 0)
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    p = e / total
    losses = (top + torch.log(total))[:, 0] - z.gather(1, at[:, None])[:, 0]
    far = torch.where(torch.isfinite(z), (z - top).abs(), torch.zeros(()).double())
    sums = (2 * (p * far).sum(1) + V / 64 + 64) * U
    zero = torch.zeros((), dtype=torch.float64)
    e_loss = torch.where(live, sums + 4 * U * (losses.abs() + top[:, 0].abs()), zero)
    losses = torch.where(live, losses, zero)
    count = max(1, int(live.sum()))
    hot = torch.zeros_like(z)
    hot[torch.arange(N), at] = 1.0
    grad = torch.where(live[:, None], (p - hot) / count, zero)
    e_grad = torch.where(live[:, None], (p * (2 * far + 8) * U + p * sums[:, None] + 8 * U * (p - hot).abs()) / count, zero)
    return {"losses": (losses, e_loss), "mean": (losses.sum() / count, e_loss.sum() / count + 4 * U * losses.abs().sum() / count),
            "grad": (grad, e_grad)}


def check(got, want, dtype, what):
    """Assert |got - value| <= the bound of a store in dtype, everywhere, and print the worst share of it."""
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    if got.numel() == 0:
        return
    share = ((got - value).abs() / stored(bound, value, dtype)).max().item()
    assert share <= 1.0, f"{what}: error is {share:.2f} of its bound"
