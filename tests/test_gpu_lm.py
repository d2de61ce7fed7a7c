"""The language-model operators on the GPU against 64-bit references (needs an MI355X)."""
import numpy as np
import pytest

import lm_reference as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
gs = pytest.importorskip("paper_2108_06004_amd")
from paper_2108_06004_amd import lm  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
IDS = ["f32", "bf16", "f16"]
NAN = float("nan")


def rnd(gen, *shape, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(shape, generator=gen) * scale + shift).to(dtype).to(DEV)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def inputs(seed, B, T, C, dtype, gate=True, h0=True, packed=False, grads=True):
    """Inputs of a recurrence; gates reach from nearly shut to nearly open (|z| <= 12)."""
    g = gen(seed)
    n = 3 if gate else 2
    xfo = rnd(g, B, T, n * C, dtype=dtype)
    x, f = xfo[:, :, :C], xfo[:, :, C:2 * C]
    f.mul_(2.5).add_(1.5).clamp_(-12, 12)
    o = xfo[:, :, 2 * C:].mul_(2.0) if gate else None
    if not packed:
        x, f, o = x.contiguous(), f.contiguous(), o.contiguous() if gate else None
    gy = rnd(g, B, T, C, dtype=dtype) if grads else None
    return dict(x=x, f=f, o=o, h0=rnd(g, B, C) if h0 else None, gy=gy, gh=rnd(g, B, C) if grads and h0 else None)


def run_and_check(i, lengths=None, what=""):
    """Forward and backward of one set of inputs against the reference; returns all outputs."""
    dt = i["x"].dtype
    y, h, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], lengths=lengths, save=True)
    dx, df, do, dh0 = lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, lengths=lengths, gh=i["gh"])
    torch.cuda.synchronize()
    want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], lengths, i["gy"], i["gh"])
    got = {"y": y, "h_last": h, "dx": dx, "df": df, "dh0": dh0}
    if i["o"] is not None:
        got["do"] = do
    else:
        assert do is None
    for name, t in got.items():
        ref.check(t, want[name], torch.float32 if name in ("h_last", "dh0") else dt, f"{what} {name}")
    only, h2, none = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], lengths=lengths)
    assert none is None and torch.equal(only, y) and torch.equal(h2, h)  # without the saved states: the same bits
    return got


# one token, a thread's steps (8), the steps between saved states (32), blocks (32, 64, 128) and the length from which
# time is split (256), each from both sides; several blocks, an odd number of them
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 1000])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_lengths_of_time(T, dtype):
    run_and_check(inputs(T, 2, T, 40, dtype), what=f"T={T}")


@pytest.mark.parametrize("C", [1, 2, 3, 31, 32, 33, 63, 64, 65, 130, 1500])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_channel_counts(C, dtype):
    run_and_check(inputs(100 + C, 3, 150, C, dtype), what=f"C={C}")
    run_and_check(inputs(200 + C, 3, 1, C, dtype), what=f"C={C}, one token")


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("h0", [True, False])
@pytest.mark.parametrize("packed", [True, False])
def test_recurrence_forms(gate, h0, packed):
    for T in (1, 5, 200):
        run_and_check(inputs(7 + T, 4, T, 96, torch.bfloat16, gate, h0, packed), what=f"T={T}")


# few channels and much time: the work is split along time and joined
@pytest.mark.parametrize("B,T,C", [(1, 5000, 64), (2, 3001, 31), (1, 20_000, 8), (3, 2048, 160)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_split_along_time(B, T, C, dtype):
    run_and_check(inputs(B * T, B, T, C, dtype, packed=True), what=f"{B}x{T}x{C}")


@pytest.mark.parametrize("B,T,C,lengths", [
    (6, 300, 48, [300, 0, 1, 128, 129, 257]),
    (5, 1, 48, [1, 0, 1, 0, 1]),
    (4, 6, 33, [0, 6, 3, 1]),
    (4, 9000, 16, [9000, 0, 5, 4500]),      # split along time: some parts hold no token
    (3, 200, 7, [-5, 500, 100]),            # outside [0, T]: taken as the nearer end
    (3, 200, 64, [0, 0, 0]),
])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_padding_is_not_used(B, T, C, lengths, dtype):
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    for packed in (False, True):
        i = inputs(B * T + C, B, T, C, dtype, packed=packed)
        clean = run_and_check(i, n, "clean")
        pad = torch.arange(T, device=DEV)[None, :] >= n[:, None]
        for name, bad in (("x", NAN), ("f", float("inf")), ("o", NAN), ("gy", -float("inf"))):
            i[name][pad] = bad
        dirty = run_and_check(i, n, "padding of NaN and infinities")
        for name in clean:
            assert torch.equal(clean[name], dirty[name]), name
        assert not dirty["y"][pad].any() and not dirty["dx"][pad].any() and not dirty["df"][pad].any()


@pytest.mark.parametrize("T", [6, 40, 300, 5000])  # no groups, one block, several, split along time
@pytest.mark.parametrize("gate", [True, False])
def test_recurrence_gradients_are_zero_at_padding(T, gate):
    # also where the state or its gradient is infinite or NaN, whose products with zero are not zero
    for dtype in TYPES:
        for gh, x in ((float("inf"), 0.0), (NAN, 0.0), (1.0, float("inf")), (1.0, NAN)):
            i = inputs(T, 4, T, 34, dtype, gate)
            n = torch.tensor([T - 3, T, 0, T // 2 + 1], dtype=torch.int32, device=DEV)
            i["gh"][:, ::2] = gh
            i["x"][:, T // 2, 1::3] += x
            _, _, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], lengths=n, save=True)
            dx, df, do, _ = lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, lengths=n, gh=i["gh"])
            pad = torch.arange(T, device=DEV)[None, :] >= n[:, None]
            for name, t in (("dx", dx), ("df", df), ("do", do)):
                if t is not None:
                    assert torch.equal(t[pad], torch.zeros_like(t[pad])), f"{dtype} {name} gh {gh} x {x}"


def test_recurrence_extreme_gates():
    # gates of exactly 0 and 1 (infinite pre-activations) and of the types' largest values
    for dtype in TYPES:
        i = inputs(3, 2, 140, 64, dtype)
        big = torch.finfo(dtype).max
        for t, z in ((0, float("inf")), (1, -float("inf")), (2, big), (3, -big), (130, float("inf")), (131, -float("inf"))):
            i["f"][:, t] = z
            i["o"][:, t + 4] = z
        run_and_check(i, what=str(dtype))


def test_recurrence_nan_gates_are_not_swallowed():
    # a NaN among the tokens reaches everything computed from it, and nothing else
    for T, t in ((1, 0), (6, 2), (200, 70), (3000, 1500)):
        i = inputs(4, 2, T, 70, torch.bfloat16)
        i["f"][1, t, 5] = NAN
        y, h, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], save=True)
        dx, df, do, dh0 = lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, gh=i["gh"])
        assert torch.isnan(y[1, t:, 5]).all() and torch.isnan(h[1, 5]) and torch.isnan(dh0[1, 5])
        assert torch.isnan(do[1, t:, 5]).all() and torch.isnan(df[1, :t + 1, 5]).all() and torch.isnan(dx[1, :t, 5]).all()
        for out in (y, dx, df, do):
            assert torch.isfinite(out[0]).all() and torch.isfinite(out[1, :, 6:]).all() and torch.isfinite(out[1, :, :5]).all()
        assert torch.isfinite(y[1, :t, 5]).all()


def test_recurrence_zero_sizes():
    for B, T, C in ((0, 5, 8), (3, 0, 8), (3, 5, 0)):
        i = inputs(1, B, T, C, torch.bfloat16)
        y, h, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], save=True)
        dx, df, do, dh0 = lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, gh=i["gh"])
        assert y.shape == dx.shape == (B, T, C)
        if T == 0:
            assert torch.equal(h, i["h0"]) and torch.equal(dh0, i["gh"])


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_recurrence_strides(dtype):
    # time-major tensors, views off their alignment, gradients into slices, an expanded gradient
    B, T, C = 3, 260, 50
    i = inputs(11, B, T, C, dtype)
    base = run_and_check(i)
    j = dict(i)
    j["x"] = i["x"].transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.empty((B, T, C + 3), dtype=dtype, device=DEV)
    wide[:, :, 1:C + 1] = i["f"]
    j["f"] = wide[:, :, 1:C + 1]
    j["o"] = torch.cat([i["o"], i["o"]], 1)[:, :T]
    again = run_and_check(j, what="views")
    for name in base:
        ref_t, got_t = base[name].double().cpu(), again[name].double().cpu()
        assert torch.allclose(ref_t, got_t, rtol=2.0 ** -6, atol=1e-3), name
    i["gy"] = torch.ones((1, 1, C), dtype=dtype, device=DEV).expand(B, T, C)
    plain = run_and_check(i, what="expanded gradient")
    out = torch.full((B, T, 3 * C), 7.0, dtype=dtype, device=DEV)
    _, _, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], save=True)
    parts = out.split(C, -1)
    lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, gh=i["gh"], dx=parts[0], df=parts[1], do=parts[2])
    for name, t in zip(("dx", "df", "do"), parts):
        assert torch.allclose(t.float(), plain[name].float(), rtol=2.0 ** -6, atol=1e-3), name


def test_recurrence_state_in_place_and_token_by_token():
    # a sequence read whole, and the same read token by token with the state updated in place
    i = inputs(5, 4, 40, 96, torch.bfloat16)
    y, h, _ = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"])
    state = i["h0"].clone()
    steps = [lm.recurrence_forward(i["x"][:, t:t + 1], i["f"][:, t:t + 1], i["o"][:, t:t + 1], h0=state, h_last=state)[0]
             for t in range(40)]
    want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], None)
    ref.check(torch.cat(steps, 1), want["y"], torch.bfloat16, "token by token")
    ref.check(state, want["h_last"], torch.float32, "state")
    for B, T, C in ((1, 4000, 40), (2, 300, 40)):  # in place where time is split, and where it is not
        i = inputs(6, B, T, C, torch.float32)
        want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], None)
        lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], h_last=i["h0"])
        ref.check(i["h0"], want["h_last"], torch.float32, f"in place, T={T}")


def test_recurrence_offsets_beyond_32_bits():
    # sequences that start more than 2^31 elements (and 2^32 bytes) apart
    stride = (1 << 31) + 64
    B, T, C = 2, 140, 64
    store = torch.empty(stride + T * 3 * C, dtype=torch.bfloat16, device=DEV)
    i = inputs(8, B, T, C, torch.bfloat16)
    views = {}
    for n, name in enumerate(("x", "f", "o")):
        views[name] = store.as_strided((B, T, C), (stride, 3 * C, 1), n * C)
        views[name].copy_(i[name])
    base = run_and_check(i)
    far = run_and_check({**i, **views})
    for name in base:
        assert torch.equal(base[name], far[name]), name


def test_recurrence_gradient_against_differences():
    # <gradient, direction> against central differences of the loss in 64 bits
    i = inputs(12, 2, 150, 24, torch.float32)
    got = run_and_check(i)
    g = gen(99)
    step = 1e-5

    def loss(k):
        r = ref.recurrence(k["x"], k["f"], k["o"], k["h0"], None)
        return float((r["y"][0] * i["gy"].cpu().double()).sum() + (r["h_last"][0] * i["gh"].cpu().double()).sum())

    for name, grad in (("x", "dx"), ("f", "df"), ("o", "do"), ("h0", "dh0")):
        v = torch.randn(i[name].shape, generator=g, dtype=torch.float64)
        there, back = dict(i), dict(i)
        there[name] = i[name].cpu().double() + step * v
        back[name] = i[name].cpu().double() - step * v
        slope = (loss(there) - loss(back)) / (2 * step)
        dot = got[grad].cpu().double() * v
        # differences: truncation of order step^2; the gradient: fp32 rounding of each term
        assert abs(slope - float(dot.sum())) <= 1e-5 * float(dot.abs().sum()), name


@pytest.mark.parametrize("gate", [True, False])
def test_recurrence_autograd(gate):
    B, T, C = 3, 70, 20
    i = inputs(21, B, T, C, torch.float32, gate=gate)
    leaves = {k: i[k].clone().requires_grad_() for k in ("x", "f", "h0") + (("o",) if gate else ())}
    lengths = torch.tensor([70, 0, 33], dtype=torch.int32, device=DEV)
    y, h = lm.gated_recurrence(leaves["x"], leaves["f"], leaves.get("o"), leaves["h0"], lengths)
    torch.autograd.backward([y, h], [i["gy"], i["gh"]])
    want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], lengths, i["gy"], i["gh"])
    for k in leaves:
        ref.check(leaves[k].grad, want["d" + k], torch.float32, k)
    packed = torch.cat([i[k] for k in ("x", "f", "o") if i[k] is not None], -1).requires_grad_()
    y2, h2 = lm.gated_recurrence_packed(packed, C, i["h0"], lengths)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    y2.backward(i["gy"])
    want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], lengths, i["gy"], None)
    for n, k in enumerate(("dx", "df", "do")[:3 if gate else 2]):
        ref.check(packed.grad[:, :, n * C:(n + 1) * C], want[k], torch.float32, k)
    # only the last state is used
    only = i["x"].clone().requires_grad_()
    lm.gated_recurrence(only, i["f"], i["o"], i["h0"])[1].sum().backward()
    want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], None, torch.zeros_like(i["gy"]), torch.ones_like(i["gh"]))
    ref.check(only.grad, want["dx"], torch.float32, "last state alone")


# ---- dropout


@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8, 9, 255, 2048, 2049, 100_003])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_dropout_bit_for_bit(n, dtype):
    g = gen(n)
    x, r = rnd(g, n, dtype=dtype), rnd(g, n, dtype=dtype)
    step = torch.tensor([77], dtype=torch.int64, device=DEV)
    for p in (0.0, 1e-6, 0.1, 0.5, 0.999, 1.0):
        for residual in (None, r):
            y = lm.dropout_forward(x, p, 1234, site=9, step=step, residual=residual)
            assert torch.equal(y.cpu(), ref.dropout(x, p, 1234, 9, 77, residual)), (p, residual is not None)
    y = lm.dropout_forward(x, 0.5, -1, site=(1 << 64) - 1)  # no step: 0; the words wrap
    assert torch.equal(y.cpu(), ref.dropout(x, 0.5, -1, (1 << 64) - 1, 0))


@pytest.mark.parametrize("rows,cols,pad", [(5, 64, 8), (7, 33, 1), (3, 1000, 24), (300, 6, 2), (2, 2050, 6), (1, 9, 4),
                                           (70_000, 3, 1)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_dropout_rows_apart(rows, cols, pad, dtype):
    # strided rows draw what the contiguous tensor draws; what lies between them stays
    g = gen(rows)
    x, r = rnd(g, rows, cols + pad, dtype=dtype)[:, :cols], rnd(g, rows, cols, dtype=dtype)
    whole = torch.full((rows, cols + pad), 5.0, dtype=dtype, device=DEV)
    y = whole[:, pad:]
    lm.dropout_forward(x, 0.3, 5, residual=r, y=y)
    assert torch.equal(y.cpu(), ref.dropout(x, 0.3, 5, residual=r))
    assert (whole[:, :pad] == 5.0).all()
    assert torch.equal(lm.dropout_forward(x, 0.3, 5, residual=r), y)


def test_dropout_unaligned_and_in_place():
    for dtype in TYPES:
        g = gen(4)
        store = rnd(g, 4101, dtype=dtype)
        want = ref.dropout(store[3:4100], 0.4, 8)
        assert torch.equal(lm.dropout_forward(store[3:4100], 0.4, 8).cpu(), want)
        x = store[3:4100].clone()
        lm.dropout_forward(x, 0.4, 8, y=x)
        assert torch.equal(x.cpu(), want)
        r = rnd(g, 4097, dtype=dtype)
        want = ref.dropout(store[3:4100], 0.4, 8, residual=r)
        lm.dropout_forward(store[3:4100], 0.4, 8, residual=r, y=r)
        assert torch.equal(r.cpu(), want)


def test_dropout_dropped_elements_are_not_used():
    x = torch.full((64, 64), NAN, dtype=torch.bfloat16, device=DEV)
    keep = torch.from_numpy(ref.draws(4096, 3, 0, 0) >= 32768).view(64, 64).to(DEV)
    x[keep] = 1.0
    y = lm.dropout_forward(x, 0.5, 3)
    assert torch.equal(y, keep.to(torch.bfloat16) * 2)
    r = torch.ones_like(x)
    assert torch.equal(lm.dropout_forward(torch.full_like(x, float("inf")), 1.0, 3, residual=r), r)


def test_dropout_masks_are_independent_and_of_the_right_density():
    n = 1 << 20
    x = torch.ones(n, device=DEV)
    a = lm.dropout_forward(x, 0.25, 1, site=0) > 0
    sets = {"site": lm.dropout_forward(x, 0.25, 1, site=1) > 0, "seed": lm.dropout_forward(x, 0.25, 2) > 0,
            "step": lm.dropout_forward(x, 0.25, 1, step=torch.ones(1, dtype=torch.int64, device=DEV)) > 0}
    five = 5 * (0.25 * 0.75 / n) ** 0.5
    assert abs(float(a.float().mean()) - 0.75) < five
    for name, b in sets.items():
        both = float((a & b).float().mean())
        assert abs(both - 0.75 ** 2) < 5 * (0.5625 * 0.4375 / n) ** 0.5, name
    for lane in range(4):
        assert abs(float(a[lane::4].float().mean()) - 0.75) < 2 * five


def test_dropout_autograd():
    g = gen(6)
    x, r = rnd(g, 33, 50).requires_grad_(), rnd(g, 33, 50).requires_grad_()
    step = torch.tensor([3], dtype=torch.int64, device=DEV)
    gy = rnd(g, 33, 50)
    lm.dropout(x, 0.3, 11, 2, step, r).backward(gy)
    assert torch.equal(x.grad.cpu(), ref.dropout(gy, 0.3, 11, 2, 3)) and torch.equal(r.grad, gy)
    y = lm.dropout(x, 0.3, 11, 2, step, r)
    step.add_(1)
    with pytest.raises(RuntimeError):  # another mask than the forward pass drew
        y.backward(gy)


def test_dropout_offsets_beyond_32_bits():
    n = (1 << 31) + 4099
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    y = lm.dropout_forward(x, 0.5, 21)
    for at in (0, (1 << 31) - 2000, n - 4000):
        at -= at % 4
        m = min(4000, n - at)
        key = np.uint64(0)
        words = np.arange(at // 4, (at + m + 3) // 4, dtype=np.uint64)
        d = ref.draws(4, 21, 0, 0)  # the generator's own check of the key below
        with np.errstate(over="ignore"):
            def mix(z):
                z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
                z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
                return z ^ (z >> np.uint64(31))
            key = mix(mix(mix(np.array([21], np.uint64))))
            w = mix(key + (words + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15))
            first = mix(key + np.uint64(0x9E3779B97F4A7C15)).view("<u2")
        assert np.array_equal(first, d)
        keep = torch.from_numpy(w.view("<u2")[:m] >= 32768)
        assert torch.equal(y[at:at + m].cpu(), keep.to(torch.bfloat16) * 2), at


# ---- cross-entropy


def logits(seed, N, V, dtype, scale=3.0):
    g = gen(seed)
    z = rnd(g, N, V, dtype=dtype, scale=scale)
    t = torch.randint(0, V, (N,), generator=g).to(DEV)
    z[torch.arange(N, device=DEV), t] += 4.0
    return z, t


def check_xent(z, t, ignore=-100, what=""):
    want = ref.cross_entropy(z, t, ignore)
    mean, losses, none = lm.cross_entropy_forward(z, t, ignore)
    assert none is None
    mean2, losses2, grad = lm.cross_entropy_forward(z, t, ignore, grad=True)
    assert torch.equal(mean, mean2) and torch.equal(losses, losses2)
    ref.check(losses, want["losses"], torch.float32, what + " losses")
    ref.check(mean, want["mean"], torch.float32, what + " mean")
    ref.check(grad, want["grad"], z.dtype, what + " grad")
    inside = z.clone()
    lm.cross_entropy_forward(inside, t, ignore, grad=inside)
    ref.check(inside, want["grad"], z.dtype, what + " in place")
    if inside.stride() == z.stride():  # the bits of a row depend on its alignment
        assert torch.equal(inside, grad), what + " in place"
    return grad


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 64, 65, 257, 1000, 1500, 2049, 4096, 9001, 22_000, 40_001])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cross_entropy_vocabularies(V, dtype):
    z, t = logits(V, 5, V, dtype)
    t[3] = -100
    check_xent(z, t, what=f"V={V}")


# rows that no workgroup can hold, few rows of many logits, many rows of few
@pytest.mark.parametrize("N,V", [(1, 200_003), (3, 131_072), (2, 131_071), (1, 65_536), (700, 65), (3000, 10), (257, 1001)])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cross_entropy_extents(N, V, dtype):
    z, t = logits(N + V, N, V, dtype)
    check_xent(z, t, what=f"{N}x{V}")


@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cross_entropy_strided_rows(dtype):
    for N, V, wide, at in ((9, 1000, 1008, 0), (9, 999, 1024, 0), (6, 501, 517, 3), (2, 70_001, 70_005, 1)):
        z, t = logits(V, N, wide, dtype)
        t = t % V
        view = z[:, at:at + V]
        grad = check_xent(view, t, what=f"{N}x{V} of {wide}")
        out = torch.full((N, wide + 2), 9.0, dtype=dtype, device=DEV)
        lm.cross_entropy_forward(view, t, grad=out[:, 1:V + 1])
        assert torch.equal(out[:, 1:V + 1], grad)
        assert (out[:, 0] == 9.0).all() and (out[:, V + 1:] == 9.0).all()


@pytest.mark.parametrize("V", [10, 3001, 70_000, 150_000])
@pytest.mark.parametrize("dtype", TYPES, ids=IDS)
def test_cross_entropy_masks(V, dtype):
    # logits of -inf and of the type's lowest value; ignored rows of NaN; rows without a softmax
    z, t = logits(V, 8, V, dtype)
    low = torch.finfo(dtype).min
    z[0, torch.arange(V, device=DEV) != t[0]] = -float("inf")  # the target alone is left
    z[1, torch.arange(V, device=DEV) % 2 != t[1] % 2] = -float("inf")
    z[2, torch.arange(V, device=DEV) % 2 != t[2] % 2] = low
    z[3] = NAN
    t[3] = -100
    z[4] = low  # all alike: uniform
    clean = z.clone()
    clean[3] = 0
    want = ref.cross_entropy(clean, t)
    mean, losses, grad = lm.cross_entropy_forward(z, t, grad=True)
    ref.check(losses, want["losses"], torch.float32, "losses")
    ref.check(mean, want["mean"], torch.float32, "mean")
    ref.check(grad, want["grad"], dtype, "grad")
    assert not grad[3].any()
    # a target of probability zero: its loss is infinite, its gradient is not
    z[5, t[5]] = -float("inf")
    _, losses, grad = lm.cross_entropy_forward(z, t, grad=True)
    assert losses[5] == float("inf") and torch.isfinite(grad[5]).all()
    # no softmax: NaN there, and nowhere else
    z[5] = -float("inf")
    z[6, V // 2] = NAN
    z[7, V - 1] = float("inf")
    _, losses, grad = lm.cross_entropy_forward(z, t, grad=True)
    assert torch.isnan(losses[5:]).all() and torch.isnan(grad[5:]).all()
    assert torch.isfinite(losses[:5]).all() and torch.isfinite(grad[:5]).all()


@pytest.mark.parametrize("V", [10, 2000, 150_000])
def test_cross_entropy_targets_outside_the_vocabulary(V):
    z, t = logits(1, 5, V, torch.bfloat16)
    t[1], t[2], t[3] = V, -1, 1 << 40
    _, losses, grad = lm.cross_entropy_forward(z, t, grad=True)
    assert torch.isnan(losses[1:4]).all() and torch.isnan(grad[1:4]).all()
    assert torch.isfinite(losses[[0, 4]]).all() and torch.isfinite(grad[[0, 4]]).all()
    t[1:4] = V  # as the index to ignore it is no fault
    check_xent(z, t, ignore=V)


def test_cross_entropy_no_row_counts():
    for N, V in ((4, 50), (2, 150_000)):
        z, _ = logits(2, N, V, torch.float32)
        t = torch.full((N,), -100, dtype=torch.int64, device=DEV)
        mean, losses, grad = lm.cross_entropy_forward(z, t, grad=True)
        assert mean == 0 and not losses.any() and not grad.any()
    mean, losses, grad = lm.cross_entropy_forward(z[:0], t[:0], grad=True)
    assert mean == 0 and losses.shape == (0,) and grad.shape == (0, V)


def test_cross_entropy_offsets_beyond_32_bits():
    N, V, stride = 2, 1001, (1 << 31) + 8
    z, t = logits(3, N, V, torch.bfloat16)
    store = torch.empty(stride + V, dtype=torch.bfloat16, device=DEV)
    view = store.as_strided((N, V), (stride, 1))
    view.copy_(z)
    check_xent(z, t)
    ref.check(lm.cross_entropy_forward(view, t, grad=True)[2], ref.cross_entropy(z, t)["grad"], torch.bfloat16, "far rows")


def test_cross_entropy_gradient_against_differences():
    z, t = logits(4, 6, 301, torch.float32)
    grad = check_xent(z, t).cpu().double()
    v = torch.randn(z.shape, generator=gen(1), dtype=torch.float64)
    step = 1e-5
    up, down = (float(ref.cross_entropy(z.cpu().double() + s * v, t)["mean"][0]) for s in (step, -step))
    assert abs((up - down) / (2 * step) - float((grad * v).sum())) <= 1e-5 * float((grad * v).abs().sum())


@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_cross_entropy_autograd_and_factor(reduction):
    z, t = logits(5, 12, 333, torch.float32)
    t[4] = -100
    want = ref.cross_entropy(z, t)
    count = int((t != -100).sum())
    leaf = z.clone().requires_grad_()
    out = lm.cross_entropy(leaf, t, reduction=reduction)
    if reduction == "mean":
        (3.0 * out).backward()
        ref.check(leaf.grad, (3 * want["grad"][0], 3 * want["grad"][1]), torch.float32, "mean")
    else:
        w = torch.arange(1.0, 13.0, device=DEV)
        out.backward(w)
        rows = w.cpu().double()[:, None] * count
        ref.check(leaf.grad, (rows * want["grad"][0], rows * want["grad"][1]), torch.float32, "rows")
    scaled = lm.cross_entropy_forward(z, t, grad=True, factor=1024.0)[2]
    assert torch.equal(scaled, 1024.0 * lm.cross_entropy_forward(z, t, grad=True)[2])


# ---- how calls are made


def everything(i, z, t, step):
    y, h, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], save=True)
    u = lm.dropout_forward(y, 0.2, 5, step=step, residual=i["x"])
    dy = lm.dropout_backward(i["gy"], 0.2, 5, step=step)
    grads = lm.recurrence_backward(dy, i["x"], i["f"], i["o"], saved, gh=i["gh"])
    return [y, h, u, dy, *grads, *lm.cross_entropy_forward(z, t, grad=True)]


@pytest.mark.parametrize("B,T,C,N,V", [(3, 200, 64, 20, 1000), (1, 4000, 64, 2, 150_000), (5, 1, 48, 5, 300)])
def test_the_same_bits_on_every_run_and_on_another_stream(B, T, C, N, V):
    i = inputs(31, B, T, C, torch.bfloat16)
    z, t = logits(6, N, V, torch.bfloat16)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    first = everything(i, z, t, step)
    for _ in range(3):
        for p, q in zip(first, everything(i, z, t, step)):
            assert torch.equal(p, q)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        there = everything(i, z, t, step)
    side.synchronize()
    for p, q in zip(first, there):
        assert torch.equal(p, q)


@pytest.mark.parametrize("B,T,C,N,V", [(3, 200, 64, 20, 1000), (1, 4000, 64, 2, 150_000), (5, 1, 48, 5, 300)])
def test_replays_of_a_captured_graph_equal_eager_calls(B, T, C, N, V):
    i = inputs(32, B, T, C, torch.bfloat16)
    z, t = logits(7, N, V, torch.bfloat16)
    step = torch.zeros(1, dtype=torch.int64, device=DEV)
    everything(i, z, t, step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = everything(i, z, t, step)
    last = None
    for n in range(4):
        step.fill_(n)  # a new mask on each replay
        i["x"].copy_(inputs(40 + n, B, T, C, torch.bfloat16)["x"])
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(outs, everything(i, z, t, step)):
            assert torch.equal(p, q), n
        if last is not None:
            assert not torch.equal(outs[3], last)
        last = outs[3].clone()


def test_refusals():
    i = inputs(41, 2, 10, 8, torch.bfloat16)
    x, f, o = i["x"], i["f"], i["o"]
    with pytest.raises(TypeError):
        lm.recurrence_forward(x.double(), f, o)
    with pytest.raises(TypeError):
        lm.recurrence_forward(x.cpu(), f, o)
    with pytest.raises(TypeError):
        lm.recurrence_forward(x, f.float(), o)
    with pytest.raises(ValueError):
        lm.recurrence_forward(x, f[:, :5], o)
    with pytest.raises(ValueError):
        lm.recurrence_forward(x.transpose(1, 2), f, o)
    with pytest.raises(ValueError):
        lm.recurrence_forward(x, f, x.new_empty(2, 8, 10).transpose(1, 2))
    with pytest.raises(ValueError):
        lm.recurrence_forward(x, f, o, h0=i["h0"][:1])
    with pytest.raises(TypeError):
        lm.recurrence_forward(x, f, o, h0=i["h0"].bfloat16())
    with pytest.raises(TypeError):
        lm.recurrence_forward(x, f, o, lengths=torch.ones(2, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        lm.recurrence_forward(x, f, o, y=x[:, :1].expand(2, 10, 8))
    _, _, saved = lm.recurrence_forward(x, f, o, save=True)
    with pytest.raises(ValueError):
        lm.recurrence_backward(i["gy"], x, f, None, saved, do=torch.empty_like(x))
    with pytest.raises(ValueError):
        lm.recurrence_backward(i["gy"], x, f, o, saved[:, :, :4].contiguous())
    wide = x.new_empty(gs.GS_RECURRENCE_MAX_STRIDE + 16).as_strided((1, 2, 8), (8, gs.GS_RECURRENCE_MAX_STRIDE + 8, 1))
    with pytest.raises(gs.GsError) as e:
        lm.recurrence_forward(wide, wide, None)
    assert e.value.status == gs.GS_ERR_UNSUPPORTED
    for p in (-0.1, 1.1, NAN):
        with pytest.raises(gs.GsError) as e:
            lm.dropout_forward(x, p, 1)
        assert e.value.status == gs.GS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        lm.dropout_forward(x.transpose(1, 2), 0.1, 1)
    with pytest.raises(ValueError):
        lm.dropout_forward(x, 0.1, 1, residual=x[:, :5])
    with pytest.raises(TypeError):
        lm.dropout_forward(x, 0.1, 1, step=torch.zeros(1, device=DEV))
    z, t = logits(1, 4, 9, torch.float32)
    with pytest.raises(TypeError):
        lm.cross_entropy_forward(z, t.int())
    with pytest.raises(ValueError):
        lm.cross_entropy_forward(z, t[:3])
    with pytest.raises(ValueError):
        lm.cross_entropy_forward(z.t(), torch.zeros(9, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError):
        lm.cross_entropy_forward(z, t, grad=z.bfloat16())
    with pytest.raises(gs.GsError):
        lm.cross_entropy_forward(z[:, :0], t)
    with pytest.raises(gs.GsError):  # rows on top of each other
        lm.cross_entropy_forward(z.as_strided((3, 9), (4, 1)), t[:3])


def test_a_written_tensor_counts_as_changed():
    # torch's own rule for its in-place operations: a backward pass that needs what was there before is an error
    i = inputs(51, 2, 12, 8, torch.float32)
    z, t = logits(51, 6, 20, torch.float32)

    def versions(**given):
        return {k: v._version for k, v in given.items()}

    def wrote(call, inputs_, **outs):
        was, kept = versions(**outs), versions(**inputs_)
        call(**outs)
        assert all(outs[k]._version > was[k] for k in outs), call
        assert versions(**inputs_) == kept

    new = lambda: torch.empty_like(i["x"])  # noqa: E731
    fixed = {k: i[k] for k in ("x", "f", "o", "gy", "gh")}
    wrote(lambda **k: lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], **k), fixed, y=new(), h_last=i["h0"].clone())
    wrote(lambda **k: lm.recurrence_forward(i["x"], i["f"], i["o"], h0=k["h_last"], **k), fixed, h_last=i["h0"].clone())
    _, _, saved = lm.recurrence_forward(i["x"], i["f"], i["o"], h0=i["h0"], save=True)
    wrote(lambda **k: lm.recurrence_backward(i["gy"], i["x"], i["f"], i["o"], saved, gh=i["gh"], **k),
          {**fixed, "saved": saved}, dx=new(), df=new(), do=new())
    wrote(lambda **k: lm.dropout_forward(i["x"], 0.5, 1, **k), fixed, y=new())
    wrote(lambda **k: lm.dropout_backward(i["gy"], 0.5, 1, **k), fixed, dx=new())
    wrote(lambda **k: lm.cross_entropy_forward(z, t, **k), dict(z=z, t=t), grad=torch.empty_like(z))
    # tensors that an earlier node saved
    for write in (lambda u: lm.dropout_forward(u, 0.5, 1, y=u),
                  lambda u: lm.recurrence_forward(i["x"], i["f"], i["o"], y=u),
                  lambda u: lm.cross_entropy_forward(u.view(-1, 8), torch.zeros(24, dtype=torch.int64, device=DEV),
                                                     grad=u.view(-1, 8))):
        u = i["x"].clone().requires_grad_() * 2
        y, _ = lm.gated_recurrence(u, i["f"], i["o"], i["h0"])
        write(u.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    with torch.inference_mode():  # tensors without a version
        u = i["x"].clone()
        assert torch.equal(lm.dropout_forward(u, 0.5, 1, y=u), lm.dropout_forward(i["x"], 0.5, 1))


def test_a_gradient_of_any_time_stride_goes_backward():
    # autograd hands over whatever layout the gradient has; here one that the kernels do not take
    wide = gs.GS_RECURRENCE_MAX_STRIDE + 8
    for C in (1, 8):
        i = inputs(52, 2, 2, C, torch.bfloat16)
        gy = torch.empty(3 * wide, dtype=torch.bfloat16, device=DEV).as_strided((2, 2, C), (wide // 2, wide, 1))
        gy.copy_(i["gy"])
        want = ref.recurrence(i["x"], i["f"], i["o"], i["h0"], None, i["gy"], None)
        leaf = i["x"].clone().requires_grad_()
        lm.gated_recurrence(leaf, i["f"], i["o"], i["h0"])[0].backward(gy)
        ref.check(leaf.grad, want["dx"], torch.bfloat16, "dx")
        leaf = torch.cat([i["x"], i["f"], i["o"]], -1).requires_grad_()
        lm.gated_recurrence_packed(leaf, C, i["h0"])[0].backward(gy)
        for n, k in enumerate(("dx", "df", "do")):
            ref.check(leaf.grad[:, :, n * C:(n + 1) * C], want[k], torch.bfloat16, k)


def test_a_packed_recurrence_without_channels():
    for T in (0, 5):
        xfo = torch.empty((3, T, 0), device=DEV, requires_grad=True)
        y, h = lm.gated_recurrence_packed(xfo, 0)
        assert y.shape == (3, T, 0) and h.shape == (3, 0)
        y.sum().backward()
        assert xfo.grad.shape == xfo.shape


def test_cross_entropy_counts_rows_past_the_whole_numbers_of_fp32():
    # 2^25 + 16 rows that count, each of loss log 2: their mean is log 2, each rounding of the loss, the count and the quotient
    # within 2^-24 of it, log 2's own evaluation within 2^-23
    N = (1 << 25) + 1024
    z = torch.zeros((N, 2), dtype=torch.bfloat16, device=DEV)
    t = torch.zeros(N, dtype=torch.int64, device=DEV)
    last = t[N - 1024:]
    last[torch.arange(1024, device=DEV) % 64 != 0] = -100
    mean, losses, _ = lm.cross_entropy_forward(z, t)
    assert (losses[:N - 1024] == losses[0]).all() and abs(float(losses[0]) - 0.6931471805599453) <= 2.0 ** -23
    assert abs(float(mean) / float(losses[0]) - 1) <= 2.0 ** -23


def test_recurrence_gates_over_the_range_of_fp32():
    # from h = 0 and x = 1 one step gives 1 - a, from h = 1 and x = 0 it gives a. The exponential's argument z log2(e) is off
    # by 1.23 u of itself (the constant's rounding and the product's), which is 1.23 |z| u of the result; the exponential, the
    # sum, the reciprocal and a product add at most 8 u. Below 2^-125 a gate may be 0.
    z = torch.linspace(-95, 95, 20_001).view(1, 1, -1).to(DEV)
    one, none = torch.ones_like(z), torch.zeros_like(z)
    f = z.double().cpu()
    for x, h0, want in ((one, none, 1 / (1 + torch.exp(f))), (none, one, 1 / (1 + torch.exp(-f)))):
        y, h, _ = lm.recurrence_forward(x, z, h0=h0[0].contiguous())
        assert torch.equal(y[0], h)
        off = (y.double().cpu() - want).abs() - 2.0 ** -125
        assert (off <= (1.25 * f.abs() + 8) * 2.0 ** -24 * want).all()
