"""The C ABI of the language-model operators on the CPU: what is refused before any device call."""
import ctypes

import pytest

import paper_2108_06004_amd as gs

FAKE = 4096  # never dereferenced: the checks fail first, or there is nothing to compute


@pytest.fixture(scope="module")
def lib():
    return gs.load_library()


def rows(data=FAKE, batch=80, time=8):
    return gs.gs_rows(data, batch, time)


def recurrence(**over):
    kw = dict(B=2, T=10, C=8, dtype=gs.GS_BF16, x=rows(), f=rows(), o=rows(), lengths=None, h0=None)
    kw.update(over)
    return gs.gs_recurrence(*(kw[n] for n, _ in gs.gs_recurrence._fields_))


INVALID, UNSUPPORTED = gs.GS_ERR_INVALID_ARG, gs.GS_ERR_UNSUPPORTED


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(C=-1), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID),
    (dict(x=rows(None)), INVALID), (dict(f=rows(None)), INVALID), (dict(x=rows(FAKE + 1)), INVALID),
    (dict(f=rows(batch=-1)), INVALID), (dict(o=rows(time=-8)), INVALID), (dict(h0=FAKE + 2), INVALID),
    (dict(lengths=FAKE + 2), INVALID), (dict(B=1 << 31), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED),
    (dict(C=1 << 31), UNSUPPORTED), (dict(x=rows(time=gs.GS_RECURRENCE_MAX_STRIDE + 1)), UNSUPPORTED),
])
def test_recurrence_refuses(lib, over, status):
    r = recurrence(**over)
    assert lib.gs_recurrence_forward(ctypes.byref(r), None, rows(), FAKE, None, FAKE) == status
    assert lib.gs_last_error(None).startswith(b"gs_recurrence_forward: ")
    assert lib.gs_recurrence_backward(ctypes.byref(r), None, rows(), None, FAKE, rows(), rows(), rows(), None,
                                      FAKE) == status
    assert lib.gs_last_error(None).startswith(b"gs_recurrence_backward: ")


def test_recurrence_refuses_its_other_arguments(lib):
    r = ctypes.byref(recurrence())
    none = rows(None)
    assert lib.gs_recurrence_forward(None, None, rows(), FAKE, None, FAKE) == INVALID
    assert lib.gs_recurrence_forward(r, None, none, FAKE, None, FAKE) == INVALID
    assert lib.gs_recurrence_forward(r, None, rows(), None, None, FAKE) == INVALID
    assert lib.gs_recurrence_forward(r, None, rows(), FAKE, FAKE + 1, FAKE) == INVALID
    back = lambda gy=rows(), states=FAKE, dx=rows(), df=rows(), do=rows(): lib.gs_recurrence_backward(  # noqa: E731
        r, None, gy, None, states, dx, df, do, None, FAKE)
    assert back(gy=none) == back(dx=none) == back(df=none) == back(do=none) == back(states=None) == INVALID
    ungated = ctypes.byref(recurrence(o=none))
    assert lib.gs_recurrence_backward(ungated, None, rows(), None, FAKE, rows(), rows(), rows(), None, FAKE) == INVALID


def test_work_split_along_time_needs_its_scratch(lib):
    r = recurrence(B=1, T=1 << 20, C=8)
    n = lib.gs_recurrence_work(1, 1 << 20, 8, gs.GS_BF16)
    # one map of two fp32 values a channel for each segment, at most 512 of them
    assert 0 < n <= 512 * 2 * 8 * 4
    assert lib.gs_recurrence_forward(ctypes.byref(r), None, rows(), FAKE, None, None) == INVALID
    assert b"work" in lib.gs_last_error(None)
    assert lib.gs_recurrence_backward(ctypes.byref(r), None, rows(), None, FAKE, rows(), rows(), rows(), None,
                                      None) == INVALID
    for T in (1, 8, gs.GS_RECURRENCE_BLOCK, gs.GS_RECURRENCE_WHOLE):  # never for so few steps
        for C in (1, 2, 63, 64, 5000):
            for dtype in (gs.GS_F32, gs.GS_BF16, gs.GS_F16):
                assert lib.gs_recurrence_work(1, T, C, dtype) == 0
    assert lib.gs_recurrence_work(1, 1, 1 << 25, gs.GS_F32) < 0  # over GS_RECURRENCE_MAX_CHANNELS


def test_nothing_to_compute_is_no_error(lib):
    none = rows(None)
    for size in (dict(B=0), dict(C=0)):
        r = ctypes.byref(recurrence(x=none, f=none, o=none, **size))
        assert lib.gs_recurrence_forward(r, None, none, None, None, None) == gs.GS_OK
        assert lib.gs_recurrence_backward(r, None, none, None, None, none, none, none, None, None) == gs.GS_OK
    assert lib.gs_dropout(None, gs.GS_F32, 0, 8, None, 8, None, 0, None, 8, 0.5, 0, 0, None) == gs.GS_OK
    x = gs.gs_xent(N=0, V=9, dtype=gs.GS_F32)
    assert lib.gs_cross_entropy(ctypes.byref(x), None) == gs.GS_OK
    assert lib.gs_last_error(None) == b""


def test_scratch_sizes(lib):
    assert lib.gs_recurrence_work(-1, 1, 1, 0) < 0 and lib.gs_recurrence_work(1, 1, 1, 9) < 0
    assert lib.gs_recurrence_work(4, 1, 1500, gs.GS_BF16) == 0  # single tokens need none
    assert lib.gs_recurrence_work(0, 0, 0, gs.GS_F32) == 0
    assert lib.gs_cross_entropy_work(1, -1, 0) < 0 and lib.gs_cross_entropy_work(1, 1, 3) < 0


@pytest.mark.parametrize("over,status", [
    (dict(dtype=4), INVALID), (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(x=None), INVALID),
    (dict(y=None), INVALID), (dict(x=FAKE + 1), INVALID), (dict(res=FAKE + 1), INVALID), (dict(xs=7), INVALID),
    (dict(ys=7), INVALID), (dict(res=FAKE, rs=7), INVALID), (dict(p=-0.01), INVALID), (dict(p=1.01), INVALID),
    (dict(p=float("nan")), INVALID), (dict(step=FAKE + 4), INVALID), (dict(rows=1 << 40, cols=1 << 40, xs=1 << 40,
                                                                           ys=1 << 40), UNSUPPORTED),
])
def test_dropout_refuses(lib, over, status):
    kw = dict(dtype=gs.GS_F16, rows=3, cols=8, x=FAKE, xs=8, res=None, rs=0, y=FAKE, ys=8, p=0.5, step=None)
    kw.update(over)
    assert lib.gs_dropout(None, kw["dtype"], kw["rows"], kw["cols"], kw["x"], kw["xs"], kw["res"], kw["rs"], kw["y"],
                          kw["ys"], kw["p"], 1, 2, kw["step"]) == status
    assert lib.gs_last_error(None).startswith(b"gs_dropout: ")


@pytest.mark.parametrize("over,status", [
    (dict(dtype=5), INVALID), (dict(N=-1), INVALID), (dict(V=-1), INVALID), (dict(V=0), INVALID), (dict(logits=None), INVALID),
    (dict(logits=FAKE + 1), INVALID), (dict(targets=None), INVALID), (dict(targets=FAKE + 4), INVALID),
    (dict(losses=None), INVALID), (dict(losses=FAKE + 2), INVALID), (dict(mean_loss=FAKE + 2), INVALID),
    (dict(logits_stride=8), INVALID), (dict(grad_stride=8), INVALID), (dict(grad=FAKE + 1), INVALID),
    (dict(scale_stride=2), INVALID), (dict(scale=FAKE + 1), INVALID), (dict(N=300, work=None), INVALID),
    (dict(work=FAKE + 4), INVALID), (dict(N=1 << 31), UNSUPPORTED), (dict(V=1 << 31), UNSUPPORTED),
])
def test_cross_entropy_refuses(lib, over, status):
    kw = dict(N=4, V=9, dtype=gs.GS_BF16, mean=1, logits=FAKE, logits_stride=9, targets=FAKE, ignore_index=-100, factor=1.0,
              scale=None, scale_stride=0, losses=FAKE, mean_loss=FAKE, grad=FAKE, grad_stride=9, work=FAKE)
    kw.update(over)
    x = gs.gs_xent(**kw)
    assert lib.gs_cross_entropy(ctypes.byref(x), None) == status
    assert lib.gs_last_error(None).startswith(b"gs_cross_entropy: ")
    assert lib.gs_cross_entropy(None, None) == INVALID


def test_constants_match_the_header():
    import os
    import re

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "gs.h")).read()
    for name in ("GS_F32", "GS_BF16", "GS_F16", "GS_RECURRENCE_BLOCK", "GS_RECURRENCE_WHOLE", "GS_RECURRENCE_MAX_STRIDE",
                 "GS_RECURRENCE_MAX_CHANNELS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(gs, name)


def test_operators_refuse_tensors_off_the_gpu():
    torch = pytest.importorskip("torch")
    from paper_2108_06004_amd import lm

    x = torch.zeros(2, 3, 4)
    with pytest.raises(TypeError):
        lm.recurrence_forward(x, x)
    with pytest.raises(TypeError):
        lm.dropout_forward(x, 0.1, 1)
    with pytest.raises(TypeError):
        lm.cross_entropy_forward(x[0], torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        lm.gated_recurrence_packed(x, 3)
    with pytest.raises(ValueError):
        lm.cross_entropy(x[0], torch.zeros(3, dtype=torch.int64), reduction="sum")
    with pytest.raises(TypeError):
        lm.RecurrentLM(10, 4, dtype=torch.float64)


def test_a_failed_generation_leaves_the_training_mode():
    torch = pytest.importorskip("torch")
    from paper_2108_06004_amd import lm

    model = lm.RecurrentLM(10, 4)
    with pytest.raises(TypeError):  # not on the GPU
        model.generate(torch.zeros((1, 2), dtype=torch.int64), 1)
    assert model.training
