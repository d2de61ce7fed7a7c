"""The language model made of the operators, trained through the compression step (needs an MI355X)."""
import os
import sys

import numpy as np
import pytest

import lm_reference as ref
import oracle
import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
gs = pytest.importorskip("paper_2108_06004_amd")
from paper_2108_06004_amd import lm  # noqa: E402
from paper_2108_06004_amd.train import DensitySchedule, GlobalSketchOptimizer  # noqa: E402

DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def reference_gradients(model, tokens, targets, worker, step):
    """Loss and parameter gradients of the same network in 64 bits on the CPU, by autograd over elementary
    operations, with the same dropout masks."""
    params = {n: p.detach().cpu().double().requires_grad_() for n, p in model.named_parameters()}
    C = model.width
    u = params["embedding.weight"][tokens.cpu()]
    below = int(np.floor(model.p * 65536 + 0.5))
    for j in range(len(model.inner)):
        x, f, o = (u @ params[f"inner.{j}.weight"].t() + params[f"inner.{j}.bias"]).split(C, -1)
        a = torch.sigmoid(f)
        h = torch.zeros(u.shape[0], C, dtype=torch.float64)
        ys = []
        for t in range(u.shape[1]):
            h = a[:, t] * h + (1 - a[:, t]) * x[:, t]
            ys.append(torch.sigmoid(o[:, t]) * h)
        keep = torch.from_numpy(ref.draws(u.numel(), model.seed, worker * len(model.inner) + j, step) >= below)
        u = u + torch.stack(ys, 1) * keep.view(u.shape) * (65536 / (65536 - below))
    z = (u @ params["outer.weight"].t() + params["outer.bias"]).flatten(0, 1)
    loss = torch.nn.functional.cross_entropy(z, targets.cpu().flatten())
    loss.backward()
    return loss.detach(), {n: p.grad for n, p in params.items()}


def test_gradients_of_the_model_and_one_compression_step():
    # every parameter gradient against 64 bits: fp32 products over sums of at most 200 terms through two layers,
    # each rounding 2^-24 of its terms; 1e-4 of the gradient's norm is far above that and far below any error
    # of a formula, a mask or an order of states. Then the optimizer's step from these gradients against the oracle.
    torch.manual_seed(7)
    P, r, c = 2, 5, 1024
    model = lm.RecurrentLM(50, 40, layers=2, p=0.25, seed=9).to(DEV)
    hp = synth.hash_params(synth.BASE_SEED + 171, r)
    opt = GlobalSketchOptimizer(model.parameters(), P, r, c, hp, DensitySchedule(0.02, 0.5), rho=0.9)
    gen = torch.Generator(device=DEV).manual_seed(8)
    model.step.fill_(5)
    for worker in range(P):
        tokens = torch.randint(50, (3, 21), generator=gen, device=DEV)
        model.worker = worker
        mean = model.loss_backward(tokens[:, :-1], tokens[:, 1:])
        loss, want = reference_gradients(model, tokens[:, :-1], tokens[:, 1:], worker, 5)
        assert abs(float(mean) - float(loss)) <= 1e-5 * float(loss)
        for n, p in model.named_parameters():
            off = (p.grad.cpu().double() - want[n]).norm() / want[n].norm()
            assert off <= 1e-4, (n, float(off))
        opt.collect(worker)
    g, w = opt.grads.cpu().numpy().copy(), opt.flat.cpu().numpy().copy()
    assert np.abs(g[0] - g[1]).max() > 0
    opt.step()
    k = opt.last_k
    idx, vals = opt.idx[:k].cpu().numpy(), opt.values[:k].cpu().numpy()
    uo, vo = np.zeros_like(g), np.zeros_like(g)
    step = oracle.step(g, uo, vo, hp, c, k, rho=0.9)
    common, gi, oi = np.intersect1d(idx, step["idx"], return_indices=True)
    assert len(common) >= 0.99 * k and np.array_equal(vals[gi], step["values"][oi])
    oracle.apply_update(w, idx, vals, 0.5 / P)
    assert np.array_equal(opt.flat.cpu().numpy(), w)
    opt.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_tokens_one_at_a_time_give_what_the_sequence_gives(dtype):
    torch.manual_seed(3)
    model = lm.RecurrentLM(60, 64, layers=3, dtype=dtype).to(DEV).eval()
    gen = torch.Generator(device=DEV).manual_seed(4)
    tokens = torch.randint(60, (5, 30), generator=gen, device=DEV)
    with torch.no_grad():
        whole, after = model(tokens)
        state, parts = None, []
        for t in range(30):
            z, state = model(tokens[:, t:t + 1], state)
            parts.append(z)
    # the same formulas in another order of sums: fp32 roundings, or bf16 ones of every layer's activations
    tol = 1e-4 if dtype == torch.float32 else 0.05
    scale = whole.float().abs().max()
    assert (torch.cat(parts, 1).float() - whole.float()).abs().max() <= tol * scale
    for p, q in zip(after, state):
        assert (p - q).abs().max() <= tol * p.abs().max()
    said = model.generate(tokens, 4)
    assert said.shape == (5, 4) and torch.equal(said[:, 0], whole[:, -1].argmax(-1)) and not model.training


def test_padding_of_a_batch_of_prompts():
    torch.manual_seed(5)
    model = lm.RecurrentLM(30, 32, layers=2).to(DEV).eval()
    gen = torch.Generator(device=DEV).manual_seed(6)
    tokens = torch.randint(30, (3, 12), generator=gen, device=DEV)
    lengths = torch.tensor([12, 5, 0], dtype=torch.int32, device=DEV)
    with torch.no_grad():
        z, state = model(tokens, lengths=lengths)
        alone, own = model(tokens[1:2, :5])
    assert torch.allclose(z[1, :5], alone[0], rtol=1e-4, atol=1e-5)
    for s, t in zip(state, own):
        assert torch.allclose(s[1], t[0], rtol=1e-4, atol=1e-5) and not s[2].any()


def test_the_example_learns_its_text():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import recurrent_lm
    finally:
        sys.path.pop(0)
    # a token's successor follows nine times in ten: log(vocab) = 4.6 before, towards 0.8 after
    got = recurrent_lm.main(["--steps", "80", "--vocab", "100", "--width", "64"])
    assert got["first"] > 4.0 and got["last"] < 0.6 * got["first"] and got["right"] > 0.5


def test_gradients_of_a_half_precision_model_of_many_words_and_tokens():
    # A uniform softmax over 20,000 words, in the mean over 2,048 tokens, is 2.4e-8 an entry of the logits' gradient: less
    # than half of fp16's smallest number. Every parameter gradient against 64 bits, after one pass and after two that add
    # up. Some sixteen roundings to 11 bits lie between the embedding and a gradient, each 2^-11 of its value at most:
    # 0.8% of the norm, with logits' errors of up to |z| <= 3 times that in the softmax's share: 2%.
    torch.manual_seed(11)
    V, B, T = 20_000, 16, 128
    model = lm.RecurrentLM(V, 16, layers=1, p=0.1, seed=4, dtype=torch.float16).to(DEV)
    gen = torch.Generator(device=DEV).manual_seed(12)
    tokens = torch.randint(V, (B, T + 1), generator=gen, device=DEV)
    loss, want = reference_gradients(model, tokens[:, :-1], tokens[:, 1:], 0, 0)
    for passes in (1, 2):
        mean = model.loss_backward(tokens[:, :-1], tokens[:, 1:])
        assert abs(float(mean) - float(loss)) <= 2.0 ** -9 * float(loss)
        for n, p in model.named_parameters():
            off = (p.grad.cpu().double() / passes - want[n]).norm() / want[n].norm()
            assert off <= 0.02, (passes, n, float(off))
    never = torch.ones(V, dtype=torch.bool, device=DEV)
    never[tokens[:, 1:].flatten()] = False
    assert (model.outer.bias.grad[never] > 0).all()


def test_a_half_precision_model_when_most_targets_are_ignored():
    # one target of 4,096 counts: the factor that holds the gradients up must not carry them over fp16's largest number
    torch.manual_seed(13)
    model = lm.RecurrentLM(500, 32, layers=2, p=0.0, dtype=torch.float16).to(DEV)
    gen = torch.Generator(device=DEV).manual_seed(14)
    tokens = torch.randint(500, (32, 129), generator=gen, device=DEV)
    targets = torch.full((32, 128), -100, dtype=torch.int64, device=DEV)
    targets[3, 100] = tokens[3, 101]
    model.loss_backward(tokens[:, :-1], targets)
    plain = lm.RecurrentLM(500, 32, layers=2, p=0.0).to(DEV)
    plain.load_state_dict(model.state_dict())
    plain.loss_backward(tokens[:, :-1], targets)
    for (n, p), q in zip(model.named_parameters(), plain.parameters()):
        assert torch.isfinite(p.grad).all(), n
        assert (p.grad - q.grad).norm() <= 0.04 * q.grad.norm(), n  # two layers: twice the roundings of the test above


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16], ids=["f32", "f16"])
def test_a_factor_of_the_logits_gradient_changes_no_other_gradient(dtype):
    # gradients of the logits 64 times as large, the states' as they are: the same gradients of parameters and states. The
    # factor is a power of two, so fp32 differs by orders of sums alone (200 terms of 2^-24), fp16 by its subnormals
    torch.manual_seed(15)
    model = lm.RecurrentLM(40, 32, layers=2, dtype=dtype).to(DEV).eval()
    gen = torch.Generator(device=DEV).manual_seed(16)
    tokens = torch.randint(40, (4, 9), generator=gen, device=DEV)
    g = torch.randn((4, 9, 40), generator=gen, device=DEV).to(dtype)
    gh = [torch.randn((4, 32), generator=gen, device=DEV) for _ in range(2)]
    got = []
    for factor in (1.0, 64.0):
        state = [torch.ones((4, 32), device=DEV, requires_grad=True) for _ in range(2)]
        logits, after = model(tokens, state, factor=factor)
        model.zero_grad()
        torch.autograd.backward([logits, *after], [g * factor, *gh])
        got.append([p.grad for p in model.parameters()] + [s.grad for s in state])
    for p, q in zip(*got):
        assert (p - q).norm() <= (1e-5 if dtype == torch.float32 else 2.0 ** -8) * p.norm()
