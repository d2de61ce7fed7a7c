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
