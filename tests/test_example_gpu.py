"""The example's model: its gradients against a 64-bit model of the same layers, what it learns, and beam search against one that keeps
every beam's tokens and runs them anew."""
import math
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import decoder_layer as ex  # noqa: E402

pytestmark = pytest.mark.gpu


def reference_logits(m, p, tokens):
    """The model's forward pass in 64 bits on the CPU (differentiable)."""
    batch, n = tokens.shape
    lam = m.lam.double().cpu()
    t = torch.arange(n)
    decay = torch.where(t[:, None] >= t[None, :], lam[:, None, None] ** (t[:, None] - t[None, :]).clamp(min=0), torch.zeros(1, dtype=torch.float64))
    norm = lambda x, w, b: torch.nn.functional.layer_norm(x, (m.width,), w, b, 1e-5)
    x = p["embed"][tokens.reshape(-1)]
    for i in range(m.layers):
        q = torch.nn.functional.silu(norm(x, p["%d.ln1_w" % i], p["%d.ln1_b" % i]) @ p["%d.qkv" % i].T)
        q, k, v = (q.view(batch, n, 3, m.heads, m.head_dim)[:, :, j].transpose(1, 2) for j in range(3))
        o = ((q @ k.transpose(2, 3)) * decay) @ v
        o = o / (o.square().mean(-1, keepdim=True) + 1e-6).sqrt()
        h = x + o.transpose(1, 2).reshape(batch * n, m.width) @ p["%d.out" % i].T
        u = torch.nn.functional.gelu(norm(h, p["%d.ln2_w" % i], p["%d.ln2_b" % i]) @ p["%d.up" % i].T + p["%d.up_b" % i])
        x = h + u @ p["%d.down" % i].T + p["%d.down_b" % i]
    return norm(x, p["ln_w"], p["ln_b"]) @ p["head"].T


def test_gradients_of_the_whole_model():
    m = ex.Model(vocab=50, layers=2, heads=2, head_dim=64, dtype=torch.float32, seed=3)
    tokens = ex.sentences(3, 34, 50, torch.Generator().manual_seed(4))
    logits, saved = m.forward(tokens[:, :-1].contiguous().cuda())
    loss, d = ex.loss_and_gradient(logits, tokens[:, 1:].reshape(-1).cuda())
    grads = m.backward(d, saved)
    p = {k: v.double().cpu().requires_grad_() for k, v in m.p.items()}
    ref = reference_logits(m, p, tokens[:, :-1])
    want = torch.nn.functional.cross_entropy(ref, tokens[:, 1:].reshape(-1))
    want.backward()
    want = want.detach()
    assert set(grads) == set(p)
    # fp32 throughout: sums of some hundred terms and a dozen operators behind one another, 1e-4 of a gradient's largest entry
    assert abs(float(loss) - float(want)) < 1e-5 * float(want)
    for k, v in grads.items():
        top = float(p[k].grad.abs().max())
        assert float((v.double().cpu() - p[k].grad).abs().max()) <= 1e-4 * top, k


@pytest.fixture(scope="module")
def trained():
    m = ex.Model(vocab=31, layers=2, heads=4, head_dim=64, seed=5)
    losses = ex.train(m, 60, 32, 48)
    return m, losses


def test_it_learns(trained):
    _, losses = trained
    assert losses[0] > 0.8 * math.log(31) and max(losses[-5:]) < 0.25 * losses[0], losses


def test_beam_search(trained):
    m, _ = trained
    prompt = ex.sentences(5, 12, 31, torch.Generator().manual_seed(6))
    said, scores = ex.beam_search(m, prompt.cuda(), beams=4, steps=5)
    assert torch.equal(scores, scores.sort(1, descending=True).values)
    going_on = (prompt[:, -1:] + (prompt[:, 1:2] - prompt[:, :1]) % 31 * torch.arange(1, 6)) % 31
    assert torch.equal(said[:, 0].cpu().long(), going_on)
    # the scores are those of the tokens, run anew from the prompt (bf16 layers: decode steps and whole passes round differently, by up to
    # some 2^-7 of logits of size 10, five times)
    full = torch.cat([prompt.cuda().repeat_interleave(4, 0), said.reshape(20, 5).long()], 1)
    logits, _ = m.forward(full[:, :-1].contiguous())
    lp = torch.log_softmax(logits.float().view(20, 16, 31), 2)[:, 11:].gather(2, full[:, 12:, None]).sum((1, 2))
    assert float((lp.view(5, 4) - scores).abs().max()) < 0.4
    one, s1 = ex.beam_search(m, prompt.cuda(), beams=1, steps=5)
    assert torch.equal(one[:, 0].cpu().long(), going_on)
    stop, _ = ex.beam_search(m, prompt[:1].cuda(), beams=3, steps=5, eos=int(going_on[0, 1]))
    assert stop[0, 0].tolist() == going_on[0, :2].tolist() + [int(going_on[0, 1])] * 3
