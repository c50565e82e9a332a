"""A small decoder-only language model on this library's entry points: trained on a toy language, then asked to go on by beam search.

    python examples/decoder_layer.py [--steps 60] [--layers 2] [--heads 4] [--head-dim 64]

A layer is  x + Wo Norm(LA2(q, k, v)),  q, k, v = silu(Wqkv LN(x)) ,  then  x + Wd gelu(Wu LN(x)).  Every product, normalisation and the
recurrence run in the library, forward and backward; torch supplies memory, the embedding, the loss and the optimiser.  Generating,
a prompt is run once (its recurrence hands out every layer's state), then token by token: the layers on rows of beams, selection over beams
and vocabulary, and the layers' states moved to where the selection wants them.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2401_04658_amd as la2  # noqa: E402
from paper_2401_04658_amd.workloads import head_decay  # noqa: E402


class Model:
    """Weights (a dict of tensors) and the passes over them.  Matrices are of `dtype`, normalisation weights and biases fp32."""

    def __init__(self, vocab, layers, heads, head_dim, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.vocab, self.layers, self.heads, self.head_dim, self.width = vocab, layers, heads, head_dim, heads * head_dim
        self.lam = head_decay(heads).to(device)
        w, wide = self.width, 4 * self.width
        draw = lambda rows, cols: (torch.randn(rows, cols, generator=g) / math.sqrt(cols)).to(dtype).to(device)
        self.p = {"embed": (torch.randn(vocab, w, generator=g) * 0.5).to(dtype).to(device), "head": draw(vocab, w),
                  "ln_w": torch.ones(w, device=device), "ln_b": torch.zeros(w, device=device)}
        for i in range(layers):
            self.p.update({"%d.ln1_w" % i: torch.ones(w, device=device), "%d.ln1_b" % i: torch.zeros(w, device=device),
                           "%d.qkv" % i: draw(3 * w, w), "%d.out" % i: draw(w, w),
                           "%d.ln2_w" % i: torch.ones(w, device=device), "%d.ln2_b" % i: torch.zeros(w, device=device),
                           "%d.up" % i: draw(wide, w), "%d.up_b" % i: torch.zeros(wide, device=device),
                           "%d.down" % i: draw(w, wide), "%d.down_b" % i: torch.zeros(w, device=device)})

    def _split(self, qkv, batch, n):
        """q, k, v as [batch, heads, n, head_dim] views of the rows [batch * n, 3 width]."""
        return tuple(qkv.view(batch, n, 3, self.heads, self.head_dim)[:, :, i].transpose(1, 2) for i in range(3))

    def forward(self, tokens):
        """Logits [batch * n, vocab], and what backward() needs."""
        p, (batch, n) = self.p, tokens.shape
        x = p["embed"][tokens.reshape(-1)]
        kept = []
        for i in range(self.layers):
            a, mean1, rstd1 = la2.la2_layer_norm_fwd(x, p["%d.ln1_w" % i], p["%d.ln1_b" % i])
            qkv, pre = la2.la2_linear_fwd(a, p["%d.qkv" % i], act="silu", want_pre=True)
            o, r = la2.la2_fwd_norm(*self._split(qkv, batch, n), self.lam)
            rows = o.transpose(1, 2).reshape(batch * n, self.width)
            h, _ = la2.la2_linear_fwd(rows, p["%d.out" % i], residual=x)
            b, mean2, rstd2 = la2.la2_layer_norm_fwd(h, p["%d.ln2_w" % i], p["%d.ln2_b" % i])
            u, pre_u = la2.la2_linear_fwd(b, p["%d.up" % i], p["%d.up_b" % i], act="gelu", want_pre=True)
            y, _ = la2.la2_linear_fwd(u, p["%d.down" % i], p["%d.down_b" % i], residual=h)
            kept.append((x, a, mean1, rstd1, qkv, pre, o, r, rows, h, b, mean2, rstd2, u, pre_u))
            x = y
        f, mean, rstd = la2.la2_layer_norm_fwd(x, p["ln_w"], p["ln_b"])
        logits, _ = la2.la2_linear_fwd(f, p["head"])
        return logits, (tokens, kept, x, f, mean, rstd)

    def backward(self, d_logits, saved):
        """Gradients of all weights, under their names."""
        tokens, kept, x, f, mean, rstd = saved
        p, grads, (batch, n) = self.p, {}, tokens.shape
        df, grads["head"], _ = la2.la2_linear_bwd(d_logits, f, p["head"], want_d_bias=False)
        dx, grads["ln_w"], grads["ln_b"] = la2.la2_layer_norm_bwd(df, x, mean, rstd, p["ln_w"])
        for i in reversed(range(self.layers)):
            x, a, mean1, rstd1, qkv, pre, o, r, rows, h, b, mean2, rstd2, u, pre_u = kept[i]
            du, grads["%d.down" % i], grads["%d.down_b" % i] = la2.la2_linear_bwd(dx, u, p["%d.down" % i])
            db, grads["%d.up" % i], grads["%d.up_b" % i] = la2.la2_linear_bwd(du, b, p["%d.up" % i], pre=pre_u, act="gelu")
            dh, grads["%d.ln2_w" % i], grads["%d.ln2_b" % i] = la2.la2_layer_norm_bwd(db, h, mean2, rstd2, p["%d.ln2_w" % i])
            dh += dx
            do, grads["%d.out" % i], _ = la2.la2_linear_bwd(dh, rows, p["%d.out" % i], want_d_bias=False)
            d_qkv = torch.empty_like(qkv)
            # o and its gradient lie as q does, three widths a row
            wide = torch.empty_like(qkv)
            o_like, do_like, _ = self._split(wide, batch, n)
            o_like.copy_(o)
            do_like.copy_(do.view(batch, n, self.heads, self.head_dim).transpose(1, 2))
            la2.la2_bwd_norm(*self._split(qkv, batch, n), o_like, r, do_like, self.lam, out=self._split(d_qkv, batch, n))
            da, grads["%d.qkv" % i], _ = la2.la2_linear_bwd(d_qkv, a, p["%d.qkv" % i], pre=pre, act="silu", want_d_bias=False)
            dx, grads["%d.ln1_w" % i], grads["%d.ln1_b" % i] = la2.la2_layer_norm_bwd(da, x, mean1, rstd1, p["%d.ln1_w" % i])
            dx += dh
        grads["embed"] = torch.zeros_like(p["embed"], dtype=torch.float32).index_add_(0, tokens.reshape(-1), dx.float()).to(dx.dtype)
        return grads

    def prefill(self, tokens):
        """Logits [batch, vocab] behind a prompt, and every layer's state."""
        p, (batch, n) = self.p, tokens.shape
        x, states = p["embed"][tokens.reshape(-1)], []
        for i in range(self.layers):
            a, _, _ = la2.la2_layer_norm_fwd(x, p["%d.ln1_w" % i], p["%d.ln1_b" % i])
            qkv, _ = la2.la2_linear_fwd(a, p["%d.qkv" % i], act="silu")
            o, _, kv = la2.la2_fwd_state_norm(*self._split(qkv, batch, n), self.lam)
            states.append(kv)
            x = self._rest(i, x, o.transpose(1, 2).reshape(batch * n, self.width))
        return self._logits(x.view(batch, n, self.width)[:, -1]), states

    def step(self, tokens, states):
        """Logits [rows, vocab] behind one more token a row; the states move on in place."""
        p, w = self.p, self.width
        x = p["embed"][tokens]
        for i in range(self.layers):
            a, _, _ = la2.la2_layer_norm_fwd(x, p["%d.ln1_w" % i], p["%d.ln1_b" % i])
            q, k, v = (la2.la2_linear_fwd(a, p["%d.qkv" % i][j * w:(j + 1) * w], act="silu")[0].view(-1, self.heads, self.head_dim)
                       for j in range(3))
            x = self._rest(i, x, la2.la2_decode_step_norm(q, k, v, self.lam, states[i]).view(-1, w))
        return self._logits(x)

    def _rest(self, i, x, rows):
        p = self.p
        h, _ = la2.la2_linear_fwd(rows, p["%d.out" % i], residual=x)
        b, _, _ = la2.la2_layer_norm_fwd(h, p["%d.ln2_w" % i], p["%d.ln2_b" % i])
        u, _ = la2.la2_linear_fwd(b, p["%d.up" % i], p["%d.up_b" % i], act="gelu")
        return la2.la2_linear_fwd(u, p["%d.down" % i], p["%d.down_b" % i], residual=h)[0]

    def _logits(self, x):
        f, _, _ = la2.la2_layer_norm_fwd(x.contiguous(), self.p["ln_w"], self.p["ln_b"])
        return la2.la2_linear_fwd(f, self.p["head"])[0]


def loss_and_gradient(logits, targets):
    """Mean cross entropy and its gradient with respect to the logits, in their type."""
    lp = torch.log_softmax(logits.float(), 1)
    at = targets.reshape(-1, 1)
    d = lp.exp()
    d.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    return -lp.gather(1, at).mean(), (d / at.numel()).to(logits.dtype)


class Adam:
    """The usual one, on fp32 copies of the weights."""

    def __init__(self, params, rate):
        self.params, self.rate, self.t = params, rate, 0
        self.master = {k: v.float() for k, v in params.items()}
        self.m = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.s = {k: torch.zeros_like(v) for k, v in self.master.items()}

    def step(self, grads):
        self.t += 1
        for k, g in grads.items():
            g = g.float()
            self.m[k].lerp_(g, 0.1)
            self.s[k].lerp_(g * g, 0.02)
            self.master[k] -= self.rate * (self.m[k] / (1 - 0.9 ** self.t)) / ((self.s[k] / (1 - 0.98 ** self.t)).sqrt() + 1e-8)
            self.params[k].copy_(self.master[k])


def sentences(batch, n, vocab, g):
    """A toy language: a sentence counts on from a token by a stride of its own, which its first two tokens tell."""
    start = torch.randint(0, vocab, (batch, 1), generator=g)
    stride = torch.randint(1, 4, (batch, 1), generator=g)
    return (start + stride * torch.arange(n)) % vocab


def beam_search(model, prompt, beams, steps, eos=-1):
    """(tokens [batch, beams, steps], scores [batch, beams]), the best first."""
    batch = prompt.shape[0]
    logits, states = model.prefill(prompt)
    states = [s.repeat_interleave(beams, 0) for s in states]
    logits = logits.repeat_interleave(beams, 0)
    scores = torch.full((batch, beams), -math.inf, device=prompt.device)
    scores[:, 0] = 0.0   # all beams are one at first
    finished = torch.zeros((batch, beams), dtype=torch.bool, device=prompt.device) if eos >= 0 else None
    said = torch.empty((batch, beams, 0), dtype=torch.int32, device=prompt.device)
    for i in range(steps):
        scores, parent, token, done = la2.la2_beam_select(logits.view(batch, beams, -1), scores, finished, eos=eos)
        finished = done if eos >= 0 else None
        said = torch.cat([said.gather(1, parent.long()[:, :, None].expand_as(said)), token[:, :, None]], 2)
        if i + 1 < steps:
            la2.la2_beam_reorder(states, parent)
            logits = model.step(token.reshape(-1).long(), states)
    return said, scores


def train(model, steps, batch, n, rate=3e-3, seed=1, say=None):
    g = torch.Generator().manual_seed(seed)
    optimiser, losses = Adam(model.p, rate), []
    for i in range(steps):
        tokens = sentences(batch, n + 1, model.vocab, g).cuda()
        logits, saved = model.forward(tokens[:, :-1].contiguous())
        loss, d = loss_and_gradient(logits, tokens[:, 1:].reshape(-1))
        optimiser.step(model.backward(d, saved))
        losses.append(loss)
        if say is not None and (i % 10 == 9 or i == 0):
            say("step %d: loss %.3f" % (i + 1, float(loss)))
    return [float(x) for x in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--head-dim", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=97)
    a = ap.parse_args()
    model = Model(a.vocab, a.layers, a.heads, a.head_dim)
    train(model, a.steps, 32, 64, say=lambda s: print(s, flush=True))
    prompt = sentences(4, 8, a.vocab, torch.Generator().manual_seed(2))
    said, scores = beam_search(model, prompt.cuda(), 4, 6)
    for b in range(4):
        print(prompt[b].tolist(), "->", said[b, 0].tolist(), "(%.2f)" % float(scores[b, 0]), flush=True)


if __name__ == "__main__":
    main()
