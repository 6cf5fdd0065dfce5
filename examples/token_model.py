"""Two modules of a token model trained with delayed gradients (Algorithm 1, K = 2) on the operators of token models.

  module 1 (delay 1): h = norm(dropout(E[token]))             ddg_join_norm without a residual
  module 2 (delay 0): x = h + dropout(h A^T), n = norm(x)     ddg_join_norm
                      f = cross entropy of n w^T              ddg_vocab_loss, with dn and dw, no logits

In iteration t module 1 back-propagates the error gradient of iteration t - 1: it takes the tokens of t - 1 again with its current
table and, since a dropout mask is a function of (seed, step), passes the step of t - 1 and gets the mask of t - 1, which nobody stored.
The data are a Markov chain over the vocabulary, so the loss can fall to the chain's entropy. At the end a pass without
dropout measures the loss, once from n in bf16 and once from n in 8 bits with a scale per 128 columns (ddg_join_norm_q8).

Run: python examples/token_model.py [iterations]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1804_10574_amd as ddg  # noqa: E402

VOCAB, DIM, TOKENS, DROP, LR, MOMENTUM, FOLLOWERS = 512, 128, 1024, 0.1, 0.5, 0.9, 4


class Param:
    """fp32 master weights with momentum, and their bf16 copy where a product takes one."""

    def __init__(self, value):
        self.w, self.v = value, torch.zeros_like(value)
        self.half = value.bfloat16()

    def update(self, grad, lr):
        self.v.mul_(MOMENTUM).add_(grad.float())
        self.w.sub_(lr * self.v)
        self.half.copy_(self.w)


class Module1:
    def __init__(self, gen):
        self.table = Param(torch.randn(VOCAB, DIM, device="cuda", generator=gen))
        self.gain = Param(torch.ones(DIM, device="cuda"))
        self.join = {p: ddg.JoinNorm(TOKENS, DIM, ddg.DDG_BF16, p=p, seed=11, stream=torch.cuda.current_stream().cuda_stream) for p in (DROP, 0.0)}
        self.space = torch.empty(self.join[DROP].workspace_bytes(), device="cuda", dtype=torch.uint8)
        self.x, self.rstd = torch.empty(TOKENS, DIM, device="cuda", dtype=torch.bfloat16), torch.empty(TOKENS, device="cuda")

    def forward(self, tokens, step, p=DROP):
        h = torch.empty_like(self.x)
        self.join[p].forward(self.table.half[tokens], None, self.gain.w, h, x_out=self.x, rstd=self.rstd, step=step)
        return h

    def backward_delayed(self, tokens, step, delta, lr):
        self.forward(tokens, step)                              # the stored input again, with the current weights and the mask of its iteration
        d_y, d_gain = torch.empty_like(self.x), torch.empty(DIM, device="cuda")
        self.join[DROP].backward(self.x, self.rstd, self.gain.w, delta, d_y=d_y, d_gain=d_gain, workspace=self.space, step=step)
        self.table.update(torch.zeros_like(self.table.w).index_add_(0, tokens, d_y.float()), lr)
        self.gain.update(d_gain, lr)


class Module2:
    def __init__(self, gen):
        self.a = Param(torch.randn(DIM, DIM, device="cuda", generator=gen) * DIM ** -0.5)
        self.w = Param(torch.randn(VOCAB, DIM, device="cuda", generator=gen) * 0.02)
        self.gain = Param(torch.ones(DIM, device="cuda"))
        stream = torch.cuda.current_stream().cuda_stream
        self.join = {p: ddg.JoinNorm(TOKENS, DIM, ddg.DDG_BF16, p=p, seed=12, group=128, stream=stream) for p in (DROP, 0.0)}
        self.head = ddg.VocabLoss(TOKENS, DIM, VOCAB, ddg.DDG_BF16, dw_f32=True, stream=stream)
        self.space = torch.empty(max(self.join[DROP].workspace_bytes(), self.head.workspace_bytes()), device="cuda", dtype=torch.uint8)

    def step(self, h, targets, step, lr):
        """Forward, backward and update of one minibatch; returns the loss and the error gradient for module 1."""
        like = torch.empty_like
        y, x, n, rstd = h @ self.a.half.T, like(h), like(h), torch.empty(TOKENS, device="cuda")
        self.join[DROP].forward(y, h, self.gain.w, n, x_out=x, rstd=rstd, step=step)
        loss, dn, dw = torch.empty(1, device="cuda"), like(h), like(self.w.w)
        self.head(n, self.w.half, targets, loss=loss, dh=dn, dw=dw, workspace=self.space)
        d_h, d_y, d_gain = like(h), like(h), torch.empty(DIM, device="cuda")
        self.join[DROP].backward(x, rstd, self.gain.w, dn, d_residual=d_h, d_y=d_y, d_gain=d_gain, workspace=self.space, step=step)
        delta = d_h + d_y @ self.a.half
        self.a.update(d_y.T.float() @ h.float(), lr)
        self.w.update(dw, lr)
        self.gain.update(d_gain, lr)
        return loss, delta

    def evaluate(self, h, targets):
        """Loss without dropout from n in bf16 and from n in 8 bits."""
        y, n = h @ self.a.half.T, torch.empty_like(h)
        q, scale = torch.empty(TOKENS, DIM, device="cuda", dtype=torch.uint8), torch.empty(TOKENS, DIM // 128, device="cuda")
        self.join[0.0].forward(y, h, self.gain.w, n)
        self.join[0.0].forward_q8(y, h, self.gain.w, q, scale)
        eight = (q.view(torch.float8_e4m3fn).float().view(TOKENS, -1, 128) * scale[:, :, None]).view(TOKENS, DIM).bfloat16()
        out = []
        for v in (n, eight):
            loss = torch.empty(1, device="cuda")
            self.head(v, self.w.half, targets, loss=loss, workspace=self.space)
            out.append(float(loss))
        return out


def train(iterations, say=None):
    """Returns the losses of the iterations, the chain's entropy, and the evaluation losses (bf16, 8 bits)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(5)
    follow = torch.randint(0, VOCAB, (VOCAB, FOLLOWERS), device="cuda", generator=gen)

    def minibatch():
        tokens = torch.randint(0, VOCAB, (TOKENS,), device="cuda", generator=gen)
        targets = follow[tokens, torch.randint(0, FOLLOWERS, (TOKENS,), device="cuda", generator=gen)]
        targets[torch.rand(TOKENS, device="cuda", generator=gen) < 0.1] = -1       # a tenth of the places has no target
        return tokens, targets.to(torch.int32)

    one, two = Module1(gen), Module2(gen)
    losses, stored = [], None                                   # stored: tokens and error gradient of the last iteration
    for t in range(iterations):
        tokens, targets = minibatch()
        h = one.forward(tokens, t)
        loss, delta = two.step(h, targets, t, LR)
        if stored is not None:                                  # t - 1 >= 0 (Eq. 8: no gradient before)
            one.backward_delayed(stored[0], t - 1, stored[1], LR)
        stored = (tokens, delta)
        losses.append(loss)
        if say and t % 50 == 0:
            say(f"iteration {t}: loss {float(loss):.3f}")
    tokens, targets = minibatch()
    counts = torch.zeros(VOCAB, VOCAB, device="cuda").scatter_add_(1, follow, torch.ones_like(follow, dtype=torch.float32)) / FOLLOWERS
    entropy = float(-(counts * counts.clamp_min(1e-30).log()).sum(1).mean())
    return [float(v) for v in losses], entropy, two.evaluate(one.forward(tokens, 0, p=0.0), targets)


if __name__ == "__main__":
    losses, entropy, (plain, eight) = train(int(sys.argv[1]) if len(sys.argv) > 1 else 400, lambda s: print(s, flush=True))
    print(f"loss {losses[0]:.3f} -> {sum(losses[-20:]) / 20:.3f} (entropy of the data {entropy:.3f}); without dropout {plain:.4f}, from 8 bits {eight:.4f}")
