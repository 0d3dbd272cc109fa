"""A small language model trained by W workers under detached error feedback, every part of a step from this library or a
plain matrix product: norms around the blocks, gated activations, 8-bit activation checkpoints and the weight gradients
taken from them, token log probabilities with their gradient -- and def_step on the gradient rows they fill.

    python -m paper_2004_05298_b200.lm_example [--steps N] [--workers W] [--ratio R]

Each worker evaluates its gradient at its own point z_w = x - lambda e_w (Algorithm 1's detach step), on its own tokens.
Data are synthetic: a random successor table, followed nine times out of ten."""
import argparse
import math

import torch

from . import binding as B

DEV = "cuda"


class Layout:
    """Where each parameter lies in the flat vector of d coordinates."""

    def __init__(self, vocab, width, hidden, blocks):
        self.vocab, self.width, self.hidden, self.blocks = vocab, width, hidden, blocks
        self.at, self.d = {}, 0
        self._add("embed", vocab, width)
        self._add("pre0", width)
        for i in range(blocks):
            self._add("gate_up%d" % i, 2 * hidden, width)
            self._add("down%d" % i, width, hidden)
            self._add("post%d" % i, width)
            self._add("gate%d" % i, 1, width)
            self._add("pre%d" % (i + 1), width)
        self._add("head", vocab, width)

    def _add(self, name, *shape):
        self.at[name] = (self.d, shape)
        self.d += math.prod(shape)

    def view(self, flat, name):
        start, shape = self.at[name]
        return flat[start:start + math.prod(shape)].view(shape)

    def initial(self, seed=0):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        x = torch.empty(self.d, device=DEV)
        for name, (_, shape) in self.at.items():
            v = self.view(x, name)
            if name.startswith(("pre", "post")):
                v.fill_(1.0)
            elif name.startswith("gate") and not name.startswith("gate_up"):
                v.fill_(0.5)
            else:
                v.normal_(0.0, 1.0 if name == "embed" else 1.0 / math.sqrt(shape[1]), generator=gen)
        return x


def shift(n, length):
    """Each token's row plus that of the token before it in its sequence."""
    out = n.clone().view(-1, length, n.shape[1])
    out[:, 1:] += n.view(-1, length, n.shape[1])[:, :-1]
    return out.view_as(n)


def shift_back(d, length):
    out = d.clone().view(-1, length, d.shape[1])
    out[:, :-1] += d.view(-1, length, d.shape[1])[:, 1:]
    return out.view_as(d)


class Pass:
    """Forward and backward pass of one worker's batch; activations between the two are kept in 8 bits.  Buffers are made
    once and used by every step."""

    def __init__(self, layout, tokens, length, dtype=torch.bfloat16, top=4):
        L, T, C, F, V = layout, tokens, layout.width, layout.hidden, layout.vocab
        self.layout, self.T, self.length, self.dtype = L, T, length, dtype

        def act(cols):
            return torch.empty(T, cols, dtype=dtype, device=DEV)

        def stat(*shape):
            return torch.empty(shape, device=DEV)

        def held(cols):
            return B.def_checkpoint_alloc(T, cols, DEV)

        k = L.blocks
        self.h, self.n = [act(C) for _ in range(k + 1)], act(C)
        self.hidden, self.hidden_ck = act(F), held(F)
        self.mixed_ck, self.gate_ck, self.up_ck = ([held(c) for _ in range(k)] for c in (C, F, F))
        self.block_ck, self.h_ck, self.n_ck = [held(C) for _ in range(k)], [held(C) for _ in range(k + 1)], held(C)
        self.rstd_pre, self.rstd_post = [stat(T) for _ in range(k + 1)], [stat(T) for _ in range(k)]
        self.logits, self.logp, self.entropy, self.lse = act(V), stat(T), stat(T), stat(T, 2)
        self.top_ids, self.top_logp = torch.empty(T, top, dtype=torch.int64, device=DEV), stat(T, top)
        self.dh, self.db, self.dboth = act(C), act(C), act(2 * F)
        self.weight = stat(T).fill_(-1.0 / T)                              # of each token's log probability in the loss
        sizes = [B.def_norm_backward_workspace(T, C)]
        for dy, cols in ((self.logits, C), (self.db, F), (self.dboth, C)):
            sizes.append(B.def_checkpoint_weight_grad_workspace(dy, cols))
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device=DEV)

    def _weights(self, z, name):
        return self.layout.view(z, name).to(self.dtype)

    def forward(self, z, tokens, targets):
        """Mean negative log probability of the targets at the parameters z [d]."""
        L, F = self.layout, self.layout.hidden
        P = lambda name: L.view(z, name)                                   # noqa: E731
        self.h[0].copy_(P("embed")[tokens])
        B.def_norm_forward(self.h[0], None, None, None, P("pre0"), None, self.n, None, self.rstd_pre[0], h_ck=self.h_ck[0])
        for i in range(L.blocks):
            mixed = shift(self.n, self.length)
            B.def_checkpoint_pack(mixed, self.mixed_ck[i])
            both = mixed @ self._weights(z, "gate_up%d" % i).t()
            B.def_gated_forward(both[:, :F], both[:, F:], self.hidden, self.gate_ck[i], self.up_ck[i])
            out = self.hidden @ self._weights(z, "down%d" % i).t()
            last = i == L.blocks - 1
            B.def_norm_forward(self.h[i], out, P("post%d" % i), P("gate%d" % i), P("pre%d" % (i + 1)), self.h[i + 1], self.n,
                               self.rstd_post[i], self.rstd_pre[i + 1], b_ck=self.block_ck[i], h_ck=self.h_ck[i + 1],
                               n_ck=self.n_ck if last else None)
        torch.matmul(self.n, self._weights(z, "head").t(), out=self.logits)
        B.def_logprob_forward(self.logits, targets, self.logp, self.entropy, self.lse, self.top_ids, self.top_logp)
        return -self.logp.mean()

    def backward(self, z, tokens, targets, grad):
        """The loss's gradient into grad [d] (fp32: a worker's row of the gradients def_step reads)."""
        L, F, W = self.layout, self.layout.hidden, self.workspace
        P, G = (lambda name: L.view(z, name)), (lambda name: L.view(grad, name))
        B.def_logprob_backward(self.logits, targets, self.lse, self.entropy, self.logits, dlogp=self.weight)   # in place
        B.def_checkpoint_weight_grad(self.logits, self.n_ck, G("head"), W)
        dn, dh = self.logits @ self._weights(z, "head"), None
        for i in reversed(range(L.blocks)):
            B.def_norm_backward(dn, dh, self.h_ck[i + 1], self.block_ck[i], P("post%d" % i), P("gate%d" % i), P("pre%d" % (i + 1)),
                                self.rstd_post[i], self.rstd_pre[i + 1], self.dh, self.db, G("post%d" % i), G("gate%d" % i),
                                G("pre%d" % (i + 1)), W)
            dh = self.dh
            dhidden = self.db @ self._weights(z, "down%d" % i)
            B.def_gated_backward(dhidden, self.gate_ck[i], self.up_ck[i], self.dboth[:, :F], self.dboth[:, F:], h_ck=self.hidden_ck)
            B.def_checkpoint_weight_grad(self.db, self.hidden_ck, G("down%d" % i), W)
            B.def_checkpoint_weight_grad(self.dboth, self.mixed_ck[i], G("gate_up%d" % i), W)
            dn = shift_back(self.dboth @ self._weights(z, "gate_up%d" % i), self.length)
        B.def_norm_backward(dn, dh, self.h_ck[0], None, None, None, P("pre0"), None, self.rstd_pre[0], self.dh, None, None, None,
                            G("pre0"), W)
        G("embed").zero_().index_add_(0, tokens, self.dh.float())

    def alternatives(self):
        """The most probable next tokens of the last forward pass, with their log probabilities."""
        return self.top_ids, self.top_logp


def batches(vocab, workers, tokens, length, seed=0):
    """Endless (tokens, targets) for each worker: sequences that follow a successor table nine times out of ten."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    table = torch.randperm(vocab, device=DEV, generator=gen)
    while True:
        out = []
        for _ in range(workers):
            s = torch.empty(tokens // length, length + 1, dtype=torch.int64, device=DEV)
            s[:, 0] = torch.randint(0, vocab, (tokens // length,), device=DEV, generator=gen)
            for j in range(length):
                jump = torch.randint(0, vocab, (tokens // length,), device=DEV, generator=gen)
                s[:, j + 1] = torch.where(torch.rand(tokens // length, device=DEV, generator=gen) < 0.9, table[s[:, j]], jump)
            out.append((s[:, :-1].reshape(-1), s[:, 1:].reshape(-1)))
        yield out


def train(steps=60, workers=4, ratio=8, vocab=512, width=256, hidden=640, blocks=2, tokens=1024, length=64, lr=0.5, momentum=0.9,
          lam=0.3, seed=0, report=None):
    """Losses (mean over the workers, at their detached points) of `steps` steps, and the model Algorithm 1 returns."""
    layout = Layout(vocab, width, hidden, blocks)
    x = layout.initial(seed)
    W, d = workers, layout.d
    grads, errors, mom = (torch.zeros(W, d, device=DEV) for _ in range(3))
    z = x.expand(W, d).contiguous()                                        # e = 0 before the first step
    ctx = B.def_create(d, W, max(1, d // ratio), B.DEF_VARIANT_DEF, lr, momentum, (lam, 0.0))
    work, losses = Pass(layout, tokens, length), []
    data = batches(vocab, W, tokens, length, seed)
    for t in range(steps):
        loss = 0.0
        for w, (tok, target) in enumerate(next(data)):
            loss = loss + work.forward(z[w], tok, target)
            work.backward(z[w], tok, target, grads[w])
        B.def_step_detach(ctx, x, grads, errors, mom, z, t, seed)
        losses.append(loss / W)
        if report and t % report == 0:
            print("step %3d  loss %.4f" % (t, float(losses[-1])))
    model = torch.empty_like(x)
    B.def_output(ctx, x, errors, model)
    B.def_destroy(ctx)
    return [float(v) for v in losses], model, layout


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--ratio", type=int, default=8)
    a = ap.parse_args()
    losses, _, layout = train(a.steps, a.workers, a.ratio, report=10)
    print("%d parameters, %d workers, ratio %d: loss %.4f -> %.4f" % (layout.d, a.workers, a.ratio, losses[0], losses[-1]))


if __name__ == "__main__":
    main()
