"""A student with 4-bit weights learns from a teacher's top logits with 0/1 Adam.

The student is two layers, z = relu(x W1^T) W2^T, whose weights live in one
binary32 shard that the optimizer updates.  Each step

* quantises weights, activations and output gradients to microscaled 4-bit
  matrices, along the axis that each product reduces over,
* takes the products of the forward and the backward pass from them,
* gets the loss and the gradient of the logits from the teacher's top logits,
* writes the weights' gradients into the flat gradient and makes an optimizer
  step: local steps, and every fourth a 1-bit compressed synchronisation (this
  worker alone: W = 1).

At the end one token goes through the trained student as a server would run it.

Run: python examples/distill_student.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2202_06009_amd as zo  # noqa: E402


class Weight:
    """A weight [n, k] of the shard in both 4-bit forms: along k for the forward
    product, along n for the gradient of the activations."""

    def __init__(self, values, grad):
        n, k = values.shape
        self.values, self.grad = values, grad
        self.q, self.qt = zo.Mx4(n, k), zo.Mx4(k, n)

    def quantize(self):
        zo.zo_mx4_quantize(self.values, self.q, self.qt)


class Layer:
    """y = x w^T over `tokens` rows, with the buffers of both directions."""

    def __init__(self, weight, tokens):
        n, k = weight.values.shape
        self.w = weight
        self.xq, self.xt = zo.Mx4(tokens, k), zo.Mx4(k, tokens)
        self.gq, self.gt = zo.Mx4(tokens, n), zo.Mx4(n, tokens)
        self.y = torch.empty((tokens, n), dtype=torch.bfloat16, device="cuda")
        self.dx = torch.empty((tokens, k), dtype=torch.bfloat16, device="cuda")

    def forward(self, x):
        zo.zo_mx4_quantize(x, self.xq, self.xt)
        zo.zo_mx4_product(self.xq, self.w.q, self.y)
        return self.y

    def backward(self, dy, need_dx):
        zo.zo_mx4_quantize(dy, self.gq if need_dx else None, self.gt)
        zo.zo_mx4_product(self.gt, self.xt, self.w.grad)
        if need_dx:
            zo.zo_mx4_product(self.gq, self.w.qt, self.dx)
            return self.dx


def run(steps=200, tokens=1024, hidden=256, inner=512, vocab=2000, top=32, tau=2.0, lr=2e-3,
        seed=0, quiet=False):
    """Trains; returns the mean loss of every step."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    # the shard: two segments, and the optimizer's state over it
    sizes = [inner * hidden, vocab * inner]
    d = sum(sizes)
    state = {k: torch.zeros(d, device="cuda")
             for k in ("x", "m", "v", "u", "err", "srv_err", "anchor")}
    state["x"].copy_(normal(d) * 0.05)
    grad = torch.zeros(d, device="cuda")
    sync = [t for t in range(steps) if t % 4 == 3]
    opt = zo.ZoAdam(beta1=0.9, beta2=0.99, eps=1e-8, world=1, chunk=2048,
                    seg_off=[0, sizes[0], d], tv=range(steps), tu=sync, state=state)
    packed = torch.empty((1, opt.nwords), dtype=torch.int64, device="cuda")
    scales = torch.empty((1, opt.nchunks), device="cuda")
    srv_packed = torch.empty(opt.nwords, dtype=torch.int64, device="cuda")
    srv_scales = torch.empty(opt.nchunks, device="cuda")

    def part(flat, i, n, k):
        o = sum(sizes[:i])
        return flat[o:o + sizes[i]].view(n, k)

    w1 = Weight(part(state["x"], 0, inner, hidden), part(grad, 0, inner, hidden))
    w2 = Weight(part(state["x"], 1, vocab, inner), part(grad, 1, vocab, inner))
    first, second = Layer(w1, tokens), Layer(w2, tokens)

    teacher = normal(vocab, hidden) * 0.25
    values = torch.empty((tokens, top), device="cuda")
    columns = torch.empty((tokens, top), dtype=torch.int32, device="cuda")
    lse, loss = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    losses = []
    for t in range(steps):
        x = normal(tokens, hidden).bfloat16()
        zo.zo_top_logits(x.float() @ teacher.t(), values, columns, lse, tau=tau)
        # the student
        w1.quantize()
        w2.quantize()
        h = first.forward(x)
        a = torch.relu(h)
        z = second.forward(a)
        # the gradient of the logits over the logits themselves
        zo.zo_distill_loss(z, values, columns, loss, z, tau=tau, teacher_lse=lse,
                           row_weight=weight)
        losses.append(loss.sum())
        da = second.backward(z, True)
        first.backward(da * (h > 0), False)
        # the optimizer
        if t in opt.cfg["tu"]:
            opt.compress_pack_ef(t, lr, grad, packed[0], scales[0])
            opt.unpack_average(t, packed, scales, srv_packed, srv_scales)
            opt.sync_update(t, srv_packed, srv_scales, grad)
        else:
            opt.local_step(t, lr, grad, grad)
        if not quiet and t % 20 == 0:
            print(f"step {t}: loss {float(losses[-1]):.4f}", flush=True)
    losses = torch.stack(losses).tolist()

    # a decode step: one token, the weights' codes kept
    w1.quantize()
    w2.quantize()
    x = normal(1, hidden).bfloat16()
    h = torch.empty((1, inner), dtype=torch.bfloat16, device="cuda")
    z = torch.empty((1, vocab), device="cuda")
    zo.zo_mx4_linear(x, w1.q, h, zo.Mx4(1, hidden))
    zo.zo_mx4_linear(torch.relu(h), w2.q, z, zo.Mx4(1, inner))
    best, at = torch.empty((1, 5), device="cuda"), torch.empty((1, 5), dtype=torch.int32,
                                                               device="cuda")
    zo.zo_top_logits(z, best, at)
    torch.cuda.synchronize()
    if not quiet:
        print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}; the student's top columns "
              f"{at[0].tolist()}, the teacher's "
              f"{torch.topk(x.float() @ teacher.t(), 5).indices[0].tolist()}")
    opt.close()
    return losses


if __name__ == "__main__":
    run(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
