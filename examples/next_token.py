"""Data-parallel training of a small language model with 2-bit gradient messages.

M workers, as slices of one GPU's memory, each see a batch of (previous token, next token) pairs of a synthetic source.
The model is a residual stream: an embedding, `layers` blocks h <- h + W norm(h), a last norm and the output matrix.  All
parameters lie in one flat binary32 vector with a list of tensors.  A worker's step:

  forward   qa_rms_norm adds the block's output to the stream, normalises it, and leaves the normalised values in bfloat16,
            for the product with W, and in 8 bits, for the backward pass: the stream and the codes are all that is kept
  loss      qa_token_logprob: log probability of the next token, entropy, and the most likely token
  backward  qa_token_logprob_grad, then per matrix qa_rows_weight_grad from the codes and a product for dy, per norm
            qa_rms_norm_grad; every weight gradient lands at its place in the worker's flat gradient
  message   qa_quantize_pack_segments, one threshold and scale per tensor
  update    qa_step_qcmd_segments on the average of all workers' messages

Run: python examples/next_token.py [steps]
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2208_05631_amd as qa  # noqa: E402

BF16 = torch.bfloat16
EPS = 1e-6


class Model:
    """The list of tensors, and one worker's forward and backward pass on the flat vector."""

    def __init__(self, vocab, width, layers, rows, device="cuda:0", group=32):
        self.vocab, self.width, self.layers, self.rows, self.dev = vocab, width, layers, rows, device
        shapes = [("embedding", (vocab, width))]
        for i in range(layers):
            shapes += [(f"norm{i}", (width,)), (f"w{i}", (width, width))]
        shapes += [("norm_out", (width,)), ("w_out", (vocab, width))]
        self.begin, self.length, self.shape, at = [], [], {}, 0
        for name, shape in shapes:                         # a tensor begins on a multiple of 16 components
            self.shape[name] = (at, shape)
            self.begin.append(at)
            self.length.append(math.prod(shape))
            at += -(-self.length[-1] // 16) * 16
        self.d = at
        self.codes = qa.CodedRows.make(rows, width, group)
        room = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=device)  # noqa: E731
        self.ws = room(max(qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, vocab),
                           qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, width),
                           qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_NORM_GRAD, qa.QA_BF16),
                           qa.qa_token_workspace_bytes(rows, vocab, 1)))
        new = lambda *shape, dtype=BF16: torch.empty(*shape, dtype=dtype, device=device)  # noqa: E731
        n = layers + 1
        self.stream = [new(rows, width) for _ in range(n)]                        # h after each addition
        self.kept = [(new(rows, self.codes.code_stride, dtype=torch.int8), new(rows, self.codes.scale_stride, dtype=torch.uint8),
                      new(rows, dtype=torch.float32)) for _ in range(n)]          # codes, scales, rstd of each norm
        self.y = new(rows, width)
        self.logprob, self.entropy = new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
        self.stats = new(rows, 2, dtype=torch.float32)
        self.top, self.top_index = new(rows, 1, dtype=torch.float32), new(rows, 1, dtype=torch.int32)
        self.weight_of_row = torch.full((rows,), -1.0 / rows, dtype=torch.float32, device=device)

    def view(self, flat, name):
        at, shape = self.shape[name]
        return flat[at:at + math.prod(shape)].view(shape)

    def initial(self, seed=0):
        gen = torch.Generator().manual_seed(seed)
        x = torch.zeros(self.d)
        for name, (at, shape) in self.shape.items():
            v = torch.ones(shape) if len(shape) == 1 else torch.randn(shape, generator=gen) * (0.5 if name == "embedding" else 0.5 / math.sqrt(self.width))
            x[at:at + math.prod(shape)] = v.reshape(-1)
        return x.to(self.dev)

    def _norm(self, i, x, residual, weight):
        K, (codes, scales, rstd) = self.width, self.kept[i]
        qa.qa_rms_norm(self.codes, qa.QA_BF16, x, K, residual, K, weight, EPS, self.stream[i], K, codes, scales, self.y, K, rstd)
        return self.y

    def _norm_grad(self, i, dy, dh, weight, dweight):
        K, dx = self.width, torch.empty_like(dy)
        qa.qa_rms_norm_grad(self.codes, qa.QA_BF16, dy, K, self.stream[i], K, None, None, weight, self.kept[i][2], dh, K, dx, K, dweight, 0, self.ws)
        return dx

    def _weight_grad(self, i, dy, dw):
        codes, scales, _ = self.kept[i]
        qa.qa_rows_weight_grad(self.codes, codes, scales, qa.QA_BF16, dy, dy.shape[1], dy.shape[1], dw, self.width, 0, self.ws)

    def gradient(self, x, g, before, after):
        """Gradient of the mean loss -log p(after | before) at the flat parameters x, into the flat g.  Returns nothing and waits for
        nothing: logprob, entropy and top_index hold the batch's numbers."""
        T, V, out = self.rows, self.vocab, self.layers
        w = {n: self.view(x, n).to(BF16) for n in self.shape if n.startswith("w")}
        h, add = self.view(x, "embedding")[before].to(BF16), None
        for i in range(self.layers):
            y = self._norm(i, h, add, self.view(x, f"norm{i}"))
            h, add = self.stream[i], y @ w[f"w{i}"].t()
        y = self._norm(out, h, add, self.view(x, "norm_out"))
        logits = y @ w["w_out"].t()
        qa.qa_token_logprob(qa.QA_BF16, T, V, logits, V, after, 1, self.logprob, self.entropy, self.stats, self.top, self.top_index, self.ws)

        qa.qa_token_logprob_grad(qa.QA_BF16, T, V, logits, V, after, self.stats, None, self.weight_of_row, None, logits, V)     # in place
        self._weight_grad(out, logits, self.view(g, "w_out"))
        dh = self._norm_grad(out, logits @ w["w_out"], None, self.view(x, "norm_out"), self.view(g, "norm_out"))
        for i in reversed(range(self.layers)):
            self._weight_grad(i, dh, self.view(g, f"w{i}"))
            dh = self._norm_grad(i, dh @ w[f"w{i}"], dh, self.view(x, f"norm{i}"), self.view(g, f"norm{i}"))
        self.view(g, "embedding").zero_().index_add_(0, before, dh.float())


def source(vocab, seed=1):
    """Transition probabilities of a source whose next token depends on the last one: a few likely successors each."""
    gen = torch.Generator().manual_seed(seed)
    return torch.softmax(3.0 * torch.randn(vocab, vocab, generator=gen), dim=1)


def train(steps=200, workers=4, rows=2048, vocab=257, width=96, layers=2, eta=0.02, lam=1e-7, say=print):
    dev = torch.device("cuda:0")
    model = Model(vocab, width, layers, rows, dev)
    x = model.initial()
    G, z = torch.zeros_like(x), None
    table = qa.qa_segment_plan_bytes(model.d, len(model.begin))
    plan = qa.qa_segment_plan_init(model.d, model.begin, model.length, torch.empty(table, dtype=torch.uint8, device=dev))
    L = qa.Layout.make(model.d, workers, 0, scale_stride=len(model.begin))
    g = torch.zeros(workers, model.d, device=dev)
    codes = torch.empty(workers, L.code_stride, dtype=torch.int32, device=dev)
    scales = torch.empty(workers, L.scale_stride, device=dev)
    ws = torch.empty(max(256, qa.qa_segment_workspace_bytes(plan, workers, qa.QA_OP_QUANTIZE)), dtype=torch.uint8, device=dev)
    p = source(vocab).to(dev)
    gen = torch.Generator(device=dev).manual_seed(2)
    losses = []
    for step in range(steps):
        loss = torch.zeros((), device=dev)
        for m in range(workers):
            before = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
            after = torch.multinomial(p[before], 1, generator=gen)[:, 0].to(torch.int32)
            model.gradient(x, g[m], before, after)
            loss -= model.logprob.mean() / workers
        qa.qa_quantize_pack_segments(L, plan, g, model.d, codes, scales, None, ws)
        qa.qa_step_qcmd_segments(L, plan, codes, scales, x, G, z, eta, lam, 1e-8, qa.QA_REQUANT_NONE, None)
        losses.append(loss)
        if say and (step % 20 == 0 or step == steps - 1):
            hit = float((model.top_index[:, 0] == after).float().mean())
            say(f"step {step:4d}  loss {float(loss):.4f}  entropy {float(model.entropy.mean()):.4f}  most likely token right {hit:.3f}")
    least = float(-(p * torch.log(p)).sum(dim=1).mean())
    if say:
        say(f"loss of the source itself: {least:.4f}, of a guess: {math.log(vocab):.4f}")
    return [float(v) for v in losses], least


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
