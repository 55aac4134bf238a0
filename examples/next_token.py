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

Two of these have another form.  Without kept logits (`keep_logits=False`) the loss is qa_output_logprob and its gradient
qa_output_logprob_grad, which multiply the output matrix themselves.  With `orthogonal` the blocks' square matrices are stepped by
qa_step_orthogonal on the average of their messages (qa_aggregate_unpack), the other tensors by QCMD.

Run: python examples/next_token.py [steps] [--no-logits] [--orthogonal]
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

    def __init__(self, vocab, width, layers, rows, device="cuda:0", group=32, keep_logits=True):
        self.vocab, self.width, self.layers, self.rows, self.dev, self.keep_logits = vocab, width, layers, rows, device, keep_logits
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
        self.output = qa.OutputLayer.make(rows, vocab, width)
        room = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device=device)  # noqa: E731
        self.ws = room(max(qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, vocab),
                           qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_WEIGHT_GRAD, qa.QA_BF16, width),
                           qa.qa_rows_workspace_bytes(self.codes, qa.QA_OP_NORM_GRAD, qa.QA_BF16),
                           qa.qa_token_workspace_bytes(rows, vocab, 1),
                           *(qa.qa_output_workspace_bytes(self.output, op, qa.QA_BF16) for op in (qa.QA_OP_LOGPROB, qa.QA_OP_LOGPROB_GRAD) if not keep_logits)))
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
        nothing: logprob, entropy and, with kept logits, top_index hold the batch's numbers."""
        T, V, out = self.rows, self.vocab, self.layers
        w = {n: self.view(x, n).to(BF16) for n in self.shape if n.startswith("w")}
        h, add = self.view(x, "embedding")[before].to(BF16), None
        for i in range(self.layers):
            y = self._norm(i, h, add, self.view(x, f"norm{i}"))
            h, add = self.stream[i], y @ w[f"w{i}"].t()
        y = self._norm(out, h, add, self.view(x, "norm_out"))
        if self.keep_logits:
            logits = y @ w["w_out"].t()
            qa.qa_token_logprob(qa.QA_BF16, T, V, logits, V, after, 1, self.logprob, self.entropy, self.stats, self.top, self.top_index, self.ws)
            qa.qa_token_logprob_grad(qa.QA_BF16, T, V, logits, V, after, self.stats, None, self.weight_of_row, None, logits, V)     # in place
            self._weight_grad(out, logits, self.view(g, "w_out"))
            dy = logits @ w["w_out"]
        else:
            dy = torch.empty_like(y)
            qa.qa_output_logprob(self.output, qa.QA_BF16, y, w["w_out"], after, self.logprob, self.entropy, self.stats, self.ws)
            qa.qa_output_logprob_grad(self.output, qa.QA_BF16, y, w["w_out"], after, self.stats, None, self.weight_of_row, None, dy, self.width,
                                      self.view(g, "w_out"), self.width, 0, self.ws)
        dh = self._norm_grad(out, dy, None, self.view(x, "norm_out"), self.view(g, "norm_out"))
        for i in reversed(range(self.layers)):
            self._weight_grad(i, dh, self.view(g, f"w{i}"))
            dh = self._norm_grad(i, dh @ w[f"w{i}"], dh, self.view(x, f"norm{i}"), self.view(g, f"norm{i}"))
        self.view(g, "embedding").zero_().index_add_(0, before, dh.float())


def source(vocab, seed=1):
    """Transition probabilities of a source whose next token depends on the last one: a few likely successors each."""
    gen = torch.Generator().manual_seed(seed)
    return torch.softmax(3.0 * torch.randn(vocab, vocab, generator=gen), dim=1)


class MatrixSteps:
    """qa_step_orthogonal for some of a model's matrices, from all workers' messages: a matrix's code words and scale lie in them where its
    components do."""

    def __init__(self, model, names, workers, layout):
        self.at = []
        for name in names:
            begin, shape = model.shape[name]
            L = qa.Layout.make(math.prod(shape), workers, 0, code_stride=layout.code_stride, scale_stride=layout.scale_stride)
            M = qa.Matrices.make(1, *shape)
            need = qa.qa_orthogonal_workspace_bytes(M, qa.QA_F32)
            mean = torch.empty(shape, device=model.dev)
            self.at.append((begin, list(model.shape).index(name), L, M, mean, torch.zeros_like(mean), torch.empty(need, dtype=torch.uint8, device=model.dev) if need else None))

    def step(self, codes, scales, x, eta):
        for begin, tensor, L, M, mean, momentum, ws in self.at:
            qa.qa_aggregate_unpack(L, codes[:, begin // 16:], scales[:, tensor:], mean)
            qa.qa_step_orthogonal(M, mean, momentum, x[begin:], 0.9, 1, 5, None, eta, 1.0, ws)


def train(steps=200, workers=4, rows=2048, vocab=257, width=96, layers=2, eta=0.02, lam=1e-7, say=print, keep_logits=True, orthogonal=False):
    dev = torch.device("cuda:0")
    model = Model(vocab, width, layers, rows, dev, keep_logits=keep_logits)
    x = model.initial()
    G, z = torch.zeros_like(x), None
    square = [f"w{i}" for i in range(layers)] if orthogonal else []
    length = [0 if name in square else n for name, n in zip(model.shape, model.length)]      # what QCMD steps
    table = qa.qa_segment_plan_bytes(model.d, len(model.begin))
    plan = qa.qa_segment_plan_init(model.d, model.begin, model.length, torch.empty(table, dtype=torch.uint8, device=dev))
    rest = plan if not square else qa.qa_segment_plan_init(model.d, model.begin, length, torch.empty(table, dtype=torch.uint8, device=dev))
    L = qa.Layout.make(model.d, workers, 0, scale_stride=len(model.begin))
    matrices = MatrixSteps(model, square, workers, L)
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
        matrices.step(codes, scales, x, eta)
        qa.qa_step_qcmd_segments(L, rest, codes, scales, x, G, z, eta, lam, 1e-8, qa.QA_REQUANT_NONE, None)
        losses.append(loss)
        if say and (step % 20 == 0 or step == steps - 1):
            hit = f"  most likely token right {float((model.top_index[:, 0] == after).float().mean()):.3f}" if keep_logits else ""
            say(f"step {step:4d}  loss {float(loss):.4f}  entropy {float(model.entropy.mean()):.4f}{hit}")
    least = float(-(p * torch.log(p)).sum(dim=1).mean())
    if say:
        say(f"loss of the source itself: {least:.4f}, of a guess: {math.log(vocab):.4f}")
    return [float(v) for v in losses], least


if __name__ == "__main__":
    numbers = [int(v) for v in sys.argv[1:] if not v.startswith("--")]
    train(*numbers[:1] or [200], keep_logits="--no-logits" not in sys.argv, orthogonal="--orthogonal" in sys.argv)
