"""A student learns from the stored top logits of a teacher that runs at another frame rate.

Nobody says which frame of the teacher a frame of the student answers to.  Soft-DTW aligns their features, with a learned
penalty on how far apart two frames' positions are; the alignment names a teacher's row for every row of the student's logits;
and the student's logits are drawn towards the teacher's top logits there.  The student attends over its frames under a learned
bias on relative positions, and its gradients are clipped to a largest norm.

    python examples/aligned_distillation.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2602_17206_amd as sdtw  # noqa: E402

RULE = dict(max_distance=64, two_sided=True)
BUCKETS, HEADS, GAMMA, TEMPERATURE, MAX_NORM = 16, 2, 0.1, 2.0, 1.0


class Attention(torch.autograd.Function):
    """q, k, v [B, H, N, D] to [B, H, N, D], with a bias table [H, buckets] by distance, each sequence within its length"""

    @staticmethod
    def forward(ctx, q, k, v, table, lengths):
        out, lse = sdtw.sdtw_attention_forward(q, k, v, table, row_len=lengths, col_len=lengths, **RULE)
        ctx.save_for_backward(q, k, v, table, lengths, out, lse)
        return out

    @staticmethod
    def backward(ctx, grad):
        q, k, v, table, lengths, out, lse = ctx.saved_tensors
        dq, dk, dv, dtable = sdtw.sdtw_attention_backward(q, k, v, out, lse, grad, table, row_len=lengths, col_len=lengths, **RULE)
        return dq, dk, dv, dtable.to(table.dtype), None


class Student(torch.nn.Module):
    def __init__(self, inputs, width, vocab, generator):
        super().__init__()

        def weight(*shape):
            return torch.nn.Parameter(torch.randn(shape, generator=generator, device="cuda") / shape[0] ** 0.5)
        self.embed, self.qkv, self.out = weight(inputs, width), weight(width, 3 * width), weight(width, width)
        self.head = weight(width, vocab)
        self.bias = torch.nn.Parameter(torch.zeros(HEADS, BUCKETS, device="cuda"))

    def forward(self, x, lengths):
        """(features [B, N, width], logits [B * N, vocab] bfloat16)"""
        B, N, _ = x.shape
        h = torch.tanh(x @ self.embed)
        q, k, v = (h @ self.qkv).view(B, N, 3, HEADS, -1).permute(2, 0, 3, 1, 4)
        mixed = Attention.apply(q, k, v, self.bias, lengths)
        h = h + mixed.permute(0, 2, 1, 3).reshape(B, N, -1) @ self.out
        return h, (h.reshape(B * N, -1) @ self.head).bfloat16()


def task(B=4, N=96, M=64, inputs=24, width=32, vocab=1000, top=8, seed=0):
    """The student's inputs [B, N, inputs] with their lengths, and of the teacher: features [B, M, width], its lengths, and the
    top logits and their tokens [B * M, top].  Both come from one hidden path that the student sees at a pace of its own."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    path = randn(B, M, inputs).cumsum(1) / 4.0
    x_len = torch.tensor([N - 7 * (b % 3) for b in range(B)], dtype=torch.int32, device="cuda")
    y_len = torch.tensor([M - 5 * (b % 2) for b in range(B)], dtype=torch.int32, device="cuda")
    pace = torch.rand((B, N), generator=gen, device="cuda") + 0.25
    at = pace.cumsum(1)
    last = at.gather(1, x_len.long()[:, None] - 1)
    at = (at / last * y_len[:, None]).long().clamp(max=M - 1)
    x = path.gather(1, at[:, :, None].expand(-1, -1, inputs)) + 0.05 * randn(B, N, inputs)
    y = torch.tanh(path @ (randn(inputs, width) / inputs ** 0.5))
    logits, ids = (4.0 * (y.reshape(B * M, width) @ randn(width, vocab)) / width ** 0.5).topk(top)
    return x, x_len, y, y_len, logits.bfloat16(), ids.int()


def train(steps=60, seed=0):
    """(divergence from the teacher, margin of the wrong alignments over the right ones) of every step"""
    vocab = 1000
    x, x_len, y, y_len, top_logits, top_ids = task(vocab=vocab, seed=seed)
    (B, N, inputs), (_, M, width) = x.shape, y.shape
    student = Student(inputs, width, vocab, torch.Generator(device="cuda").manual_seed(seed + 1))
    # the penalty on cells off the diagonal: 0 nearby, more with each bucket of distance
    penalty = torch.nn.Parameter(0.02 * (torch.arange(BUCKETS, device="cuda") % (BUCKETS // 2)).float()[None])
    parameters = [*student.parameters(), penalty]
    optimizer = torch.optim.Adam(parameters, lr=0.01)
    inside = torch.arange(N, device="cuda") < x_len[:, None]
    row_weight = (inside / inside.sum()).reshape(-1).float()
    # every student with its own teacher, and with its neighbour's
    both_y, both_y_len = torch.cat([y, y.roll(1, 0)]), torch.cat([y_len, y_len.roll(1, 0)])
    both_x_len = torch.cat([x_len, x_len])
    history = []
    for _ in range(steps):
        optimizer.zero_grad()
        features, logits = student(x, x_len)
        both_x = torch.cat([features, features])
        pairs, table = both_x.detach(), penalty.detach()
        value, state, workspace = sdtw.sdtw_forward_biased(pairs, both_y, table, GAMMA, x_len=both_x_len, y_len=both_y_len, **RULE)
        # the right alignment should cost less per frame than the wrong one: loss = mean softplus((right - wrong) / N + 1)
        margin = (value[B:] - value[:B]) / N
        pull = torch.sigmoid(1.0 - margin) / (B * N)
        d_pairs, _, d_penalty, E = sdtw.sdtw_backward_biased(state, pairs, both_y, table, workspace, x_len=both_x_len,
                                                             y_len=both_y_len, grad_value=torch.cat([pull, -pull]), want_E=True)
        # the teacher's row that most of a student's row is aligned with; none beyond the student's length
        teacher_row = E[:B].argmax(2) + M * torch.arange(B, device="cuda")[:, None]
        teacher_row = torch.where(inside, teacher_row, -1).int().reshape(-1)
        loss, d_logits = sdtw.sdtw_distill_step(logits.detach(), top_logits, top_ids, grad_loss=row_weight, temperature=TEMPERATURE,
                                                teacher_row=teacher_row)
        torch.autograd.backward([both_x, logits], [d_pairs, d_logits])
        penalty.grad = d_penalty
        sdtw.sdtw_gradient_clip([p.grad for p in parameters], MAX_NORM)
        optimizer.step()
        history.append((float((loss * row_weight).sum()), float(margin.mean())))
    return history


if __name__ == "__main__":
    for step, (loss, margin) in enumerate(train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)):
        if step % 10 == 9 or step == 0:
            print("step %3d  divergence %.4f  margin %.4f" % (step + 1, loss, margin), flush=True)
