"""Teaching a network that will run on ciphertexts from a network that need not (sequencing and buffers only).

A network for encrypted evaluation has polynomial activations and few levels, and is trained in the clear: by the labels
and by what a trained teacher of any shape answers.  The teacher's last steps are a residual addition and a
root-mean-square norm, written as 8-bit codes, and the product of those codes with its 8-bit table of classes (or of a
vocabulary).  Of each row of its logits only the k largest and the log-sum-exp of the others are kept, to be stored beside
the inputs or used at once.  The student's loss compares that with its own logits; its gradient goes on into autograd:

    head = TeacherHead(ctx, table, norm_weight, rows, k=64, tau=2.0)
    answers = head(x, residual)                       # Answers(values, index, rest)
    loss = distill_loss(ctx, student(images), answers, 2.0, labels, alpha=0.3).mean()
    loss.backward()

`ctx` is an HEContext; its calls go to the stream that was current at its creation, so these functions want that stream to
be the current one.
"""
from collections import namedtuple

import torch

BLOCK, F8, F8_MAX = 128, torch.float8_e4m3fn, 448.0

Answers = namedtuple("Answers", "values index rest")           # [rows][k] f32, [rows][k] i32, [rows] f32


def _same_stream(ctx):
    if torch.cuda.current_stream() != ctx.stream:
        raise ValueError("the context works on another stream than the current one")


def _code_rows(rows, cols, device):
    """Rows of codes begin at multiples of 16 bytes."""
    return torch.empty((rows, -(-cols // 16) * 16), dtype=F8, device=device)[:, :cols]


def quantize_table(w):
    """W [N][K] as codes and one scale for each 128 x 128 block, the largest number of a block at the largest code."""
    n, k = w.shape
    nb, kb = -(-n // BLOCK), -(-k // BLOCK)
    whole = torch.zeros((nb * BLOCK, kb * BLOCK), dtype=torch.float32, device=w.device)
    whole[:n, :k] = w
    blocks = whole.view(nb, BLOCK, kb, BLOCK)
    scales = blocks.abs().amax(dim=(1, 3)) / F8_MAX
    by = torch.where(scales == 0, 1.0, scales)[:, None, :, None]         # a quotient: the inverse of the smallest scales is no number
    codes = _code_rows(n, k, w.device)
    codes.copy_((blocks / by).clamp_(-F8_MAX, F8_MAX).reshape(nb * BLOCK, kb * BLOCK)[:n, :k].to(F8))
    return codes, scales


class TeacherHead:
    """The last steps of a teacher and its answers, for up to `rows` rows at a time; what lies between stays in buffers made here.

    fast_sums: whether the product's sums may lose what he_matmul_q8 says; None: where the logits have 16 bits."""

    def __init__(self, ctx, table, norm_weight, rows, k, tau, eps=1e-6, dtype=torch.bfloat16, fast_sums=None):
        self.ctx, self.k, self.tau, self.eps, self.norm_weight = ctx, k, tau, eps, norm_weight
        self.fast_sums = dtype != torch.float32 if fast_sums is None else fast_sums
        self.table, self.table_scales = quantize_table(table)
        vocab, dim = table.shape
        self.codes = _code_rows(rows, dim, table.device)
        self.scales = torch.empty((rows, -(-dim // BLOCK)), device=table.device)
        self.logits = torch.empty((rows, -(-vocab // 8) * 8), dtype=dtype, device=table.device)[:, :vocab]

    def __call__(self, x, residual=None, sum_out=None):
        """x, residual, sum_out [rows][dim]; the answers are new tensors, the logits are self.logits until the next call."""
        _same_stream(self.ctx)
        n = x.shape[0]
        if n > self.codes.shape[0]:
            raise ValueError("more rows than the head was made for")
        codes, scales, logits = self.codes[:n], self.scales[:n], self.logits[:n]
        self.ctx.he_rmsnorm_q8(x, codes, scales, self.eps, residual=residual, weight=self.norm_weight, sum_out=sum_out)
        self.ctx.he_matmul_q8(codes, scales, self.table, self.table_scales, logits, fast_sums=self.fast_sums)
        f32 = dict(dtype=torch.float32, device=x.device)
        answers = Answers(torch.empty((n, self.k), **f32), torch.empty((n, self.k), dtype=torch.int32, device=x.device), torch.empty(n, **f32))
        self.ctx.he_top_logits(logits, self.tau, *answers)
        return answers


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(run, z, ctx, answers, tau, labels, alpha):
        _same_stream(ctx)
        loss = torch.empty(z.shape[0], dtype=torch.float32, device=z.device)
        stats = torch.empty((z.shape[0], 4), dtype=torch.float32, device=z.device) if run.needs_input_grad[0] else None
        ctx.he_distill_loss(z, *answers, tau, loss, labels=labels, alpha=alpha, stats=stats)
        run.save_for_backward(z, stats, labels, *answers)
        run.ctx, run.tau, run.alpha = ctx, tau, alpha
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(run, weights):
        z, stats, labels, *answers = run.saved_tensors
        _same_stream(run.ctx)
        grad = torch.empty_like(z)
        run.ctx.he_distill_grad(z, *answers, run.tau, stats, weights.contiguous(), grad, labels=labels, alpha=run.alpha)
        return grad, None, None, None, None, None


def distill_loss(ctx, z, answers, tau, labels=None, alpha=0.0):
    """One loss for each row of the student's logits z, differentiable by z; tau as it was for the answers.  Labels are int32, or int64 as torch's
    losses take them: a negative one is padding, one beyond the vocabulary is not there."""
    if labels is not None and labels.dtype == torch.int64:
        labels = labels.clamp(-1, z.shape[-1]).to(torch.int32)
    own = z.dim() == 2 and z.stride(1) == 1 and (z.shape[0] <= 1 or z.stride(0) >= z.shape[1])       # rows in one piece that share nothing
    return _DistillLoss.apply(z if own else z.contiguous(), ctx, answers, tau, labels, alpha)
