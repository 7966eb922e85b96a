"""Adapting a model to SpargeAttention2 by velocity distillation (Sec. 4.2; Alg. 2), on a toy scale.

The paper fine-tunes video diffusion models whose weights are not available here; what can be exercised
without them is the training step itself: a frozen teacher with full attention, a student that shares its
initialisation and differs only in the attention operator, identical noisy inputs x_t = t x_1 + (1 - t) x_0
for both, and the loss ||u_sparse - u_full||^2 back-propagated through the block-sparse backward kernels.
`ToyBlock` is one pre-norm attention block that stands in for the velocity network; on request with what such a network has
around its attention: the norm of q and k with the rotation by position, attention to a prompt, dropout of its branches.
"""
from __future__ import annotations

import copy
from typing import Callable, Dict, Iterable, Optional, Sequence, Tuple, Union

import torch

from . import binding as _b
from .autograd import _operator, _plain, sparge_attn2
from .block import cross_attention, dropout_add, qk_norm_rotate, rotary_table


class ToyBlock(torch.nn.Module):
    """x -> x + proj(attention(norm(x))): fp32 parameters, bf16 attention on [B, N, H, d] activations that reach
    the kernels as permuted views (no copy).  `k_frac`, `top_p` None means full attention (the teacher).

    grid: extents of the tokens' grid (frames, height, width): the heads of q and k are normed and rotated by position.
    context_dim: a second branch attends to `context` [B, M, context_dim], of which sample b has `lengths[b]` rows (a batch of
    prompts, padded).  dropout: of both branches, in training mode; the masks' seed comes from PyTorch's default generator, in
    a captured step from the GPU's, so that every replay draws other masks."""

    def __init__(self, dim: int, heads: int, k_frac: Optional[float] = None, top_p: Optional[float] = None,
                 grid: Optional[Sequence[int]] = None, context_dim: Optional[int] = None, dropout: float = 0.0):
        super().__init__()
        assert dim % heads == 0 and dim // heads in (64, 128)
        self.heads, self.k_frac, self.top_p, self.dropout = heads, k_frac, top_p, float(dropout)
        self.norm = torch.nn.LayerNorm(dim)
        self.qkv = torch.nn.Linear(dim, 3 * dim)
        self.proj = torch.nn.Linear(dim, dim)
        self.grid, self.context_dim = grid, context_dim
        if grid is not None:
            self.q_weight, self.k_weight = (torch.nn.Parameter(torch.ones(dim // heads)) for _ in range(2))
            for name, table in zip(("cos", "sin"), rotary_table(grid, dim // heads)):
                self.register_buffer(name, table, persistent=False)
        if context_dim is not None:
            self.context_norm = torch.nn.LayerNorm(dim)
            self.context_q = torch.nn.Linear(dim, dim)
            self.context_kv = torch.nn.Linear(context_dim, 2 * dim)
            self.context_proj = torch.nn.Linear(dim, dim)
        self._full = None                     # the all-ones pattern, built once per input shape

    def _attention(self, q, k, v):
        if self.k_frac is not None:
            return sparge_attn2(q, k, v, self.k_frac, self.top_p)
        B, H, N, _ = q.shape
        if self._full is None or self._full.mask.shape[:3] != (B, H, -(-N // _b.BQ)) or self._full.mask.device != q.device:
            self._full = _b.alloc_pattern(B, H, N, q.device)
            _b.spa2_pattern_full(q.detach(), self._full)
        return sparge_attn2(q, k, v, 0.0, 0.0, pattern=self._full)

    def _seed(self, x: torch.Tensor) -> Union[None, int, torch.Tensor]:
        """Of this call's masks: a number, or under capture, where that would be the same on every replay, a (seed, offset) on
        the GPU for each of the two branches."""
        if not self.training or self.dropout <= 0.0:
            return None
        if x.is_cuda and torch.cuda.is_current_stream_capturing():
            return torch.randint(2 ** 63 - 1, (2, 2), device=x.device)
        return int(torch.randint(2 ** 63 - 1, ()).item())

    def _add(self, x: torch.Tensor, branch: torch.Tensor, seed: Union[None, int, torch.Tensor], number: int) -> torch.Tensor:
        """x plus a branch, dropped in places (each branch draws with an offset of its own)."""
        if seed is None:
            return x + branch
        return dropout_add(branch, x, self.dropout, *((seed, number) if isinstance(seed, int) else (seed[number],)))

    def forward(self, x: torch.Tensor, context: Optional[torch.Tensor] = None,
                lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
        B, N, C = x.shape
        d = C // self.heads
        seed = self._seed(x)
        qkv = self.qkv(self.norm(x))
        if self.grid is None:
            qkv = qkv.to(torch.bfloat16).view(B, N, 3, self.heads, d)
            q, k, v = (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3))         # [B, H, N, d] views
        else:                                 # (the norm reads the projection in fp32 and writes what the attention takes)
            q, k, v = (t.permute(0, 2, 1, 3) for t in qkv.view(B, N, 3, self.heads, d).unbind(2))
            q, k = qk_norm_rotate(q, k, self.q_weight, self.k_weight, self.cos, self.sin, interleaved=True)
            v = v.to(torch.bfloat16)
        o = self._attention(q, k, v)                                            # strides of q
        x = self._add(x, self.proj(o.permute(0, 2, 1, 3).reshape(B, N, C).float()), seed, 0)
        if self.context_dim is None:
            return x
        q = self.context_q(self.context_norm(x)).to(torch.bfloat16).view(B, N, self.heads, d).permute(0, 2, 1, 3)
        k, v = (t.permute(0, 2, 1, 3) for t in
                self.context_kv(context).to(torch.bfloat16).view(B, -1, 2, self.heads, d).unbind(2))
        o = cross_attention(q, k, v, lengths)
        return self._add(x, self.context_proj(o.permute(0, 2, 1, 3).reshape(B, N, C).float()), seed, 1)


def make_student(teacher: ToyBlock, k_frac: float, top_p: float, dropout: float = 0.0) -> ToyBlock:
    """Alg. 2 steps 3-4: same weights, attention replaced by SpargeAttn2(., ., ., k%, p%); the teacher is frozen.  `dropout` is
    the student's (the teacher keeps its own)."""
    student = copy.deepcopy(teacher)
    student.k_frac, student.top_p, student._full, student.dropout = float(k_frac), float(top_p), None, float(dropout)
    for p in teacher.parameters():
        p.requires_grad_(False)
    return student


def noisy_latent(x1: torch.Tensor, x0: torch.Tensor, t: torch.Tensor) -> torch.Tensor:
    """x_t = t x_1 + (1 - t) x_0 (Alg. 2 step 7), t of shape [B]."""
    t = t.view(-1, *([1] * (x1.dim() - 1)))
    return t * x1 + (1.0 - t) * x0


class _VelocityDistillationLoss(torch.autograd.Function):
    """weight * ||u_sparse - u_full||^2 through the fused kernels: one pass for the loss, one for the gradient."""

    @staticmethod
    def forward(ctx, u_sparse, u_full, weight):
        u_full = u_full.detach()
        loss = torch.empty((), dtype=torch.float64, device=u_sparse.device)
        ws = torch.empty(_b.spa2_vd_loss_workspace_bytes(), dtype=torch.uint8, device=u_sparse.device)
        _b.spa2_vd_loss(u_sparse.detach(), u_full, weight, loss, ws)
        ctx.save_for_backward(u_sparse, u_full)
        ctx.weight = weight
        return loss

    @staticmethod
    def backward(ctx, upstream):
        u_sparse, u_full = ctx.saved_tensors
        grad = torch.empty_like(u_sparse)
        _b.spa2_vd_loss_grad(u_sparse.detach(), u_full, ctx.weight, upstream.contiguous(), grad)
        return grad, None, None


def velocity_distillation_loss(u_sparse: torch.Tensor, u_full: torch.Tensor, reduction: str = "mean") -> torch.Tensor:
    """L_VD = ||u_sparse - u_full||^2 (Sec. 4.2; Alg. 2), a float64 scalar.  `reduction`: "mean" divides by the
    number of elements; "batch" divides by the size of the leading dimension, which is the paper's expectation over
    training samples of the squared norm.  The teacher's prediction gets no gradient (it is frozen)."""
    if reduction == "mean":
        weight = 1.0 / u_sparse.numel()
    elif reduction == "batch":
        weight = 1.0 / u_sparse.shape[0]
    else:
        raise ValueError('reduction is "mean" or "batch"')
    if not u_sparse.is_cuda:
        raise ValueError("spa2 runs on the GPU only: predictions must be CUDA tensors")
    u_full = u_full.to(u_sparse.dtype)
    if _plain(u_sparse, u_full):
        return _operator().velocity_loss(u_sparse, u_full, weight)
    return _VelocityDistillationLoss.apply(u_sparse.contiguous(), u_full.contiguous(), weight)


def distill(student: torch.nn.Module, teacher: torch.nn.Module, batches: Iterable[Tuple[torch.Tensor, ...]],
            lr: float = 1e-3, on_step: Optional[Callable[[int, float], None]] = None) -> Dict[str, list]:
    """The loop of Alg. 2 over `batches` of (x_1, x_0, t): teacher and student see the same x_t, only the student
    is updated.  What a batch holds behind these three (a context and its lengths) both get too.  Returns the loss per step."""
    opt = torch.optim.Adam([p for p in student.parameters() if p.requires_grad], lr=lr)
    losses = []
    for step, (x1, x0, t, *more) in enumerate(batches):
        xt = noisy_latent(x1, x0, t)
        with torch.no_grad():
            u_full = teacher(xt, *more)
        loss = velocity_distillation_loss(student(xt, *more), u_full)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(float(loss.item()))
        if on_step is not None:
            on_step(step, losses[-1])
    return {"loss": losses}
