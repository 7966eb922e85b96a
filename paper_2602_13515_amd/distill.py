"""Adapting a model to SpargeAttention2 by velocity distillation (Sec. 4.2; Alg. 2), on a toy scale.

The paper fine-tunes video diffusion models whose weights are not available here; what can be exercised
without them is the training step itself: a frozen teacher with full attention, a student that shares its
initialisation and differs only in the attention operator, identical noisy inputs x_t = t x_1 + (1 - t) x_0
for both, and the loss ||u_sparse - u_full||^2 back-propagated through the block-sparse backward kernels.
`ToyBlock` is one pre-norm attention block that stands in for the velocity network; on request with what such a network has
around its attention: the norm of q and k with the rotation by position, attention to a prompt, dropout of its branches, gates and
modulated norms; the student's attention may be one over a window instead, and the loop clips the gradients, on request.
"""
from __future__ import annotations

import copy
from typing import Callable, Dict, Iterable, Optional, Sequence, Tuple, Union

import torch

from . import binding as _b
from .autograd import _operator, _plain, sparge_attn2
from .block import cross_attention, dropout_add, gate_add_norm, qk_norm_rotate, rotary_table, window_attention
from .gradients import clip_gradients

Window = Tuple[Optional[int], Optional[int], int]


class ToyBlock(torch.nn.Module):
    """x -> x + proj(attention(norm(x))): fp32 parameters, bf16 attention on [B, N, H, d] activations that reach
    the kernels as permuted views (no copy).  `k_frac`, `top_p` None means full attention (the teacher).

    grid: extents of the tokens' grid (frames, height, width): the heads of q and k are normed and rotated by position.
    context_dim: a second branch attends to `context` [B, M, context_dim], of which sample b has `lengths[b]` rows (a batch of
    prompts, padded).  dropout: of both branches, in training mode; the masks' seed comes from PyTorch's default generator, in
    a captured step from the GPU's, so that every replay draws other masks.

    window: (left, right, sinks) of `window_attention`, which then takes the place of the block-sparse attention.  gated: each
    branch is added through a gate, a vector that is learnt, in the pass that norms the sum for the next branch
    (`gate_add_norm`).  condition_dim: with `gated`, each sample's gates, and a scale and a shift of its norms, come from a
    projection of `condition` [B, condition_dim] instead."""

    def __init__(self, dim: int, heads: int, k_frac: Optional[float] = None, top_p: Optional[float] = None,
                 grid: Optional[Sequence[int]] = None, context_dim: Optional[int] = None, dropout: float = 0.0,
                 window: Optional[Window] = None, gated: bool = False, condition_dim: Optional[int] = None):
        super().__init__()
        assert condition_dim is None or gated
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
        self.window, self.gated, self.condition_dim = window, gated, condition_dim
        branches = 1 if context_dim is None else 2
        if condition_dim is not None:         # (gate, scale and shift of each branch)
            self.modulation = torch.nn.Linear(condition_dim, 3 * branches * dim)
        elif gated:
            self.gates = torch.nn.Parameter(torch.ones(branches, dim))
        self._full = None                     # the all-ones pattern, built once per input shape

    def _attention(self, q, k, v):
        if self.window is not None:
            return window_attention(q, k, v, *self.window)
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

    def _modulated(self, condition: Optional[torch.Tensor]) -> Sequence[Tuple[Optional[torch.Tensor], ...]]:
        """(gate, scale, shift) of each branch."""
        if self.condition_dim is None:
            return [(gate, None, None) for gate in self.gates]
        return list(zip(*[iter(self.modulation(condition).chunk(3 * (1 if self.context_dim is None else 2), dim=-1))] * 3))

    def _self_branch(self, h: torch.Tensor) -> torch.Tensor:
        """Of the normed tokens h: attention among them, projected."""
        B, N, C = h.shape
        d = C // self.heads
        qkv = self.qkv(h)
        if self.grid is None:
            qkv = qkv.to(torch.bfloat16).view(B, N, 3, self.heads, d)
            q, k, v = (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3))         # [B, H, N, d] views
        else:                                 # (the norm reads the projection in fp32 and writes what the attention takes)
            q, k, v = (t.permute(0, 2, 1, 3) for t in qkv.view(B, N, 3, self.heads, d).unbind(2))
            q, k = qk_norm_rotate(q, k, self.q_weight, self.k_weight, self.cos, self.sin, interleaved=True)
            v = v.to(torch.bfloat16)
        o = self._attention(q, k, v)                                            # strides of q
        return self.proj(o.permute(0, 2, 1, 3).reshape(B, N, C).float())

    def _context_branch(self, h: torch.Tensor, context: torch.Tensor, lengths: Optional[torch.Tensor]) -> torch.Tensor:
        B, N, C = h.shape
        d = C // self.heads
        q = self.context_q(h).to(torch.bfloat16).view(B, N, self.heads, d).permute(0, 2, 1, 3)
        k, v = (t.permute(0, 2, 1, 3) for t in
                self.context_kv(context).to(torch.bfloat16).view(B, -1, 2, self.heads, d).unbind(2))
        o = cross_attention(q, k, v, lengths)
        return self.context_proj(o.permute(0, 2, 1, 3).reshape(B, N, C).float())

    def _dropped(self, branch: torch.Tensor, seed: Union[None, int, torch.Tensor], number: int) -> torch.Tensor:
        if seed is None:
            return branch
        return dropout_add(branch, None, self.dropout, *((seed, number) if isinstance(seed, int) else (seed[number],)))

    def _gated_forward(self, x, context, lengths, condition) -> torch.Tensor:
        seed = self._seed(x)
        mods, norm = self._modulated(condition), self.norm
        gate, scale, shift = mods[0]
        _, h = gate_add_norm(x, weight=norm.weight, bias=norm.bias, scale=scale, shift=shift, eps=norm.eps)
        branch = self._dropped(self._self_branch(h), seed, 0)
        if self.context_dim is None:
            return gate_add_norm(x, branch, gate, kind=None)[0]
        norm, (next_gate, scale, shift) = self.context_norm, mods[1]
        x, h = gate_add_norm(x, branch, gate, weight=norm.weight, bias=norm.bias, scale=scale, shift=shift, eps=norm.eps)
        branch = self._dropped(self._context_branch(h, context, lengths), seed, 1)
        return gate_add_norm(x, branch, next_gate, kind=None)[0]

    def forward(self, x: torch.Tensor, context: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                condition: Optional[torch.Tensor] = None) -> torch.Tensor:
        if self.gated:
            return self._gated_forward(x, context, lengths, condition)
        seed = self._seed(x)
        x = self._add(x, self._self_branch(self.norm(x)), seed, 0)
        if self.context_dim is None:
            return x
        return self._add(x, self._context_branch(self.context_norm(x), context, lengths), seed, 1)


def make_student(teacher: ToyBlock, k_frac: Optional[float], top_p: Optional[float], dropout: float = 0.0,
                 window: Optional[Window] = None) -> ToyBlock:
    """Alg. 2 steps 3-4: same weights, attention replaced by SpargeAttn2(., ., ., k%, p%), or by attention over a window (k_frac and
    top_p are then not looked at); the teacher is frozen.  `dropout` is the student's (the teacher keeps its own)."""
    student = copy.deepcopy(teacher)
    student._full, student.dropout, student.window = None, float(dropout), window
    if window is None:
        student.k_frac, student.top_p = float(k_frac), float(top_p)
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
            lr: float = 1e-3, on_step: Optional[Callable[[int, float], None]] = None,
            max_norm: Optional[float] = None) -> Dict[str, list]:
    """The loop of Alg. 2 over `batches` of (x_1, x_0, t): teacher and student see the same x_t, only the student
    is updated.  What a batch holds behind these three (a context, its lengths, a condition) both get too.  max_norm: the gradients are
    clipped to it before every update.  Returns the loss per step, and with max_norm the gradients' norm ("norm")."""
    opt = torch.optim.Adam([p for p in student.parameters() if p.requires_grad], lr=lr)
    losses, norms = [], []
    for step, (x1, x0, t, *more) in enumerate(batches):
        xt = noisy_latent(x1, x0, t)
        with torch.no_grad():
            u_full = teacher(xt, *more)
        loss = velocity_distillation_loss(student(xt, *more), u_full)
        opt.zero_grad(set_to_none=True)
        loss.backward()
        if max_norm is not None:
            norms.append(clip_gradients([p.grad for p in student.parameters() if p.grad is not None], max_norm))
        opt.step()
        losses.append(float(loss.item()))
        if on_step is not None:
            on_step(step, losses[-1])
    return {"loss": losses} if max_norm is None else {"loss": losses, "norm": [float(n) for n in norms]}
