"""The operators around the block-sparse attention of a transformer block, differentiable:

* `qk_norm_rotate`   in front of it: the norm of every head of q and k and the rotation by position, in one pass
                     (`rotary_table` makes the tables of cosines and sines);
* `cross_attention`  beside it: dense attention to another sequence, a prompt or a cache, whose samples have lengths of
                     their own;
* `dropout_add`      behind it: dropout of a branch and the sum with the residual stream, the mask drawn from a counter-based
                     generator and never stored.

They take plain CUDA tensors, in eager mode and under HIP graph capture; tracing, compilation and function transforms are
refused, and so is a captured call with gradients while an eager graph of its inputs, made on the default stream, is alive
(PyTorch would end the process in the captured backward pass).  The C entry points are in `binding` under their C names.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence, Tuple, Union

import torch

from .autograd import _operator, _plain


def _refuse_others(name: str, *tensors: Optional[torch.Tensor]) -> None:
    given = [t for t in tensors if t is not None]
    if _plain(*given):
        return
    if not all(isinstance(t, torch.Tensor) for t in given):
        raise TypeError(f"{name} takes tensors")
    if not all(t.is_cuda for t in given):
        raise ValueError(f"{name} runs on the GPU only: it has no CPU path")
    raise RuntimeError(f"{name} takes plain CUDA tensors, outside tracing, compilation and function transforms")


def rotary_table(sizes: Union[int, Sequence[int]], d: int, theta: float = 10000.0,
                 device=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Cosines and sines, fp32 [tokens, d / 2], of the rotation of d channels.  `sizes`: the number of positions, or the
    extents of a grid whose tokens are numbered row by row (frames, height, width): the channel pairs are then shared out
    to the axes, evenly and what is left to the first, and each pair turns with its axis' coordinate.  Pair i of an
    axis' m turns by coordinate * theta^(-i / m); the angles are taken in 64 bits."""
    sizes = (int(sizes),) if isinstance(sizes, int) else tuple(int(s) for s in sizes)
    if not sizes or min(sizes) < 1 or d < 2 * len(sizes) or d % 2:
        raise ValueError("sizes are at least 1, d is even and has a channel pair for each axis")
    each = d // 2 // len(sizes)
    pairs = [d // 2 - each * (len(sizes) - 1)] + [each] * (len(sizes) - 1)
    angles = []
    for axis, (size, m) in enumerate(zip(sizes, pairs)):
        at = torch.arange(size, dtype=torch.float64, device=device)
        turn = at[:, None] * float(theta) ** (-torch.arange(m, dtype=torch.float64, device=device) / m)
        shape = [1] * len(sizes) + [m]
        shape[axis] = size
        angles.append(turn.reshape(shape).expand(*sizes, m))
    angle = torch.cat(angles, dim=-1).reshape(-1, d // 2)
    return angle.cos().float(), angle.sin().float()


def qk_norm_rotate(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor] = None,
                   k_weight: Optional[torch.Tensor] = None, cos: Optional[torch.Tensor] = None,
                   sin: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                   interleaved: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """Every head of q and k over its root mean square, times a weight per channel, rotated by its token's position.

    q [B, Hq, N, d], k [B, Hk, N, d]: bf16 or fp32 views with rows on 16-byte boundaries, d in {64, 128} contiguous; Hk may differ
    from Hq.
    q_weight, k_weight [d]: bf16 or fp32, or None.  cos, sin: fp32 [rows, r / 2], contiguous from a 16-byte boundary, for the
    rotation of the first r channels, r a multiple of 16 (None: no rotation); pair i is (i, i + r / 2), or (2 i, 2 i + 1) if
    `interleaved`.  positions: contiguous int32 or int64 [N] or [B, N], the row of the tables that a token uses (clamped to them);
    None: token n uses row n.
    Returns bf16 tensors of the shapes of q and k without gaps, tokens outside the heads where the inputs have them so: what
    `sparge_attn2` and `cross_attention` take.  Gradients: q, k (in their type) and the weights; tables that require one, or
    carry a tangent, are refused."""
    _refuse_others("qk_norm_rotate", q, k, q_weight, k_weight, cos, sin, positions)
    return _operator().norm_rotate(q, k, q_weight, k_weight, cos, sin, positions, float(eps), bool(interleaved))


def cross_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lengths: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None) -> torch.Tensor:
    """softmax(scale q k^T) v over the first lengths[b] keys of sample b (None: all of them).

    q [B, Hq, Nq, d], k, v [B, Hk, Nk, d]: bf16 views with rows on 16-byte boundaries, d in {64, 128} contiguous; Hq is a multiple
    of Hk, and query head h reads key head h // (Hq // Hk).  Any Nq, Nk >= 1: one query against a long cache as well as many against a short prompt.
    lengths: contiguous int32 [B] on the GPU, clamped to [0, Nk]; what lies behind them in k and v is not read, and a sample
    without keys gives zeros and zero gradients.  (Keys whose score is minus infinity take no part; a row with no other is NaN, as
    softmax has it.)  scale: 1 / sqrt(d) if None.  Returns bf16 with q's shape (and memory order).
    Gradients: q, k, v; those of k and v are zero behind the lengths and summed over the query heads in fp32.  (A q with gaps
    between its heads and v with other strides than k are copied first.)"""
    _refuse_others("cross_attention", q, k, v, lengths)
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1]) if q.dim() and q.shape[-1] else 1.0      # (those are refused there)
    return _operator().cross_attention(q, k, v, lengths, float(scale))


def _signed(x: int) -> int:
    x = int(x) % 2 ** 64
    return x - 2 ** 64 if x >= 2 ** 63 else x


def dropout_add(x: torch.Tensor, residual: Optional[torch.Tensor], p: float, seed: Union[int, torch.Tensor],
                offset: int = 0) -> torch.Tensor:
    """residual + dropout(x): x is kept with probability 1 - p and then divided by it (p taken to the nearest multiple of
    2^-16), and the result rounded once.

    x: bf16 or fp32 of any shape.  residual: None, or of x's shape and of its type or fp32; the result has its type.
    seed, offset: numbers of 64 bits; the mask is a function of them and of an element's number (row-major) alone, the same
    on every call.  A program counts one of them up from call to call.  `seed` may also be an int64 CUDA tensor (seed,
    offset), read when the kernels run: a captured graph then draws another mask on every replay, if the program changes the
    tensor between them (not between a forward pass and its backward pass, which autograd refuses outside graphs).
    Gradients: x, from the same mask drawn again, and residual."""
    on_device = seed if isinstance(seed, torch.Tensor) else None
    _refuse_others("dropout_add", x, residual, on_device)
    if on_device is not None and offset:
        raise ValueError("a seed on the device brings its offset along")
    return _operator().dropout_add(x, residual, float(p), 0 if on_device is not None else _signed(seed), _signed(offset),
                                   on_device)
