"""Algorithm 1 of the paper on ONE GPU: the query block visits N key/value blocks in turn.

The distributed schedule keeps each K/V block on its worker and passes (Q_j, O_j, L_j) around a
ring; each visit is FlashAttention(Q_j, K_i, V_i) followed by Rescale.  Here the send/recv steps
are dropped and the N blocks are N windows of one GPU's K/V tensors, so the loop is

    (O, L) <- (0, -inf);  for n in blocks:  (dO, dL) <- lvx_xattn_fwd(Q, K[n], V[n]);
                                             (O, L) <- lvx_xattn_merge((O, L), (dO, dL))

and the backward pass runs lvx_xattn_bwd once per block with the FINAL (O, L): dK/dV of a block
are complete after its call, dQ accumulates over blocks (no rescaling appears in backward).

This module only sequences C-ABI calls and owns the buffers between them (allocated once, in
the constructor, so the timed loop allocates nothing); all arithmetic is in the kernels.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import binding as B


@dataclass
class MediaMask:
    allow: torch.Tensor      # uint8 device tensor [n_q_chunks, n_kv_blocks] (or [B, ., .])
    q_chunk: int
    kv_block: int


def _covers(t: torch.Tensor, like: torch.Tensor) -> bool:
    """t has an element wherever `like` has one (addressed with like's strides and element size)."""
    return t.shape == like.shape and t.dtype == like.dtype or (
        t.dim() == like.dim() and t.element_size() == like.element_size()
        and all(a >= b for a, b in zip(t.shape, like.shape)))


def _same_strides(t: torch.Tensor, like: torch.Tensor) -> bool:
    """Equal where they address anything: the stride of a single batch or head does not."""
    return all(a == b for n, a, b in zip(like.shape, t.stride(), like.stride()) if n > 1)


def _apart(buf: torch.Tensor, *ts):
    """The tensors, as copies where they lie in `buf`: a result handed out that comes back as an input."""
    first, last = buf.data_ptr(), buf.data_ptr() + buf.numel() * buf.element_size()
    return tuple(t.new_empty_strided(t.size(), t.stride()).copy_(t.detach()) if first <= t.data_ptr() < last else t for t in ts)


class BlockLoop:
    def __init__(self, q_shape, kv_shape, dtype: torch.dtype, n_blocks: int = 1,
                 mask: Optional[MediaMask] = None, softmax_scale: float = 0.0,
                 device: str = "cuda", bwd_flags: int = 0):
        if not torch.cuda.is_available():
            raise RuntimeError("BlockLoop needs a GPU: there is no CPU fallback")
        B.load()
        self.Bsz, self.Hq, self.Sq, self.D = q_shape
        _, self.Hkv, self.Skv, _ = kv_shape
        assert self.Skv % n_blocks == 0, "blocks must be equal (the paper's Skv/n)"
        self.n_blocks = n_blocks
        self.bwd_flags = bwd_flags      # B.LVX_BWD_FUSED / B.LVX_BWD_SPLIT: which backward kernels (0: the library's choice)
        self.blk = self.Skv // n_blocks
        if mask is not None and n_blocks > 1:
            assert self.blk % mask.kv_block == 0, "block boundaries must fall on mask blocks"
        self.dtype, self.mask, self.scale, self.dev = dtype, mask, softmax_scale, device
        f32 = dict(dtype=torch.float32, device=device)
        rows = (self.Bsz, self.Hq, self.Sq)
        self.lse = torch.empty(rows, **f32)
        self.o = torch.empty(q_shape, dtype=dtype, device=device)
        # Running O_j of Algorithm 1 (L_j lives in self.lse) and the dQ sums.  Both are float32: a float32
        # problem's are its results already, with nothing left to round.  The last visit writes the results (float32: every
        # visit) while the inputs are still read, which _apart sees to where an input is an earlier result.
        self.dq_accum = torch.empty(q_shape, **f32)
        if dtype == torch.float32:
            self.o_acc, self.dq = self.o, self.dq_accum
        else:
            self.o_acc = torch.empty(q_shape, **f32) if n_blocks > 1 else None
            self.dq = torch.empty(q_shape, dtype=dtype, device=device)
        # one workspace sized for the larger of the two passes
        qd = torch.empty(q_shape, dtype=dtype, device="meta")
        kd = torch.empty((self.Bsz, self.Hkv, self.blk, self.D), dtype=dtype, device="meta")
        p = B.make_problem(qd, kd, softmax_scale)
        p.kv_sh = self.Skv * self.D
        p.kv_sb = self.Hkv * self.Skv * self.D
        code = B.dtype_code(dtype)
        nbytes = max(B.lvx_xattn_workspace_bytes(p, code, B.LVX_WS_FWD),
                     B.lvx_xattn_workspace_bytes(p, code, B.LVX_WS_FWD_MERGE),
                     B.lvx_xattn_workspace_bytes(p, code, B.LVX_WS_BWD))
        if nbytes == 0:
            raise B.LvxError(-2, "lvx_xattn_workspace_bytes")
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)

    def _mask_for(self, n: int) -> Optional[B.lvx_mask]:
        if self.mask is None:
            return None
        per = self.blk // self.mask.kv_block if self.n_blocks > 1 else 0
        nkb = (self.blk + self.mask.kv_block - 1) // self.mask.kv_block
        return B.make_mask(self.mask.allow, self.mask.q_chunk, self.mask.kv_block, n * per, nkb)

    def _blocks(self, q, k, like_k, like_q=()):
        """The problem that the blocks share (they differ in where their keys start and, the last one, in how
        many they are: _keys_of) and the bytes from one block's keys to the next's.  The library gets
        addresses: what it is told to read or write has to be there."""
        if not q.is_cuda:
            raise RuntimeError("BlockLoop needs device tensors")
        if not all(_covers(t, k) for t in like_k) or not all(_covers(t, q) for t in like_q):
            raise ValueError("V, dK and dV have to be as large as K; O and dO as large as Q")
        rows = q.shape[0] * q.shape[1] * q.shape[2]
        if rows > self.lse.numel() or 1 + sum((n - 1) * s for n, s in zip(q.shape, q.stride())) > self.o.numel():
            raise ValueError("Q is larger than this loop's results")
        return B.make_problem(q, k, self.scale), self.blk * k.stride(2) * k.element_size()

    def _keys_of(self, n: int, k) -> int:
        """Keys of block n: as many as K has left (a K shorter than the loop was made for ends earlier)."""
        return max(0, min(self.blk, k.shape[2] - n * self.blk))

    def forward(self, q, k, v) -> Tuple[torch.Tensor, torch.Tensor]:
        """Returns (O in the input dtype, L float32); both are buffers owned by this object."""
        # (the running O of the block loop is written with Q's strides by the first visit and read as
        # a contiguous tensor by the others)
        assert self.n_blocks == 1 or q.is_contiguous(), "the block loop needs a contiguous Q"
        p, step = self._blocks(q, k, (v,))
        if self.n_blocks > 1:
            q, k, v = _apart(self.o, q, k, v)
        call = B.Calls(p, q.dtype, self.ws)
        qp, kp, vp, lp = q.data_ptr(), k.data_ptr(), v.data_ptr(), self.lse.data_ptr()
        if self.n_blocks == 1:
            call.fwd(qp, kp, vp, self._mask_for(0), self.o.data_ptr(), self.o.dtype, lp)
            return self.o, self.lse
        op = self.o_acc.data_ptr()
        p.Skv = self._keys_of(0, k)
        # merging with the identity (0, -inf) is a no-op: the first visit writes the state directly
        call.fwd(qp, kp, vp, self._mask_for(0), op, torch.float32, lp)
        for n in range(1, self.n_blocks):       # the FlashAttention call and Rescale of Algorithm 1 in one call
            p.Skv = self._keys_of(n, k)
            if n == self.n_blocks - 1 and self.o_acc is not self.o:          # ... which rounds to the output dtype, the last time
                call.fwd_merge_last(qp, kp + n * step, vp + n * step, self._mask_for(n), op, lp, self.o.data_ptr())
            else:
                call.fwd_merge(qp, kp + n * step, vp + n * step, self._mask_for(n), op, lp)
        return self.o, self.lse

    def backward(self, q, k, v, o, lse, d_o, dk, dv) -> torch.Tensor:
        """dk/dv (same shape and strides as k) are overwritten; returns dQ in the input dtype."""
        assert dk.stride() == k.stride() and dv.stride() == k.stride() and _same_strides(v, k)
        assert o.stride() == q.stride() and d_o.stride() == q.stride()
        p, step = self._blocks(q, k, (v, dk, dv), (o, d_o))
        if lse.numel() < q.shape[0] * q.shape[1] * q.shape[2]:
            raise ValueError("L has to have a value for every row of Q")
        q, k, v, o, lse, d_o = _apart(self.dq, q, k, v, o, lse, d_o)
        call = B.Calls(p, q.dtype, self.ws)
        qp, kp, vp, dkp, dvp = q.data_ptr(), k.data_ptr(), v.data_ptr(), dk.data_ptr(), dv.data_ptr()
        op, lp, gp, ap = o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), self.dq_accum.data_ptr()
        if not self.bwd_flags & B.LVX_BWD_FUSED:
            # (the first visit overwrites the dQ sums and leaves delta in the workspace, the last one rounds the sums)
            last = self.dq.data_ptr() if self.dq is not self.dq_accum else None
            for n in range(self.n_blocks):
                p.Skv = self._keys_of(n, k)
                call.bwd_visit(qp, kp + n * step, vp + n * step, op, lp, gp, self._mask_for(n), ap, dkp + n * step, dvp + n * step,
                               n == 0, last if n == self.n_blocks - 1 else None)
            return self.dq
        self.dq_accum.zero_()
        for n in range(self.n_blocks):
            # delta = rowsum(dO * O) depends on the query block only: the first visit computes it
            # into the workspace, the others reuse it
            stages = (B.LVX_BWD_ALL if n == 0 else (B.LVX_BWD_DKDV | B.LVX_BWD_DQ)) | self.bwd_flags
            p.Skv = self._keys_of(n, k)
            call.bwd(qp, kp + n * step, vp + n * step, op, lp, gp, self._mask_for(n), ap, dkp + n * step, dvp + n * step, stages)
        if self.dq is not self.dq_accum:
            B.lvx_xattn_dq_finalize(p, self.dq_accum, self.dq)
        return self.dq


@dataclass
class Norm:
    """The weights of a norm of token features: gamma and (or None) beta, [E], of the features' type."""
    gamma: torch.Tensor
    beta: Optional[torch.Tensor] = None


class _Features:
    """n tokens of E features on their way into a product, `at_once` at a time: normalised (norm = "layer" or "rms"), kept in 8 bits
    (packed), or both; made again for the backward pass, from their 8-bit form where they have one.  With neither they pass through."""

    def __init__(self, n, E, at_once, dtype, norm, packed, eps, device):
        if norm not in (None, "layer", "rms"):
            raise ValueError('norm is None, "layer" or "rms"')
        self.norm, self.eps, self.rms = norm, eps, norm == "rms"
        self.packed = B.Packed(n, E, device) if packed else None
        self.plain = norm is None and not packed
        if not self.plain:
            self.out = torch.empty((at_once, E), dtype=dtype, device=device)
        if norm is not None:
            self.stats = torch.empty((n, 2), dtype=torch.float32, device=device)
            self.dparam = torch.empty((2, E), dtype=torch.float32, device=device)
            self.ws = torch.empty(B.lvx_norm_workspace_bytes(at_once, E), dtype=torch.uint8, device=device)

    def _check(self, weights):
        if (weights is None) != (self.norm is None):
            raise ValueError("a norm's weights are given where there is a norm, and only there")

    def forward(self, t, first, shape, weights):
        """The features of the tokens t (`shape`, the first of them is token `first` of n); t None: of what was packed before."""
        self._check(weights)
        if t is None and self.packed is None:
            raise ValueError("only packed features can be made again from nothing")
        if self.plain:
            return t
        n = shape.numel() // shape[-1]
        out = self.out[:n].view(shape)
        pk = self.packed.rows(first, first + n) if self.packed is not None else None
        if self.norm is not None:
            B.lvx_norm_fwd(t, weights.gamma, weights.beta, out, self.stats[first:first + n], self.rms, self.eps, pk)
            return out
        if t is not None:
            B.lvx_pack(t, pk)
        B.lvx_unpack(pk, out)
        return out

    def again(self, t, first, shape, weights):
        """The same features once more, bit for bit (t is not read where they are packed)."""
        return self.forward(t if self.packed is None else None, first, shape, weights)

    def check_rows(self, t, name):
        """The backward pass writes gradients whose rows follow each other, with the strides of the tokens that it reads."""
        if self.packed is None and t is not None and not t.is_contiguous():
            raise ValueError(f"backward: {name} has to be contiguous (a window of a wider tensor: packed layers do not read it again)")

    def start_backward(self):
        if self.norm is not None:
            self.dparam.zero_()

    def backward(self, t, first, weights, grad):
        """grad, the gradient of the features, becomes that of the tokens in place; the norm's weights' gradients are added up."""
        if self.norm is None:
            return
        n = grad.numel() // grad.shape[-1]
        pk = self.packed.rows(first, first + n) if self.packed is not None else None
        B.lvx_norm_bwd(t if pk is None else None, weights.gamma, self.stats[first:first + n], grad, grad, self.dparam[0],
                       self.dparam[1] if weights.beta is not None else None, self.ws, self.rms, self.eps, pk)

    def gradients(self, weights):
        return () if self.norm is None else (self.dparam[0], self.dparam[1] if weights.beta is not None else None)


class RecomputeLayer:
    """One cross-attention layer under the activation recomputation of Section 3.2, on one GPU: the
    forward pass keeps the token features x, y and (O, L) and nothing else; the backward pass makes
    Q again from x and, block by block, K and V again from the block's visual tokens, runs the
    attention backward on them, and carries dQ, dK, dV on through the projections to dx, dy and the
    weights' gradients.  K and V exist for one block at a time.

    x [B, Sq, E] text tokens, y [B, Skv, E] visual tokens (B > 1: n_blocks must be 1, the
    projection entry points want the batches of a call to follow each other), wq [Hq D, E],
    wkv [2 Hkv D, E] (W_K^T on top of W_V^T).  The forward pass reads x and y as windows of wider tensors too; the backward
    pass asks for contiguous ones, where it reads them again (not where the layer keeps them packed).  Only sequences C-ABI calls.

    norm = "layer" or "rms": the projections read the norm of x and of y; forward and backward take the two norms'
    weights, and backward returns their gradients behind the others.
    packed: the layer keeps x and y in 8 bits (33 / 64 of their bf16 size) and the caller need not: the forward pass works from
    the values that these stand for, so what the backward pass makes again from them, x and y None, is the forward
    pass's bit for bit.  The gradients are those with respect to these values.

    With norm or packed the object also owns room for the features of x and of one block of y that the projections read (with n_blocks = 1: of
    all of y), in either case dx and dy.  What packing saves is the caller's copy of x and y, where nobody else needs it: one such object a layer
    keeps 33 / 64 of a copy each, and layers that read the same y may share the caller's one copy instead."""

    def __init__(self, Bsz, Sq, Skv, E, Hq, Hkv, D, dtype: torch.dtype, n_blocks: int = 1,
                 softmax_scale: float = 0.0, device: str = "cuda", norm: Optional[str] = None, packed: bool = False,
                 eps: float = 1e-5):
        assert Skv % n_blocks == 0 and (Bsz == 1 or n_blocks == 1)
        self.n_blocks, self.blk = n_blocks, Skv // n_blocks
        self.loop = BlockLoop((Bsz, Hq, Sq, D), (Bsz, Hkv, self.blk, D), dtype, 1, None, softmax_scale, device)
        kw = dict(dtype=dtype, device=device)
        self.q = torch.empty((Bsz, Hq, Sq, D), **kw)
        self.k = torch.empty((Bsz, Hkv, self.blk, D), **kw)
        self.v = torch.empty_like(self.k)
        self.dk, self.dv = torch.empty_like(self.k), torch.empty_like(self.k)
        self.o_acc = torch.empty((Bsz, Hq, Sq, D), dtype=torch.float32, device=device)
        self.dx = torch.empty((Bsz, Sq, E), **kw)
        self.dy = torch.empty((Bsz, Skv, E), **kw)
        self.dwq = torch.empty((Hq * D, E), dtype=torch.float32, device=device)
        self.dwkv = torch.empty((2 * Hkv * D, E), dtype=torch.float32, device=device)
        self.fx = _Features(Bsz * Sq, E, Bsz * Sq, dtype, norm, packed, eps, device)
        self.fy = _Features(Bsz * Skv, E, Bsz * self.blk, dtype, norm, packed, eps, device)

    def _kv_of_block(self, y, wkv, n, norm_y, again=False):
        """The block's tokens and their features, of which K and V are made."""
        yb = y[:, n * self.blk:(n + 1) * self.blk] if y is not None else None
        shape = torch.Size((self.dy.shape[0], self.blk, self.dy.shape[2]))
        feat = (self.fy.again if again else self.fy.forward)(yb, n * self.blk, shape, norm_y)
        B.lvx_xattn_project(feat, wkv, [self.k, self.v])
        return yb, feat

    def forward(self, x, y, wq, wkv, norm_x: Optional[Norm] = None, norm_y: Optional[Norm] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(O in the input dtype, L float32); Q, K, V are not kept."""
        lp = self.loop
        B.lvx_xattn_project(self.fx.forward(x, 0, self.dx.shape, norm_x), wq, [self.q])
        p = B.make_problem(self.q, self.k, lp.scale)
        for n in range(self.n_blocks):
            self._kv_of_block(y, wkv, n, norm_y)
            if self.n_blocks == 1:
                B.lvx_xattn_fwd(p, self.q, self.k, self.v, None, lp.o, lp.lse, lp.ws)
                return lp.o, lp.lse
            if n == 0:
                B.lvx_xattn_fwd(p, self.q, self.k, self.v, None, self.o_acc, lp.lse, lp.ws)
            elif n < self.n_blocks - 1 or self.q.dtype == torch.float32:
                B.lvx_xattn_fwd_merge(p, self.q, self.k, self.v, None, self.o_acc, lp.lse, lp.ws)
            else:
                B.lvx_xattn_fwd_merge_last(p, self.q, self.k, self.v, None, self.o_acc, lp.lse, lp.o, lp.ws)
                return lp.o, lp.lse
        B.lvx_xattn_merge([self.o_acc], [lp.lse], lp.o, lp.lse)
        return lp.o, lp.lse

    def backward(self, x, y, wq, wkv, o, lse, d_o, norm_x: Optional[Norm] = None, norm_y: Optional[Norm] = None):
        """(dx, dy in the input dtype, dW_Q, dW_KV float32) from x, y (None where the layer keeps them packed), (O, L) and dO alone;
        with norms followed by the gradients (float32, or None) of norm_x's gamma and beta and of norm_y's."""
        lp = self.loop
        self.fx.check_rows(x, "x")
        self.fy.check_rows(y, "y")
        feat_x = self.fx.again(x, 0, self.dx.shape, norm_x)
        B.lvx_xattn_project(feat_x, wq, [self.q])                  # Q again
        self.dwq.zero_()
        self.dwkv.zero_()
        self.fx.start_backward()
        self.fy.start_backward()
        p = B.make_problem(self.q, self.k, lp.scale)
        last = lp.dq if lp.dq is not lp.dq_accum else None
        for n in range(self.n_blocks):
            yb, feat = self._kv_of_block(y, wkv, n, norm_y, again=True)       # K, V of the block again
            B.lvx_xattn_bwd_visit(p, self.q, self.k, self.v, o, lse, d_o, None, lp.dq_accum, self.dk, self.dv, lp.ws, n == 0,
                                  last if n == self.n_blocks - 1 else None)
            dyb = self.dy[:, n * self.blk:(n + 1) * self.blk]
            B.lvx_xattn_project_bwd(feat, wkv, [self.dk, self.dv], dx=dyb, dw=self.dwkv)
            self.fy.backward(yb, n * self.blk, norm_y, dyb)
        B.lvx_xattn_project_bwd(feat_x, wq, [lp.dq], dx=self.dx, dw=self.dwq)
        self.fx.backward(x, 0, norm_x, self.dx)
        return (self.dx, self.dy, self.dwq, self.dwkv) + self.fx.gradients(norm_x) + self.fy.gradients(norm_y)


class LossHead:
    """The end of a training step on one GPU: the norm of the last hidden features (norm = "layer" or "rms", or None), their product
    with a vocabulary's weights, and the cross entropy of every token, without the logits.  Between the passes it keeps the norm's
    statistics and lse, and (packed) the features in 8 bits, so that the caller need not keep them; the rest is made again.

    h [n, E] or [B, S, E], contiguous, w [V, E], labels int64 (negative: the token takes no part).  Only sequences C-ABI calls."""

    def __init__(self, n, E, V, dtype: torch.dtype, norm: Optional[str] = None, packed: bool = False, eps: float = 1e-5,
                 device: str = "cuda"):
        if not torch.cuda.is_available():
            raise RuntimeError("LossHead needs a GPU: there is no CPU fallback")
        nbytes = B.lvx_xent_workspace_bytes(n, E, V, B.dtype_code(dtype))
        if nbytes == 0:
            raise B.LvxError(-2, "lvx_xent_workspace_bytes")
        self.f = _Features(n, E, n, dtype, norm, packed, eps, device)
        self.ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.loss = torch.empty(n, dtype=torch.float32, device=device)
        self.lse = torch.empty(n, dtype=torch.float32, device=device)
        self.dh = torch.empty((n, E), dtype=dtype, device=device)
        self.dw = torch.empty((V, E), dtype=dtype, device=device)

    def _tokens(self, h):
        if h is None:
            return None
        if h.numel() != self.dh.numel() or h.shape[-1] != self.dh.shape[1] or not h.is_contiguous():
            raise ValueError("h has to be contiguous, of as many tokens and features as this object was made for")
        return h.view(self.dh.shape)

    def forward(self, h, w, labels, norm: Optional[Norm] = None) -> torch.Tensor:
        """The tokens' losses (float32 [n], a buffer of this object; 0 without a label)."""
        feat = self.f.forward(self._tokens(h), 0, self.dh.shape, norm)
        B.lvx_xent_fwd(feat, w, labels, self.loss, self.lse, self.ws)
        return self.loss

    def backward(self, h, w, labels, d_loss, norm: Optional[Norm] = None):
        """(dh [n, E], dw in the input dtype) of sum(loss * d_loss), d_loss float32 [n]; h None where it is kept packed.  With a norm
        followed by the gradients (float32, or None) of its gamma and beta."""
        h = self._tokens(h)
        feat = self.f.again(h, 0, self.dh.shape, norm)
        self.f.start_backward()
        B.lvx_xent_bwd(feat, w, labels, self.lse, d_loss, self.dh, self.dw, self.ws)
        self.f.backward(h, 0, norm, self.dh)
        return (self.dh, self.dw) + self.f.gradients(norm)
