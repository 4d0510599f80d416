"""Sequencing of the library calls for a multi-level encoder (conv3x3x3 -> ReLU -> 2x2x2
max-pool per level) and for an attention block on a level, forward and backward.  Only call order and buffer ownership live here;
every arithmetic step is a call into libhch.so."""
from __future__ import annotations

import torch

from . import binding as B


def _aligned_bytes(nbytes, device):
    t = torch.empty(int(nbytes) + 256, dtype=torch.uint8, device=device)
    off = (-t.data_ptr()) % 256
    return t[off: off + int(nbytes)]


class Encoder:
    """channels = [c0, c1, ..., cL]: level l runs conv c_l -> c_{l+1}, ReLU, pool to level l+1.
    `levels` must hold L+1 levels.  All buffers are allocated once here."""

    def __init__(self, levels, channels, algo=B.HCH_ALGO_COLUMNS, device="cuda", fuse_pointwise=True,
                 two_streams=False, keep_columns=True):
        self.levels, self.channels, self.algo = levels, list(channels), algo
        # columns algorithm: every level keeps the column matrix of its forward pass (1 GB in all
        # for the 256^3 x 8 workload) and the weight gradient reads it instead of gathering again
        self.keep_columns = keep_columns and algo == B.HCH_ALGO_COLUMNS
        self.fuse_pointwise = fuse_pointwise       # ReLU+pool (and their backward) as one call each
        # backward: the weight gradient of a level runs on a second stream (default priority)
        # beside the data gradient; both only read dY of that level
        self.two_streams = two_streams
        self.L = len(channels) - 1
        assert levels.n_levels >= self.L + 1
        self.n = [levels.n(l) for l in range(self.L + 1)]
        f32 = dict(dtype=torch.float32, device=device)
        ch = self.channels
        self.X = [torch.empty((self.n[l], ch[l]), **f32) for l in range(self.L + 1)]    # level inputs
        self.Y = [torch.empty((self.n[l], ch[l + 1]), **f32) for l in range(self.L)]    # conv outputs
        # the rectified rows are kept only when ReLU and pooling run as separate calls: the
        # fused calls take the sign for the backward pass from Y
        self.A = [None if fuse_pointwise else torch.empty((self.n[l], ch[l + 1]), **f32)
                  for l in range(self.L)]
        self.sw = [torch.empty((self.n[l + 1], ch[l + 1]), dtype=torch.int32, device=device)
                   for l in range(self.L)]
        self.W = [torch.empty((27, ch[l], ch[l + 1]), **f32) for l in range(self.L)]
        self.dW = [torch.empty((27, ch[l], ch[l + 1]), **f32) for l in range(self.L)]
        self.dX = [torch.empty((self.n[l], ch[l]), **f32) for l in range(self.L + 1)]   # dX[L] = upstream
        self.dA = [None if fuse_pointwise else torch.empty((self.n[l], ch[l + 1]), **f32)
                   for l in range(self.L)]
        self.dY = [torch.empty((self.n[l], ch[l + 1]), **f32) for l in range(self.L)]
        need = 256
        for l in range(self.L):
            for kind in (B.HCH_WS_FWD, B.HCH_WS_BWD_DATA, B.HCH_WS_BWD_WEIGHT):
                need = max(need, B.hch_conv_workspace_bytes(levels, l, ch[l], ch[l + 1], B.HCH_F32, kind, algo))
        self.ws = _aligned_bytes(need, device)
        self.ws_col = None
        if self.keep_columns:
            self.ws_col = [_aligned_bytes(max(B.hch_conv_workspace_bytes(levels, l, ch[l], ch[l + 1], B.HCH_F32, k, algo)
                                              for k in (B.HCH_WS_FWD, B.HCH_WS_BWD_WEIGHT)), device)
                           for l in range(self.L)]
        if two_streams:
            need_w = max(B.hch_conv_workspace_bytes(levels, l, ch[l], ch[l + 1], B.HCH_F32, B.HCH_WS_BWD_WEIGHT, algo)
                         for l in range(self.L))
            self.ws_side = _aligned_bytes(max(256, need_w), device)
            self.side = torch.cuda.Stream(device=device)
            self.ready = [torch.cuda.Event() for _ in range(self.L)]
            self.begin, self.coarse_ready = torch.cuda.Event(), torch.cuda.Event()

    def flops_per_step(self):
        """paper-method count: forward, data-gradient and weight-gradient products, each
        2 * 27 * c_in * c_out * N_l."""
        return sum(3 * 2 * 27 * self.channels[l] * self.channels[l + 1] * self.n[l] for l in range(self.L))

    def build_indices(self):
        if not self.two_streams:
            if self.algo == B.HCH_ALGO_COLUMNS:       # its products take the voxels as they come: no row orders
                B.hch_build_index_lists(self.levels, 0, self.levels.n_levels)
            else:
                B.hch_build_neighbours(self.levels, -1)
            return
        # the finest level's lists on the main stream, the coarser levels' beside it; the main
        # stream picks them up before the first pooling (forward)
        main = torch.cuda.current_stream()
        self.begin.record(main)
        self.side.wait_event(self.begin)          # the side stream's previous work is in order anyway
        B.hch_build_neighbours_range(self.levels, 0, 1)
        B.hch_build_neighbours_range(self.levels, 1, self.levels.n_levels - 1, stream=self.side.cuda_stream)
        self.coarse_ready.record(self.side)

    def forward(self):
        ch = self.channels
        for l in range(self.L):
            B.hch_conv_fwd(self.levels, l, B.HCH_F32, self.X[l], self.W[l], self.Y[l], ch[l], ch[l + 1],
                           self.ws_col[l] if self.keep_columns else self.ws, self.algo)
            if l == 0 and self.two_streams:
                torch.cuda.current_stream().wait_event(self.coarse_ready)
            if self.fuse_pointwise:
                B.hch_relu_pool_fwd(self.levels, l, self.Y[l], None, self.X[l + 1], self.sw[l], ch[l + 1])
            else:
                B.hch_relu_fwd(self.Y[l], self.A[l], self.A[l].numel())
                B.hch_pool_fwd(self.levels, l, self.A[l], self.X[l + 1], self.sw[l], ch[l + 1])

    def backward(self):
        ch = self.channels
        main = torch.cuda.current_stream()
        for l in reversed(range(self.L)):
            if self.fuse_pointwise:
                B.hch_pool_relu_bwd_pooled(self.levels, l, self.dX[l + 1], self.sw[l], self.X[l + 1], self.dY[l], ch[l + 1])
            else:
                B.hch_pool_bwd(self.levels, l, self.dX[l + 1], self.sw[l], self.dA[l], ch[l + 1])
                B.hch_relu_bwd(self.A[l], self.dA[l], self.dY[l], self.dY[l].numel())
            walgo = B.HCH_ALGO_COLUMNS_RESIDENT if self.keep_columns else self.algo
            if self.two_streams:
                self.ready[l].record(main)
                self.side.wait_event(self.ready[l])
                B.hch_conv_bwd_weight(self.levels, l, B.HCH_F32, self.X[l], self.dY[l], self.dW[l], ch[l], ch[l + 1],
                                      self.ws_col[l] if self.keep_columns else self.ws_side, walgo,
                                      stream=self.side.cuda_stream)
            else:
                B.hch_conv_bwd_weight(self.levels, l, B.HCH_F32, self.X[l], self.dY[l], self.dW[l], ch[l], ch[l + 1],
                                      self.ws_col[l] if self.keep_columns else self.ws, walgo)
            B.hch_conv_bwd_data(self.levels, l, B.HCH_F32, self.dY[l], self.W[l], self.dX[l], ch[l], ch[l + 1], self.ws,
                                self.algo)
        if self.two_streams:
            main.wait_stream(self.side)     # the next pass overwrites what the side stream reads

    def step(self):
        """One pass of the whole hot path: index lists by hash lookup, forward, backward."""
        self.build_indices()
        self.forward()
        self.backward()


def _by_eights(n, width, dtype, device):
    """An empty [n][width] tensor, and its memory as rows of 8 elements (a few more than there are)."""
    t = torch.empty(((n * width + 7) // 8, 8), dtype=dtype, device=device)
    return t.view(-1)[: n * width].view(n, width), t


class AttentionBlock:
    """A pre-norm attention block over the voxels of one level, each shape by itself, forward and backward:

        h = norm1(X);  q, k, v = h Wqkv with rotary positions from the voxels;  S = X + attention(q, k, v) Wo;  Y = norm2(S)

    S is the block's result on the residual path, Y what the next layer takes.  X, S, Y and all gradients
    of them are fp32 [n][channels]; with dtype = HCH_BF16 what goes into products is bf16.  The linear layers are
    convolutions with F = 1.  `sections`: pairs of a head turned by x, y and z (default: a third each).  All buffers are
    allocated once here; key_mask (bytes, nonzero = seen) may be set between passes."""

    def __init__(self, levels, level, channels, heads_q, heads_kv, head_dim, dtype=B.HCH_F32, sections=None, base=10000.0,
                 eps=1e-5, device="cuda"):
        self.levels, self.level, self.c, self.dtype = levels, level, channels, dtype
        self.hq, self.hkv, self.d, self.eps, self.base = heads_q, heads_kv, head_dim, eps, base
        third = head_dim // 6
        self.sections = (head_dim // 2 - 2 * third, third, third) if sections is None else tuple(sections)
        self.scale = head_dim ** -0.5
        n = self.n = levels.n(level)
        self.wide = (heads_q + 2 * heads_kv) * head_dim
        wq, wk, c = heads_q * head_dim, heads_kv * head_dim, channels
        f32 = dict(dtype=torch.float32, device=device)
        t = dict(dtype=torch.bfloat16 if dtype == B.HCH_BF16 else torch.float32, device=device)
        self.offsets, self.positions = levels.device_offsets(level, device), levels.device_positions(level, device)
        self.key_mask = None
        self.field = torch.empty((n, 1), dtype=torch.int32, device=device)
        self.field_t = torch.empty((n, 1), dtype=torch.int32, device=device)
        B.hch_field_build(levels, level, 1, 1, 0, self.field, self.field_t)
        # weights (in the products' type) and their gradients
        self.gamma, self.beta = [torch.ones(c, **f32) for _ in range(2)], [torch.zeros(c, **f32) for _ in range(2)]
        self.Wqkv, self.Wo = torch.empty((1, c, self.wide), **t), torch.empty((1, wq, c), **t)
        self.dgamma, self.dbeta = [torch.empty(c, **f32) for _ in range(2)], [torch.empty(c, **f32) for _ in range(2)]
        self.dWqkv, self.dWo = torch.empty((1, c, self.wide), **f32), torch.empty((1, wq, c), **f32)
        # forward
        self.X, self.S, self.Y, self.P = (torch.empty((n, c), **f32) for _ in range(4))
        self.h, self.O = torch.empty((n, c), **t), torch.empty((n, wq), **t)
        self.stats = [torch.empty((n, 2), **f32) for _ in range(2)]
        self.proj = torch.empty((n, self.wide), **f32)
        self.qkv = self.proj if dtype == B.HCH_F32 else torch.empty((n, self.wide), **t)
        self.q, self.k, self.v = self.qkv[:, :wq], self.qkv[:, wq: wq + wk], self.qkv[:, wq + wk:]
        self.lse = torch.empty((n, heads_q), **f32)
        # backward; in fp32 the gradients go into products as they are
        same = dtype == B.HCH_F32
        self.dY, self.dX, self.dh = (torch.empty((n, c), **f32) for _ in range(3))
        (self.dS, dS8), (self.dO32, dO32_8) = _by_eights(n, c, **f32), _by_eights(n, wq, **f32)
        self.dP, dP8 = (self.dS, None) if same else _by_eights(n, c, **t)
        self.dO, dO8 = (self.dO32, None) if same else _by_eights(n, wq, **t)
        self._to_products = (dS8, dP8), (dO32_8, dO8)
        self.dqkv = torch.empty((n, self.wide), **t)
        self.dq, self.dk, self.dv = self.dqkv[:, :wq], self.dqkv[:, wq: wq + wk], self.dqkv[:, wq + wk:]
        b = self.offsets.numel() - 1
        need = [B.hch_layernorm_workspace_bytes(n, c)]
        need += [B.hch_attn_workspace_bytes(k, dtype, b, n, n, heads_q, heads_kv, head_dim) for k in (B.HCH_WS_FWD, B.HCH_WS_BWD_DATA)]
        for kind in (B.HCH_WS_FWD, B.HCH_WS_BWD_DATA, B.HCH_WS_BWD_WEIGHT):
            need += [B.hch_sconv_workspace_bytes(levels, level, 1, 1, ci, co, dtype, kind) for ci, co in ((c, self.wide), (wq, c))]
        self.ws = _aligned_bytes(max(need), device)

    def _convert(self, x8, y8):
        """y = x in the products' type, all elements in rows of 8 whatever the width: rotary positions that turn nothing."""
        if y8 is not None:
            B.hch_rope_fwd(B.HCH_F32, x8, self.dtype, y8, None, x8.shape[0], 1, 0, 8, (0, 0, 0))

    def forward(self):
        """X -> S, Y"""
        n, c, wq, dt, lv = self.n, self.c, self.hq * self.d, self.dtype, (self.levels, self.level, 1, 1)
        B.hch_layernorm_fwd(B.HCH_F32, self.X, None, None, self.gamma[0], self.beta[0], dt, self.h, self.stats[0], n, c, self.eps)
        B.hch_sconv_fwd(*lv, dt, self.h, self.Wqkv, self.proj, self.field, c, self.wide, self.ws)
        B.hch_rope_fwd(B.HCH_F32, self.proj, dt, self.qkv, self.positions, n, self.hq + 2 * self.hkv, self.hq + self.hkv, self.d,
                       self.sections, self.base)
        B.hch_attn_fwd(dt, self.q, self.k, self.v, self.O, self.lse, self.offsets, self.offsets, self.key_mask, self.hq, self.hkv,
                       self.d, self.scale, self.ws)
        B.hch_sconv_fwd(*lv, dt, self.O, self.Wo, self.P, self.field, wq, c, self.ws)
        B.hch_layernorm_fwd(B.HCH_F32, self.X, self.P, self.S, self.gamma[1], self.beta[1], B.HCH_F32, self.Y, self.stats[1], n, c,
                            self.eps)

    def backward(self, dS=None):
        """dY (and the gradient dS that reaches S by itself) -> dX and the weights' gradients"""
        n, c, wq, dt, lv = self.n, self.c, self.hq * self.d, self.dtype, (self.levels, self.level, 1, 1)
        B.hch_layernorm_bwd(B.HCH_F32, self.S, self.stats[1], self.gamma[1], B.HCH_F32, self.dY, dS, self.dS, self.dgamma[1],
                            self.dbeta[1], n, c, self.ws)
        self._convert(*self._to_products[0])
        B.hch_sconv_bwd_weight(*lv, dt, self.O, self.dP, self.dWo, self.field, wq, c, self.ws)
        B.hch_sconv_bwd_data(*lv, dt, self.dP, self.Wo, self.dO32, self.field_t, wq, c, self.ws)
        self._convert(*self._to_products[1])
        B.hch_attn_bwd(dt, self.q, self.k, self.v, self.O, self.lse, self.dO, self.dq, self.dk, self.dv, self.offsets, self.offsets,
                       self.key_mask, self.hq, self.hkv, self.d, self.scale, self.ws)
        B.hch_rope_bwd(dt, self.dqkv, dt, self.dqkv, self.positions, n, self.hq + 2 * self.hkv, self.hq + self.hkv, self.d,
                       self.sections, self.base)
        B.hch_sconv_bwd_weight(*lv, dt, self.h, self.dqkv, self.dWqkv, self.field, c, self.wide, self.ws)
        B.hch_sconv_bwd_data(*lv, dt, self.dqkv, self.Wqkv, self.dh, self.field_t, c, self.wide, self.ws)
        B.hch_layernorm_bwd(B.HCH_F32, self.X, self.stats[0], self.gamma[0], B.HCH_F32, self.dh, self.dS, self.dX, self.dgamma[0],
                            self.dbeta[0], n, c, self.ws)
