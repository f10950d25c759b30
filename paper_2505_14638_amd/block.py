"""The decoder-block linear stack (QKV -> O -> gate|up -> SiLU*mul -> down) on the HIP path.

Orchestration only: every tensor operation is one call into the C-ABI library (activation quantization, linear
layer, SiLU*mul); PyTorch provides buffers and views.  The O projection reads the first `hidden` columns of the QKV
output (a strided view -- the quantizer takes a row stride), standing in for attention, which is not part of the
quantized-linear path.  Intermediates are bf16, each linear layer's input is quantized to FP8 with its own static
per-tensor scale (Eq. 13; all linear layers of a block are quantized, Sec. 4.1).

`fused=True` runs the same computation with the quantization of each intermediate folded into the kernel that produces
it (w4a8_linear_fp8_out for QKV and O, w4a8_linear_silu_mul_fp8_out for gate|up with SiLU*mul, on a row-interleaved
copy of the gate|up weights) and, up to eight tokens, the quantization of the block input folded into the QKV layer
(w4a8_linear_quantize_in_fp8_out): four or five launches instead of nine, the same bytes at every layer input and the
same block output.

`DecoderBlock` has attention in that place: queries and keys are rotated, keys and values go to a paged cache, and whole prompts or single
tokens of a batch attend; with `fused=True` attention writes the E4M3 bytes that the O projection reads.  Neither class has norms or residual
additions: they are the quantized layers, and attention, of a block.
"""
from __future__ import annotations

import torch

from . import binding as B

LAYERS = ("qkv", "o", "gate_up", "down")


class DecoderBlockLinears:
    def __init__(self, hidden: int, ffn: int, qkv_out: int, group_size: int = 128, device: str = "cuda:0",
                 fused: bool = False):
        self.hidden, self.ffn, self.group_size, self.device, self.fused = hidden, ffn, group_size, device, fused
        self.dims = {"qkv": (hidden, qkv_out), "o": (hidden, hidden), "gate_up": (hidden, 2 * ffn), "down": (ffn, hidden)}
        self.weights = {}
        self.scales_x = {}
        self._buffers = {}
        self.quantize_in_up_to = 8                               # tokens up to which the QKV layer quantizes its own input
        self._workspace = None                                   # scratch of w4a8_linear (K ranges across workgroups), grown on demand
        self._retired = []                                       # outgrown workspaces, kept for launches already captured

    def load_layer(self, name: str, w_f32: torch.Tensor) -> None:
        """Quantize (round-to-nearest INT4) and pack one [N, K] float32 weight matrix on the device."""
        k, n = self.dims[name]
        assert tuple(w_f32.shape) == (n, k)
        w_dev = w_f32.to(self.device)
        self.weights[name] = B.pack_weights(w_dev, self.group_size, B.LAYOUT_TILED)
        if name == "gate_up":                                    # row-interleaved copy for the fused gate|up + SiLU*mul layer
            self.weights["gate_up_interleaved"] = B.pack_weights(B.interleave_gate_up(w_dev), self.group_size, B.LAYOUT_TILED)

    def set_act_scale(self, name: str, s_x: float) -> None:
        self.scales_x[name] = torch.tensor([s_x], dtype=torch.float32, device=self.device)

    def _buf(self, key, shape, dtype):
        b = self._buffers.get(key)
        if b is None or tuple(b.shape) != tuple(shape):
            b = torch.empty(shape, dtype=dtype, device=self.device)
            self._buffers[key] = b
        return b

    def _ws(self, name: str, m: int):
        """The workspace w4a8_linear asks for on this layer at this batch size (None where it asks for none)."""
        k, n = self.dims[name]
        need = B.linear_workspace_bytes(m, k, n, self.group_size)
        if need == 0:
            return None
        if self._workspace is None or self._workspace.numel() < need:
            if self._workspace is not None:
                self._retired.append(self._workspace)            # a captured graph may still write to it: never freed
            self._workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
        return self._workspace

    def _linear(self, name: str, x: torch.Tensor, m: int) -> torch.Tensor:
        k, n = self.dims[name]
        x8 = self._buf((name, "x8", m), (m, k), torch.uint8)
        y = self._buf((name, "y", m), (m, n), torch.bfloat16)
        B.quantize_act(x, self.scales_x[name], out=x8)
        packed, scales = self.weights[name]
        # only the last layer takes the workspace: the fused forms of the others take none, and with one w4a8_linear may add
        # the ranges of K in another order than they do
        ws = self._ws(name, m) if name == "down" else None
        B.linear(x8, self.scales_x[name], packed, scales, n, self.group_size, B.LAYOUT_TILED, out=y, workspace=ws)
        return y

    def _forward_fused(self, x: torch.Tensor, keep: dict | None) -> torch.Tensor:
        m, g, sx, w = x.shape[0], self.group_size, self.scales_x, self.weights
        x8 = self._buf(("qkv", "x8", m), (m, self.hidden), torch.uint8)
        qkv8 = self._buf(("qkv", "y8", m), (m, self.dims["qkv"][1]), torch.uint8)
        if m <= self.quantize_in_up_to and m * self.hidden <= 65536:   # every workgroup quantizes x itself: one launch fewer
            B.linear_quantize_in_fp8_out(x, sx["qkv"], *w["qkv"], self.dims["qkv"][1], g, sx["o"], out=qkv8,
                                         x8_out=x8 if keep is not None else None)
        else:
            B.quantize_act(x, sx["qkv"], out=x8)
            B.linear_fp8_out(x8, sx["qkv"], *w["qkv"], self.dims["qkv"][1], g, sx["o"], out=qkv8)
        if keep is not None:
            keep.update(qkv_x8=x8, o_x8=qkv8[:, :self.hidden])
        return self._from_o_fused(qkv8[:, :self.hidden], m, keep)

    def _from_o_fused(self, o_x8: torch.Tensor, m: int, keep: dict | None) -> torch.Tensor:
        """The O projection's E4M3 input to the block's output."""
        g, sx, w = self.group_size, self.scales_x, self.weights
        o8 = B.linear_fp8_out(o_x8, sx["o"], *w["o"], self.hidden, g, sx["gate_up"],
                              out=self._buf(("o", "y8", m), (m, self.hidden), torch.uint8))
        h8 = self._buf(("h8", m), (m, self.ffn), torch.uint8)
        B.linear_silu_mul_fp8_out(o8, sx["gate_up"], *w["gate_up_interleaved"], self.ffn, g, sx["down"], out=h8)
        y = B.linear(h8, sx["down"], *w["down"], self.hidden, g, B.LAYOUT_TILED,
                     out=self._buf(("down", "y", m), (m, self.hidden), torch.bfloat16), workspace=self._ws("down", m))
        if keep is not None:
            keep.update(gate_up_x8=o8, down_x8=h8, down=y)
        return y

    def forward(self, x: torch.Tensor, keep: dict | None = None) -> torch.Tensor:
        """x: bf16 [M, hidden] on the device.  `keep`, if given, receives every intermediate tensor."""
        if self.fused:
            return self._forward_fused(x, keep)
        m = x.shape[0]
        qkv = self._linear("qkv", x, m)
        y = self._from_o(qkv[:, :self.hidden], m, keep)
        if keep is not None:
            keep.update(qkv=qkv, qkv_x8=self._buffers[("qkv", "x8", m)])
        return y

    def _from_o(self, attended: torch.Tensor, m: int, keep: dict | None) -> torch.Tensor:
        """The O projection's bf16 input to the block's output."""
        o = self._linear("o", attended, m)
        gu = self._linear("gate_up", o, m)
        h = B.silu_mul(gu, out=self._buf(("h", m), (m, self.ffn), torch.bfloat16))
        y = self._linear("down", h, m)
        if keep is not None:
            keep.update(o=o, gate_up=gu, h=h, down=y, **{nm + "_x8": self._buffers[(nm, "x8", m)] for nm in LAYERS[1:]})
        return y


class DecoderBlock(DecoderBlockLinears):
    """A block with attention between QKV and O: `heads` query heads and `kv_heads` key and value heads of hidden / heads channels."""

    def __init__(self, hidden: int, ffn: int, heads: int, kv_heads: int, cos_sin: torch.Tensor, rope: int = B.ROPE_HALVES,
                 group_size: int = 128, device: str = "cuda:0", fused: bool = False):
        """cos_sin: float32 [positions, head_dim], the table of w4a8_rope_cache_write (rotary_table makes one)."""
        if hidden % heads != 0 or heads % kv_heads != 0:
            raise ValueError(f"hidden {hidden}, heads {heads}, kv_heads {kv_heads} do not divide")
        self.heads, self.kv_heads, self.head_dim, self.cos_sin, self.rope = heads, kv_heads, hidden // heads, cos_sin, rope
        super().__init__(hidden, ffn, hidden + 2 * kv_heads * self.head_dim, group_size, device, fused)

    def forward(self, x: torch.Tensor, keep: dict | None = None) -> torch.Tensor:
        raise TypeError("attention needs to know what x is: forward_prompt or forward_decode")

    def _qkv(self, x: torch.Tensor, m: int, keep: dict | None) -> torch.Tensor:
        if self.fused and m <= self.quantize_in_up_to and m * self.hidden <= 65536:
            return B.linear_quantize_in(x, self.scales_x["qkv"], *self.weights["qkv"], self.dims["qkv"][1], self.group_size,
                                        out=self._buf(("qkv", "y", m), (m, self.dims["qkv"][1]), torch.bfloat16),
                                        x8_out=self._buf(("qkv", "x8", m), (m, self.hidden), torch.uint8) if keep is not None else None)
        return self._linear("qkv", x, m)

    def _rows(self, name: str, m: int, heads: int) -> torch.Tensor:
        return self._buf((name, m), (m, heads * self.head_dim), torch.bfloat16)

    def _attended(self, m: int):
        """(output of attention, its scale): E4M3 for the O projection where the quantization is folded in."""
        if self.fused:
            return self._buf(("o", "x8", m), (m, self.hidden), torch.uint8), self.scales_x["o"]
        return self._rows("attended", m, self.heads), None

    def _finish(self, out: torch.Tensor, qkv: torch.Tensor, m: int, keep: dict | None) -> torch.Tensor:
        if keep is not None:
            keep.update(qkv=qkv, qkv_x8=self._buffers[("qkv", "x8", m)], **({"o_x8": out} if self.fused else {"attended": out}))
        return self._from_o_fused(out, m, keep) if self.fused else self._from_o(out, m, keep)

    def forward_prompt(self, x: torch.Tensor, starts: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache,
                       keep: dict | None = None) -> torch.Tensor:
        """Whole prompts, packed: x bf16 [M, hidden], starts int32 [sequences + 1] (rows of no sequence get what their buffer held);
        positions and slots int32 [M], where each token goes in `cache` = (keys, values, scales or None).  A row attends to rows of this call
        alone, so its sequence holds nothing before them: PagedCache.grow's positions behind tokens are refused (a copy of them is not known as such).
        Sequences that hold tokens take further ones by forward_decode, or by a prompt of all of them as a new sequence."""
        if getattr(positions, "behind_tokens", False):
            raise ValueError("forward_prompt: a sequence holds tokens already, which its new rows would not see")
        m, (k_cache, v_cache, kv_scales) = x.shape[0], cache
        qkv = self._qkv(x, m, keep)
        q, k = self._rows("q", m, self.heads), self._rows("k", m, self.kv_heads)
        B.rope_cache_write(qkv, self.cos_sin, positions, slots, k_cache, v_cache, kv_scales, self.rope, q_out=q, k_out=k)
        out, y_scale = self._attended(m)
        shape = (self.kv_heads, self.head_dim)
        B.attention_prompt(q.view(m, self.heads, self.head_dim), k.view(m, *shape), qkv[:, -self.kv_heads * self.head_dim:].unflatten(1, shape),
                           starts, out=out, y_scale=y_scale)
        return self._finish(out, qkv, m, keep)

    def forward_decode(self, x: torch.Tensor, positions: torch.Tensor, slots: torch.Tensor, cache, tables: torch.Tensor, lengths: torch.Tensor,
                       prefix_pages: torch.Tensor | None = None, prefix_length: int = 0, keep: dict | None = None) -> torch.Tensor:
        """One token of each sequence: x bf16 [M, hidden]; its keys and values go to `slots` first, so `lengths` count it."""
        m, (k_cache, v_cache, kv_scales) = x.shape[0], cache
        qkv = self._qkv(x, m, keep)
        q = B.rope_cache_write(qkv, self.cos_sin, positions, slots, k_cache, v_cache, kv_scales, self.rope, q_out=self._rows("q", m, self.heads))
        out, y_scale = self._attended(m)
        B.attention_decode(q.view(m, self.heads, self.head_dim), k_cache, v_cache, tables, lengths, prefix_pages, prefix_length, kv_scales,
                           out=out, y_scale=y_scale)
        return self._finish(out, qkv, m, keep)


def rotary_table(positions: int, head_dim: int, base: float = 10000.0, device: str = "cuda:0") -> torch.Tensor:
    """float32 [positions, head_dim]: cosines, then sines of position * base^(-2i / head_dim), the angles in 64 bits."""
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, head_dim, 2, dtype=torch.float64) / head_dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().to(device)
