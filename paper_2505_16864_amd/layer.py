"""Buffers for one attention layer: torch owns the device memory and the stream, the library does the work."""
import torch

from . import binding as B


class CarveLayer:
    """Allocates the curve-side tensors, index lists and workspaces of one configuration once and
    runs the four calls, or all of them as one (forward), on torch's current stream."""

    def __init__(self, w, device="cuda:0", text_bias=None, flags=None, want_mask=False, want_lse=False, rotary=None):
        """rotary: None, or the keyword arguments of make_rotary() behind head_dim: dims, theta, origin, step, flags.  forward() then
        turns Q and K by their positions."""
        self.plan = None
        self.w = dict(w)
        if text_bias is None:
            text_bias = w.get("text_bias", 0.0)
        if flags is None:
            flags = w.get("flags", 7)
        self.device = torch.device(device)
        self.cfg = B.make_config(w["T"], w["H"], w["W"], w["n_text"], w["batch"], w["heads"], w["head_dim"],
                                 w["block"], w["topk"], w["p"], text_bias, flags)
        with torch.cuda.device(self.device):
            self.plan = B.jenga_plan_create(self.cfg)
        self.info = B.jenga_plan_info(self.plan)
        i, dev = self.info, self.device
        shape_c = (w["batch"], w["heads"], i.N_pad, w["head_dim"])
        self.q_c, self.k_c, self.v_c, self.o_c = [torch.empty(shape_c, dtype=torch.bfloat16, device=dev)
                                                  for _ in range(4)]
        self.sel_count = torch.empty((w["batch"], w["heads"], i.M), dtype=torch.int32, device=dev)
        self.sel_index = torch.full((w["batch"], w["heads"], i.M, i.M), -1, dtype=torch.int32, device=dev)
        self.mask = torch.zeros((w["batch"], w["heads"], i.M, i.M), dtype=torch.uint8, device=dev) if want_mask else None
        self.lse = torch.empty((w["batch"], w["heads"], i.N_pad), dtype=torch.float32, device=dev) if want_lse else None
        self.ws_select = torch.empty(max(1, i.select_workspace_bytes), dtype=torch.uint8, device=dev)
        self.ws_attn = torch.empty(max(1, i.attn_workspace_bytes), dtype=torch.uint8, device=dev)
        self.rotary = None
        if rotary is not None:
            self.rotary = B.make_rotary(w["T"], w["H"], w["W"], w["head_dim"], **rotary)
            table = torch.empty(sum(n * d for n, d in zip((w["T"], w["H"], w["W"]), self.rotary.dim)), dtype=torch.float32)
            B.jenga_rotary_table(self.rotary, table)
            self.rotary_table = table.to(dev)
        self.out_thw = torch.empty((w["batch"], i.N_v + w["n_text"], w["heads"], w["head_dim"]),
                                   dtype=torch.bfloat16, device=dev)

    def _stream(self):
        # the raw handle, without building a Stream object (2 us) for every call
        index = self.device.index
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index)

    def permute_in(self, q, k, v):
        B.jenga_curve_permute_qkv(self.plan, q, k, v, self.q_c, self.k_c, self.v_c, self._stream())

    def select(self):
        B.jenga_select_blocks(self.plan, self.q_c, self.k_c, self.sel_count, self.sel_index, self.mask,
                              self.ws_select, self.ws_select.numel(), self._stream())

    def attend(self):
        B.jenga_block_sparse_attn(self.plan, self.q_c, self.k_c, self.v_c, self.sel_count, self.sel_index,
                                  self.o_c, self.lse, self.ws_attn, self.ws_attn.numel(), self._stream())

    def pack(self):
        B.jenga_pack_kv(self.plan, self.k_c, self.v_c, self.ws_attn, self.ws_attn.numel(), self._stream())

    def attend_packed(self):
        B.jenga_block_sparse_attn_packed(self.plan, self.q_c, self.ws_attn, self.ws_attn.numel(), self.sel_count,
                                         self.sel_index, self.o_c, self.lse, self._stream())

    def permute_out(self):
        B.jenga_unpermute(self.plan, self.o_c, self.out_thw, self._stream())

    def forward(self, q, k, v):
        """Whole path on thw-side bf16 tensors [batch, N_v+N_c, heads, d]; returns the thw-side output.  With rotary positions they may
        be columns of one projection."""
        if self.rotary is not None:
            if q.shape != self.out_thw.shape:   # the plan's sizes are not the call's to see
                raise ValueError("q, k and v of shape %s, not %s" % (tuple(q.shape), tuple(self.out_thw.shape)))
            B.jenga_forward_rotary(self.plan, self.rotary, self.rotary_table, q, k, v, self.q_c, self.k_c, self.v_c, self.sel_count,
                                   self.sel_index, self.mask, self.ws_select, self.ws_select.numel(), self.o_c, self.lse, self.ws_attn,
                                   self.ws_attn.numel(), self.out_thw, self._stream())
            return self.out_thw
        B.jenga_forward(self.plan, q, k, v, self.q_c, self.k_c, self.v_c, self.sel_count, self.sel_index, self.mask,
                        self.ws_select, self.ws_select.numel(), self.o_c, self.lse, self.ws_attn, self.ws_attn.numel(),
                        self.out_thw, self._stream())
        return self.out_thw

    def close(self):
        if self.plan is not None:
            B.jenga_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class CarveBlock:
    """The attention half of a transformer block on hidden states: a modulated layer norm straight to 8 bits, one 8-bit product for Q, K
    and V, a CarveLayer with rotary positions, an 8-bit output projection.  Owns the weights in 8 bits and every buffer."""

    def __init__(self, w, w_qkv, b_qkv, w_out, b_out, rotary, device="cuda:0", eps=1e-6, **layer):
        """w: a workload of CarveLayer.  w_qkv [3 * heads * head_dim, hidden] (rows of Q, K, V), w_out [hidden, heads * head_dim] in
        bf16, fp16 or float32; b_qkv, b_out float32 or None.  rotary and **layer: of CarveLayer."""
        inner, hidden = w["heads"] * w["head_dim"], w_out.shape[0]
        if tuple(w_qkv.shape) != (3 * inner, hidden) or w_out.shape[1] != inner:
            raise ValueError("weights of shapes %s and %s for %d heads x %d" % (tuple(w_qkv.shape), tuple(w_out.shape), w["heads"],
                                                                              w["head_dim"]))
        if rotary is None:
            raise ValueError("a CarveBlock turns Q and K: rotary positions are wanted")
        self.eps, self.hidden, self.inner = eps, hidden, inner
        self.layer = CarveLayer(w, device, rotary=rotary, **layer)
        dev = self.device = self.layer.device
        self.batch, self.tokens = w["batch"], self.layer.info.N_v + w["n_text"]
        rows = self.batch * self.tokens
        with torch.cuda.device(dev):
            self.w_qkv, self.s_qkv = self._quantized(w_qkv.to(dev), 128)
            self.w_out, self.s_out = self._quantized(w_out.to(dev), 128)
            self.b_qkv, self.b_out = [None if b is None else b.to(dev, torch.float32).contiguous() for b in (b_qkv, b_out)]
            self.x, self.s_x = self._room(rows, hidden)
            self.o, self.s_o = self._room(rows, inner)
            self.qkv = torch.empty((self.batch, self.tokens, 3, w["heads"], w["head_dim"]), dtype=torch.bfloat16, device=dev)
            self.out = torch.empty((self.batch, self.tokens, hidden), dtype=torch.bfloat16, device=dev)

    def _room(self, rows, cols, block_rows=1):
        return (torch.empty((rows, B.padded_columns(cols)), dtype=torch.float8_e4m3fn, device=self.device),
                torch.empty((-(-rows // block_rows), B.scale_columns(cols)), dtype=torch.uint8, device=self.device))

    def _quantized(self, weight, block_rows):
        q, scale = self._room(*weight.shape, block_rows)
        B.jenga_quantize(weight.contiguous(), q, scale, block_rows, stream=self.layer._stream())
        return q, scale

    def project(self, x, scale=None, shift=None):
        """x bf16 [batch, tokens, hidden]; scale, shift bf16 or float32 [batch, hidden], any stride between batch entries.  Returns Q, K and V before
        their turn, [batch, tokens, heads, head_dim] each, columns of one tensor."""
        stream = self.layer._stream()
        B.jenga_layer_norm(x.reshape(-1, self.hidden), self.x, scale, shift, y_scale=self.s_x, group_rows=self.tokens, weight_offset=1.0,
                           eps=self.eps, stream=stream)
        B.jenga_matmul(self.x, self.s_x, self.w_qkv, self.s_qkv, self.qkv.view(-1, self.w_qkv.shape[0]), self.b_qkv, stream=stream)
        return self.qkv.unbind(2)

    def forward(self, x, scale=None, shift=None):
        """What the block adds to x, before its gate: bf16 [batch, tokens, hidden], overwritten by the next call."""
        stream = self.layer._stream()
        o = self.layer.forward(*self.project(x, scale, shift))
        B.jenga_quantize(o.view(-1, self.inner), self.o, self.s_o, stream=stream)
        B.jenga_matmul(self.o, self.s_o, self.w_out, self.s_out, self.out.view(-1, self.hidden), self.b_out, stream=stream)
        return self.out

    def close(self):
        self.layer.close()
