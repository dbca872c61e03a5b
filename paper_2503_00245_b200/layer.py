"""Conveniences over the C ABI: pack weights once, own a context and its workspace.

No arithmetic of the layer happens here; every call forwards to libcosmoe.so.
"""
from __future__ import annotations

import threading

import torch

from . import binding as B


def pack_dense(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor):
    """[E,d,f], [E,d,f], [E,f,d] bf16 (maths layout) -> gud [E,f,3,d]."""
    E, d, f = w_gate.shape
    gud = torch.empty((E, f, 3, d), dtype=torch.bfloat16, device=w_gate.device)
    B.moe_pack_dense(d, f, E, w_gate, w_up, w_down, gud)
    return gud


def pack_wd(gL, gR, uL, uR, dL, dR):
    """Eq. 1 factors in maths layout -> (wd_a [E,r,2,d], wd_b [E,f,2,r], wd_c [E,r,f], wd_d [E,d,r])."""
    E, d, r = gL.shape
    f = gR.shape[2]
    dev, bf = gL.device, torch.bfloat16
    wd_a = torch.empty((E, r, 2, d), dtype=bf, device=dev)
    wd_b = torch.empty((E, f, 2, r), dtype=bf, device=dev)
    wd_c = torch.empty((E, r, f), dtype=bf, device=dev)
    wd_d = torch.empty((E, d, r), dtype=bf, device=dev)
    B.moe_pack_wd(d, f, r, E, gL, gR, uL, uR, dL, dR, wd_a, wd_b, wd_c, wd_d)
    return wd_a, wd_b, wd_c, wd_d


# ---- 4-bit rows and experts -------------------------------------------------------------
class Fp4Rows:
    """A matrix in MXFP4: codes uint8 [rows, 16 ceil(n / 32)] and scales uint8 [ceil(n / 128), rows rounded up to 4, 4] (the layout of
    moe_fp4 in cosmoe.h)."""

    __slots__ = ("_codes", "_scales", "_buf", "device", "rows", "n", "c")

    def __init__(self, codes, scales, n):
        rows, nb = codes.shape[0], -(-n // 32)
        if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
            raise TypeError("codes and scales are uint8")
        if tuple(codes.shape) != (rows, 16 * nb) or tuple(scales.shape) != (-(-nb // 4), -(-rows // 4) * 4, 4):
            raise ValueError(f"codes {tuple(codes.shape)} and scales {tuple(scales.shape)} are not those of {rows} rows of {n} values")
        if codes.device != scales.device:
            raise ValueError("codes and scales lie on different devices")
        self._codes, self._scales, self._buf, self.device, self.rows, self.n = codes, scales, None, codes.device, rows, n
        self.c = B.make_fp4(codes, scales, rows, n)

    @classmethod
    def empty(cls, rows, n, device="cuda"):
        return cls._over(torch.empty(cls._bytes(rows, B._i32(n)), dtype=torch.uint8, device=device), rows, n)

    @staticmethod
    def _bytes(rows, n):
        nb = -(-n // 32)
        return 16 * (rows * nb + -(-nb // 4) * -(-rows // 4))

    @classmethod
    def _over(cls, buf, rows, n):
        """In one buffer, codes first; the two tensors are made when somebody asks for them (each takes as long as a small launch)."""
        q = object.__new__(cls)
        at = buf.data_ptr()
        q._codes = q._scales = None
        q._buf, q.device, q.rows, q.n = buf, buf.device, rows, n
        q.c = B.moe_fp4(at, at + 16 * rows * -(-n // 32), rows, n)
        return q

    @property
    def codes(self):
        if self._codes is None:
            nb = -(-self.n // 32)
            self._codes = self._buf[:16 * self.rows * nb].view(self.rows, 16 * nb)
        return self._codes

    @property
    def scales(self):
        if self._scales is None:
            nb = -(-self.n // 32)
            self._scales = self._buf[16 * self.rows * nb:].view(-(-nb // 4), -(-self.rows // 4) * 4, 4)
        return self._scales

    @property
    def _tensor(self):
        return self._codes if self._buf is None else self._buf

    def dequantize(self, dtype=torch.bfloat16):
        """The values, [rows, n] (n a multiple of 8)."""
        out = self._tensor.new_empty((self.rows, self.n), dtype=dtype)
        _here(out)
        B.moe_fp4_dequantize_rows(self.c, out)
        return out


def _here(*tensors):
    """Calls go to the current device's current stream: their tensors have to lie there."""
    here = B._current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor on {t.device}, but the current device is cuda:{here}")


def fp4_quantize(x, row_of=None, row_div=1):
    """x [src_rows, n] float32 or bfloat16, any strides -> Fp4Rows; with row_of (int32): row i is x[row_of[i] // row_div]."""
    if x.dim() != 2:
        raise ValueError("x is a matrix of rows")
    rows = x.shape[0]
    if row_of is not None:
        if row_of.dtype != torch.int32 or row_of.dim() != 1:
            raise TypeError("row_of is a vector of int32")
        rows = row_of.shape[0]
    _here(x, row_of)
    n = x.shape[1]
    q = Fp4Rows._over(x.new_empty(Fp4Rows._bytes(rows, n), dtype=torch.uint8), rows, n)
    B.moe_fp4_quantize_rows(x, row_of, row_div, rows, q.c.codes, q.c.scales)
    return q


def pack_fp4(w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor):
    """[E,d,f], [E,d,f], [E,f,d] bf16 (maths layout) -> the experts in MXFP4: (gu, down)."""
    E, d, f = w_gate.shape
    if any(w.dtype != torch.bfloat16 for w in (w_gate, w_up, w_down)):
        raise TypeError("the experts' matrices are bfloat16")
    if w_up.shape != (E, d, f) or w_down.shape != (E, f, d):
        raise ValueError(f"w_gate {tuple(w_gate.shape)}, w_up {tuple(w_up.shape)} and w_down {tuple(w_down.shape)} are not [E,d,f], [E,d,f] and [E,f,d]")
    _here(w_gate, w_up, w_down)
    gu, down = Fp4Rows.empty(E * 64 * -(-f // 32), d, w_gate.device), Fp4Rows.empty(E * d, f, w_gate.device)
    B.moe_fp4_pack_dense(d, f, E, w_gate, w_up, w_down, gu.c, down.c)
    return gu, down


_shared = {}  # device index -> a ctx for calls that need no more of one than its status word
_shared_lock = threading.Lock()


def _shared_ctx():
    here = B._current_device()
    ctx = _shared.get(here)
    if ctx is None:
        with _shared_lock:  # (one for all threads: whose status fp4_check reads)
            ctx = _shared.get(here)
            if ctx is None:
                ctx = _shared[here] = B.moe_create(B.make_config(8, 8, 1, 1))
    return ctx


def fp4_check() -> int:
    """What moe_check says of the current device's calls of fp4_product that had no ctx: 0, or the first failure since the last check (an
    expired wait: that call's output is undefined).  Waits for the current stream; what runs on others has to be waited for before."""
    ctx = _shared.get(B._current_device())
    return B.MOE_OK if ctx is None else B.moe_check(ctx)


def fp4_product(a: Fp4Rows, w: Fp4Rows, expert_offsets, out=None, out_dtype=torch.bfloat16, ctx=None):
    """out[s] = a[s] times the matrix of the expert e with expert_offsets[e] <= s < expert_offsets[e + 1]; w holds the experts'
    matrices, w.rows / E rows each.  Rows outside the offsets are left as they are.  out: rows may lie apart.  Without a ctx (its
    status word is what moe_check reads) the library's own for this device is used, whose status fp4_check() reads, made by the first
    call on it: let that one come before a stream is captured."""
    E = expert_offsets.shape[0] - 1
    if expert_offsets.dtype != torch.int32 or E < 1:
        raise TypeError("expert_offsets is a vector of E + 1 int32")
    N = w.rows // E
    _here(a._tensor, w._tensor, expert_offsets, out)
    if out is None:
        out = expert_offsets.new_empty((a.rows, N), dtype=out_dtype)
        stride = N
    else:
        if tuple(out.shape) != (a.rows, N) or out.stride(1) != 1:
            raise ValueError(f"out has to be [{a.rows}, {N}] with contiguous rows")
        stride = out.stride(0) if a.rows > 1 else max(N, out.stride(0))
    B.moe_fp4_product(_shared_ctx() if ctx is None else ctx, a.c, w.c, expert_offsets, E, out, stride)
    return out


class SelectRule:
    """How experts are chosen from logits (moe_select): scoring "softmax" or "sigmoid"; `groups` of which `groups_kept` stay, judged by
    their `group_top` largest keys; renormalised weights times `scale`."""

    def __init__(self, n_experts, top_k, scoring="softmax", groups=1, groups_kept=1, group_top=1, renorm=True, scale=1.0):
        self.E, self.k = n_experts, top_k
        self.c = B.make_select_config(n_experts, top_k, {"softmax": B.MOE_SCORE_SOFTMAX, "sigmoid": B.MOE_SCORE_SIGMOID}[scoring], groups,
                                      groups_kept, group_top, int(renorm), scale)


def select_experts(logits, rule: SelectRule, bias=None):
    """logits [T, E] float32 or bfloat16 (rows may lie apart), bias [E] float32 -> (topk_idx int32 [T, k], topk_w float32 [T, k])."""
    shape = logits.shape
    if len(shape) != 2 or shape[1] != rule.E or (rule.E > 1 and logits.stride(1) != 1):
        raise ValueError(f"logits have to be [T, {rule.E}] with contiguous rows")
    if bias is not None and (bias.dtype != torch.float32 or bias.shape != (rule.E,)):
        raise ValueError(f"the bias has to be float32 [{rule.E}]")
    _here(logits, bias)
    T = shape[0]
    idx = logits.new_empty((T, rule.k), dtype=torch.int32)
    w = logits.new_empty((T, rule.k), dtype=torch.float32)
    B.moe_select(rule.c, logits, T, bias, idx.data_ptr(), w.data_ptr(), logits.stride(0) if T > 1 else rule.E)
    return idx, w


class Fp4Experts:
    """Experts in MXFP4 (pack_fp4) with a context and a workspace for up to max_tokens: the FFN for a given routing."""

    def __init__(self, d_model, d_ff, n_experts, top_k, gu: Fp4Rows, down: Fp4Rows, x_dtype=torch.bfloat16, max_tokens=1, ctx=None):
        self.d, self.k, self.x_dtype, self.max_tokens = d_model, top_k, x_dtype, max_tokens
        self.gu, self.down, self.device = gu, down, gu.device
        self.cfg = B.make_config(d_model, d_ff, n_experts, top_k, 0, B.dtype_of(x_dtype))
        self.ctx, self.lent = ctx, ctx is not None  # (a layer lends its own)
        _here(gu._tensor, down._tensor)
        if ctx is None:
            self.ctx = B.moe_create(self.cfg)
        self.ws = torch.empty(B.moe_fp4_workspace_bytes(self.cfg, max_tokens), dtype=torch.uint8, device=self.device)

    def forward(self, x, topk_idx, topk_w, y=None):
        """x [T, d], topk_idx int32 [T, k], topk_w float32 [T, k] -> y [T, d]."""
        T = x.shape[0]
        if T > self.max_tokens:
            raise ValueError(f"T={T} exceeds max_tokens={self.max_tokens} this workspace was sized for")
        if x.shape != (T, self.d) or x.dtype != self.x_dtype:
            raise ValueError(f"x has to be {self.x_dtype} [T, {self.d}]")
        if topk_idx.shape != (T, self.k) or topk_w.shape != (T, self.k) or topk_idx.dtype != torch.int32 or topk_w.dtype != torch.float32:
            raise ValueError(f"the routing has to be int32 and float32 [{T}, {self.k}]")
        _here(x, topk_idx, topk_w, y, self.ws)
        if y is None:
            y = torch.empty((T, self.d), dtype=self.x_dtype, device=self.device)
        elif y.shape != (T, self.d) or y.dtype != self.x_dtype:
            raise ValueError(f"y has to be {self.x_dtype} [{T}, {self.d}]")
        B.moe_fp4_experts(self.ctx, x, T, self.gu.c, self.down.c, topk_idx, topk_w, y, self.ws)
        return y

    def check(self) -> int:
        return B.moe_check(self.ctx)

    def close(self):
        if self.ctx and not self.lent:
            B.moe_destroy(self.ctx)
        self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MoELayer:
    """One MoE layer's packed weights plus a context and workspace sized for up to max_tokens.

    Experts: dense (pack_dense), wd (pack_wd) or fp4 (pack_fp4).  renorm (True): a token's weights are rescaled to sum to 1.  select: a
    SelectRule that chooses the experts from the router's logits, with select_bias seen by the selection alone, in place of the paper's
    softmax and top-k; whether weights are rescaled is then the rule's to say."""

    by_steps, select, fp4, ctx = False, None, None, None

    def __init__(self, d_model, d_ff, n_experts, top_k, w_router, b_router=None, *, dense=None, wd=None, fp4=None,
                 x_dtype=torch.bfloat16, renorm=None, path=B.MOE_PATH_AUTO, max_tokens=1, expert_slot=None, select=None,
                 select_bias=None):
        assert (dense is not None) + (wd is not None) + (fp4 is not None) == 1
        if select is not None and (select.E, select.k) != (n_experts, top_k):
            raise ValueError("the selection rule is for other numbers of experts")
        if select is None and select_bias is not None:
            raise ValueError("select_bias without a selection rule")
        if select is not None:
            if renorm is not None and bool(renorm) != bool(select.c.renorm):
                raise ValueError(f"renorm={renorm}, but the selection rule, which makes the weights, has renorm={bool(select.c.renorm)}")
            renorm = select.c.renorm
        elif renorm is None:
            renorm = True
        if fp4 is not None and (path != B.MOE_PATH_AUTO or expert_slot is not None):
            raise ValueError("4-bit experts take neither a path nor expert_slot")
        self.select, self.select_bias = select, select_bias
        self.d, self.f, self.E, self.k = d_model, d_ff, n_experts, top_k
        self.x_dtype = x_dtype
        self.device = w_router.device
        self._cuda_index = self.device.index if self.device.type == "cuda" else None
        self.rank = 0 if wd is None else wd[0].shape[1]
        self.cfg = B.make_config(d_model, d_ff, n_experts, top_k, self.rank,
                                 B.dtype_of(x_dtype), int(renorm), path)
        if dense is not None:
            self.weights = B.make_weights(w_router, b_router, gud=dense, expert_slot=expert_slot)
        elif wd is not None:
            self.weights = B.make_weights(w_router, b_router, wd_a=wd[0], wd_b=wd[1], wd_c=wd[2], wd_d=wd[3],
                                          expert_slot=expert_slot)
        else:
            self.weights = B.make_weights(w_router, b_router)
        self.by_steps = fp4 is not None or select is not None
        self.ctx = B.moe_create(self.cfg)
        self.max_tokens = max_tokens
        if fp4 is not None:
            self.fp4 = Fp4Experts(d_model, d_ff, n_experts, top_k, fp4[0], fp4[1], x_dtype, max_tokens, ctx=self.ctx)
        self.ws = self.fp4.ws if self.fp4 else torch.empty(B.moe_workspace_bytes(self.cfg, max_tokens), dtype=torch.uint8, device=self.device)

    @classmethod
    def from_math_layout(cls, shape_kw: dict, tensors: dict, **kw):
        """tensors: the dict synth.workloads.make_layer returns (already on the device)."""
        if "w_gate" in tensors:
            dense, wd = pack_dense(tensors["w_gate"], tensors["w_up"], tensors["w_down"]), None
        else:
            dense, wd = None, pack_wd(*(tensors[n] for n in ("gL", "gR", "uL", "uR", "dL", "dR")))
        return cls(shape_kw["d_model"], shape_kw["d_ff"], shape_kw["n_experts"], shape_kw["top_k"],
                   tensors["w_router"], tensors["b_router"], dense=dense, wd=wd, **kw)

    def _need(self, T):
        if T > self.max_tokens:
            raise ValueError(f"T={T} exceeds max_tokens={self.max_tokens} this layer's workspace was sized for")

    # ---- step-by-step calls -------------------------------------------------------------
    def logits(self, x):
        """x [T, d] -> the router's logits, float32 [T, E]."""
        if x.dim() != 2 or x.shape[1] != self.d or x.dtype != self.x_dtype:
            raise ValueError(f"x has to be {self.x_dtype} [T, {self.d}]")
        _here(x)
        out = torch.empty((x.shape[0], self.E), dtype=torch.float32, device=self.device)
        B.moe_route_logits(self.ctx, x, x.shape[0], self.weights, out)
        return out

    def route(self, x, want_probs=False):
        T = x.shape[0]
        if self.select is not None:
            if want_probs:
                raise ValueError("a selection rule has no probabilities to return")
            return (*select_experts(self.logits(x), self.select, self.select_bias), None)
        idx = torch.empty((T, self.k), dtype=torch.int32, device=self.device)
        w = torch.empty((T, self.k), dtype=torch.float32, device=self.device)
        probs = torch.empty((T, self.E), dtype=torch.float32, device=self.device) if want_probs else None
        B.moe_route(self.ctx, x, T, self.weights, idx, w, probs)
        return idx, w, probs

    def permute(self, topk_idx):
        T = topk_idx.shape[0]
        offsets = torch.empty(self.E + 1, dtype=torch.int32, device=self.device)
        perm = torch.empty(T * self.k, dtype=torch.int32, device=self.device)
        inv = torch.empty(T * self.k, dtype=torch.int32, device=self.device)
        B.moe_permute(self.ctx, topk_idx, T, offsets, perm, inv)
        return offsets, perm, inv

    def expert_ffn(self, x, offsets, perm):
        if self.fp4:
            raise ValueError("4-bit experts: forward, or fp4.forward for a given routing")
        T = x.shape[0]
        self._need(T)
        out = torch.empty((T * self.k, self.d), dtype=torch.float32, device=self.device)
        B.moe_expert_ffn(self.ctx, x, T, self.weights, offsets, perm, out, self.ws)
        return out

    def combine(self, out_slots, topk_w, inv):
        T = topk_w.shape[0]
        y = torch.empty((T, self.d), dtype=self.x_dtype, device=self.device)
        B.moe_combine(self.ctx, out_slots, topk_w, inv, T, y)
        return y

    # ---- the whole layer ------------------------------------------------------------------
    def forward(self, x, y=None, topk_idx=None, topk_w=None):
        shape = x.shape
        T = shape[0]
        if T > self.max_tokens:
            self._need(T)
        if self.by_steps:
            return self._forward_by_steps(x, y, topk_idx, topk_w)
        if y is None:
            # one token's layer takes about as long as a few calls into PyTorch: y is allocated the cheapest way where that
            # gives the same tensor (a plain one on the layer's device)
            if (x.get_device() == self._cuda_index and type(x) is torch.Tensor and len(shape) == 2 and shape[1] == self.d
                    and x.dtype == self.x_dtype):
                y = torch.empty_like(x)
            else:
                y = torch.empty((T, self.d), dtype=self.x_dtype, device=self.device)
        B.moe_layer_forward(self.ctx, x, T, self.weights, y, topk_idx, topk_w, self.ws)
        return y

    def _forward_by_steps(self, x, y, topk_idx, topk_w):
        idx, w, _ = self.route(x)
        if topk_idx is not None:
            topk_idx.copy_(idx)
        if topk_w is not None:
            topk_w.copy_(w)
        if self.fp4:
            return self.fp4.forward(x, idx, w, y)
        offsets, perm, inv = self.permute(idx)
        out = self.combine(self.expert_ffn(x, offsets, perm), w, inv)
        return out if y is None else y.copy_(out)

    def check(self) -> int:
        return B.moe_check(self.ctx)

    def close(self):
        if self.fp4:
            self.fp4.close()
        if self.ctx:
            B.moe_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class OffloadedStack:
    """n_layers stacked MoE layers whose experts live in pinned host memory (packed gud layout); the device
    keeps `slots` experts per layer.  Owns the pinned master copy, the device slots, a ctx and its workspace."""

    def __init__(self, d_model, d_ff, n_experts, top_k, slots, layers, x_dtype=torch.bfloat16, device="cuda", fp8=False):
        """layers: iterable of dicts with w_router, b_router and gud [E,f,3,d] (device tensors, consumed one by one).
        fp8: keep the host copies as FP8 codes + row scales (half the bytes per fetch)."""
        import ctypes
        self.fp8 = fp8
        self.d, self.f, self.E, self.k, self.slots = d_model, d_ff, n_experts, top_k, slots
        self.cfg = B.make_config(d_model, d_ff, n_experts, top_k, 0,
                                 B.dtype_of(x_dtype), 1, B.MOE_PATH_STREAM)
        self.slot_bytes = d_ff * 3 * d_model * 2
        self.host, self.routers_t = [], []
        ptrs = []
        self.blob_bytes = d_ff * 3 * d_model + d_ff * 3 * 4 if fp8 else self.slot_bytes
        for lay in layers:
            if fp8:
                gud = lay["gud"]
                rows = n_experts * d_ff * 3
                codes = torch.empty((n_experts, d_ff * 3 * d_model), dtype=torch.uint8, device=gud.device)
                scales = torch.empty((n_experts, d_ff * 3), dtype=torch.float32, device=gud.device)
                B.moe_fp8_quantize_rows(gud, rows, d_model, codes, scales)
                hg = torch.empty((n_experts, self.blob_bytes), dtype=torch.uint8, pin_memory=True)
                hg[:, :d_ff * 3 * d_model].copy_(codes)
                hg[:, d_ff * 3 * d_model:].copy_(scales.view(torch.uint8).reshape(n_experts, -1))
                del codes, scales
            else:
                hg = torch.empty(lay["gud"].shape, dtype=torch.bfloat16, pin_memory=True)
                hg.copy_(lay["gud"])
            self.host.append(hg)
            self.routers_t.append((lay["w_router"], lay["b_router"]))
            ptrs += [hg.data_ptr() + e * self.blob_bytes for e in range(n_experts)]
        self.n_layers = len(self.host)
        torch.cuda.synchronize()
        self.device_slots = torch.empty(self.n_layers * slots * self.slot_bytes, dtype=torch.uint8, device=device)
        self.off = B.moe_offload_create(self.cfg, self.n_layers, slots, ptrs, self.device_slots, self.slot_bytes, fp8=fp8)
        self.ctx = B.moe_create(self.cfg)
        self.ws = torch.empty(B.moe_workspace_bytes(self.cfg, 1), dtype=torch.uint8, device=device)
        self.routers = (B.moe_weights * self.n_layers)()
        for l, (wr, br) in enumerate(self.routers_t):
            self.routers[l].w_router = wr.data_ptr()
            self.routers[l].b_router = br.data_ptr() if br is not None else None
        self._ctypes = ctypes

    def step(self, h):
        """h: fp32 [d] device tensor, updated in place.  Returns the per-layer selections."""
        return B.moe_stack_decode_step(self.off, self.ctx, self.routers, h, self.n_layers, self.k, self.ws)

    def step_trace(self, h, sel):
        """The same step with every layer's expert set given (sel [n_layers][k]); no host wait between layers."""
        B.moe_stack_decode_step_trace(self.off, self.ctx, self.routers, h, sel, self.ws)

    def stats(self):
        return B.moe_offload_stats(self.off)

    def resident(self, layer):
        return B.moe_offload_resident(self.off, layer, self.slots)

    def check(self):
        return B.moe_check(self.ctx)

    def close(self):
        if self.off:
            B.moe_offload_destroy(self.off)
            self.off = None
        if self.ctx:
            B.moe_destroy(self.ctx)
            self.ctx = None
