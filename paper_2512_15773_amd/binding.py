"""ctypes binding of libtsdp.so: argument marshalling only, every step runs in the HIP kernels.

torch is used for device memory and streams.  The library must have been built in-tree
(`python -m paper_2512_15773_amd.build` or `__graft_entry__.build()`); there is no fallback.

Calls only enqueue work on the given (default: torch's current) stream.  The binding passes raw pointers: a tensor
handed to a call must stay alive until that stream has run the call -- torch's caching allocator does not know of the
use and would hand a freed tensor's memory out again (keep a reference, or call Tensor.record_stream yourself).
"""
import ctypes as C
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtsdp.so")

EXPORTS = ["tsdp_create", "tsdp_destroy", "tsdp_load_weights", "tsdp_set_cond", "tsdp_draft", "tsdp_verify",
           "tsdp_accept", "tsdp_round", "tsdp_accept_threshold", "tsdp_round_threshold", "tsdp_chain", "tsdp_chain_staged",
           "tsdp_chain_enqueue", "tsdp_prepare",
           "tsdp_distill_loss", "tsdp_distill_loss_noalloc", "tsdp_status", "tsdp_kernel_timing", "tsdp_kernel_ms", "tsdp_path_name",
           "tsdp_cache_write", "tsdp_cache_read", "tsdp_attend_prompt", "tsdp_attend_paged", "tsdp_attend_scratch",
           "tsdp_last_error"]


class TsdpConfig(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("H", C.c_int32), ("A", C.c_int32), ("cond_mode", C.c_int32),
                ("cond_dim", C.c_int32), ("cond_tokens", C.c_int32),
                ("base_layers", C.c_int32), ("base_d", C.c_int32), ("base_heads", C.c_int32), ("base_mlp_ratio", C.c_int32),
                ("draft_layers", C.c_int32), ("draft_d", C.c_int32), ("draft_heads", C.c_int32), ("draft_mlp_ratio", C.c_int32),
                ("T", C.c_int32), ("schedule", C.c_int32), ("beta0", C.c_float), ("beta1", C.c_float),
                ("clip_x0", C.c_int32), ("clip_val", C.c_float), ("B_max", C.c_int32), ("K_max", C.c_int32),
                ("seed", C.c_uint64), ("sampler", C.c_int32), ("eta", C.c_float),
                ("bonus_row", C.c_int32), ("norm", C.c_int32)]


class TsdpHeads(C.Structure):
    _fields_ = [("type", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("causal", C.c_int32), ("scale", C.c_float)]


class TsdpKvCache(C.Structure):
    _fields_ = [("type", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32),
                ("pages", C.c_int32), ("B", C.c_int32), ("columns", C.c_int32), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("d_k_scale", C.c_void_p), ("d_v_scale", C.c_void_p), ("d_page_table", C.c_void_p)]


_lib = None


def load_library():
    """Loads libtsdp.so and declares the prototypes; raises if the library has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_15773_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32 = C.c_void_p, C.c_int
    lib.tsdp_create.argtypes = [C.POINTER(TsdpConfig), C.POINTER(vp)]
    lib.tsdp_destroy.argtypes = [vp]; lib.tsdp_destroy.restype = None
    lib.tsdp_load_weights.argtypes = [vp, i32, vp, C.c_size_t]
    lib.tsdp_set_cond.argtypes = [vp, vp, i32, vp]
    lib.tsdp_draft.argtypes = [vp, i32] + [vp] * 12 + [vp]
    lib.tsdp_verify.argtypes = [vp, i32, i32] + [vp] * 5 + [vp]
    lib.tsdp_accept.argtypes = [vp, i32] + [vp] * 16 + [vp]
    lib.tsdp_round.argtypes = [vp, i32] + [vp] * 7 + [vp]
    lib.tsdp_accept_threshold.argtypes = [vp, i32] + [vp] * 15 + [vp]
    lib.tsdp_round_threshold.argtypes = [vp, i32] + [vp] * 8 + [vp]
    lib.tsdp_chain.argtypes = [vp, i32] + [vp] * 6 + [i32, i32] + [vp] * 3 + [C.POINTER(C.c_int32), vp]
    lib.tsdp_chain_staged.argtypes = [vp, i32] + [vp] * 5 + [i32, i32, vp, i32, i32] + [vp] * 3 + [C.POINTER(C.c_int32), vp]
    lib.tsdp_chain_enqueue.argtypes = [vp, i32] + [vp] * 5 + [i32, i32, i32, vp, i32] + [vp] * 4 + [vp]
    lib.tsdp_prepare.argtypes = [vp]
    lib.tsdp_distill_loss.argtypes = [vp, i32, vp, vp, vp, vp, C.c_float, C.c_float, vp, vp]
    lib.tsdp_distill_loss_noalloc.argtypes = lib.tsdp_distill_loss.argtypes
    lib.tsdp_status.argtypes = [vp, vp, C.POINTER(C.c_int32)]
    lib.tsdp_kernel_timing.argtypes = [vp, i32]
    lib.tsdp_kernel_ms.argtypes = [vp, i32, C.POINTER(C.c_float)]
    lib.tsdp_path_name.argtypes = [vp, i32]; lib.tsdp_path_name.restype = C.c_char_p
    i64 = C.c_int64
    lib.tsdp_cache_write.argtypes = [vp, C.POINTER(TsdpKvCache), i32, i32, i32, vp, vp, vp, i64, vp, i64, vp]
    lib.tsdp_cache_read.argtypes = lib.tsdp_cache_write.argtypes
    lib.tsdp_attend_prompt.argtypes = [vp, C.POINTER(TsdpHeads), i32, i32, i32, vp, vp] + [vp, i64] * 4 + [vp, vp]
    lib.tsdp_attend_paged.argtypes = [vp, C.POINTER(TsdpHeads), C.POINTER(TsdpKvCache), i32, i32, i32, vp, vp, i64, i32, vp, i64, vp,
                                      vp, i64, vp]
    lib.tsdp_attend_scratch.argtypes = [C.POINTER(TsdpHeads), i32, i32, i32]; lib.tsdp_attend_scratch.restype = i64
    lib.tsdp_last_error.argtypes = [vp]; lib.tsdp_last_error.restype = C.c_char_p
    for name in EXPORTS:
        if getattr(lib, name).restype is C.c_int:
            getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


class TsdpError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"tsdp error {code}: {msg}")
        self.code = code


def _ptr(t, dtype=None):
    if t is None:
        return None
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous"
    if dtype is not None:
        assert t.dtype == dtype, f"expected {dtype}, got {t.dtype}"
    return t.data_ptr()


def _stream(stream):
    # the handle alone: building torch's Stream object takes 3 us
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()) if stream is None else stream.cuda_stream


def _memory_of(stream, make, *args, **kwargs):
    """make(...) with the memory of the stream that the call runs on: nothing that another stream still uses."""
    if stream is None:
        return make(*args, **kwargs)
    with torch.cuda.stream(stream):
        return make(*args, **kwargs)


_TYPE = {torch.float32: 0, torch.bfloat16: 1}


def _rows(t, heads, dim, dtype, dev):
    """Pointer and row stride of packed rows [rows, heads, dim]; the rows may be slices of wider ones."""
    assert t.dtype is dtype and t.dim() == 3, f"expected [rows, {heads}, {dim}] of {dtype}, got {tuple(t.shape)} of {t.dtype}"
    rows, h, d = t.shape
    assert h == heads and d == dim, f"expected [rows, {heads}, {dim}], got {tuple(t.shape)}"
    assert t.get_device() == dev, "packed rows must be on the current device"
    if t.is_contiguous():
        return t.data_ptr(), heads * dim
    row, head, one = t.stride()
    assert one == 1 and (head == dim or heads == 1), "the heads of a row must be next to each other"
    return t.data_ptr(), row if rows > 1 else heads * dim


def _table(t, n, dev):
    """Pointer of an int32 device tensor of n entries."""
    assert t.dtype is torch.int32 and t.get_device() == dev and t.is_contiguous() and t.numel() == n, f"expected {n} contiguous int32 on the current device"
    return t.data_ptr()


class KvCache:
    """A paged cache of keys / values (tsdp_kv_cache): pools k, v [pages, kv_heads, page_tokens, head_dim] in float32, bfloat16
    or uint8 (8 bits, with scale pools [pages, kv_heads, page_tokens, head_dim // 32] in uint8) and the int32 page table
    [B, columns].  The tensors are the caller's and stay the cache's memory: change the table in place."""

    def __init__(self, k, v, page_table, k_scale=None, v_scale=None):
        held = {**_TYPE, torch.uint8: 2}
        assert k.dtype in held, f"a cache holds float32, bfloat16 or uint8, not {k.dtype}"
        assert k.dim() == 4 and k.shape == v.shape and k.dtype == v.dtype, "k and v must be alike, [pages, kv_heads, page_tokens, head_dim]"
        assert page_table.dim() == 2 and k.get_device() == v.get_device() == page_table.get_device(), "pools and table must be on one device"
        pages, kv, page, dim = k.shape
        assert (k_scale is None) == (v_scale is None) == (held[k.dtype] != 2), "scale pools belong to 8 bits, and to nothing else"
        for s in (k_scale, v_scale):
            assert s is None or (tuple(s.shape) == (pages, kv, page, dim // 32) and s.get_device() == k.get_device()), "scale pools must be [pages, kv_heads, page_tokens, head_dim // 32]"
        self.k, self.v, self.k_scale, self.v_scale, self.page_table = k, v, k_scale, v_scale, page_table
        self.kv_heads, self.head_dim, self.device, self.B = kv, dim, k.get_device(), page_table.shape[0]
        self.c = TsdpKvCache(type=held[k.dtype], kv_heads=kv, head_dim=dim, page_tokens=page, pages=pages, B=page_table.shape[0],
                             columns=page_table.shape[1], d_k=_ptr(k), d_v=_ptr(v), d_k_scale=_ptr(k_scale, torch.uint8),
                             d_v_scale=_ptr(v_scale, torch.uint8), d_page_table=_ptr(page_table, torch.int32))
        self.ref = C.byref(self.c)

    @classmethod
    def alloc(cls, dtype, pages, kv_heads, page_tokens, head_dim, page_table):
        """Pools of zeros; dtype float32, bfloat16, or uint8 for 8 bits."""
        f = lambda d, dt: torch.zeros(pages, kv_heads, page_tokens, d, dtype=dt, device=page_table.device)
        scales = [f(head_dim // 32, torch.uint8) for _ in "kv"] if dtype == torch.uint8 else [None, None]
        return cls(f(head_dim, dtype), f(head_dim, dtype), page_table, *scales)


class Tsdp:
    """One library context.  Methods carry the names of the C entry points."""

    def __init__(self, *, dtype, H, A, cond_mode, cond_dim, cond_tokens, base, draft, T, schedule,
                 beta0=1e-4, beta1=0.02, clip=None, B_max, K_max, seed, sampler=0, eta=1.0, bonus_row=False, norm=0):
        """base / draft: (layers, d, heads, mlp_ratio)."""
        self.lib = load_library()
        self.cfg = TsdpConfig(dtype=dtype, H=H, A=A, cond_mode=cond_mode, cond_dim=cond_dim, cond_tokens=cond_tokens,
                              base_layers=base[0], base_d=base[1], base_heads=base[2], base_mlp_ratio=base[3],
                              draft_layers=draft[0], draft_d=draft[1], draft_heads=draft[2], draft_mlp_ratio=draft[3],
                              T=T, schedule=schedule, beta0=beta0, beta1=beta1, clip_x0=0 if clip is None else 1,
                              clip_val=0.0 if clip is None else float(clip), B_max=B_max, K_max=K_max, seed=seed,
                              sampler=sampler, eta=eta, bonus_row=1 if bonus_row else 0, norm=norm)
        self.ctx = C.c_void_p()
        rc = self.lib.tsdp_create(C.byref(self.cfg), C.byref(self.ctx))
        if rc != 0:
            self.ctx = C.c_void_p()
            raise TsdpError(rc, "tsdp_create rejected the configuration")
        self.H, self.A, self.D, self.K_max, self.B_max = H, A, H * A, K_max, B_max
        self.rows_per_env = K_max + (1 if bonus_row else 0)

    @classmethod
    def from_workload(cls, wl, *, B_max=None, K_max=None, clip=None, seed=None, sampler=0, eta=1.0, bonus_row=False, norm=0):
        return cls(dtype=0 if wl.dtype == "fp32" else 1, H=wl.H, A=wl.A, cond_mode=wl.cond_mode, cond_dim=wl.cond_dim,
                   cond_tokens=wl.cond_tokens, base=(wl.base.layers, wl.base.d, wl.base.heads, wl.base.mlp_ratio),
                   draft=(wl.draft.layers, wl.draft.d, wl.draft.heads, wl.draft.mlp_ratio), T=wl.T,
                   schedule=wl.schedule, beta0=wl.beta0 or 1e-4, beta1=wl.beta1 or 0.02, clip=clip,
                   B_max=wl.B if B_max is None else B_max, K_max=wl.K_max if K_max is None else K_max,
                   seed=wl.philox_seed if seed is None else seed, sampler=sampler, eta=eta,
                   bonus_row=bonus_row, norm=norm)

    def close(self):
        if self.ctx:
            self.lib.tsdp_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, rc):
        if rc != 0:
            raise TsdpError(rc, self.lib.tsdp_last_error(self.ctx).decode())

    def path_name(self, which):
        return self.lib.tsdp_path_name(self.ctx, which).decode()

    def tsdp_load_weights(self, which, blob):
        blob = np.ascontiguousarray(blob, dtype=np.float32)
        self._chk(self.lib.tsdp_load_weights(self.ctx, which, blob.ctypes.data, blob.nbytes))

    def tsdp_set_cond(self, cond, stream=None):
        self._chk(self.lib.tsdp_set_cond(self.ctx, _ptr(cond, torch.float32), cond.shape[0], _stream(stream)))

    def alloc_rows(self, B, device="cuda"):
        """Caller-side ragged buffers for tsdp_draft / tsdp_verify / tsdp_accept (R_cap = B*(K_max + bonus_row) rows)."""
        R, D = B * self.rows_per_env, self.D
        f = lambda *s: torch.zeros(*s, dtype=torch.float32, device=device)
        i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=device)
        return dict(row_ptr=i(B + 1), row_t=i(R), row_env=i(R), states=f(R, self.H, self.A), eps_p=f(R, self.H, self.A),
                    eps_q=f(R, self.H, self.A), xi=f(R, self.H, self.A), y_last=f(B, self.H, self.A))

    def tsdp_draft(self, x, t0, K, sigma_scale, env_id, rows, stream=None):
        B = x.shape[0]
        self._chk(self.lib.tsdp_draft(self.ctx, B, _ptr(x, torch.float32), _ptr(t0, torch.int32), _ptr(K, torch.int32),
                                      _ptr(sigma_scale, torch.float32), _ptr(env_id, torch.int32),
                                      _ptr(rows["row_ptr"]), _ptr(rows["row_t"]), _ptr(rows["row_env"]),
                                      _ptr(rows["states"]), _ptr(rows["eps_p"]), _ptr(rows["xi"]), _ptr(rows["y_last"]),
                                      _stream(stream)))

    def tsdp_verify(self, B, rows, R_cap=None, stream=None):
        R_cap = rows["row_t"].shape[0] if R_cap is None else R_cap
        self._chk(self.lib.tsdp_verify(self.ctx, B, R_cap, _ptr(rows["row_ptr"], torch.int32), _ptr(rows["row_t"], torch.int32),
                                       _ptr(rows["row_env"], torch.int32), _ptr(rows["states"], torch.float32),
                                       _ptr(rows["eps_q"], torch.float32), _stream(stream)))

    def tsdp_accept(self, B, sigma_scale, env_id, rows, diagnostics=True, stream=None):
        dev = rows["states"].device
        R = rows["row_t"].shape[0]
        out = dict(x_out=torch.empty(B, self.H, self.A, dtype=torch.float32, device=dev),
                   t_next=torch.empty(B, dtype=torch.int32, device=dev),
                   n_accept=torch.empty(B, dtype=torch.int32, device=dev),
                   n_adv=torch.empty(B, dtype=torch.int32, device=dev))
        if diagnostics:
            out.update(flags=torch.zeros(R, dtype=torch.uint8, device=dev),
                       logratio=torch.zeros(R, dtype=torch.float32, device=dev),
                       logu=torch.zeros(R, dtype=torch.float32, device=dev))
        self.tsdp_accept_into(B, sigma_scale, env_id, rows, out, stream)
        return out

    def tsdp_accept_into(self, B, sigma_scale, env_id, rows, out, stream=None):
        self._chk(self.lib.tsdp_accept(self.ctx, B, _ptr(rows["row_ptr"], torch.int32), _ptr(rows["row_t"], torch.int32),
                                       _ptr(env_id, torch.int32), _ptr(sigma_scale, torch.float32),
                                       _ptr(rows["states"], torch.float32), _ptr(rows["eps_p"], torch.float32),
                                       _ptr(rows["eps_q"], torch.float32), _ptr(rows["xi"], torch.float32),
                                       _ptr(rows["y_last"], torch.float32), _ptr(out["x_out"]), _ptr(out["t_next"]),
                                       _ptr(out["n_accept"]), _ptr(out.get("n_adv")), _ptr(out.get("flags")),
                                       _ptr(out.get("logratio")), _ptr(out.get("logu")), _stream(stream)))

    def tsdp_accept_threshold(self, B, sigma_scale, lam, rows, stream=None):
        dev = rows["states"].device
        R = rows["row_t"].shape[0]
        out = dict(x_out=torch.empty(B, self.H, self.A, dtype=torch.float32, device=dev),
                   t_next=torch.empty(B, dtype=torch.int32, device=dev), n_accept=torch.empty(B, dtype=torch.int32, device=dev),
                   n_adv=torch.empty(B, dtype=torch.int32, device=dev), flags=torch.zeros(R, dtype=torch.uint8, device=dev),
                   logratio=torch.zeros(R, dtype=torch.float32, device=dev))
        self._chk(self.lib.tsdp_accept_threshold(self.ctx, B, _ptr(rows["row_ptr"], torch.int32), _ptr(rows["row_t"], torch.int32),
                                                 _ptr(sigma_scale, torch.float32), _ptr(lam, torch.float32),
                                                 _ptr(rows["states"], torch.float32), _ptr(rows["eps_p"], torch.float32),
                                                 _ptr(rows["eps_q"], torch.float32), _ptr(rows["xi"], torch.float32),
                                                 _ptr(rows["y_last"], torch.float32), _ptr(out["x_out"]), _ptr(out["t_next"]),
                                                 _ptr(out["n_accept"]), _ptr(out["n_adv"]), _ptr(out["flags"]),
                                                 _ptr(out["logratio"]), _stream(stream)))
        return out

    def tsdp_round_threshold(self, x, t, K, sigma_scale, env_id, lam, n_accept=None, n_advanced=None, stream=None):
        self._chk(self.lib.tsdp_round_threshold(self.ctx, x.shape[0], _ptr(x, torch.float32), _ptr(t, torch.int32),
                                                _ptr(K, torch.int32), _ptr(sigma_scale, torch.float32),
                                                _ptr(env_id, torch.int32), _ptr(lam, torch.float32),
                                                _ptr(n_accept, torch.int32), _ptr(n_advanced, torch.int32), _stream(stream)))

    def tsdp_chain(self, x, t, K, sigma_scale, env_id, lam=None, max_rounds=1000, check_every=4, totals=True, stream=None):
        """Runs rounds until every environment finishes; returns (rounds, totals dict or None)."""
        B = x.shape[0]
        tot = None
        if totals:
            tot = {k: torch.zeros(B, dtype=torch.int32, device=x.device) for k in ("accept", "drafts", "rounds")}
        n = C.c_int32(0)
        self._chk(self.lib.tsdp_chain(self.ctx, B, _ptr(x, torch.float32), _ptr(t, torch.int32), _ptr(K, torch.int32),
                                      _ptr(sigma_scale, torch.float32), _ptr(env_id, torch.int32), _ptr(lam, torch.float32),
                                      max_rounds, check_every, _ptr(tot["accept"]) if tot else None,
                                      _ptr(tot["drafts"]) if tot else None, _ptr(tot["rounds"]) if tot else None,
                                      C.byref(n), _stream(stream)))
        return n.value, tot

    def tsdp_chain_staged(self, x, t, K3, sigma_scale3, lam3, t_hi, t_lo, env_id, max_rounds=1000, check_every=4,
                          totals=True, stream=None):
        """tsdp_chain with [B,3] stage tables; returns (rounds, totals dict or None)."""
        B = x.shape[0]
        tot = None
        if totals:
            tot = {k: torch.zeros(B, dtype=torch.int32, device=x.device) for k in ("accept", "drafts", "rounds")}
        n = C.c_int32(0)
        self._chk(self.lib.tsdp_chain_staged(self.ctx, B, _ptr(x, torch.float32), _ptr(t, torch.int32),
                                             _ptr(K3, torch.int32), _ptr(sigma_scale3, torch.float32),
                                             _ptr(lam3, torch.float32), t_hi, t_lo, _ptr(env_id, torch.int32),
                                             max_rounds, check_every, _ptr(tot["accept"]) if tot else None,
                                             _ptr(tot["drafts"]) if tot else None, _ptr(tot["rounds"]) if tot else None,
                                             C.byref(n), _stream(stream)))
        return n.value, tot

    def tsdp_chain_enqueue(self, x, t, K, sigma_scale, lam, env_id, n_rounds, *, stages=None, totals=None,
                           rounds_run=None, stream=None):
        """Enqueues exactly n_rounds rounds with no host round trip.  stages = (t_hi, t_lo) makes K, sigma_scale and
        lam [B,3] stage tables.  totals: dict of caller-allocated int32[B] device tensors (accept, drafts, rounds) or
        None; rounds_run: caller-allocated int32[1] device tensor or None."""
        tot = totals or {}
        self._chk(self.lib.tsdp_chain_enqueue(self.ctx, x.shape[0], _ptr(x, torch.float32), _ptr(t, torch.int32),
                                              _ptr(K, torch.int32), _ptr(sigma_scale, torch.float32),
                                              _ptr(lam, torch.float32), 0 if stages is None else 1,
                                              0 if stages is None else stages[0], 0 if stages is None else stages[1],
                                              _ptr(env_id, torch.int32), n_rounds, _ptr(tot.get("accept")),
                                              _ptr(tot.get("drafts")), _ptr(tot.get("rounds")),
                                              _ptr(rounds_run, torch.int32), _stream(stream)))

    def tsdp_prepare(self):
        self._chk(self.lib.tsdp_prepare(self.ctx))

    def tsdp_distill_loss(self, R, rows, lambda1, lambda2, stream=None):
        loss = torch.zeros(3, dtype=torch.float64, device=rows["states"].device)
        self._chk(self.lib.tsdp_distill_loss(self.ctx, R, _ptr(rows["row_t"], torch.int32), _ptr(rows["states"], torch.float32),
                                             _ptr(rows["eps_p"], torch.float32), _ptr(rows["eps_q"], torch.float32),
                                             lambda1, lambda2, _ptr(loss), _stream(stream)))
        return loss

    def tsdp_distill_loss_noalloc(self, R, rows, lambda1, lambda2, loss, stream=None):
        """`loss`: caller-allocated float64[3] device tensor (this entry point allocates nothing)."""
        self._chk(self.lib.tsdp_distill_loss_noalloc(self.ctx, R, _ptr(rows["row_t"], torch.int32),
                                                     _ptr(rows["states"], torch.float32), _ptr(rows["eps_p"], torch.float32),
                                                     _ptr(rows["eps_q"], torch.float32), lambda1, lambda2,
                                                     _ptr(loss, torch.float64), _stream(stream)))

    def tsdp_round(self, x, t, K, sigma_scale, env_id, n_accept=None, n_advanced=None, stream=None):
        self._chk(self.lib.tsdp_round(self.ctx, x.shape[0], _ptr(x, torch.float32), _ptr(t, torch.int32),
                                      _ptr(K, torch.int32), _ptr(sigma_scale, torch.float32), _ptr(env_id, torch.int32),
                                      _ptr(n_accept, torch.int32), _ptr(n_advanced, torch.int32), _stream(stream)))

    def _cache_rows(self, call, cache, row_ptr, start, k, v, stream):
        dev = torch.cuda.current_device()
        dtype, rows, B = k.dtype, k.shape[0], start.shape[0]
        assert cache.device == dev, "the cache must be on the current device"
        assert dtype in _TYPE and v.shape[0] == rows, "rows of keys and values must be alike, float32 or bfloat16"
        kp, k_row = _rows(k, cache.kv_heads, cache.head_dim, dtype, dev)
        vp, v_row = _rows(v, cache.kv_heads, cache.head_dim, dtype, dev)
        rc = call(self.ctx, cache.ref, B, rows, _TYPE[dtype], _table(row_ptr, B + 1, dev), _table(start, B, dev), kp, k_row, vp, v_row, _stream(stream))
        if rc:
            self._chk(rc)

    def tsdp_cache_write(self, cache, row_ptr, start, k, v, stream=None):
        """Rows row_ptr[b] .. of k, v [rows, kv_heads, head_dim] to positions start[b] .. of environment b."""
        self._cache_rows(self.lib.tsdp_cache_write, cache, row_ptr, start, k, v, stream)

    def tsdp_cache_read(self, cache, row_ptr, start, rows, dtype, out=None, stream=None):
        """Positions start[b] .. of every environment as packed rows (k, v); out: such a pair to write into."""
        if out is None:
            out = _memory_of(stream, row_ptr.new_empty, (2, rows, cache.kv_heads, cache.head_dim), dtype=dtype).unbind()
        assert out[0].dtype is dtype and out[0].shape[0] == rows, "out must hold `rows` rows of the given type"
        self._cache_rows(self.lib.tsdp_cache_read, cache, row_ptr, start, out[0], out[1], stream)
        return out

    @staticmethod
    def _lse(lse, rows, heads, dev):
        if lse is None:
            return None
        assert tuple(lse.shape) == (rows, heads) and lse.get_device() == dev, f"lse must be [{rows}, {heads}]"
        return _ptr(lse, torch.float32)

    def tsdp_attend_prompt(self, q, k, v, q_ptr, k_ptr=None, *, causal=True, scale=None, out=None, lse=None, stream=None):
        """q [rows, q_heads, head_dim] (float32 or bfloat16), k, v [rows of keys, kv_heads, head_dim]; returns out."""
        dev = torch.cuda.current_device()
        dtype = q.dtype
        (rows, heads, dim), (k_rows, kv, _) = q.shape, k.shape
        assert dtype in _TYPE and v.shape[0] == k_rows, "q, k and v must be of one type, float32 or bfloat16, and k and v alike"
        if out is None:
            out = _memory_of(stream, torch.empty_like, q, memory_format=torch.contiguous_format)
        assert out.shape[0] == rows, "out must be alike q"
        qp, q_row = _rows(q, heads, dim, dtype, dev)
        kp, k_row = _rows(k, kv, dim, dtype, dev)
        vp, v_row = _rows(v, kv, dim, dtype, dev)
        op, out_row = _rows(out, heads, dim, dtype, dev)
        n = q_ptr.shape[0]
        rc = self.lib.tsdp_attend_prompt(self.ctx, TsdpHeads(_TYPE[dtype], heads, kv, dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale),
                                         n - 1, rows, k_rows, _table(q_ptr, n, dev), None if k_ptr is None else _table(k_ptr, n, dev),
                                         qp, q_row, kp, k_row, vp, v_row, op, out_row, self._lse(lse, rows, heads, dev), _stream(stream))
        if rc:
            self._chk(rc)
        return out

    def alloc_scratch(self, cache, q_heads, tokens, max_len, B=None):
        """Scratch of tsdp_attend_paged for B environments (default: as many as the page table has), uint8, or None.  A cache of 8
        bits: for queries of either type (fp32 ones need the most)."""
        h = TsdpHeads(1 if cache.c.type == 1 else 0, q_heads, cache.kv_heads, cache.head_dim, 1, 1.0)
        n = self.lib.tsdp_attend_scratch(h, cache.B if B is None else B, tokens, max_len)
        if n < 0:
            raise TsdpError(int(n), "tsdp_attend_scratch rejected the sizes")
        return cache.k.new_empty(n, dtype=torch.uint8) if n else None

    def tsdp_attend_paged(self, q, cache, length, max_len, *, tokens=1, causal=True, scale=None, out_dtype=None, out=None, lse=None,
                          scratch=None, stream=None):
        """q [B * tokens, q_heads, head_dim] over the first length[b] tokens of the cache; returns out (out_dtype: float32 or
        that of q).  scratch: from alloc_scratch (allocated for the call where it is left out)."""
        dev = torch.cuda.current_device()
        dtype, B = q.dtype, length.shape[0]
        rows, heads, dim = q.shape
        assert cache.device == dev, "the cache must be on the current device"
        assert dtype in _TYPE and rows == B * tokens and dim == cache.head_dim, "q must be [B * tokens, q_heads, head_dim], float32 or bfloat16"
        if out is None:
            out = _memory_of(stream, torch.empty_like, q, dtype=out_dtype, memory_format=torch.contiguous_format)
        assert out.dtype in _TYPE and out.shape[0] == rows and out_dtype in (None, out.dtype), "out must be alike q, float32 or bfloat16"
        assert scratch is None or scratch.get_device() == dev, "scratch must be on the current device"
        if scratch is None:
            scratch = _memory_of(stream, self.alloc_scratch, cache, heads, tokens, max_len, B)
        qp, q_row = _rows(q, heads, dim, dtype, dev)
        op, out_row = _rows(out, heads, dim, out.dtype, dev)
        rc = self.lib.tsdp_attend_paged(self.ctx, TsdpHeads(_TYPE[dtype], heads, cache.kv_heads, dim, 1 if causal else 0, dim ** -0.5 if scale is None else scale),
                                        cache.ref, B, tokens, max_len, _table(length, B, dev), qp, q_row, _TYPE[out.dtype], op, out_row,
                                        self._lse(lse, rows, heads, dev), _ptr(scratch),
                                        0 if scratch is None else scratch.numel() * scratch.element_size(), _stream(stream))
        if rc:
            self._chk(rc)
        return out

    def tsdp_kernel_timing(self, enable):
        """False / 0 = off, True / 1 = all stages, 2 * mask = chosen stages (mask bit 0 drafter, 1 verify, 2 accept)."""
        self._chk(self.lib.tsdp_kernel_timing(self.ctx, int(enable)))

    def tsdp_kernel_ms(self, stage):
        ms = C.c_float(0)
        self._chk(self.lib.tsdp_kernel_ms(self.ctx, stage, C.byref(ms)))
        return ms.value

    def tsdp_status(self, stream=None):
        st = C.c_int32(0)
        self._chk(self.lib.tsdp_status(self.ctx, _stream(stream), C.byref(st)))
        return st.value
