"""ctypes binding of the Qwen3-shaped adapter step (include/qwen3.h and
include/qwen3_prompt.h) in libgpt2_mi355x.so.

Argument marshalling only: torch supplies the device buffers and the stream,
every step runs in the library's HIP kernels. Also maps the per-projection
tensors of the oracle's parameter dictionaries to the library's packed
layouts (q|k|v and gate|up stacked, adapter ranks zero-padded) and back.
"""
from __future__ import annotations

import ctypes
import functools

import numpy as np

from .binding import (GPT2_ERR_INVALID_ARG, LibError, Muon, i32, lib as _lib_gpt2, muon_settings, on_stream,
                      stream_buffer)

RP = 64   # padded adapter rank of the library
# kernel classes of the timing probes (QWEN3_K_* in include/qwen3.h)
FUSION = dict(swiglu=0)
KCLASS = dict(gemm_fwd=0, gemm_dx=1, gemm_adapter=2, attn_fwd=3, attn_bwd=4, norm=5, cross_entropy=6, optimizer=7,
              other=8)
GROUPS = {"qkv": 1, "o": 2, "gate_up": 4, "down": 8}
_GROUP_TARGETS = {"qkv": ("q", "k", "v"), "o": ("o",), "gate_up": ("gate", "up"), "down": ("down",)}


class Qwen3Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layer", "d_model", "n_head", "n_kv_head", "head_dim", "d_ff",
                                              "vocab", "max_seq_len", "B", "T")] + [
        ("rms_eps", ctypes.c_float), ("rope_theta", ctypes.c_float), ("lora_rank", ctypes.c_int32),
        ("lora_alpha", ctypes.c_float), ("lora_groups", ctypes.c_int32), ("loss_from", ctypes.c_float),
        ("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("adam_eps", ctypes.c_float),
        ("weight_decay", ctypes.c_float), ("grad_clip", ctypes.c_float)]


_BUFS = ("base_bf16", "lora_f32", "lora_grads", "adam_m", "adam_v", "lora_bf16", "activations", "workspace")


class Qwen3Sizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in _BUFS]


class Qwen3Buffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in _BUFS]


class Rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_tokens", "n_head", "n_kv_head", "head_dim", "n_axes")] + [
        ("sections", ctypes.c_int32 * 4), ("interleaved", ctypes.c_int32), ("theta", ctypes.c_float),
        ("rms_eps", ctypes.c_float)]


class PrefixConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_head", "n_kv_head", "head_dim", "prefix_len", "n_seq",
                                              "prefix_queries")]


_lib = None


def lib():
    """The shared library with the qwen3_* prototypes declared."""
    global _lib
    if _lib is not None:
        return _lib
    L = _lib_gpt2()
    P, I32, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_float
    protos = {
        "qwen3_query_sizes": (I32, [ctypes.POINTER(Qwen3Config), ctypes.POINTER(Qwen3Sizes)]),
        "qwen3_tensor_info": (I32, [ctypes.POINTER(Qwen3Config), I32, I32, ctypes.c_char_p,
                                    ctypes.POINTER(ctypes.c_size_t), ctypes.POINTER(I32), ctypes.POINTER(I32)]),
        "qwen3_init": (I32, [ctypes.POINTER(Qwen3Config), ctypes.POINTER(Qwen3Buffers), P, ctypes.POINTER(P)]),
        "qwen3_sync_weights": (I32, [P]),
        "qwen3_forward": (I32, [P, P, P]),
        "qwen3_backward": (I32, [P]),
        "qwen3_adamw_step": (I32, [P, ctypes.c_int64, P]),
        "qwen3_rotary_forward": (I32, [ctypes.POINTER(Rotary), P, P, P, P, P, P]),
        "qwen3_rotary_backward": (I32, [ctypes.POINTER(Rotary), P, P, P, P, P, P, P]),
        "qwen3_set_positions": (I32, [P, P, I32, ctypes.POINTER(I32), I32]),
        "qwen3_prefix_size": (I32, [ctypes.POINTER(PrefixConfig), ctypes.POINTER(I32),
                                    ctypes.POINTER(ctypes.c_size_t)]),
        "qwen3_prefix_create": (I32, [ctypes.POINTER(PrefixConfig), ctypes.POINTER(I32), P, ctypes.c_size_t, P,
                                      ctypes.POINTER(P)]),
        "qwen3_prefix_forward": (I32, [P, P, P, P, P]),
        "qwen3_prefix_backward": (I32, [P, P, P, P, P, P, P]),
        "qwen3_prefix_destroy": (None, [P]),
        "qwen3_layout_size": (I32, [P, I32, I32, ctypes.POINTER(I32), ctypes.POINTER(ctypes.c_size_t)]),
        "qwen3_set_layout": (I32, [P, I32, I32, ctypes.POINTER(I32), P, ctypes.c_size_t]),
        "qwen3_muon_size": (I32, [ctypes.POINTER(Qwen3Config), ctypes.POINTER(ctypes.c_size_t)]),
        "qwen3_muon_step": (I32, [P, ctypes.POINTER(Muon), P, ctypes.c_size_t, P]),
        "qwen3_loss": (I32, [P, ctypes.POINTER(F32), P]),
        "qwen3_set_fusion": (I32, [P, I32, I32]),
        "qwen3_destroy": (None, [P]),
        "qwen3_last_error": (ctypes.c_char_p, [P]),
        "qwen3_probe_enable": (I32, [P, ctypes.c_uint32]),
        "qwen3_probe_reset": (I32, [P]),
        "qwen3_probe_read": (I32, [P, I32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64),
                                   ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]),
    }
    for name, (res, args) in protos.items():
        f = getattr(L, name)
        f.restype, f.argtypes = res, args
    _lib = L
    return L


def make_config(w: dict, optim: dict | None = None) -> Qwen3Config:
    """Library config from a workload dict and optimiser settings (the
    oracle's field names); adapter targets become whole groups."""
    src = dict(w)
    src.update(optim or {})
    c = Qwen3Config()
    for f, _ in Qwen3Config._fields_:
        if f != "lora_groups" and f in src:
            setattr(c, f, src[f])
    targets = tuple(src.get("lora_targets", ("q", "k", "v", "o")))
    groups = 0
    for g, ts in _GROUP_TARGETS.items():
        present = [t in targets for t in ts]
        if any(present):
            if not all(present):
                raise ValueError(f"adapter targets must cover the whole group {ts}")
            groups |= GROUPS[g]
    c.lora_groups = groups
    return c


def out_widths(cfg: Qwen3Config) -> dict:
    qd, kvd = cfg.n_head * cfg.head_dim, cfg.n_kv_head * cfg.head_dim
    return {"q": qd, "k": kvd, "v": kvd, "o": cfg.d_model, "gate": cfg.d_ff, "up": cfg.d_ff, "down": cfg.d_model}


def targets_of(cfg: Qwen3Config) -> tuple:
    return tuple(t for g, ts in _GROUP_TARGETS.items() if cfg.lora_groups & GROUPS[g] for t in ts)


def _check(status, handle=None):
    if status != 0:
        msg = lib().qwen3_last_error(handle)
        raise LibError(status, msg.decode() if msg else "")


def query_sizes(cfg: Qwen3Config) -> Qwen3Sizes:
    s = Qwen3Sizes()
    _check(lib().qwen3_query_sizes(ctypes.byref(cfg), ctypes.byref(s)))
    return s


def tensor_table(cfg: Qwen3Config, which: int):
    """[(name, offset, shape)] of the base (0) or adapter (1) layout."""
    out, i = [], 0
    name = ctypes.create_string_buffer(64)
    off = ctypes.c_size_t()
    shape = (ctypes.c_int32 * 3)()
    nd = ctypes.c_int32()
    while lib().qwen3_tensor_info(ctypes.byref(cfg), which, i, name, ctypes.byref(off), shape, ctypes.byref(nd)) == 0:
        out.append((name.value.decode(), off.value, tuple(shape[k] for k in range(nd.value))))
        i += 1
    return out


def pack_base(base: dict) -> dict:
    """The library's base tensors from the oracle's: q|k|v and gate|up stacked."""
    p = dict(base)
    p["qkv"] = np.concatenate([base["q"], base["k"], base["v"]], axis=1)
    p["gate_up"] = np.concatenate([base["gate"], base["up"]], axis=1)
    return p


def pack_lora(lora: dict, shapes: dict, r: int) -> dict:
    """Padded group tensors (name -> array of the library's shape) from the
    oracle's per-projection A [L, r, in] and B [L, out, r]."""
    out = {}
    for g, ts in _GROUP_TARGETS.items():
        if g + "_A" not in shapes:
            continue
        A = np.zeros(shapes[g + "_A"], dtype=np.float32)
        B = np.zeros(shapes[g + "_B"], dtype=np.float32)
        row = 0
        for j, t in enumerate(ts):
            A[:, j * RP:j * RP + r, :] = lora[t + "_A"]
            o = lora[t + "_B"].shape[1]
            B[:, row:row + o, :r] = lora[t + "_B"]
            row += o
        out[g + "_A"], out[g + "_B"] = A, B
    return out


def unpack_lora(packed: dict, targets, r: int, out_widths: dict) -> dict:
    """The oracle's per-projection tensors from the library's padded groups."""
    res = {}
    for g, ts in _GROUP_TARGETS.items():
        if g + "_A" not in packed:
            continue
        row = 0
        for j, t in enumerate(ts):
            o = out_widths[t]
            res[t + "_A"] = packed[g + "_A"][:, j * RP:j * RP + r, :]
            res[t + "_B"] = packed[g + "_B"][:, row:row + o, :r]
            row += o
    return {k: v for k, v in res.items() if k[:-2] in targets}


def _device_rows(t, name, dtype, like=None, shape=None):
    """A contiguous device tensor of the dtype, on like's device, or ValueError."""
    try:
        if (t.dtype is dtype and (t.device == like.device if like is not None else t.is_cuda)
                and (shape is None or t.shape == shape) and t.is_contiguous()):
            return t
    except AttributeError:   # not a tensor
        pass
    raise ValueError(f"{name} must be a contiguous {dtype} device tensor"
                     + (f" of shape {tuple(shape)}" if shape is not None else "")
                     + (" on the other tensors' device" if like is not None else ""))


@functools.lru_cache(maxsize=256)
def _rotary_desc(n, n_head, n_kv_head, width, sections, interleaved, theta, eps):
    """The call's description, made once per shape, and head_dim."""
    if n_head < 1 or n_kv_head < 1 or width % (n_head + 2 * n_kv_head) or not 1 <= len(sections) <= 4:
        raise ValueError("rows of q | k | v are (n_head + 2 n_kv_head) head_dim wide, with 1 to 4 sections")
    hd = width // (n_head + 2 * n_kv_head)
    return ctypes.byref(Rotary(i32(n), i32(n_head), i32(n_kv_head), i32(hd), len(sections),
                               (ctypes.c_int32 * 4)(*map(i32, sections)),
                               int(bool(interleaved)), theta, eps)), hd


def _rotary_args(qkv, positions, n_head, n_kv_head, sections, theta, q_norm, k_norm, eps, interleaved):
    import torch
    _device_rows(qkv, "q | k | v", torch.bfloat16)
    if qkv.dim() != 2:
        raise ValueError("rows of q | k | v [tokens, (n_head + 2 n_kv_head) head_dim]")
    n, width = qkv.shape
    # plain numbers: descriptions are kept by value, and a tensor's would be its identity
    sections = tuple(map(int, sections))
    r, hd = _rotary_desc(n, int(n_head), int(n_kv_head), width, sections, bool(interleaved), float(theta), float(eps))
    _device_rows(positions, "positions", torch.int32, qkv, (len(sections), n))
    for name, g in (("q_norm", q_norm), ("k_norm", k_norm)):
        if g is not None:
            _device_rows(g, name, torch.bfloat16, qkv, (hd,))
    return r


def _ptr(t):
    return None if t is None else t.data_ptr()


def rotary(qkv, positions, *, n_head, n_kv_head, sections, theta=1e6, q_norm=None, k_norm=None, eps=1e-6,
           interleaved=False, out=None):
    """Head norm (with gains q_norm and k_norm) and rotary embedding of the
    query and key heads of qkv, bf16 [tokens, (n_head + 2 n_kv_head) head_dim],
    at positions int32 [axes, tokens]; sections: pairs per axis
    (qwen3_rotary_forward). On the current stream; out may be qkv."""
    import torch
    r = _rotary_args(qkv, positions, n_head, n_kv_head, sections, theta, q_norm, k_norm, eps, interleaved)
    out = torch.empty_like(qkv) if out is None else _device_rows(out, "out", torch.bfloat16, qkv, qkv.shape)
    _check(on_stream(qkv.device, lib().qwen3_rotary_forward, r, qkv.data_ptr(), positions.data_ptr(), _ptr(q_norm),
                     _ptr(k_norm), out.data_ptr()))
    return out


def rotary_backward(dout, qkv, positions, *, n_head, n_kv_head, sections, theta=1e6, q_norm=None, k_norm=None,
                    eps=1e-6, interleaved=False, out=None):
    """The gradient of rotary's qkv from that of its result
    (qwen3_rotary_backward); out may be dout."""
    import torch
    r = _rotary_args(qkv, positions, n_head, n_kv_head, sections, theta, q_norm, k_norm, eps, interleaved)
    _device_rows(dout, "dout", torch.bfloat16, qkv, qkv.shape)
    out = torch.empty_like(qkv) if out is None else _device_rows(out, "out", torch.bfloat16, qkv, qkv.shape)
    _check(on_stream(qkv.device, lib().qwen3_rotary_backward, r, dout.data_ptr(), qkv.data_ptr(),
                     positions.data_ptr(), _ptr(q_norm), _ptr(k_norm), out.data_ptr()))
    return out


class SharedPrefix:
    """Attention over packed sequences that share one prefix
    (qwen3_prefix_*): tokens of the prefix, then of each sequence. The layout
    is made once and its calls run one at a time, on the current stream."""

    def __init__(self, n_head, n_kv_head, head_dim, prefix_len, seq_lens, prefix_queries=True, device="cuda"):
        import torch
        self.torch = torch
        self.h = ctypes.c_void_p()
        lens = [i32(n) for n in seq_lens]
        n_head, n_kv_head, head_dim, prefix_len = map(i32, (n_head, n_kv_head, head_dim, prefix_len))
        cfg = PrefixConfig(n_head, n_kv_head, head_dim, prefix_len, len(lens), int(bool(prefix_queries)))
        c_lens = (ctypes.c_int32 * len(lens))(*lens)
        n = ctypes.c_size_t()
        _check(lib().qwen3_prefix_size(ctypes.byref(cfg), c_lens, ctypes.byref(n)))
        self.tokens = prefix_len + sum(lens)
        self.rows = self.tokens if prefix_queries else sum(lens)
        self.n_head, self.width, self.out_width = n_head, (n_head + 2 * n_kv_head) * head_dim, n_head * head_dim
        self.plan = torch.empty(n.value, dtype=torch.uint8, device=device)
        with torch.cuda.device(self.plan.device):
            self.stream = torch.cuda.current_stream().cuda_stream
            _check(lib().qwen3_prefix_create(ctypes.byref(cfg), c_lens, self.plan.data_ptr(), n.value, self.stream,
                                             ctypes.byref(self.h)))

    def close(self):
        if self.h:
            lib().qwen3_prefix_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _run(self, fn, *args):
        def call(*args):
            if args[-1] != self.stream:   # the buffer is another stream's: it stays until this one is done with it
                self.plan.record_stream(self.torch.cuda.current_stream(self.plan.device))
            return fn(self.h, *args)
        _check(on_stream(self.plan.device, call, *args))

    def _rows(self, t, name, shape, dtype=None):
        return _device_rows(t, name, dtype or self.torch.bfloat16, self.plan, shape)

    def forward(self, qkv, out=None, lse=None):
        """(out [rows, n_head head_dim] bf16, lse [n_head, rows] fp32) of qkv
        [tokens, (n_head + 2 n_kv_head) head_dim] bf16; rows: the tokens with
        queries."""
        torch = self.torch
        self._rows(qkv, "q | k | v", (self.tokens, self.width))
        shapes = (self.rows, self.out_width), (self.n_head, self.rows)
        out = qkv.new_empty(shapes[0]) if out is None else self._rows(out, "out", shapes[0])
        lse = (qkv.new_empty(shapes[1], dtype=torch.float32) if lse is None
               else self._rows(lse, "lse", shapes[1], torch.float32))
        self._run(lib().qwen3_prefix_forward, qkv.data_ptr(), out.data_ptr(), lse.data_ptr())
        return out, lse

    def backward(self, dout, qkv, out, lse, dqkv=None):
        """The gradient of qkv from dout, that of out, and the forward's qkv,
        out and lse."""
        torch = self.torch
        self._rows(qkv, "q | k | v", (self.tokens, self.width))
        self._rows(dout, "dout", (self.rows, self.out_width))
        self._rows(out, "out", (self.rows, self.out_width))
        self._rows(lse, "lse", (self.n_head, self.rows), torch.float32)
        dqkv = torch.empty_like(qkv) if dqkv is None else self._rows(dqkv, "dqkv", (self.tokens, self.width))
        self._run(lib().qwen3_prefix_backward, qkv.data_ptr(), out.data_ptr(), lse.data_ptr(), dout.data_ptr(),
                  dqkv.data_ptr())
        return dqkv


class Qwen3:
    """One model instance on a torch-owned set of device buffers."""

    def __init__(self, cfg: Qwen3Config, device="cuda"):
        import torch
        self.torch = torch
        self.cfg = cfg
        sizes = query_sizes(cfg)
        self.bufs = {n: torch.zeros(getattr(sizes, n), dtype=torch.uint8, device=device) for n in _BUFS}
        self.base_table = {n: (o, s) for n, o, s in tensor_table(cfg, 0)}
        self.lora_table = {n: (o, s) for n, o, s in tensor_table(cfg, 1)}
        self.n_lora = sum(int(np.prod(s)) for _, s in self.lora_table.values())
        self.stream = torch.cuda.current_stream(device)
        b = Qwen3Buffers(**{n: t.data_ptr() for n, t in self.bufs.items()})
        self._positions = self._plan = self._in_use = None
        self.h = ctypes.c_void_p()
        _check(lib().qwen3_init(ctypes.byref(cfg), ctypes.byref(b), ctypes.c_void_p(self.stream.cuda_stream),
                                ctypes.byref(self.h)))

    def close(self):
        if self.h:
            lib().qwen3_destroy(self.h)
            self.h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _view(self, buf, dtype, table, name):
        torch = self.torch
        off, shape = table[name]
        esz = 2 if dtype == torch.bfloat16 else 4
        n = int(np.prod(shape))
        return self.bufs[buf][off * esz:(off + n) * esz].view(dtype).view(*shape)

    def set_base(self, base: dict):
        """Copy the oracle's base parameters (rounded to bf16) to the device."""
        torch = self.torch
        p = pack_base(base)
        for name in self.base_table:
            v = self._view("base_bf16", torch.bfloat16, self.base_table, name)
            v.copy_(torch.from_numpy(np.ascontiguousarray(p[name], dtype=np.float32)).to(torch.bfloat16))

    def set_lora(self, lora: dict):
        """Copy the oracle's adapter parameters (fp32) and refresh their bf16 copy."""
        self.set_packed("lora_f32", lora)
        _check(lib().qwen3_sync_weights(self.h), self.h)

    def packed(self, which="lora_f32") -> dict:
        """Group tensors of an adapter-layout buffer (lora_f32, lora_grads,
        adam_m, adam_v: fp32; lora_bf16: bf16), copied to the host as fp32."""
        torch = self.torch
        torch.cuda.synchronize()
        dt = torch.bfloat16 if which == "lora_bf16" else torch.float32
        return {n: self._view(which, dt, self.lora_table, n).float().cpu().numpy() for n in self.lora_table}

    def adapters(self, which="lora_f32") -> dict:
        """Per-projection tensors of an adapter-layout buffer, oracle names."""
        return unpack_lora(self.packed(which), targets_of(self.cfg), self.cfg.lora_rank, out_widths(self.cfg))

    def flat(self, which="lora_grads"):
        """An fp32 adapter-layout buffer as one flat device tensor."""
        return self.bufs[which][:self.n_lora * 4].view(self.torch.float32)

    def set_packed(self, which: str, per_projection: dict):
        """Write per-projection fp32 tensors (oracle names) into an fp32
        adapter-layout buffer, padding zero."""
        torch = self.torch
        shapes = {n: s for n, (_, s) in self.lora_table.items()}
        for name, arr in pack_lora(per_projection, shapes, self.cfg.lora_rank).items():
            self._view(which, torch.float32, self.lora_table, name).copy_(torch.from_numpy(arr))


    def forward(self, ids, targets=None):
        torch = self.torch
        self._ids = ids.to(torch.int32).cuda().contiguous()
        self._tgt = None if targets is None else targets.to(torch.int32).cuda().contiguous()
        status = lib().qwen3_forward(self.h, ctypes.c_void_p(self._ids.data_ptr()),
                                     ctypes.c_void_p(self._tgt.data_ptr() if self._tgt is not None else 0))
        if status != GPT2_ERR_INVALID_ARG:
            # a backward takes its forward's positions and layout, whatever is set in between; those
            # of the forward before stay where this one is refused
            self._in_use = (self._positions, self._plan)
        _check(status, self.h)

    def backward(self):
        _check(lib().qwen3_backward(self.h), self.h)

    def adamw_step(self, step: int, norm_out=None):
        ptr = ctypes.c_void_p(norm_out.data_ptr() if norm_out is not None else 0)
        _check(lib().qwen3_adamw_step(self.h, step, ptr), self.h)

    def set_positions(self, positions=None, sections=(64,), interleaved=False):
        """Positions int32 [axes, B*T] of the tokens from the next forward on,
        with the pairs per axis (qwen3_set_positions); None: the default. What
        the current stream has enqueued is done before the model reads them."""
        if positions is not None:
            _device_rows(positions, "positions", self.torch.int32, self.bufs["workspace"],
                         (len(sections), self.cfg.B * self.cfg.T))
        sec = (ctypes.c_int32 * len(sections))(*map(i32, sections))
        _check(lib().qwen3_set_positions(self.h, _ptr(positions), len(sections), sec, int(bool(interleaved))), self.h)
        if positions is not None:
            # the model's stream reads them: after what the current one has to do with them, and before they are freed
            now = self.torch.cuda.current_stream(positions.device)
            if now != self.stream:
                self.stream.wait_stream(now)
            positions.record_stream(self.stream)
        self._positions = positions

    def set_layout(self, prefix_len=0, seq_lens=None):
        """The tokens as a prefix and sequences over it (qwen3_set_layout),
        from the next forward on; without seq_lens: B sequences of T tokens.
        Not in a capture, and a graph captured with a layout (or positions) is
        replayed only until others are set, when these are let go."""
        if seq_lens is None:
            _check(lib().qwen3_set_layout(self.h, 0, 0, None, None, 0), self.h)
            self._plan = None
            return
        lens, prefix_len = [i32(n) for n in seq_lens], i32(prefix_len)
        c_lens = (ctypes.c_int32 * len(lens))(*lens)
        n = ctypes.c_size_t()
        _check(lib().qwen3_layout_size(self.h, prefix_len, len(lens), c_lens, ctypes.byref(n)), self.h)
        plan = stream_buffer(n.value, self.bufs["workspace"].device, self.stream)
        _check(lib().qwen3_set_layout(self.h, prefix_len, len(lens), c_lens, plan.data_ptr(), n.value), self.h)
        self._plan = plan

    def muon_step(self, norm_out=None, momentum=0.95, nesterov=True, iterations=5, scale=0.2):
        """Clip and an orthogonalised update with momentum of every adapter
        matrix (qwen3_muon_step). Its workspace is allocated on the first call
        and kept."""
        if getattr(self, "muon_workspace", None) is None:
            n = ctypes.c_size_t()
            _check(lib().qwen3_muon_size(ctypes.byref(self.cfg), ctypes.byref(n)))
            self.muon_workspace = stream_buffer(n.value, self.bufs["workspace"].device, self.stream)
        how = muon_settings(momentum, nesterov, iterations, scale)
        _check(lib().qwen3_muon_step(self.h, ctypes.byref(how), self.muon_workspace.data_ptr(),
                                     self.muon_workspace.numel(),
                                     norm_out.data_ptr() if norm_out is not None else None), self.h)

    def loss(self, token_losses=None) -> float:
        v = ctypes.c_float()
        ptr = ctypes.c_void_p(token_losses.data_ptr() if token_losses is not None else 0)
        _check(lib().qwen3_loss(self.h, ctypes.byref(v), ptr), self.h)
        return v.value

    # ---- probes -------------------------------------------------------------
    def set_fusion(self, fusion: str, mode: int):
        """Select an alternative kernel arrangement (qwen3_set_fusion)."""
        _check(lib().qwen3_set_fusion(self.h, FUSION[fusion], int(mode)), self.h)

    def probe_enable(self, classes):
        mask = 0
        for c in classes:
            mask |= 1 << KCLASS[c]
        _check(lib().qwen3_probe_enable(self.h, mask), self.h)

    def probe_reset(self):
        _check(lib().qwen3_probe_reset(self.h), self.h)

    def probe_read(self, cls: str) -> dict:
        ms, fl, by = ctypes.c_double(), ctypes.c_double(), ctypes.c_double()
        n = ctypes.c_int64()
        _check(lib().qwen3_probe_read(self.h, KCLASS[cls], ctypes.byref(ms), ctypes.byref(n), ctypes.byref(fl),
                                      ctypes.byref(by)), self.h)
        return {"ms": ms.value, "launches": n.value, "flops": fl.value, "bytes": by.value}
