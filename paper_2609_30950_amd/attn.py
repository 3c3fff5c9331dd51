"""Python binding of the attention layers' entry points (argument marshalling
only; see include/kda.h for layouts and contracts).

Tensors are torch tensors on the current HIP device; calls are enqueued on
torch's current stream.  Row-strided inputs (slices of a fused projection)
are taken as they are; everything else is contiguous.
"""
import ctypes
from dataclasses import dataclass, fields
from math import sqrt
from typing import Optional

import torch

from ._lib import KdaError, kda_attn_config, kda_latent_config, kda_pages, load
from .api import _check

_TYPES = {"bf16": (0, torch.bfloat16), "f16": (1, torch.float16)}
_E4M3 = (2, torch.float8_e4m3fn)
_I32 = torch.int32


def _int32(**numbers):
    """ctypes would cut a wider number to its low 32 bits."""
    for name, x in numbers.items():
        if not -2**31 <= x < 2**31:
            raise KdaError(f"{name}: {x} does not fit 32 bits")


class _Value:
    """Copies and pickles are made from the fields alone (the C structure and
    its reference are formed anew)."""

    def __reduce__(self):
        return type(self), tuple(getattr(self, f.name) for f in fields(self))


@dataclass(frozen=True)
class Pages(_Value):
    """Requests and the page pool they share."""
    B: int
    page: int
    n_pages: int
    max_pages: int

    def __post_init__(self):
        _int32(B=self.B, page=self.page, n_pages=self.n_pages, max_pages=self.max_pages)
        object.__setattr__(self, "_c", kda_pages(self.B, self.page, self.n_pages, self.max_pages))
        object.__setattr__(self, "_ref", ctypes.byref(self._c))


def _element(cfg):
    if cfg.dtype not in _TYPES:
        raise KdaError(f"dtype: expected one of {sorted(_TYPES)}, got {cfg.dtype!r}")
    return _TYPES[cfg.dtype]


@dataclass(frozen=True)
class AttnConfig(_Value):
    """Grouped-query attention; cache "same" (as dtype) or "e4m3"."""
    pages: Pages
    H_q: int
    H_kv: int
    d: int
    dtype: str = "bf16"
    cache: str = "same"
    scale: Optional[float] = None   # None: 1 / sqrt(d)

    def __post_init__(self):
        code, t = _element(self)
        if self.cache not in ("same", "e4m3"):
            raise KdaError(f"cache: expected 'same' or 'e4m3', got {self.cache!r}")
        held = _E4M3 if self.cache == "e4m3" else (code, t)
        _int32(H_q=self.H_q, H_kv=self.H_kv, d=self.d)
        if self.d < 1:
            raise KdaError("invalid config")
        scale = 1.0 / sqrt(self.d) if self.scale is None else float(self.scale)
        for name, value in (("_c", kda_attn_config(self.pages._c, self.H_q, self.H_kv, self.d, code,
                                                   held[0], scale)), ("_t", t), ("_held", held[1])):
            object.__setattr__(self, name, value)
        object.__setattr__(self, "_ref", ctypes.byref(self._c))

        p = self.pages
        for name, value in (("key_shape", (p.n_pages, self.H_kv, p.page, self.d)),
                            ("value_shape", (p.n_pages, self.H_kv, p.page // 8, self.d, 8)),
                            ("_table", (p.B, p.max_pages)), ("_out", (p.B, self.H_q, self.d)),
                            ("_need", int(load().kda_attn_workspace_bytes(self._ref)))):
            object.__setattr__(self, name, value)


@dataclass(frozen=True)
class LatentConfig(_Value):
    """Latent attention: H heads over cached rows [c (d_c), r (d_r)]."""
    pages: Pages
    H: int
    d_n: int
    d_r: int
    d_c: int
    d_v: int
    dtype: str = "bf16"
    scale: Optional[float] = None   # None: 1 / sqrt(d_n + d_r)

    def __post_init__(self):
        code, t = _element(self)
        _int32(H=self.H, d_n=self.d_n, d_r=self.d_r, d_c=self.d_c, d_v=self.d_v)
        if self.d_n < 1 or self.d_r < 1:
            raise KdaError("invalid config")
        scale = 1.0 / sqrt(self.d_n + self.d_r) if self.scale is None else float(self.scale)
        for name, value in (("_c", kda_latent_config(self.pages._c, self.H, self.d_n, self.d_r, self.d_c, self.d_v,
                                                     code, scale)), ("_t", t)):
            object.__setattr__(self, name, value)
        object.__setattr__(self, "_ref", ctypes.byref(self._c))

        p = self.pages
        for name, value in (("cache_shape", (p.n_pages, p.page, self.d_c + self.d_r)),
                            ("_table", (p.B, p.max_pages)), ("_uk", (self.H, self.d_n, self.d_c)),
                            ("_uv", (self.H, self.d_v, self.d_c)),
                            ("_need", int(load().kda_latent_workspace_bytes(self._ref)))):
            object.__setattr__(self, name, value)


# The checks below take one comparison chain per tensor where all is well and
# say what is wrong only afterwards: a decode step makes ten of them.

def _refuse(t, dtype, shape, dev, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise KdaError(f"{name}: expected a device tensor")
    if t.dtype != dtype:
        raise KdaError(f"{name}: expected {dtype}, got {t.dtype}")
    if t.get_device() != dev:
        raise KdaError(f"{name}: on {t.device}, but the current device is {dev}")
    if t.shape != shape:
        raise KdaError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    raise KdaError(f"{name}: expected contiguous {'rows' if name in _ROWS else 'memory'}, got strides {t.stride()}")


_ROWS = ("q", "k", "v", "c", "r", "q_n", "q_r")


def _dense(t, dtype, shape, dev, name):
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        return t.data_ptr()
    _refuse(t, dtype, shape, dev, name)


def _dense_or_none(t, dtype, shape, dev, name):
    return None if t is None else _dense(t, dtype, shape, dev, name)


def _rows(t, dtype, shape, dev, name):
    """Pointer and row stride of rows that are each contiguous."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev:
        n, width = shape[0], 1
        for x in shape[1:]:
            width *= x
        if t.is_contiguous():
            return t.data_ptr(), width
        want, good = 1, True
        for x, s in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
            good = good and (x == 1 or s == want)
            want *= x
        if good:
            return t.data_ptr(), t.stride(0) if n > 1 else width
    _refuse(t, dtype, shape, dev, name)


def _heads(t, dtype, shape, dev, name):
    """Pointer, row stride and head stride of [rows, heads, d], d contiguous."""
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev:
        n, H, d = shape
        row, head, one = t.stride()
        if one == 1:
            head = head if H > 1 else d
            return t.data_ptr(), row if n > 1 else (H - 1) * head + d, head
    _refuse(t, dtype, shape, dev, name)


def _count(t, dim=None):
    """Elements, or the size of a dimension; 0 for what the checks refuse."""
    if not isinstance(t, torch.Tensor):
        return 0
    return t.numel() if dim is None else t.shape[dim] if t.dim() > dim else 0


def _scratch(ws, need, dev, name="ws"):
    if need == 0:
        raise KdaError("invalid config")
    if not isinstance(ws, torch.Tensor) or ws.dtype is not torch.uint8 or ws.get_device() != dev:
        _refuse(ws, torch.uint8, (need,), dev, name)
    if ws.numel() < need or not ws.is_contiguous():
        raise KdaError(f"{name}: expected at least {need} contiguous bytes, got {ws.numel()}")
    return ws.data_ptr()


# torch's current stream as a handle, without the Stream object around it
# (0.1 against 1.1 us of a call's eight)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _here():
    """The current device and torch's current stream on it."""
    try:
        dev = torch.cuda.current_device()
        return dev, _raw_stream(dev)
    except (RuntimeError, AssertionError) as e:
        raise KdaError(f"no HIP device to hold a device tensor: {e}") from e


def _new_workspace(need, device):
    if need == 0:
        raise KdaError("invalid config")
    return torch.empty(need, dtype=torch.uint8, device=device)


def kda_pages_plan(pages, lens, new_tokens, n_free, free_pages, tables, lens_out, n_free_out, cu, slots, ok):
    dev, stream = _here()
    B = pages.B
    per = (B,)
    n = _count(slots)
    if n >= 2**31:
        _int32(slots=n)
    _check(load().kda_pages_plan(
        pages._ref, n, _dense(lens, _I32, per, dev, "lens"), _dense(new_tokens, _I32, per, dev, "new_tokens"),
        _dense(n_free, _I32, (1,), dev, "n_free"), _dense(free_pages, _I32, (pages.n_pages,), dev, "free_pages"),
        _dense(tables, _I32, (B, pages.max_pages), dev, "tables"), _dense(lens_out, _I32, per, dev, "lens_out"),
        _dense(n_free_out, _I32, (1,), dev, "n_free_out"), _dense(cu, _I32, (B + 1,), dev, "cu"),
        _dense(slots, _I32, (n,), dev, "slots"), _dense(ok, _I32, per, dev, "ok"), stream))


def new_attn_caches(cfg, device="cuda"):
    """Zero-filled (keys, values) of the pool."""
    raw = torch.uint8 if cfg.cache == "e4m3" else torch.int16
    return tuple(torch.zeros(s, dtype=raw, device=device).view(cfg._held)
                 for s in (cfg.key_shape, cfg.value_shape))


def new_attn_workspace(cfg, device="cuda"):
    return _new_workspace(cfg._need, device)


def _only_e4m3(cfg, k_scale, v_scale):
    if cfg.cache != "e4m3" and (k_scale is not None or v_scale is not None):
        raise KdaError("k_scale, v_scale: only with an e4m3 cache")


def _scales(cfg, k_scale, v_scale, dev):
    return (_dense_or_none(k_scale, torch.float32, (cfg.H_kv,), dev, "k_scale"),
            _dense_or_none(v_scale, torch.float32, (cfg.H_kv,), dev, "v_scale"))


def kda_attn_append(cfg, k, v, slots, k_cache, v_cache, k_scale=None, v_scale=None):
    """Rows k, v [n, H_kv, d] (row-strided) into the pages of slots [n]."""
    _only_e4m3(cfg, k_scale, v_scale)
    dev, stream = _here()
    n = _count(slots)
    shape = (n, cfg.H_kv, cfg.d)
    ks, vs = _scales(cfg, k_scale, v_scale, dev)
    _check(load().kda_attn_append(
        cfg._ref, n, *_rows(k, cfg._t, shape, dev, "k"), *_rows(v, cfg._t, shape, dev, "v"),
        _dense(slots, _I32, (n,), dev, "slots"), ks, vs, _dense(k_cache, cfg._held, cfg.key_shape, dev, "k_cache"),
        _dense(v_cache, cfg._held, cfg.value_shape, dev, "v_cache"), stream))


def kda_attn_step(cfg, q, k_cache, v_cache, tables, lens, o, ws, lse=None, k_scale=None, v_scale=None):
    """q [B, H_q, d] (row-strided) over the first lens [B] tokens of each
    request; o [B, H_q, d], lse [B, H_q] float32 or None."""
    _only_e4m3(cfg, k_scale, v_scale)
    dev, stream = _here()
    t, out = cfg._t, cfg._out
    ks, vs = _scales(cfg, k_scale, v_scale, dev)
    _check(load().kda_attn_step(
        cfg._ref, *_rows(q, t, out, dev, "q"), _dense(k_cache, cfg._held, cfg.key_shape, dev, "k_cache"),
        _dense(v_cache, cfg._held, cfg.value_shape, dev, "v_cache"), _dense(tables, _I32, cfg._table, dev, "tables"),
        _dense(lens, _I32, out[:1], dev, "lens"), ks, vs, _dense(o, t, out, dev, "o"),
        _dense_or_none(lse, torch.float32, out[:2], dev, "lse"), _scratch(ws, cfg._need, dev), stream))


def new_latent_cache(cfg, device="cuda"):
    """Zero-filled latent rows of the pool."""
    return torch.zeros(cfg.cache_shape, dtype=cfg._t, device=device)


def new_latent_workspace(cfg, device="cuda"):
    return _new_workspace(cfg._need, device)


def _prefill_bytes(cfg, max_kv):
    _int32(max_kv=max_kv)
    return int(load().kda_latent_prefill_workspace_bytes(cfg._ref, max_kv))


def new_latent_prefill_workspace(cfg, max_kv, device="cuda"):
    return _new_workspace(_prefill_bytes(cfg, max_kv), device)


def kda_latent_append(cfg, c, r, slots, cache):
    """Rows c [n, d_c] and r [n, d_r] (row-strided) into the pages of slots [n]."""
    dev, stream = _here()
    n = _count(slots)
    _check(load().kda_latent_append(
        cfg._ref, n, *_rows(c, cfg._t, (n, cfg.d_c), dev, "c"), *_rows(r, cfg._t, (n, cfg.d_r), dev, "r"),
        _dense(slots, _I32, (n,), dev, "slots"), _dense(cache, cfg._t, cfg.cache_shape, dev, "cache"), stream))


def kda_latent_step(cfg, q_n, q_r, w_uk, w_uv, cache, tables, lens, o, ws):
    """q_n [B, H, d_n], q_r [B, H, d_r] (row- and head-strided) over the first
    lens [B] tokens of each request; o [B, H, d_v]."""
    dev, stream = _here()
    t, B, H = cfg._t, cfg.pages.B, cfg.H
    _check(load().kda_latent_step(
        cfg._ref, *_heads(q_n, t, (B, H, cfg.d_n), dev, "q_n"), *_heads(q_r, t, (B, H, cfg.d_r), dev, "q_r"),
        _dense(w_uk, t, cfg._uk, dev, "w_uk"), _dense(w_uv, t, cfg._uv, dev, "w_uv"),
        _dense(cache, t, cfg.cache_shape, dev, "cache"), _dense(tables, _I32, cfg._table, dev, "tables"),
        _dense(lens, _I32, (B,), dev, "lens"), _dense(o, t, (B, H, cfg.d_v), dev, "o"),
        _scratch(ws, cfg._need, dev), stream))


def kda_latent_prefill(cfg, max_kv, q_n, q_r, cu, w_uk, w_uv, cache, tables, lens, o, ws):
    """Packed prompt rows q_n [n, H, d_n], q_r [n, H, d_r] (row- and
    head-strided), request b's in cu[b] .. cu[b + 1] - 1; o [n, H, d_v]."""
    dev, stream = _here()
    t, B, H, n = cfg._t, cfg.pages.B, cfg.H, _count(q_n, 0)
    need = _prefill_bytes(cfg, max_kv)
    _check(load().kda_latent_prefill(
        cfg._ref, n, max_kv, *_heads(q_n, t, (n, H, cfg.d_n), dev, "q_n"),
        *_heads(q_r, t, (n, H, cfg.d_r), dev, "q_r"), _dense(cu, _I32, (B + 1,), dev, "cu"),
        _dense(w_uk, t, cfg._uk, dev, "w_uk"), _dense(w_uv, t, cfg._uv, dev, "w_uv"),
        _dense(cache, t, cfg.cache_shape, dev, "cache"), _dense(tables, _I32, cfg._table, dev, "tables"),
        _dense(lens, _I32, (B,), dev, "lens"), _dense(o, t, (n, H, cfg.d_v), dev, "o"),
        _scratch(ws, need, dev), stream))
