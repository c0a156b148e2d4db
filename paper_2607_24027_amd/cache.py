"""ctypes binding of the serving operators (C ABI in include/sol_cache.h).

Argument marshalling only, as in ``binding``: torch tensors supply device memory and the current stream, every step of
the computation runs in the library's HIP kernels.  A step of autoregressive generation for a ragged batch::

    new = cache.tables(lens, add, table, ring, state, rows)
    q, k = cache.qk_norm_rope(q, k, q_weight, k_weight, cos, sin, new.positions[None])
    cache.append(k[0], v, store, new.slots)
    out = cache.forward(q[0], store, table, new.lens, new.row_start, new.positions, max_rows=max_rows)

Tensors of tokens are heads first ([B, H, N, d], [H, T, d]) with any strides as long as the channels of a head are
contiguous: pass the projection's output through ``transpose`` and it is read where it is.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from . import binding as _b

PAGE = 64
HALVES, PAIRS = 0, 1

_P, _I, _F, _S = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
_L = ctypes.POINTER(ctypes.c_longlong)
# (restype, argtypes) for every symbol of include/sol_cache.h
SIGNATURES = {
    "sol_qk_norm_rope": (_I, [_P] * 4 + [_L] * 4 + [_P] * 5 + [_I] * 8 + [_F, _I, _I, _P]),
    "sol_cache_tables": (_I, [_P] * 10 + [_I] * 4 + [_P]),
    "sol_cache_append": (_I, [_P] * 2 + [_L] * 2 + [_P] * 2 + [_I] * 5 + [_P]),
    "sol_cache_read": (_I, [_P] * 4 + [_L] * 2 + [_I] * 5 + [_P]),
    "sol_cache_bytes": (_S, [_I] * 3),
    "sol_cache_workspace_bytes": (_S, [_I] * 7),
    "sol_cache_forward": (_I, [_P, _L, _P, _L] + [_P] * 5 + [_I] * 10 + [_P, _S, _P]),
}
_INVALID = ctypes.c_size_t(-1).value
_INT_MAX = 2 ** 31 - 1

_lib = None


def lib() -> ctypes.CDLL:
    """libsolattn.so with the signatures of this module (raises if it has not been built)."""
    global _lib
    if _lib is None:
        handle = _b.lib()
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _call(fn, device, *args):
    """One call of the library on the tensors' device and its current stream.  The library launches on the current device:
    another one is made current for the call."""
    if device.index is None or device.index == torch.cuda.current_device():
        rc = fn(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            rc = fn(*args, _stream(device))
    if rc != _b.SOL_OK:
        raise _b.SolAttnError(rc, _b.last_error())


_DTYPES = {torch.bfloat16: _b.SOL_BF16, torch.float32: _b.SOL_F32}
_F32_ONLY = (torch.float32,)


@functools.lru_cache(maxsize=4096)
def _stride_array(shape, stride):
    """Strides of all dimensions but the last, as a C array (of a dimension of one element: 0)."""
    s = [st if n > 1 else 0 for st, n in zip(stride[:-1], shape[:-1])]
    return (ctypes.c_longlong * len(s))(*s)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _strides(t):
    return None if t is None else _stride_array(t.shape, t.stride())


# The current stream's handle without a Stream object around it (0.2 instead of 4 us a call), where torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device) -> int:
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _check_heads(name, t, dim, ref=None, writable=False):
    # the common case first: these checks are a good part of what a short call costs
    if t.dim() == dim and t.stride(-1) == 1 and t.dtype in _DTYPES and not writable and \
            (ref is None or (t.dtype is ref.dtype and t.device == ref.device)):
        return
    if t.dim() != dim:
        raise ValueError(f"{name} must have {dim} dimensions (got {tuple(t.shape)})")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"the channels of {name} must be contiguous")
    _b._dtype_code(t)
    if ref is not None:
        if t.dtype != ref.dtype:
            raise ValueError(f"{name} must have dtype {ref.dtype} (got {t.dtype})")
        if t.device != ref.device:
            raise ValueError(f"{name} must be on {ref.device} (got {t.device})")
    if writable:
        rows = sorted((st, n) for st, n in zip(t.stride()[:-1], t.shape[:-1]) if n > 1)
        reach = t.shape[-1]
        for st, n in rows:
            if st < reach:
                raise ValueError(f"rows of {name} overlap")
            reach = st * (n - 1) + reach


def _check_floats(name, t, shape, dtypes, device):
    if t.dtype in dtypes and t.shape == shape and t.device == device and t.is_contiguous():
        return
    _b._check_buffer(name, t, shape, dtypes, device)


def _check_ints(name, t, shape, device):
    if t.dtype is torch.int32 and t.shape == shape and t.device == device and t.is_contiguous():
        return
    _b._check_buffer(name, t, shape, (torch.int32,), device)


def _overlap(a, b):
    """Whether two tensors share memory: False, or True where they may.  They do not if their outermost bytes lie apart, or if both
    repeat with one stride, as parts of each row of one buffer do, and lie apart inside of it."""
    if a.device != b.device or not a.numel() or not b.numel():
        return False
    dims = [[(st * t.element_size(), n) for st, n in zip(t.stride(), t.shape) if n > 1] for t in (a, b)]

    def reach(t, steps):
        return sum(st * (n - 1) for st, n in steps) + t.element_size()
    a0, b0 = a.data_ptr(), b.data_ptr()
    if a0 + reach(a, dims[0]) <= b0 or b0 + reach(b, dims[1]) <= a0:
        return False
    for period in {st for steps in dims for st, _ in steps if st}:
        ra, rb = (reach(t, [(st, n) for st, n in steps if st % period]) for t, steps in zip((a, b), dims))
        if (b0 - a0) % period >= ra and (a0 - b0) % period >= rb:
            return False
    return True


def _disjoint(name, t, **others):
    for other, o in others.items():
        if o is not None and t is not None and _overlap(t, o):
            raise ValueError(f"{name} must not overlap {other}")


def qk_norm_rope(q, k, q_weight=None, k_weight=None, cos=None, sin=None, positions=None, eps: float = 1e-6,
                 interleaved: bool = False, q_out=None, k_out=None):
    """RMS norm of each head of q [B,Hq,N,d] and k [B,Hk,N,d] (either may be None) and the rotation by position, in one pass.

    q_weight, k_weight: [d] (bf16 or f32, one dtype) or None for ones.  cos, sin: f32 [P, rot / 2] tables (None: no rotation)
    whose row is the token's position; positions: int32 [B, N], or None for 0 ... N - 1.  Tokens whose position is not a
    row of the tables are left out (their rows of given outputs stay as they were, those of new ones are undefined).
    interleaved: channels 2i and 2i + 1 are a pair, otherwise i and i + rot / 2.  q_out, k_out: any strides; new contiguous
    tensors by default, as forward() takes them.  Returns (q_out, k_out)."""
    ref = q if q is not None else k
    if ref is None:
        raise ValueError("one of q and k must be given")
    _check_heads("k" if q is None else "q", ref, 4)
    B, _, N, d = ref.shape
    if q is not None and k is not None:
        _check_heads("k", k, 4, q)
        if (k.shape[0], k.shape[2], k.shape[3]) != (B, N, d):
            raise ValueError(f"q and k must agree in B, N and d (got {tuple(q.shape)} and {tuple(k.shape)})")
    device = ref.device
    wdtype = None
    for name, x, w in (("q_weight", q, q_weight), ("k_weight", k, k_weight)):
        if w is not None:
            if x is None:
                raise ValueError(f"{name} needs {name[0]}")
            _check_floats(name, w, (d,), _DTYPES, device)
            if wdtype is not None and w.dtype != wdtype:
                raise ValueError("q_weight and k_weight must have one dtype")
            wdtype = w.dtype
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin must be given together")
    P = rot = 0
    if cos is not None:
        if cos.dim() != 2:
            raise ValueError("cos and sin must be [P, rot / 2]")
        P, rot = cos.shape[0], 2 * cos.shape[1]
        _check_floats("cos", cos, cos.shape, _F32_ONLY, device)
        _check_floats("sin", sin, cos.shape, _F32_ONLY, device)
    if positions is not None:
        _check_ints("positions", positions, (B, N), device)
    if q_out is not None or k_out is not None:
        for name, x, out in (("q_out", q, q_out), ("k_out", k, k_out)):
            if out is None:
                continue
            if x is None:
                raise ValueError(f"{name} needs {name[0]}")
            if out.shape != x.shape:
                raise ValueError(f"{name} must have shape {tuple(x.shape)} (got {tuple(out.shape)})")
            _check_heads(name, out, 4, x, writable=True)
            _disjoint(name, out, q=q, k=k, cos=cos, sin=sin, positions=positions, q_weight=q_weight, k_weight=k_weight)
        _disjoint("q_out", q_out, k_out=k_out)
    _b._require_gpu(ref)
    if P > _INT_MAX or rot > _INT_MAX:
        raise ValueError("cos and sin are too large")
    if q is not None and q_out is None:
        q_out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if k is not None and k_out is None:
        k_out = torch.empty_like(k, memory_format=torch.contiguous_format)
    if B == 0 or N == 0:
        return q_out, k_out
    _call(lib().sol_qk_norm_rope, device, _ptr(q), _ptr(k), _ptr(q_out), _ptr(k_out), _strides(q), _strides(k), _strides(q_out),
          _strides(k_out), _ptr(q_weight), _ptr(k_weight), _ptr(cos), _ptr(sin), _ptr(positions), B,
          0 if q is None else q.shape[1], 0 if k is None else k.shape[1], N, d, P, rot, PAIRS if interleaved else HALVES, eps,
          _DTYPES[ref.dtype], _b.SOL_F32 if wdtype is torch.float32 else _b.SOL_BF16)
    return q_out, k_out


class Step(NamedTuple):
    """What tables() gives: row_start [S + 1], slots and positions [rows], lens [S] and state [2] after the step."""
    row_start: "object"
    slots: "object"
    positions: "object"
    lens: "object"
    state: "object"


def tables(lens, add, table, ring, state, rows: int, out: Optional[Step] = None) -> Step:
    """Pages, slots and positions of one step: int32 lens [S] (tokens held), add [S] (tokens to add, or below 0 to take
    back), table [S, max_pages] and ring [P] (both updated), state [2] (place and number of the free pages in the ring);
    rows: the rows of slots and positions to fill, at least the sum of the positive adds.  The rules are in
    include/sol_cache.h.  out: tensors of an earlier step to write into (not lens and state themselves)."""
    if lens.dim() != 1 or table.dim() != 2 or ring.dim() != 1:
        raise ValueError("lens, table and ring must be [S], [S, max_pages] and [P]")
    S, MP = lens.shape[0], table.shape[1]
    device = lens.device
    _check_ints("lens", lens, (S,), device)
    _check_ints("add", add, (S,), device)
    _check_ints("table", table, (S, MP), device)
    _check_ints("ring", ring, ring.shape, device)
    _check_ints("state", state, (2,), device)
    if not 0 <= rows <= 1 << 30:
        raise ValueError(f"rows must be from 0 to 2^30 (got {rows})")
    if out is not None:
        shapes = {"row_start": (S + 1,), "slots": (rows,), "positions": (rows,), "lens": (S,), "state": (2,)}
        for name, shape in shapes.items():
            _check_ints(f"out.{name}", getattr(out, name), shape, lens.device)
        for name in shapes:
            _disjoint(f"out.{name}", getattr(out, name), lens=lens, add=add, table=table, ring=ring, state=state,
                      **{f"out.{o}": getattr(out, o) for o in shapes if o != name})
    _b._require_gpu(lens)
    if out is None:
        flat = torch.empty(S + 1 + 2 * rows + S + 2, dtype=torch.int32, device=device)
        out = Step(*torch.split_with_sizes(flat, (S + 1, rows, rows, S, 2)))
    _call(lib().sol_cache_tables, device, lens.data_ptr(), add.data_ptr(), table.data_ptr(), ring.data_ptr(), state.data_ptr(),
          out[3].data_ptr(), out[4].data_ptr(), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(), S, MP, ring.shape[0], rows)
    return out


def cache_bytes(pages: int, heads: int, d: int) -> int:
    """Bytes of a store of that many pages (of 64 tokens) and key/value heads."""
    n = int(lib().sol_cache_bytes(pages, heads, d))
    if n == _INVALID:
        raise ValueError(f"no store of {pages} pages, {heads} heads of {d} channels")
    return n


def empty(pages: int, heads: int, d: int, device):
    """A store [pages, heads, 68 d] of bytes for append(); its contents are undefined."""
    cache_bytes(pages, heads, d)
    return torch.empty((pages, heads, 68 * d), dtype=torch.uint8, device=device)


def _check_store(store):
    """(pages, heads, d) of a store."""
    shape = store.shape
    if len(shape) != 3 or shape[2] not in (68 * 64, 68 * 128):
        raise ValueError(f"store must be [pages, heads, 68 d] bytes with d = 64 or 128 (got {tuple(shape)})")
    if store.dtype is not torch.uint8 or not store.is_contiguous():
        _b._check_buffer("store", store, shape, (torch.uint8,), store.device)
    return shape[0], shape[1], shape[2] // 68


def append(k, v, store, slots):
    """Writes k, v [heads, T, d] into the slots (int32 [T], slot = 64 page + token; others are left out) of the store."""
    P, H, d = _check_store(store)
    _check_heads("k", k, 3)
    _check_heads("v", v, 3, k)
    if tuple(k.shape) != tuple(v.shape):
        raise ValueError(f"k and v must have one shape (got {tuple(k.shape)} and {tuple(v.shape)})")
    if (k.shape[0], k.shape[2]) != (H, d):
        raise ValueError(f"k and v must have {H} heads of {d} channels as the store has (got {tuple(k.shape)})")
    device = k.device
    if store.device != device:
        raise ValueError(f"store must be on {device} (got {store.device})")
    T = k.shape[1]
    _check_ints("slots", slots, (T,), device)
    _b._require_gpu(k)
    if T == 0:
        return
    _call(lib().sol_cache_append, device, k.data_ptr(), v.data_ptr(), _strides(k), _strides(v), store.data_ptr(), slots.data_ptr(),
          T, H, d, P, _DTYPES[k.dtype])


def read(store, slots, dtype=None, k_out=None, v_out=None):
    """(k, v) [heads, T, d] of the slots (int32 [T]), as the values that their codes stand for; zeros for slots outside the
    store.  dtype: bf16 (default) or f32.  With k_out or v_out given, only what is given is read."""
    P, H, d = _check_store(store)
    if slots.dim() != 1:
        raise ValueError("slots must be [T]")
    T = slots.shape[0]
    _check_ints("slots", slots, (T,), store.device)
    given = () if k_out is None and v_out is None else [t for t in (k_out, v_out) if t is not None]
    if given:
        if dtype is not None and dtype != given[0].dtype:
            raise ValueError(f"dtype is {dtype}, that of the outputs {given[0].dtype}")
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            if t is None:
                continue
            _check_heads(name, t, 3, given[0], writable=True)
            if tuple(t.shape) != (H, T, d):
                raise ValueError(f"{name} must have shape {(H, T, d)} (got {tuple(t.shape)})")
            if t.device != store.device:
                raise ValueError(f"{name} must be on {store.device} (got {t.device})")
            _disjoint(name, t, store=store, slots=slots)
        _disjoint("k_out", k_out, v_out=v_out)
    dt = given[0].dtype if given else torch.bfloat16 if dtype is None else dtype
    if dt not in _DTYPES:
        raise TypeError(f"unsupported dtype {dt}")
    _b._require_gpu(store)
    device = store.device
    if not given:
        k_out = torch.empty((H, T, d), dtype=dt, device=device)
        v_out = torch.empty((H, T, d), dtype=dt, device=device)
    if T == 0:
        return k_out, v_out
    _call(lib().sol_cache_read, device, store.data_ptr(), slots.data_ptr(), _ptr(k_out), _ptr(v_out), _strides(k_out),
          _strides(v_out), T, H, d, P, _DTYPES[dt])
    return k_out, v_out


def workspace_bytes(S: int, T: int, max_rows: int, Hq: int, Hk: int, d: int, max_pages: int) -> int:
    """Scratch bytes of forward() for S requests with T rows in all, max_rows of one at most."""
    n = int(lib().sol_cache_workspace_bytes(S, T, max_rows, Hq, Hk, d, max_pages))
    if n == _INVALID:
        raise ValueError(_b.last_error())
    return n


def forward(q, store, table, lens, row_start, positions, causal_granule: int = 1, max_rows: Optional[int] = None, out=None,
            workspace=None):
    """Attention of the rows q [Hq, T, d] of S requests over their tokens in the store.

    table [S, max_pages], lens [S] (with the new tokens), row_start [S + 1], positions [T]: int32, as tables() gives them.
    causal_granule: 1 is token-causal, the tokens of a frame frame-causal, the longest length or more no mask.  max_rows:
    rows of the request that has most, or a bound of them.  The call is planned for it: by default it is T, and a batch of single tokens
    then starts work for requests of many rows too and takes a larger workspace (48 requests of 32 heads, 200 to 32,000
    tokens: 75 us and 26 MB with it, 84 us and 69 MB without; 1,000 tokens each in a table of 512 pages: 18 and 24 us).  out: like q, any strides; by default with q's order of
    dimensions in memory, rows outside the requests undefined.  workspace: 1-D uint8 tensor of workspace_bytes(...)
    bytes, by default a new one of torch's allocator (inside a graph capture: of the graph's own pool).  Returns out."""
    P, Hk, d = _check_store(store)
    _check_heads("q", q, 3)
    Hq, T = q.shape[0], q.shape[1]
    if q.shape[2] != d:
        raise ValueError(f"q must have {d} channels as the store has (got {q.shape[2]})")
    device = q.device
    if store.device != device:
        raise ValueError(f"store must be on {device} (got {store.device})")
    if lens.dim() != 1 or table.dim() != 2:
        raise ValueError("lens and table must be [S] and [S, max_pages]")
    S, MP = lens.shape[0], table.shape[1]
    _check_ints("lens", lens, (S,), device)
    _check_ints("table", table, (S, MP), device)
    _check_ints("row_start", row_start, (S + 1,), device)
    _check_ints("positions", positions, (T,), device)
    if out is not None:
        if tuple(out.shape) != tuple(q.shape):
            raise ValueError(f"out must have shape {tuple(q.shape)} (got {tuple(out.shape)})")
        _check_heads("out", out, 3, q, writable=True)
        _disjoint("out", out, q=q, store=store, table=table, lens=lens, row_start=row_start, positions=positions,
                  workspace=workspace)
    if workspace is not None:
        if workspace.dim() != 1:
            raise ValueError("workspace must be a 1-D uint8 tensor")
        _b._check_buffer("workspace", workspace, workspace.shape, (torch.uint8,), q.device)
        _disjoint("workspace", workspace, q=q, store=store, table=table, lens=lens, row_start=row_start, positions=positions)
    _b._require_gpu(q)
    rows = T if max_rows is None else min(int(max_rows), T)
    granule = min(int(causal_granule), _INT_MAX)   # longer than any sequence
    call = lib()
    if workspace is None and T > 0:
        need = call.sol_cache_workspace_bytes(S, T, rows, Hq, Hk, d, MP)
        if need and need != _INVALID:   # invalid arguments are the call's to report
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
    given = out is not None or not _dense(q.shape, q.stride())   # whether out's strides may be others than q's
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=device) if given else torch.empty_like(q)
    if T == 0:
        return out
    strides = _strides(q)
    _call(call.sol_cache_forward, device, q.data_ptr(), strides, out.data_ptr(), _strides(out) if given else strides,
          store.data_ptr(), table.data_ptr(), lens.data_ptr(), row_start.data_ptr(), positions.data_ptr(), S, T, rows, Hq, Hk, d, P,
          MP, granule, _DTYPES[q.dtype], None if workspace is None else workspace.data_ptr(),
          0 if workspace is None else workspace.numel())
    return out


@functools.lru_cache(maxsize=4096)
def _dense(shape, stride):
    """Whether a tensor of that shape and strides fills its memory without holes or overlaps."""
    reach = 1
    for st, n in sorted((st, n) for st, n in zip(stride, shape) if n > 1):
        if st != reach:
            return False
        reach *= n
    return True
