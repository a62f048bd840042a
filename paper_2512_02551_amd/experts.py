"""Binding of the expert-layer operators of include/hgemm.h: products of 8-bit floats with block scales (plain and by groups of rows),
quantising, routing and combining.  Argument marshalling only.

The ``*Plan`` classes take raw device pointers and a stream, as :class:`~paper_2512_02551_amd.Plan` does; the lower-case functions take
torch tensors on the current device, allocate the results and run on torch's current stream.  A function makes its plan in the call: route, route_backward and a
scaled_product whose K is split own a workspace and wait for their result before they give it back, so these are not for the capture of a graph; plans are.
"""
from __future__ import annotations

import ctypes
from typing import Optional

SCALE_BLOCK = 128                                    # HGEMM_SCALE_BLOCK
_BYTE = {"e4m3": 0, "e5m2": 1}
_TYPE = {"f16": 0, "bf16": 1, "f32": 2}
_SCALE = {"f32": 0, "e8m0": 1}
_GROUP = {"none": 0, "rows": 1, "depth": 2}

_i32, _i64, _vp, _ci = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_int


class _Scaled(ctypes.Structure):
    _fields_ = [("a", _ci), ("c", _ci), ("scale", _ci), ("b_block_rows", _i32), ("group", _ci), ("groups", _i32), ("a_rows", _i64),
                ("lda", _i64), ("ldb", _i64), ("ldc", _i64), ("ld_scale_a", _i64), ("ld_scale_b", _i64)]


class _Quantise(ctypes.Structure):
    _fields_ = [("x", _ci), ("q", _ci), ("scale", _ci), ("block_rows", _i32), ("M", _i64), ("K", _i64), ("x_rows", _i64),
                ("ldx", _i64), ("ldq", _i64), ("lds", _i64), ("ldqt", _i64), ("ldst", _i64)]


class _Route(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("experts", _i32), ("k", _i32), ("logits", _ci), ("ld", _i64), ("sigmoid", _i32), ("groups", _i32), ("keep", _i32), ("top2", _i32),
                ("renormalise", _i32), ("factor", ctypes.c_float), ("align", _i32)]


class _Combine(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("N", _i64), ("y_rows", _i64), ("k", _i32), ("y", _ci), ("out", _ci), ("ldy", _i64), ("ldo", _i64)]


def declare(lib) -> None:
    """Argument types of the entry points (called once, by binding.load)."""
    def of(name, *args, result=_ci):
        f = getattr(lib, name)
        f.restype, f.argtypes = result, list(args)

    p = ctypes.POINTER
    of("hgemm_scaled_plan", p(_vp), _i64, _i64, _i64, p(_Scaled))
    of("hgemm_scaled_plan_override", p(_vp), _i64, _i64, _i64, p(_Scaled), ctypes.c_char_p)
    of("hgemm_scaled_run", *[_vp] * 9)
    of("hgemm_scaled_destroy", _vp)
    of("hgemm_scaled_workspace_bytes", _vp, result=ctypes.c_size_t)
    of("hgemm_scaled_describe", _vp, ctypes.c_char_p, ctypes.c_size_t)
    of("hgemm_quantise", p(_Quantise), *[_vp] * 7)
    of("hgemm_route_plan", p(_vp), p(_Route))
    of("hgemm_route_run", *[_vp] * 9)
    of("hgemm_route_backward", *[_vp] * 6)
    of("hgemm_route_destroy", _vp)
    of("hgemm_route_capacity", p(_Route), result=_i64)
    of("hgemm_combine", p(_Combine), *[_vp] * 5)
    of("hgemm_combine_backward", p(_Combine), *[_vp] * 8)


def _lib():
    from . import binding
    return binding.load()


def _check(status: int, what: str) -> None:
    if status != 0:
        from .binding import HgemmError
        raise HgemmError(status, what)


def _kind(table: dict, value: str, what: str) -> int:
    if value not in table:
        raise ValueError(f"{what}: {value!r} is none of {', '.join(table)}")
    return table[value]


class _Handle:
    """Owns one plan of the library."""

    _destroy = ""

    def __init__(self):
        self._h = _vp()

    def destroy(self) -> None:
        if self._h:
            getattr(_lib(), self._destroy)(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()


class ScaledPlan(_Handle):
    """C = A B^T over 8-bit floats with a scale for each block of 128 (hgemm_scaled_plan).

    a: "e4m3" or "e5m2"; c: "f16", "bf16" or "f32"; scale: "f32" or "e8m0"; b_rows: rows of B that share a scale, 128 or 1.
    groups, along: experts, as blocks of rows ("rows") or ranges of K ("depth"); a_rows: rows of an A that an index gathers from.
    spec: the kernel, as describe() names it, instead of the library's choice.
    """

    _destroy = "hgemm_scaled_destroy"

    def __init__(self, M: int, N: int, K: int, a: str = "e4m3", c: str = "f16", scale: str = "f32", b_rows: int = 128, groups: int = 0, along: str = "rows", a_rows: int = 0,
                 lda: int = 0, ldb: int = 0, ldc: int = 0, ld_scale_a: int = 0, ld_scale_b: int = 0, spec: Optional[str] = None):
        super().__init__()
        d = _Scaled(_kind(_BYTE, a, "a"), _kind(_TYPE, c, "c"), _kind(_SCALE, scale, "scale"), b_rows, _kind(_GROUP, along if groups else "none", "along"), groups, a_rows,
                    lda, ldb, ldc, ld_scale_a, ld_scale_b)
        lib = _lib()
        if spec is None:
            _check(lib.hgemm_scaled_plan(ctypes.byref(self._h), M, N, K, ctypes.byref(d)), "hgemm_scaled_plan")
        else:
            _check(lib.hgemm_scaled_plan_override(ctypes.byref(self._h), M, N, K, ctypes.byref(d), spec.encode()), f"hgemm_scaled_plan_override({spec!r})")
        self._run = lib.hgemm_scaled_run

    def run(self, a: int, scale_a: int, b: int, scale_b: int, c: int, stream: int = 0, offsets: int = 0, index: int = 0) -> None:
        status = self._run(self._h, a, scale_a, b, scale_b, c, offsets, index, stream)
        if status:
            _check(status, "hgemm_scaled_run")

    def workspace_bytes(self) -> int:
        return int(_lib().hgemm_scaled_workspace_bytes(self._h))

    def describe(self) -> str:
        buf = ctypes.create_string_buffer(256)
        _check(_lib().hgemm_scaled_describe(self._h, buf, len(buf)), "hgemm_scaled_describe")
        return buf.value.decode()


class QuantisePlan:
    """What hgemm_quantise needs besides pointers.  x: type of the matrix; q: "e4m3" or "e5m2"; scale: "f32" or "e8m0"; block_rows: 1 or 128;
    x_rows: rows of an X that an index gathers from."""

    def __init__(self, M: int, K: int, x: str = "f16", q: str = "e4m3", scale: str = "f32", block_rows: int = 1, x_rows: int = 0,
                 ldx: int = 0, ldq: int = 0, lds: int = 0, ldqt: int = 0, ldst: int = 0):
        self._d = _Quantise(_kind(_TYPE, x, "x"), _kind(_BYTE, q, "q"), _kind(_SCALE, scale, "scale"), block_rows, M, K, x_rows, ldx, ldq, lds, ldqt, ldst)
        self._ref, self._run = ctypes.byref(self._d), _lib().hgemm_quantise

    def run(self, x: int, q: int, s: int, qt: int = 0, st: int = 0, stream: int = 0, index: int = 0) -> None:
        status = self._run(self._ref, x, index, q, s, qt, st, stream)
        if status:
            _check(status, "hgemm_quantise")


class RoutePlan(_Handle):
    """The choice of k experts per token and the order of the rows (hgemm_route_plan).  score: "softmax" or "sigmoid"."""

    _destroy = "hgemm_route_destroy"

    def __init__(self, tokens: int, experts: int, k: int, logits: str = "f16", score: str = "softmax", groups: int = 1, keep: int = 1, top2: bool = False,
                 renormalise: bool = True, factor: float = 1.0, align: int = 1, ld: int = 0):
        super().__init__()
        d = _Route(tokens, experts, k, _kind(_TYPE, logits, "logits"), ld, _kind({"softmax": 0, "sigmoid": 1}, score, "score"), groups, keep, int(top2), int(renormalise), factor, align)
        lib = _lib()
        _check(lib.hgemm_route_plan(ctypes.byref(self._h), ctypes.byref(d)), "hgemm_route_plan")
        self.capacity = int(lib.hgemm_route_capacity(ctypes.byref(d)))
        self._run, self._backward = lib.hgemm_route_run, lib.hgemm_route_backward

    def run(self, logits: int, bias: int, weights: int, experts: int, offsets: int = 0, rows: int = 0, tokens_of: int = 0, stream: int = 0) -> None:
        status = self._run(self._h, logits, bias, weights, experts, offsets, rows, tokens_of, stream)
        if status:
            _check(status, "hgemm_route_run")

    def backward(self, logits: int, experts: int, dweights: int, dlogits: int, stream: int = 0) -> None:
        status = self._backward(self._h, logits, experts, dweights, dlogits, stream)
        if status:
            _check(status, "hgemm_route_backward")


class CombinePlan:
    """What hgemm_combine and hgemm_combine_backward need besides pointers."""

    def __init__(self, tokens: int, k: int, N: int, y_rows: int, y: str = "f16", out: str = "f16", ldy: int = 0, ldo: int = 0):
        self._d = _Combine(tokens, N, y_rows, k, _kind(_TYPE, y, "y"), _kind(_TYPE, out, "out"), ldy, ldo)
        lib = _lib()
        self._ref, self._run, self._backward = ctypes.byref(self._d), lib.hgemm_combine, lib.hgemm_combine_backward

    def run(self, rows: int, weights: int, y: int, out: int, stream: int = 0) -> None:
        status = self._run(self._ref, rows, weights, y, out, stream)
        if status:
            _check(status, "hgemm_combine")

    def backward(self, rows: int, tokens_of: int, weights: int, y: int, dout: int, dy: int, dweights: int, stream: int = 0) -> None:
        status = self._backward(self._ref, rows, tokens_of, weights, y, dout, dy, dweights, stream)
        if status:
            _check(status, "hgemm_combine_backward")


# ---- torch tensors -----------------------------------------------------------------------------------------------------------------

def _type_name(t) -> str:
    import torch

    names = {torch.float16: "f16", torch.bfloat16: "bf16", torch.float32: "f32", torch.float8_e4m3fn: "e4m3", torch.float8_e5m2: "e5m2", torch.uint8: "e8m0",
             torch.float8_e8m0fnu: "e8m0"}
    if t.dtype not in names:
        raise TypeError(f"no operator takes {t.dtype}")
    return names[t.dtype]


def _torch_type(name: str):
    import torch

    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "e8m0": torch.uint8}[name]


def _on_device(t, what: str) -> None:
    """The kernels go to the current device's stream: its memory is what they reach."""
    import torch

    if not t.is_cuda:
        raise TypeError(f"{what}: a CUDA tensor is needed")
    if t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{what}: on cuda:{t.get_device()}, and the current device is cuda:{torch.cuda.current_device()}")


def _rows(t, what: str, dims: int = 2):
    """(tensor, leading dimension) of a CUDA tensor whose rows are contiguous.  Rows that share memory -- one repeated by expand(), say -- have no leading
    dimension: they are copied apart.  The caller holds the tensor until its kernel is enqueued."""
    _on_device(t, what)
    if t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what}: {dims} dimensions with contiguous rows are needed")
    if t.shape[-2] > 1 and t.stride(-2) < t.shape[-1]:
        t = t.contiguous()
    if not t.shape[-1]:
        return t, 0                                       # no columns: packed, whatever its strides
    ld = max(t.stride(-2), t.shape[-1])
    if dims == 3 and t.shape[0] > 1 and t.stride(0) != t.shape[1] * ld:
        raise ValueError(f"{what}: packed groups are needed")
    return t, ld


def _whole(t, what: str, dtype: str, shape) -> int:
    """Address of a contiguous CUDA tensor of one type and shape; None: a null pointer."""
    import torch

    if t is None:
        return 0
    if t.dtype != getattr(torch, dtype) or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != tuple(shape):
        raise TypeError(f"{what}: a contiguous {dtype} CUDA tensor of shape {tuple(shape)} is needed")
    _on_device(t, what)
    return t.data_ptr()


def _ints(t, what: str, *shape) -> int:
    return _whole(t, what, "int32", shape)


def _floats(t, what: str, *shape) -> int:
    return _whole(t, what, "float32", shape)


def _stream() -> int:
    import torch

    return torch.cuda.current_stream().cuda_stream


def _blocks(n: int) -> int:
    return -(-n // SCALE_BLOCK)


def _up16(n: int) -> int:
    return -(-n // 16) * 16


def quantise(x, q: str = "e4m3", scale: str = "f32", block_rows: int = 1, rows: bool = True, transposed: bool = False, index=None):
    """x [M][K] (or rows of it by `index`) -> (Q, S) and, `transposed`, (QT, ST); None for a form that is not asked for.
    Q is [M][K rounded up to 16], its tail zeros; S is [blocks of K][M], for block_rows = 128 [blocks of M][blocks of K]."""
    import torch

    x, ldx = _rows(x, "x")
    m, k = (x.shape[0] if index is None else index.shape[0]), x.shape[1]
    pi = 0 if index is None else _ints(index, "index", m)
    if index is not None and not x.shape[0]:
        x, ldx = x.new_zeros((1, k)), k                   # an index into no rows: the library takes no rows for no index
    p = QuantisePlan(m, k, _type_name(x), q, scale, block_rows, x_rows=0 if index is None else x.shape[0], ldx=ldx)
    bytes_, kind = _torch_type(q), _torch_type(scale)
    new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=x.device)  # noqa: E731
    qs = ss = qt = st = None
    if rows:
        qs, ss = new((m, _up16(k)), bytes_), new((_blocks(m), _blocks(k)) if block_rows > 1 else (_blocks(k), m), kind)
    if transposed:
        qt, st = new((k, _up16(m)), bytes_), new((_blocks(k), _blocks(m)) if block_rows > 1 else (_blocks(m), k), kind)
    at = lambda t: 0 if t is None else t.data_ptr()  # noqa: E731
    p.run(x.data_ptr(), at(qs), at(ss), at(qt), at(st), _stream(), pi)
    return qs, ss, qt, st


def scaled_product(a, scale_a, b, scale_b, K: Optional[int] = None, c: str = "f16", offsets=None, along: str = "rows", index=None, spec: Optional[str] = None):
    """C = A B^T of 8-bit floats.  a [M][>= K]; scale_a [blocks of K][M] in float32, or of a byte in uint8 or float8_e8m0fnu; b [N][>= K] with scale_b [blocks of N][blocks of K] or
    [blocks of K][N].  With `offsets` [groups + 1]: along = "rows": b [groups][N][>= K], scale_b [groups][blocks of N][blocks of K], and
    `index` [rows] gathers the rows of a; along = "depth": C is [groups][M][N].  K defaults to the width of a."""
    import torch

    if a.dtype not in (torch.float8_e4m3fn, torch.float8_e5m2) or b.dtype != torch.float8_e4m3fn or _type_name(scale_a) != _type_name(scale_b):
        raise TypeError("scaled_product needs a in e4m3 or e5m2, b in e4m3 and scales of one type")
    K = min(a.shape[1], b.shape[-1]) if K is None else K
    if K > a.shape[1] or K > b.shape[-1]:
        raise ValueError("a and b are narrower than K")
    by_rows = offsets is not None and along == "rows"
    groups = 0 if offsets is None else offsets.shape[0] - 1
    po = 0 if offsets is None else _ints(offsets, "offsets", groups + 1)
    M, N = (a.shape[0] if index is None else index.shape[0]), b.shape[-2]
    pi = 0 if index is None else _ints(index, "index", M)
    if index is not None and not by_rows:
        raise ValueError("an index needs groups of rows")
    (a, lda), (b, ldb) = _rows(a, "a"), _rows(b, "b", 3 if by_rows else 2)
    (scale_a, ldsa), (scale_b, ldsb) = _rows(scale_a, "scale_a"), _rows(scale_b, "scale_b", 3 if by_rows else 2)
    by_block = tuple(scale_b.shape[-2:]) == (_blocks(N), _blocks(K))
    if by_rows and (b.shape[0] != groups or scale_b.shape[0] != groups):
        raise ValueError("b and scale_b hold one matrix for each group")
    if not by_block and (by_rows or tuple(scale_b.shape) != (_blocks(K), N)):
        raise ValueError("scale_b has another shape")
    # a scale for each row of a single block of rows reads the same both ways only where N = 1
    if tuple(scale_a.shape) != (_blocks(K), a.shape[0]):
        raise ValueError("scale_a has another shape")
    if index is not None and not a.shape[0]:              # as in quantise
        a, scale_a, ldsa = torch.zeros((1, lda), dtype=torch.uint8, device=a.device).view(a.dtype), scale_a.new_zeros((_blocks(K), 1)), 1
    out = torch.empty((groups, M, N) if groups and not by_rows else (M, N), dtype=_torch_type(c), device=a.device)
    with ScaledPlan(M, N, K, _type_name(a), c, _type_name(scale_a), SCALE_BLOCK if by_block else 1, groups, along, a.shape[0] if index is not None else 0, lda, ldb, 0, ldsa, ldsb, spec) as p:
        p.run(a.data_ptr(), scale_a.data_ptr(), b.data_ptr(), scale_b.data_ptr(), out.data_ptr(), _stream(), po, pi)
        if p.workspace_bytes():
            torch.cuda.current_stream().synchronize()     # the plan's workspace is freed on exit
    return out


def route(logits, k: int, bias=None, score: str = "softmax", groups: int = 1, keep: int = 1, top2: bool = False, renormalise: bool = True, factor: float = 1.0, align: int = 1):
    """logits [tokens][experts] -> weights [tokens][k], experts [tokens][k], offsets [experts + 1], rows [tokens][k], tokens_of [capacity]."""
    import torch

    logits, ld = _rows(logits, "logits")
    t, e = logits.shape
    new = lambda dtype, *shape: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
    pb = _floats(bias, "bias", e)
    with RoutePlan(t, e, k, _type_name(logits), score, groups, keep, top2, renormalise, factor, align, ld) as p:
        weights, experts = new(torch.float32, t, k), new(torch.int32, t, k)
        offsets, rows, tokens_of = new(torch.int32, e + 1), new(torch.int32, t, k), new(torch.int32, p.capacity)
        p.run(logits.data_ptr(), pb, weights.data_ptr(), experts.data_ptr(), offsets.data_ptr(), rows.data_ptr(), tokens_of.data_ptr(), _stream())
        torch.cuda.current_stream().synchronize()         # the plan's workspace is freed on exit
    return weights, experts, offsets, rows, tokens_of


def route_backward(logits, experts, dweights, score: str = "softmax", renormalise: bool = True, factor: float = 1.0):
    """dlogits from the gradient of route()'s weights, given its choice."""
    import torch

    logits, ld = _rows(logits, "logits")
    t, k = experts.shape
    pe = _ints(experts, "experts", logits.shape[0], k)
    pw = _floats(dweights, "dweights", t, k)
    dlogits = torch.empty_strided(logits.shape, (ld, 1), dtype=logits.dtype, device=logits.device)
    with RoutePlan(t, logits.shape[1], k, _type_name(logits), score, renormalise=renormalise, factor=factor, ld=ld) as p:
        p.backward(logits.data_ptr(), pe, pw, dlogits.data_ptr(), _stream())
        torch.cuda.current_stream().synchronize()         # the plan's workspace is freed on exit
    return dlogits


def combine(y, rows, weights=None, out: Optional[str] = None):
    """out[t] = sum over j of weights[t][j] * y[rows[t][j]]; weights None: ones."""
    import torch

    y, ldy = _rows(y, "y")
    t, k = rows.shape
    pr, pw = _ints(rows, "rows", t, k), _floats(weights, "weights", t, k)
    found = torch.empty((t, y.shape[1]), dtype=y.dtype if out is None else _torch_type(out), device=y.device)
    CombinePlan(t, k, y.shape[1], y.shape[0], _type_name(y), _type_name(found), ldy).run(pr, pw, y.data_ptr(), found.data_ptr(), _stream())
    return found


def combine_backward(y, rows, tokens_of, weights, dout):
    """(dY, dweights) of combine(y, rows, weights)."""
    import torch

    y, ldy = _rows(y, "y")
    dout, ldo = _rows(dout, "dout")
    t, k = rows.shape
    pr, pt, pw = _ints(rows, "rows", t, k), _ints(tokens_of, "tokens_of", y.shape[0]), _floats(weights, "weights", t, k)
    if tuple(dout.shape) != (t, y.shape[1]):
        raise ValueError("dout has another shape")
    dy = torch.empty_strided(y.shape, (ldy, 1), dtype=y.dtype, device=y.device)
    dw = torch.empty((t, k), dtype=torch.float32, device=y.device)
    CombinePlan(t, k, y.shape[1], y.shape[0], _type_name(y), _type_name(dout), ldy, ldo).backward(
        pr, pt, pw, y.data_ptr(), dout.data_ptr(), dy.data_ptr(), dw.data_ptr(), _stream())
    return dy, dw
