"""What the tensor functions of the expert-layer operators hand to the library: addresses and leading dimensions that reach the tensors' own values.  A stand-in
for the library reads them back from host memory, behind tensors that claim to be on the GPU.  No GPU."""
import ctypes
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2512_02551_amd as hg  # noqa: E402
from paper_2512_02551_amd import experts  # noqa: E402

DTYPES = [torch.float16, torch.bfloat16, torch.float32]          # of hgemm_type_t


class Device(torch.Tensor):
    """A host tensor that claims to be on a GPU."""

    is_cuda = property(lambda self: True)
    get_device = lambda self: 0  # noqa: E731


class OtherDevice(Device):
    get_device = lambda self: 1  # noqa: E731


def device(t):
    return t.as_subclass(Device)


def values(address, rows, cols, ld, dtype):
    """The matrix that a kernel finds at `address`."""
    if not rows or not cols:
        return torch.empty((rows, cols), dtype=dtype)
    size = torch.empty((), dtype=dtype).element_size()
    raw = bytearray(ctypes.string_at(address, ((rows - 1) * ld + cols) * size))
    return torch.frombuffer(raw, dtype=dtype).as_strided((rows, cols), (ld, 1)).clone()


class Library:
    """Keeps what a kernel would read, under the operands' names, and the descriptions."""

    def __init__(self):
        self.seen, self.launches = {}, 0

    def hgemm_quantise(self, d, x, index, q, s, qt, st, stream):
        d = self.desc = d._obj
        self.launches += 1
        self.seen["x"] = values(x, d.x_rows if index else d.M, d.K, d.ldx, DTYPES[d.x])
        return 0

    def hgemm_scaled_plan(self, handle, m, n, k, d):
        self.desc, self.shape = d._obj, (m, n, k)
        return 0

    def hgemm_scaled_workspace_bytes(self, handle):
        return 0

    def hgemm_scaled_run(self, handle, a, scale_a, b, scale_b, c, offsets, index, stream):
        d, (m, n, k) = self.desc, self.shape
        self.launches += 1
        groups, blocks = d.groups if d.group == 1 else 1, experts._blocks(k)
        rows = d.a_rows if index else m
        kind = torch.float32 if d.scale == 0 else torch.uint8
        self.seen["a"], self.seen["b"] = values(a, rows, k, d.lda, torch.uint8), values(b, groups * n, k, d.ldb, torch.uint8)
        self.seen["scale_a"] = values(scale_a, blocks, rows, d.ld_scale_a, kind)
        self.seen["scale_b"] = values(scale_b, *((blocks, n) if d.b_block_rows == 1 else (groups * experts._blocks(n), blocks)), d.ld_scale_b, kind)
        return 0

    def hgemm_route_plan(self, handle, d):
        self.desc = d._obj
        return 0

    def hgemm_route_capacity(self, d):
        return 64

    def _logits(self, address):
        d = self.desc
        self.launches += 1
        self.seen["logits"] = values(address, d.tokens, d.experts, d.ld, DTYPES[d.logits])
        return 0

    def hgemm_route_run(self, handle, logits, *rest):
        return self._logits(logits)

    def hgemm_route_backward(self, handle, logits, *rest):
        return self._logits(logits)

    def hgemm_combine(self, d, rows, weights, y, out, stream):
        d = self.desc = d._obj
        self.launches += 1
        self.seen["y"] = values(y, d.y_rows, d.N, d.ldy, DTYPES[d.y])
        return 0

    def hgemm_combine_backward(self, d, rows, tokens_of, weights, y, dout, dy, dweights, stream):
        d = d._obj
        self.seen["dout"] = values(dout, d.tokens, d.N, d.ldo, DTYPES[d.out])
        return self.hgemm_combine(ctypes.byref(d), rows, weights, y, None, stream)


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(experts, "_lib", lambda: lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=0, synchronize=lambda: None))
    return lib


ROWS, COLS = 6, 32
LAYOUTS = {                                                       # rows, columns, distance of the rows
    "packed": (ROWS, COLS, COLS), "apart": (ROWS, COLS, COLS + 16), "repeated": (ROWS, COLS, 0), "overlapping": (ROWS, COLS, 16), "one row": (1, COLS, 7),
    "a repeated element": (ROWS, 1, 0), "no rows": (0, COLS, 0),
}


def view(name, dtype=torch.float32):
    """A view of a buffer that goes on behind it, with other values."""
    rows, cols, distance = LAYOUTS[name]
    return device(torch.as_strided((torch.arange(4096) % 241 + 1).to(dtype), (rows, cols), (distance, 1)))


def ints(*shape):
    return device(torch.zeros(shape, dtype=torch.int32))


def same(got, want):
    return torch.equal(got.view(torch.uint8) if got.element_size() == 1 else got, want.as_subclass(torch.Tensor).contiguous().view(torch.uint8) if want.element_size() == 1 else want.as_subclass(torch.Tensor))


@pytest.mark.parametrize("name", list(LAYOUTS))
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_rows_of_any_distance_reach_the_kernels_of_16_and_32_bits(library, name, dtype):
    x = view(name, dtype)
    rows, cols = x.shape
    hg.quantise(x)
    assert same(library.seen["x"], x)
    if rows:
        hg.quantise(x, index=ints(9))
        assert same(library.seen["x"], x)
    hg.route(x, 1)
    assert same(library.seen["logits"], x)
    dx = hg.route_backward(x, ints(rows, 1), device(torch.zeros(rows, 1)))
    assert same(library.seen["logits"], x) and dx.shape == x.shape
    assert rows == 0 or dx.untyped_storage().nbytes() >= ((rows - 1) * library.desc.ld + cols) * dx.element_size()
    hg.combine(x, ints(3, 2))
    assert same(library.seen["y"], x)
    dy, dw = hg.combine_backward(x, ints(rows, 2), ints(rows), None, x)
    assert same(library.seen["y"], x) and same(library.seen["dout"], x) and dy.shape == x.shape and dw.shape == (rows, 2)
    assert rows == 0 or dy.untyped_storage().nbytes() >= ((rows - 1) * library.desc.ldy + cols) * dy.element_size()      # every row of the gradient has a place


@pytest.mark.parametrize("name", ["packed", "apart", "repeated", "overlapping"])
def test_rows_of_any_distance_reach_the_products(library, name):
    q = view(name, torch.uint8).view(torch.float8_e4m3fn)
    packed = device(torch.ones((5, COLS), dtype=torch.float8_e4m3fn))
    one = lambda *shape: device(torch.rand(shape))  # noqa: E731
    hg.scaled_product(q, one(1, ROWS), packed, one(1, 1))
    assert same(library.seen["a"], q)
    hg.scaled_product(packed, one(1, 5), q, one(1, 1))
    assert same(library.seen["b"], q)
    a, b = device(torch.ones((9, 3 * 128), dtype=torch.float8_e4m3fn)), device(torch.ones((7, 3 * 128), dtype=torch.float8_e4m3fn))
    by_row = [device(torch.rand(1, r)).expand(3, r) for r in (9, 7)]                # one scale for all blocks of a row
    assert by_row[0].stride() == (0, 1)
    hg.scaled_product(a, by_row[0], b, by_row[1])
    assert same(library.seen["scale_a"], by_row[0]) and same(library.seen["scale_b"], by_row[1]) and library.desc.b_block_rows == 1


def test_groups_have_to_be_packed(library):
    a, offsets = device(torch.ones((4, COLS), dtype=torch.float8_e4m3fn)), ints(3)
    b, scales = torch.ones((1, 8, COLS), dtype=torch.float8_e4m3fn), device(torch.ones(2, 1, 1))
    hg.scaled_product(a, device(torch.ones(1, 4)), device(b.repeat(2, 1, 1)), scales, offsets=offsets)
    for shared in (b.expand(2, 8, COLS), torch.ones((4, 8, COLS), dtype=torch.float8_e4m3fn)[::2]):
        before = library.launches
        with pytest.raises(ValueError, match="packed groups"):
            hg.scaled_product(a, device(torch.ones(1, 4)), device(shared), scales, offsets=offsets)
        assert library.launches == before


@pytest.mark.parametrize("wrong", ["on the host", "of another type", "of another shape", "not contiguous"])
@pytest.mark.parametrize("function", ["combine", "combine_backward", "route", "route_backward"])
def test_weights_are_checked_before_a_kernel_sees_them(library, function, wrong):
    t, k = 4, 2
    good = (3,) if function == "route" else (t, k)
    bad = {"on the host": torch.ones(good), "of another type": device(torch.ones(good, dtype=torch.float16)), "of another shape": device(torch.ones(5, 7)),
           "not contiguous": device(torch.ones(*good, 2)[..., 0])}[wrong]
    y, logits = view("packed"), device(torch.randn(t, 3))
    call = {"combine": lambda w: hg.combine(y, ints(t, k), w), "combine_backward": lambda w: hg.combine_backward(y, ints(t, k), ints(ROWS), w, device(torch.ones(t, COLS))),
            "route": lambda w: hg.route(logits, k, w), "route_backward": lambda w: hg.route_backward(logits, ints(t, k), w)}[function]
    with pytest.raises(TypeError):
        call(bad)
    assert library.launches == 0
    call(device(torch.ones(good)))
    assert library.launches == 1


def test_tensors_of_another_device_are_refused(library, monkeypatch):
    """Each operand in turn on device 1 with device 0 current, and all of them on device 0 with device 1 current."""
    q = lambda *shape: device(torch.ones(shape, dtype=torch.float8_e4m3fn))  # noqa: E731
    f = lambda *shape: device(torch.ones(shape))  # noqa: E731
    calls = [
        (lambda x, index: hg.quantise(x, index=index), [f(4, COLS), ints(6)]),
        (hg.scaled_product, [q(4, COLS), f(1, 4), q(5, COLS), f(1, 1)]),
        (lambda a, sa, b, sb, o, i: hg.scaled_product(a, sa, b, sb, offsets=o, index=i), [q(4, COLS), f(1, 4), q(2, 5, COLS), f(2, 1, 1), ints(3), ints(6)]),
        (lambda x, b: hg.route(x, 2, b), [f(4, 8), f(8)]), (hg.route_backward, [f(4, 8), ints(4, 2), f(4, 2)]),
        (hg.combine, [f(6, COLS), ints(4, 2), f(4, 2)]), (hg.combine_backward, [f(6, COLS), ints(4, 2), ints(6), f(4, 2), f(4, COLS)]),
    ]
    for n, (function, operands) in enumerate(calls):
        function(*operands)
        assert library.launches == n + 1
    for function, operands in calls:
        for i in range(len(operands)):
            with pytest.raises(ValueError, match="cuda:1"):
                function(*operands[:i], operands[i].as_subclass(OtherDevice), *operands[i + 1:])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for function, operands in calls:
        with pytest.raises(ValueError, match="cuda:1"):
            function(*operands)
    assert library.launches == len(calls)


def test_an_index_into_no_rows_gives_rows_of_zeros(library):
    """The library takes a source without rows for one that is not indexed: it is handed a row of zeros, which every index inside it reads."""
    hg.quantise(device(torch.ones(0, 48)), index=ints(6))
    assert library.desc.x_rows == 1 and library.desc.M == 6 and same(library.seen["x"], device(torch.zeros(1, 48)))
    for k in (48, 300):
        blocks, width = experts._blocks(k), experts._up16(k)
        out = hg.scaled_product(device(torch.ones((0, width), dtype=torch.float8_e4m3fn)), device(torch.ones(blocks, 0)), device(torch.ones((2, 5, width), dtype=torch.float8_e4m3fn)),
                                device(torch.ones(2, 1, blocks)), K=k, offsets=ints(3), index=ints(6))
        assert out.shape == (6, 5) and library.desc.a_rows == 1 and library.desc.lda % 16 == 0
        assert (library.seen["a"] == 0).all() and library.seen["a"].shape == (1, k) and (library.seen["scale_a"] == 0).all() and library.seen["scale_a"].shape == (blocks, 1)


@pytest.mark.parametrize("mixed", [False, True])
def test_scales_of_a_byte_may_have_torchs_type_for_them(library, mixed):
    a, b = (device(torch.ones((r, 256), dtype=torch.float8_e4m3fn)) for r in (6, 5))
    sa, sb = (torch.randint(120, 130, s, dtype=torch.uint8, generator=torch.Generator().manual_seed(1)) for s in ((2, 6), (2, 5)))
    hg.scaled_product(a, device(sa.view(torch.float8_e8m0fnu)), b, device(sb if mixed else sb.view(torch.float8_e8m0fnu)))
    assert library.desc.scale == 1 and same(library.seen["scale_a"], device(sa)) and same(library.seen["scale_b"], device(sb))
    shared = device(sa[:1].view(torch.float8_e8m0fnu)).expand(2, 6)
    hg.scaled_product(a, shared, b, device(sb))
    assert same(library.seen["scale_a"], device(sa[:1].expand(2, 6).contiguous()))
    for wrong in (torch.ones(2, 6), torch.ones((2, 6), dtype=torch.float16)):
        with pytest.raises((TypeError, ValueError)):
            hg.scaled_product(a, device(wrong), b, device(sb))


def test_matrices_without_columns_are_packed(library):
    """No K, no N: nothing is read, whatever strides torch gives such tensors; products give zeros."""
    q = lambda *shape: device(torch.ones(shape, dtype=torch.float8_e4m3fn))  # noqa: E731
    f = lambda *shape: device(torch.ones(shape))  # noqa: E731
    assert hg.scaled_product(q(4, 0), f(0, 4), q(6, 0), f(1, 0)).shape == (4, 6) and library.desc.lda == library.desc.ldb == 0 and library.desc.ld_scale_b == 0
    assert hg.scaled_product(q(4, 0), f(0, 4), q(2, 6, 0), f(2, 1, 0), offsets=ints(3)).shape == (4, 6) and library.desc.ldb == 0
    assert hg.scaled_product(q(4, 0), f(0, 4), q(6, 0), f(0, 6), offsets=ints(3), along="depth").shape == (2, 4, 6) and library.desc.b_block_rows == 1
    hg.quantise(f(4, 0), transposed=True)
    assert library.desc.ldx == 0
    hg.combine(f(6, 0), ints(4, 2))
    assert library.desc.ldy == 0
    dy, dw = hg.combine_backward(f(6, 0), ints(4, 2), ints(6), None, f(4, 0))
    assert library.desc.ldy == library.desc.ldo == 0 and dy.shape == (6, 0) and dw.shape == (4, 2)
