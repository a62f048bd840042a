"""Products by groups in every kernel, type of C and kind of scale, against 64 bits: rows of groups that end around halves of tiles and around tiles, with and
without an index; ranges of K of several blocks; and what the library chooses for groups of many rows."""
import functools

import pytest

torch = pytest.importorskip("torch")

import experts_ref as ref  # noqa: E402
import paper_2512_02551_amd as hg  # noqa: E402
from test_gpu_experts import TILES, blocks, check, gen, random_bytes, random_scales, run_product  # noqa: E402

pytestmark = pytest.mark.gpu

SPECS = [s for s in TILES if "sk=" not in s]
TYPES = ["f16", "bf16", "f32"]


def scales(g, shape, kind, low=0):
    """e8m0: results of an fp16 C stay below its largest value."""
    s = random_scales(g, shape, kind)
    return s - low if kind == "e8m0" else s


def has_no(spec, k, error):
    """256 x 256 tiles have not all kinds of sums, and phased ones take whole 16-byte chunks of K."""
    return error.status == 2 and ("bm=256,bn=256" in spec or spec.startswith("phased") and k % 16)


LENGTHS = [1, 127, 128, 0, 129, 255, 256, 257, 300, 0, 64, 32]      # a tile of 256 rows ends in its first half, at it, in its second, and behind it


@functools.lru_cache(maxsize=None)
def problem_of_rows(lengths, n, k, kind, scale, indexed, rest=21):
    g = gen("rows", lengths, n, k, kind, scale, indexed)
    e = len(lengths)
    offsets = torch.tensor((0,) + lengths).cumsum(0).to(torch.int32)
    m, source = int(offsets[-1]) + rest, 333
    index = torch.randint(0, source, (m,), generator=g).to(torch.int32)
    index[::7], index[1::11] = -1, source
    a = random_bytes(g, source if indexed else m, k, kind)
    b = torch.stack([random_bytes(g, n, k, "e4m3") for _ in range(e)])
    sa, sb = scales(g, (blocks(k), a.shape[0]), scale, 10), scales(g, (e, blocks(n), blocks(k)), scale)
    va, vb = ref.by_rows(a, sa, k), ref.by_blocks(b, sb, k)
    if indexed:
        ok = (index >= 0) & (index < source)
        va = torch.where(ok[:, None], va[index.long().clamp(0, source - 1)], torch.zeros((), dtype=torch.float64))
    want, size = torch.zeros((m, n), dtype=torch.float64), torch.zeros((m, n), dtype=torch.float64)
    for i in range(e):
        lo, hi = int(offsets[i]), int(offsets[i + 1])
        want[lo:hi], size[lo:hi] = va[lo:hi] @ vb[i].t(), va[lo:hi].abs() @ vb[i].abs().t()
    return offsets, index if indexed else None, a, sa, b, sb, want, size, source


def bound_of(size, want, c, n_blocks):
    """ref.product_bound, of the sums of magnitudes."""
    one = torch.ones((1, 1), dtype=torch.float64)
    return ref.product_bound(one, one, torch.zeros((1, 1), dtype=torch.float64), c, n_blocks) * size + ref.product_bound(0 * one, one, want, c, n_blocks)


def run_rows(lengths, n, k, kind, scale, indexed, c, spec=None):
    offsets, index, a, sa, b, sb, want, size, source = problem_of_rows(lengths, n, k, kind, scale, indexed)
    got, desc = run_product(a, sa, b, sb, want.shape[0], n, k, c, ldc=n + 1, offsets=offsets, index=index, a=kind, scale=scale, groups=len(lengths), along="rows",
                            a_rows=source if indexed else 0, spec=spec)
    check(got, want, bound_of(size, want, c, blocks(k)), (desc, c))
    assert (got[int(offsets[-1]):] == 0).all()
    return desc


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("indexed", [False, True])
@pytest.mark.parametrize("c", TYPES)
@pytest.mark.parametrize("spec", SPECS)
def test_rows_of_groups_in_every_kernel(spec, c, indexed, scale):
    ran = 0
    for n, k, kind in ((333, 656, "e4m3"), (260, 1280, "e5m2"), (140, 203, "e4m3")):
        try:
            assert run_rows(tuple(LENGTHS), n, k, kind, scale, indexed, c, spec).startswith(spec)
            ran += 1
        except hg.HgemmError as error:
            assert has_no(spec, k, error)
    assert ran or "bm=256,bn=256" in spec


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("c", TYPES)
@pytest.mark.parametrize("spec", SPECS)
def test_ranges_of_k_in_every_kernel(spec, c, b_rows, scale):
    ran, m, n = 0, 300, 270
    for k, lengths in ((1520, (128, 0, 384, 256, 640, 112)), (1280, (1152, 128)), (845, (768, 0, 77))):
        want, size, a, sa, b, sb, offsets = problem_of_ranges(k, lengths, m, n, b_rows, scale)
        try:
            got, desc = run_product(a, sa, b, sb, m, n, k, c, ldc=n + 2, offsets=offsets, out_shape=(len(lengths), m, n), a="e5m2", scale=scale, b_rows=b_rows, groups=len(lengths),
                                    along="depth", spec=spec)
        except hg.HgemmError as error:
            assert has_no(spec, k, error)
            continue
        ran += 1
        assert desc.startswith(spec)
        check(got, want, bound_of(size, want, c, max(blocks(x) for x in lengths)), (desc, c, k))
        assert all((got[i] == 0).all() for i, x in enumerate(lengths) if x == 0)
    assert ran or "bm=256,bn=256" in spec


@functools.lru_cache(maxsize=None)
def problem_of_ranges(k, lengths, m, n, b_rows, scale):
    g = gen("ranges", k, lengths, b_rows, scale)
    offsets = torch.tensor((0,) + lengths).cumsum(0).to(torch.int32)
    a, b = random_bytes(g, m, k, "e5m2"), random_bytes(g, n, k, "e4m3")
    sa, sb = scales(g, (blocks(k), m), scale, 10), scales(g, (blocks(k), n) if b_rows == 1 else (blocks(n), blocks(k)), scale)
    va, vb = ref.by_rows(a, sa, k), (ref.by_rows if b_rows == 1 else ref.by_blocks)(b, sb, k)
    parts = [(va[:, offsets[i]:offsets[i + 1]], vb[:, offsets[i]:offsets[i + 1]]) for i in range(len(lengths))]
    return torch.stack([x @ y.t() for x, y in parts]), torch.stack([x.abs() @ y.abs().t() for x, y in parts]), a, sa, b, sb, offsets


# ---- what the library chooses -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("indexed", [False, True])
@pytest.mark.parametrize("c", ["f16", "bf16"])
@pytest.mark.parametrize("lengths,kernel", [((2100, 3, 0, 1025, 256, 511, 130, 2954), "phased,bm=256"), ((700, 3, 0, 325, 256, 511, 130, 54), "phased,bm=128")], ids=str)
def test_groups_of_many_rows_as_the_library_runs_them(lengths, kernel, c, indexed, scale):
    assert run_rows(lengths, 2048, 512, "e4m3", scale, indexed, c).startswith(kernel)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("lengths", [(1, 0, 2, 3, 1, 0, 0, 1), (37,), (0, 300, 1, 64, 65, 0, 127, 129)], ids=str)
@pytest.mark.parametrize("c", ["f16", "bf16"])
def test_groups_of_few_rows_as_the_library_runs_them(c, lengths, scale):
    for indexed in (False, True):
        for k in (384, 272, 203):
            run_rows(lengths, 200, k, "e4m3", scale, indexed, c)


@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("c", TYPES)
def test_ranges_of_k_as_the_library_runs_them(c, scale):
    lengths, m, n = (1024, 0, 2048, 128, 512, 384), 520, 760
    want, size, a, sa, b, sb, offsets = problem_of_ranges(4096, lengths, m, n, 1, scale)
    got, desc = run_product(a, sa, b, sb, m, n, 4096, c, offsets=offsets, out_shape=(len(lengths), m, n), a="e5m2", scale=scale, b_rows=1, groups=len(lengths), along="depth")
    check(got, want, bound_of(size, want, c, 16), (desc, c))


@pytest.mark.parametrize("c", ["f32", "bf16"])
@pytest.mark.parametrize("spec", [None] + SPECS)
def test_ranges_behind_a_k_that_ends_inside_a_block_are_empty(spec, c):
    """An expert without rows behind the last one that has some: zeros, not the last block once more.  Offsets past K count as K."""
    m, n = 70, 90
    for k, lengths, past in ((336, (256, 80, 0, 0), 0), (336, (0, 336, 0), 500), (48, (48, 0), 0), (333, (256, 77, 0), 3)):
        want, size, a, sa, b, sb, offsets = problem_of_ranges(k, lengths, m, n, 1, "f32")
        offsets = offsets.clone()
        offsets[-1] += past
        try:
            got, desc = run_product(a, sa, b, sb, m, n, k, c, offsets=offsets, out_shape=(len(lengths), m, n), a="e5m2", b_rows=1, groups=len(lengths), along="depth", spec=spec)
        except hg.HgemmError as error:
            assert spec and has_no(spec, k, error)
            continue
        check(got, want, bound_of(size, want, c, 3), (desc, c, k))


# ---- sums whose large products cancel -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("scale", ["f32", "e8m0"])
@pytest.mark.parametrize("c", TYPES)
@pytest.mark.parametrize("spec", [None] + SPECS)
def test_cancelling_products(spec, c, scale):
    """Within every block of 128 each large product comes with its negative, at places dealt at random, beside small ones that are what is left: a 16-bit C keeps them to
    2^-10 of the magnitudes, an fp32 C to roundings of fp32."""
    g = gen("cancel", scale)
    m, n, k = 70, 150, 384

    def half(rows):
        big = torch.exp2(torch.randint(-6, 9, (rows, k // 128, 48), generator=g).float()) * torch.where(torch.rand((rows, k // 128, 48), generator=g) < 0.5, -1.75, 1.0)
        return big, torch.exp2(torch.randint(-6, 1, (rows, k // 128, 32), generator=g).float())

    (a, small_a), (b, small_b) = half(m), half(n)
    order = torch.stack([torch.randperm(128, generator=g) for _ in range(k // 128)])
    a, b = (torch.cat(parts, 2).gather(2, order.expand(len(parts[0]), -1, -1)).flatten(1).to(torch.float8_e4m3fn) for parts in ((a, -a, small_a), (b, b, small_b)))
    sa, sb = scales(g, (blocks(k), m), scale, 10), scales(g, (blocks(n), blocks(k)), scale)
    va, vb = ref.by_rows(a, sa, k), ref.by_blocks(b, sb, k)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    assert (want.abs() < 0.05 * size).all()
    try:
        got, desc = run_product(a, sa, b, sb, m, n, k, c, scale=scale, spec=spec)
    except hg.HgemmError as error:
        assert spec and has_no(spec, k, error)
        return
    check(got, want, bound_of(size, want, c, blocks(k)), (desc, c))
