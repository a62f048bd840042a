"""The expert-layer operators on inputs off the ordinary: rows that share memory, no K, the most tokens, infinite logits, no tokens, types, new weights under a captured step, new plans beside a busy stream."""
import zlib

import pytest

torch = pytest.importorskip("torch")

import paper_2512_02551_amd as hg  # noqa: E402

pytestmark = pytest.mark.gpu


def gen(*seed):
    g = torch.Generator()
    g.manual_seed(zlib.crc32(repr(seed).encode()))
    return g


def same(got, want):
    """Bit for bit (no NaN among them)."""
    return all(a is b is None or torch.equal(a.float(), b.float()) for a, b in zip(got, want))


# ---- rows that share memory: the results of the same values in rows of their own -----------------------------------------------------

SHARED = {"repeated": 0, "overlapping": 40}


def shared(name, rows, cols, dtype, g):
    base = torch.randn(rows * 40 + cols, generator=g).to(dtype).cuda()
    x = torch.as_strided(base, (rows, cols), (SHARED[name], 1))
    return x, x.contiguous()


@pytest.mark.parametrize("name", list(SHARED))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
def test_rows_that_share_memory(name, dtype):
    g = gen("shared", name, dtype)
    x, own = shared(name, 70, 256, dtype, g)
    assert same(hg.quantise(x, transposed=True), hg.quantise(own, transposed=True))
    assert same(hg.quantise(x, block_rows=128, transposed=True), hg.quantise(own, block_rows=128, transposed=True))
    found, want = hg.route(x, 4), hg.route(own, 4)
    assert same(found, want)
    dw = torch.randn((70, 4), generator=g).cuda()
    assert torch.equal(hg.route_backward(x, found[1], dw), hg.route_backward(own, found[1], dw))
    rows = torch.randperm(70, generator=g).to(torch.int32).view(35, 2).cuda()
    tokens = torch.empty(70, dtype=torch.int32, device="cuda")
    tokens[rows.flatten().long()] = torch.arange(35, dtype=torch.int32, device="cuda").repeat_interleave(2)
    w = torch.rand((35, 2), generator=g).cuda()
    assert torch.equal(hg.combine(x, rows, w), hg.combine(own, rows, w))
    dout, dout_own = shared(name, 35, 256, dtype, g)
    assert same(hg.combine_backward(x, rows, tokens, w, dout), hg.combine_backward(own, rows, tokens, w, dout_own))


@pytest.mark.parametrize("name", list(SHARED))
def test_operands_of_a_product_that_share_memory(name):
    g = gen("shared operands", name)
    a, b = (torch.as_strided((torch.randn(8192, generator=g) * 4).to(torch.float8_e4m3fn).cuda(), (r, 384), (SHARED[name] // 16 * 16, 1)) for r in (50, 60))
    own = [t.view(torch.uint8).contiguous().view(torch.float8_e4m3fn) for t in (a, b)]
    sa, sb = (torch.rand((1, r), generator=g).cuda().expand(3, r) for r in (50, 60))      # one scale for all blocks of a row
    found = hg.scaled_product(a, sa, b, sb, c="f32")
    assert torch.equal(found, hg.scaled_product(own[0], sa.contiguous(), own[1], sb.contiguous(), c="f32")) and found.abs().max() > 0


# ---- no K -------------------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("c", ["f16", "f32"])
@pytest.mark.parametrize("spec", ["tile,bm=16,bn=64,sk=2", "tile,bm=64,bn=64,sk=16", "rows,bm=16,bn=16", "phased,bm=128,bn=128"])
def test_no_depth_gives_zeros_whatever_the_kernel(spec, c):
    m, n = 40, 100
    out = torch.full((m, n), float("nan"), dtype={"f16": torch.float16, "f32": torch.float32}[c], device="cuda")
    with hg.ScaledPlan(m, n, 0, c=c, spec=spec) as p:
        p.run(0, 0, 0, 0, out.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    assert (out == 0).all()


@pytest.mark.parametrize("c", ["f16", "f32"])
def test_no_depth_gives_zeros_from_tensors(c):
    q, s, qt, st = hg.quantise(torch.ones((5, 0), device="cuda"), transposed=True)
    assert q.shape == (5, 0) and s.shape == (0, 5) and qt.shape == (0, 16) and st.shape == (1, 0)
    new = lambda *shape: torch.empty(shape, device="cuda")  # noqa: E731
    b = new(6, 0).to(torch.float8_e4m3fn)
    assert torch.equal(hg.scaled_product(q, s, b, new(1, 0), c=c).float(), torch.zeros((5, 6), device="cuda"))
    offsets = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    assert torch.equal(hg.scaled_product(q, s, torch.stack([b, b]), new(2, 1, 0), c=c, offsets=offsets).float(), torch.zeros((5, 6), device="cuda"))
    assert torch.equal(hg.scaled_product(q, s, b, new(0, 6), c=c, offsets=0 * offsets, along="depth").float(), torch.zeros((2, 5, 6), device="cuda"))


# ---- as many tokens as there may be -------------------------------------------------------------------------------------------------------

def test_the_gradient_of_the_most_tokens():
    t, e = (1 << 26) - 1, 4
    x = torch.randn((t, e), dtype=torch.float16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    chosen = (torch.arange(t, dtype=torch.int32, device="cuda") % e)[:, None].contiguous()
    dw = torch.ones((t, 1), device="cuda")
    dx = torch.full((t, e), float("nan"), dtype=torch.float16, device="cuda")
    with hg.RoutePlan(t, e, 1, renormalise=False) as p:
        p.backward(x.data_ptr(), chosen.data_ptr(), dw.data_ptr(), dx.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
    assert not dx.isnan().any()
    at = torch.tensor([0, 1, 4, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, (1 << 25) + 4, t - 4, t - 3, t - 2, t - 1], device="cuda")
    p64 = torch.softmax(x[at].double(), 1)
    one = torch.nn.functional.one_hot(chosen[at, 0].long(), e).double()
    want = p64 * (one - (p64 * one).sum(1, keepdim=True))
    assert ((dx[at].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -20).all()      # one rounding, and fp32 on numbers below 1


# ---- infinite logits ----------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", [torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("e", [8, 200])
def test_a_softmax_over_an_infinite_logit_is_no_number(e, renormalise, kind):
    """exp(inf - inf) over its sum: no weight of such a token is a number, as in the formula.  The choice goes by the logits and stays."""
    x = torch.randn((40, e), generator=gen("infinite", e)).to(kind)
    x[7, 5] = float("inf")
    weights, chosen = (v.cpu() for v in hg.route(x.cuda(), 3, renormalise=renormalise)[:2])
    assert torch.equal(chosen, x.float().sort(stable=True, dim=1, descending=True).indices[:, :3].to(torch.int32)) and chosen[7, 0] == 5
    bad = torch.zeros(40, dtype=torch.bool)
    bad[7] = True
    assert torch.equal(weights.isnan(), bad[:, None].expand(40, 3))
    dx = hg.route_backward(x.cuda(), chosen.cuda(), torch.ones((40, 3), device="cuda"), renormalise=renormalise).cpu()
    assert torch.equal(dx.isnan(), bad[:, None].expand(40, e))


def test_a_sigmoid_of_an_infinite_logit_is_one():
    x = torch.randn((40, 64), generator=gen("infinite sigmoid"))
    x[7, 5] = float("inf")
    weights, chosen = (v.cpu() for v in hg.route(x.cuda(), 3, score="sigmoid", renormalise=False)[:2])
    assert chosen[7, 0] == 5 and weights[7, 0] == 1 and torch.isfinite(weights).all()
    dx = hg.route_backward(x.cuda(), chosen.cuda(), torch.ones((40, 3), device="cuda"), "sigmoid", False).cpu()
    assert torch.isfinite(dx).all() and dx[7, 5] == 0


# ---- no tokens ------------------------------------------------------------------------------------------------------------------------------

def test_an_index_into_no_rows_gives_zeros():
    index = torch.tensor([-1, 0, 5, -1], dtype=torch.int32, device="cuda")
    q, s, qt, st = hg.quantise(torch.ones((0, 200), device="cuda"), index=index, transposed=True)
    assert q.shape == (4, 208) and (q.float() == 0).all() and (qt.float() == 0).all() and torch.equal(s, torch.full_like(s, 2.0 ** -96 / 448)) and torch.equal(st, torch.full_like(st, 2.0 ** -96 / 448))
    b, sb, _, _ = hg.quantise(torch.randn((2 * 128, 200), device="cuda"), block_rows=128)
    offsets = torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda")
    for c in ("f16", "f32"):
        out = hg.scaled_product(q[:0], s[:, :0], b.view(2, 128, 208), sb.view(2, 1, 2), K=200, c=c, offsets=offsets, index=index)
        assert out.shape == (4, 128) and (out == 0).all()


def test_a_layer_without_tokens():
    """Rows of padding alone: an empty result, and weight gradients of zeros."""
    import test_gpu_expert_layer as layers

    e, k, width, hidden = 4, 2, 256, 384
    g = gen("no tokens")
    new = lambda *shape: (0.05 * torch.randn(shape, generator=g)).to(torch.bfloat16).cuda()  # noqa: E731
    layer = layers.example.ExpertLayer(new(e, hidden, width), new(e, width, hidden), k)
    out = layer.forward(new(0, width), torch.randn((0, e), device="cuda"))
    dx, dlogits, dup, ddown = layer.backward(new(0, width))
    assert out.shape == dx.shape == (0, width) and dlogits.shape == (0, e)
    assert dup.shape == (e, hidden, width) and ddown.shape == (e, width, hidden) and (dup == 0).all() and (ddown == 0).all()


# ---- types ------------------------------------------------------------------------------------------------------------------------------------

def test_scales_of_a_byte_in_torchs_type():
    g = gen("e8m0")
    a, sa, _, _ = hg.quantise(torch.randn((50, 300), generator=g).cuda(), scale="e8m0")
    b, sb, _, _ = hg.quantise(torch.randn((70, 300), generator=g).cuda(), scale="e8m0", block_rows=128)
    own = torch.float8_e8m0fnu
    want = hg.scaled_product(a, sa, b, sb, K=300)
    assert torch.equal(hg.scaled_product(a, sa.view(own), b, sb.view(own), K=300), want) and torch.equal(hg.scaled_product(a, sa.view(own), b, sb, K=300), want)
    one = sa[:1].view(own)
    assert torch.equal(hg.scaled_product(a, one.expand(3, 50), b, sb, K=300), hg.scaled_product(a, sa[:1].repeat(3, 1), b, sb, K=300))


# ---- new weights --------------------------------------------------------------------------------------------------------------------------------

def test_a_captured_step_goes_on_with_the_weights_that_are_loaded():
    import test_gpu_expert_layer as layers

    t, e, k, width, hidden = 12, 4, 2, 256, 384
    g = gen("load")
    weights = lambda: [(0.05 * torch.randn(s, generator=g)).to(torch.bfloat16).cuda() for s in ((e, hidden, width), (e, width, hidden))]  # noqa: E731
    first, second = weights(), weights()
    x, logits = torch.randn((t, width), generator=g).to(torch.bfloat16).cuda(), torch.randn((t, e), generator=g).cuda()
    layer = layers.example.ExpertLayer(*first, k)
    step = layers.example.DecodeStep(layer, t, e, width, hidden)
    want = [layers.example.ExpertLayer(*w, k).forward(x, logits) for w in (first, second)]
    assert not torch.equal(*want)
    for i in (0, 1, 0, 1):
        layer.load(*(first, second)[i])
        held = [torch.full((e, hidden, width), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]      # on what the old weights gave back, if they did
        assert torch.equal(step(x, logits), want[i]) and torch.equal(layer.forward(x, logits), want[i]), i
        del held


# ---- streams ------------------------------------------------------------------------------------------------------------------------------------

def test_a_new_plan_runs_on_a_stream_beside_a_busy_null_stream():
    """Its counters are cleared in the null stream; the other stream does not wait for that, so the plan has to."""
    g = gen("busy")
    m, n, k, t, e = 64, 512, 8192, 32, 64
    a, sa, _, _ = hg.quantise(torch.randn((m, k), generator=g).cuda())
    b, sb, _, _ = hg.quantise(torch.randn((n, k), generator=g).cuda(), block_rows=128)
    x, w = torch.randn((m, k), generator=g).half().cuda(), torch.randn((k, n), generator=g).half().cuda()
    logits = torch.randn((t, e), generator=g).cuda()
    new = lambda *shape, dtype=torch.int32: torch.full(shape, -7, dtype=dtype, device="cuda")  # noqa: E731
    want = hg.scaled_product(a, sa, b, sb, spec="tile,bm=64,bn=64,sk=8"), hg.hgemm(x, w, spec="skinny,sk=8,fr=1"), *hg.route(logits, 4)
    big, side = torch.randn((8192, 8192), device="cuda").half(), torch.cuda.Stream()
    c, d = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    order = torch.zeros_like(want[2]), new(t, 4), new(e + 1), new(t, 4), new(t * 4)
    torch.cuda.synchronize()
    for _ in range(20):
        big @ big                                                 # some milliseconds ahead of the clearing
    with hg.ScaledPlan(m, n, k, spec="tile,bm=64,bn=64,sk=8") as p, hg.Plan(m, n, k, spec="skinny,sk=8,fr=1") as q, hg.RoutePlan(t, e, 4, "f32") as r:
        assert p.workspace_bytes() > 0 and q.workspace_bytes() > 0
        s = side.cuda_stream
        p.run(a.data_ptr(), sa.data_ptr(), b.data_ptr(), sb.data_ptr(), c.data_ptr(), s)
        q.run(x.data_ptr(), w.data_ptr(), d.data_ptr(), s)
        r.run(logits.data_ptr(), 0, *[o.data_ptr() for o in order], s)
        torch.cuda.synchronize()
    for got, expected in zip((c, d, *order), want):
        assert torch.equal(got, expected)
