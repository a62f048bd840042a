"""What the expert-layer operators allocate and launch, read from the host code on a machine without a GPU (fake_experts.py)."""
import pytest

from fake_experts import ask


@pytest.mark.parametrize("spec", ["tile,bm=16,bn=64,sk=2", "tile,bm=64,bn=64,sk=16", "tile,bm=128,bn=128,sk=1", None])
def test_nothing_is_split_where_there_is_no_k(spec):
    """Zeros all the same: one launch, no workspace."""
    for c in (0, 2):
        (r,) = ask([{"op": "scaled", "M": 40, "N": 100, "K": 0, "c": c, **({"spec": spec} if spec else {})}])
        assert r["plan"] == 0 and r["run"] == 0 and r["workspace"] == 0 and len(r["launches"]) == 1, r
        assert spec is None or r["describe"].endswith("sk=1")


@pytest.mark.parametrize("k,splits", [(1, 1), (128, 1), (129, 2), (256, 2), (385, 2), (1024, 2)])
def test_a_split_has_no_empty_range(k, splits):
    (r,) = ask([{"op": "scaled", "M": 40, "N": 100, "K": k, "spec": "tile,bm=16,bn=64,sk=2"}])
    assert r["plan"] == 0 and r["launches"] == [["scaled_tile_kernel", 6, splits]] and (r["workspace"] > 0) == (splits > 1)


@pytest.mark.parametrize("tokens", [1, 4, 5, (1 << 26) - 4, (1 << 26) - 3, (1 << 26) - 1])
def test_every_launch_of_the_routing_has_fewer_than_2_32_threads_along_x(tokens):
    (r,) = ask([{"op": "route", "tokens": tokens, "experts": 8, "k": 1}])
    assert r["plan"] == r["run"] == r["backward"] == 0
    for name, x, y in r["launches"]:
        assert x * 1024 < 1 << 32
    ((name, x, y),) = r["backward_launches"]
    assert x * 256 < 1 << 32 and y < 1 << 16 and tokens <= 4 * x * y < tokens + 8


@pytest.mark.parametrize("question", [
    {"op": "scaled", "M": 64, "N": 512, "K": 8192, "spec": "tile,bm=64,bn=64,sk=8"}, {"op": "route", "tokens": 32, "experts": 64, "k": 4}, {"op": "route", "tokens": 500, "experts": 64, "k": 4},
    {"op": "plan", "M": 64, "N": 512, "K": 8192, "spec": "skinny,sk=8,fr=1"},
], ids=lambda q: "-".join(map(str, q.values())))
def test_a_run_finds_the_counters_of_a_new_plan_cleared(question):
    """They are cleared in the null stream, which other streams do not wait for, and a clearing returns before it has run."""
    (r,) = ask([question])
    assert r["plan"] == r["run"] == 0 and r.get("workspace", 1) > 0 and r["overtaken"] == 0
