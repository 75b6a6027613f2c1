"""Values and sizes at the edges of the operators around the cache, against their definitions in 64 bits."""
import pytest
import torch

from tests import rope_reference as rope_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    import __graft_entry__ as ge
    ge.build()
    import paper_2504_09261_b200 as pkg
    return pkg


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ norms and rotation
def _same_numbers(out, want, size):
    """NaN where the definition has NaN, the same infinities, and everything else within the bound of roundings."""
    out, finite = out.double(), torch.isfinite(want)
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    infinite = torch.isinf(want)
    assert torch.equal(out[infinite], want[infinite])
    return ((out - want).abs() - size)[finite]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("dim,rotary,layout", [(128, 128, 0), (64, 32, 1), (64, 20, 0), (128, 0, 0)])
def test_rows_with_no_numbers_and_infinities(hb, dtype, norm, dim, rotary, layout):
    """A NaN or an infinity in a row is in the result what the definition makes of it, and the rows beside it do not see it."""
    g = _gen(dim + norm)
    b, h, n = 2, 5, 9
    x = torch.randn(b, h, n, dim, generator=g, device="cuda").to(dtype)
    x[0, 1, 3, 5] = float("nan")
    x[0, 2, 4, dim - 1] = float("nan")
    x[1, 0, 0, 7] = float("inf")
    x[1, 4, 8, 0] = -float("inf")
    x[1, 3, 2] = 0                                           # a row without length beside them
    out = torch.empty_like(x)
    weight = 1 + 0.3 * torch.rand(dim, generator=g, device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") + 3
    plan = hb.hack_rope_plan(dim, rotary, layout=layout) if rotary else None
    hb.hack_qk_norm_rope(plan, x, None, None, out, None, None, pos if rotary else None, norm=norm, eps=1e-6, q_weight=weight)
    want = rope_ref.normalise(x, norm, 1e-6, weight)
    size = want.abs()
    if rotary:
        want, size = rope_ref.rotate(want, pos, rotary, layout, 1, *rope_ref.frequencies(rotary, 1))
    assert _same_numbers(out, want, rope_ref.bound(want, size, dtype)).max() <= 0


# ------------------------------------------------------------------ attention over 4 bits
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,kv_heads,group,tokens,length", [(64, 32, 1, 1, 4096), (64, 32, 7, 1, 4096), (64, 16, 13, 1, 3000), (64, 2, 3, 5, 900),
                                                              (128, 32, 1, 1, 4096), (128, 3, 5, 3, 1000)])
def test_clusters_whose_warps_have_rows_for_some_of_their_threads(hb, dtype, dim, kv_heads, group, tokens, length):
    """At head_dim 64 half a warp adds up a row: with an odd number of rows the other half is done first."""
    from tests.test_gpu_kv4 import Planes, _check
    kv4 = Planes(1, dim)
    kv4 = hb.HackKv4(*(t.expand(kv_heads * length, -1).contiguous() for t in kv4.all()), batch=1, n_kv_heads=kv_heads, cap=length)
    q = torch.empty(1, kv_heads * group, tokens, dim, dtype=dtype, device="cuda")
    # no workspace: one launch, in clusters (a single CTA for so many rows takes two to three times as long as a few)
    assert kv4.hack_kv4_workspace(q, length) == 0
    _check(hb, _gen(group), dtype, dim, 1, kv_heads, group, tokens, length, [length] + [length * i // kv_heads for i in range(1, kv_heads)])


@pytest.mark.parametrize("kv_heads,group,tokens,cap", [(1, 1, 129, 300), (2, 3, 43, 1500), (1, 1, 1, 700), (150, 1, 255, 131)])
def test_tiles_whose_warps_have_rows_for_some_of_their_threads(hb, kv_heads, group, tokens, cap):
    """Tiles of 128 query rows of which one, 127 or a few in a warp are there, head_dim 128 (the output leaves in two halves), with the
    blocks of a unit on one CTA and shared."""
    from tests.test_gpu_kv4 import _check
    _check(hb, _gen(cap), torch.bfloat16, 128, 1, kv_heads, group, tokens, cap, [cap] + [cap * i // kv_heads for i in range(1, kv_heads)], form=2)


# ------------------------------------------------------------------ a layer's rows
def test_launches_are_counted_as_they_are_made(hb):
    from tests.parity_util import make_cache
    from tests.test_gpu_kv4 import Planes
    from workloads import SyntheticQKV, get_config
    cfg = get_config(1, n_layers=1)
    cache = make_cache(cfg, SyntheticQKV(cfg).head_is_contextual.numpy())
    b, h, d = cfg.batch, cfg.n_heads, cfg.head_dim
    planes = Planes(b * h * 4, d)
    kv4, lens = planes.handle(hb, b, h, 4), torch.zeros(b * h, dtype=torch.int32, device="cuda")
    cache.hack_store_kv4(0, kv4, lens)                       # a layer without rows: nothing to launch
    assert cache.hack_launch_count() == 0
    assert all((p == 0x5a).all() for p in planes.all())
    q = torch.randn(b, h, 1, d, generator=_gen(2), device="cuda").to(torch.bfloat16)
    out, pos = torch.empty_like(q), _ints(0)
    cache.hack_scale_step_qkv(0, 0, hb.hack_rope_plan(d), q, q, q, out, pos)
    steps = cache.hack_launch_count()
    cache.hack_store_kv4(0, kv4, lens)
    assert steps >= 2 and cache.hack_launch_count() == steps + 1
    cache.close()
