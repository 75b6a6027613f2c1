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


# ------------------------------------------------------------------ which form serves a call
@pytest.mark.parametrize("dim,heads,tokens,cap,many", [(128, 16, 32, 10521, False), (128, 16, 64, 10521, True), (128, 64, 64, 2240, True),
                                                       (64, 4, 64, 700, False), (128, 16, 1024, 64, True), (64, 256, 256, 680, True)])
def test_the_form_that_was_faster(hb, dim, heads, tokens, cap, many):
    """At sizes timed in both forms.  They add up in different orders, so that some of a call's many results differ in a bit: the
    library's own choice has all the bits of one of them."""
    from tests.test_gpu_kv4 import Planes
    g = _gen(heads + tokens)
    planes = Planes(heads * cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, heads, cap)
    q = torch.randn(1, heads, tokens, dim, generator=g, device="cuda").to(torch.bfloat16)
    lens, outs = _ints(*([cap] * heads)), []
    for form in (0, hb.HACK_KV4_FEW, hb.HACK_KV4_MANY):
        work = torch.empty(kv4.hack_kv4_workspace(q, cap, form=form), dtype=torch.uint8, device="cuda")
        outs.append(torch.empty_like(q))
        kv4.hack_kv4_attend(q, outs[-1], lens, cap, workspace=work, form=form)
    assert not torch.equal(outs[1], outs[2])
    assert torch.equal(outs[0], outs[2 if many else 1])
    kv4.hack_kv4_poll_status()


# ------------------------------------------------------------------ queries that are no numbers
@pytest.mark.parametrize("dtype,form", [(torch.float32, 1), (torch.bfloat16, 1), (torch.bfloat16, 2)])
@pytest.mark.parametrize("dim,tokens,length", [(64, 5, 300), (128, 3, 1000), (64, 150, 200), (128, 140, 90)])
def test_queries_with_no_numbers_and_infinities(hb, dtype, form, dim, tokens, length):
    """A query with a NaN has NaN for its result, and zeros where it sees no row at all; the queries beside it, in the same tile and the
    same warp, are what they would be without it."""
    from tests import kv4_reference as ref
    from tests.test_gpu_kv4 import Planes
    g, group = _gen(tokens + dim), 2
    planes = Planes(length, dim)
    planes.randomise(g)
    # no element of a key is 0: an infinity in a query gives logits of both signs, of which one is certain to be +inf
    planes.k_codes[planes.k_codes & 15 == 8] += 1
    planes.k_codes[planes.k_codes >> 4 == 8] += 16
    kv4 = planes.handle(hb, 1, 1, length)
    q = torch.randn(1, group, tokens, dim, generator=g, device="cuda").to(dtype)
    q[0, 0, 1, 3], q[0, 1, tokens - 1, dim - 1], q[0, 1, 0, 5] = float("nan"), float("inf"), float("nan")
    bad = torch.zeros(group, tokens, dtype=torch.bool, device="cuda")
    bad[0, 1] = bad[1, tokens - 1] = bad[1, 0] = True
    for causal, rows in ((False, length), (True, length), (True, tokens - 1)):      # the last: the first query of all sees nothing
        rows = min(rows, length)
        out = torch.full_like(q, 77.0)
        work = torch.empty(kv4.hack_kv4_workspace(q, length, causal=causal, form=form), dtype=torch.uint8, device="cuda")
        kv4.hack_kv4_attend(q, out, _ints(rows), length, workspace=work, causal=causal, form=form)
        want = ref.attend(q[0].masked_fill(bad[..., None], 0), ref.values(planes.k_codes, planes.k_scales),
                          ref.values(planes.v_codes, planes.v_scales), rows, tokens, dim ** -0.5, causal)
        sees = torch.ones(tokens, dtype=torch.bool, device="cuda")
        if causal:
            sees = torch.arange(tokens, device="cuda") + rows - tokens >= 0
        assert torch.isnan(out[0][bad & sees]).all()
        assert (out[0][:, ~sees] == 0).all()
        over = (out[0].double() - want[0]).abs() - ref.bound(*want, dtype, dim, rows)
        assert over[~bad].max() <= 0
    kv4.hack_kv4_poll_status()


# ------------------------------------------------------------------ windows of few queries
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens,group", [(1, 1), (5, 2), (33, 1)])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (7, 4), (32, 0), (33, 40), (100, 3), (1000, 5)])
@pytest.mark.parametrize("causal", [True, False])
def test_windows_of_few_queries(hb, dtype, tokens, group, window, n_sink, causal):
    from tests.test_gpu_kv4 import _check
    _check(hb, _gen(window), dtype, 128, 1, 3, group, tokens, 400, [400, 190, 12], causal=causal, window=window, n_sink=n_sink, form=1)


# ------------------------------------------------------------------ calls that the header allows
@pytest.mark.parametrize("dtype,form,tokens,cap", [(torch.float32, 1, 1, 60000), (torch.float32, 1, 40, 3000), (torch.bfloat16, 1, 1, 60000), (torch.bfloat16, 1, 7, 2000),
                                                   (torch.bfloat16, 2, 300, 200), (torch.bfloat16, 2, 130, 9000)])
def test_attention_in_place(hb, dtype, form, tokens, cap):
    """The output is the queries' own tensor, with one CTA to a tile, a cluster, and partial results."""
    from tests.test_gpu_kv4 import Planes
    g, heads, dim = _gen(tokens), 2, 64
    planes = Planes(heads * cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, heads, cap)
    q = torch.randn(1, heads * 3, tokens, dim, generator=g, device="cuda").to(dtype)
    out, lens = torch.empty_like(q), _ints(cap, cap // 2)
    work = torch.empty(kv4.hack_kv4_workspace(q, cap, form=form), dtype=torch.uint8, device="cuda")
    kv4.hack_kv4_attend(q, out, lens, cap, workspace=work, form=form)
    kv4.hack_kv4_attend(q, q, lens, cap, workspace=work, form=form)
    assert torch.equal(q, out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_and_rotation_in_place(hb, dtype):
    """All three parts where they lie in the projection's output."""
    g = _gen(17)
    qkv = torch.randn(2, 19, 8 + 2 * 2, 128, generator=g, device="cuda").to(dtype)
    parts = lambda x: [x[:, :, a:b].transpose(1, 2) for a, b in ((0, 8), (8, 10), (10, 12))]   # noqa: E731
    plan, pos = hb.hack_rope_plan(128, 96), torch.arange(19, dtype=torch.int32, device="cuda")
    outs = [torch.empty(x.shape, dtype=dtype, device="cuda") for x in parts(qkv)]
    hb.hack_qk_norm_rope(plan, *parts(qkv), *outs, pos)
    before = qkv.clone()
    hb.hack_qk_norm_rope(plan, *parts(qkv), *parts(qkv), pos)
    assert all(torch.equal(x, y) for x, y in zip(parts(qkv), outs))
    assert torch.equal(qkv[:, :, 10:], before[:, :, 10:])


def test_threads_on_streams_of_their_own(hb):
    """Calls of several threads at once, each of sizes that the binding has not seen and of sizes that it has."""
    import threading
    plan, wrong = hb.hack_rope_plan(64), []
    f = rope_ref.frequencies(64, 1)

    def work(i):
        try:
            stream, g = torch.cuda.Stream(), _gen(i)
            with torch.cuda.stream(stream):
                for r in range(60):
                    n = 1 + (7 * r + i) % 25
                    x = torch.randn(1, 3, n, 64, generator=g, device="cuda")
                    y, pos = torch.empty_like(x), torch.arange(n, dtype=torch.int32, device="cuda")
                    hb.hack_rope(plan, x, y, pos, stream=stream.cuda_stream)
                    want, size = rope_ref.rotate(x, pos, 64, 0, 1, *f)
                    assert ((y.double() - want).abs() <= rope_ref.bound(want, size, x.dtype)).all()
        except Exception as e:                               # noqa: BLE001  (told to the test's own thread)
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong, wrong
