"""hack_rope and hack_qk_norm_rope against their definitions in 64 bits."""
import math

import pytest
import torch

from tests import rope_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hb():
    import __graft_entry__ as ge
    ge.build()
    import paper_2504_09261_b200 as pkg
    return pkg


def _gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def _close(out, want, size):
    err = (out.double() - want).abs()
    over = err - ref.bound(want, size, out.dtype)
    assert torch.isfinite(out).all() and over.max() <= 0, (err.max().item(), over.max().item())


CASES = [  # dim, rotary, layout, axes, tokens, heads, batch
    (128, 128, 0, 1, 1, 1, 1), (128, 128, 0, 1, 17, 3, 2), (128, 128, 1, 1, 33, 5, 1), (64, 64, 0, 2, 169, 3, 2),
    (64, 64, 1, 2, 16, 30, 1), (128, 64, 0, 1, 5, 2, 3), (128, 64, 1, 2, 9, 33, 1), (128, 2, 0, 1, 4, 2, 1), (64, 2, 1, 1, 3, 1, 1),
    (64, 36, 0, 1, 40, 4, 1), (128, 124, 0, 2, 31, 7, 2), (64, 4, 0, 2, 8, 1, 1), (128, 6, 1, 1, 2, 1, 5), (64, 62, 1, 1, 50, 2, 2),
    (128, 56, 0, 1, 12, 70, 1), (64, 8, 0, 1, 1000, 2, 1),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,rotary,layout,axes,tokens,heads,batch", CASES)
@pytest.mark.parametrize("transpose", [False, True])
def test_rotation(hb, dtype, dim, rotary, layout, axes, tokens, heads, batch, transpose):
    g = _gen(dim + rotary + tokens)
    x = torch.randn(batch, heads, tokens, dim, generator=g, device="cuda").to(dtype)
    y = torch.full_like(x, float("nan"))
    if axes == 2:
        pos = torch.rand(tokens, 2, generator=g, device="cuda") * 70
    else:
        pos = torch.randint(-500, 1_000_000, (batch, tokens), generator=g, device="cuda", dtype=torch.int32)
    plan = hb.hack_rope_plan(dim, rotary, layout=layout, axes=axes)
    hb.hack_rope(plan, x, y, pos, transpose=transpose)
    f, gain = ref.frequencies(rotary, axes)
    _close(y, *ref.rotate(x, pos, rotary, layout, axes, f, gain, transpose))


@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
@pytest.mark.parametrize("rotary,axes", [(128, 1), (64, 2), (4, 2), (2, 1)])
def test_frequencies_of_long_contexts(hb, scaling, rotary, axes):
    plan = hb.hack_rope_plan(128, rotary, axes=axes, base=500000.0, scaling=scaling, factor=16.0, trained_length=8192)
    f, gain = ref.frequencies(rotary, axes, 500000.0, scaling, 16.0, 8192)
    pairs = rotary // 2 // axes
    for a in range(axes):
        got = torch.tensor(list(plan.freq)[a * pairs:(a + 1) * pairs], dtype=torch.float64)
        assert ((got - f).abs() <= 1e-13 * f).all()
    assert abs(plan.gain - gain) <= 2 ** -24 * gain * 2
    # positions next to the ends of what 32 bits hold
    pos = torch.tensor([0, 1, 2 ** 24 + 1, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    if axes == 2:
        pos = torch.stack([pos, pos.flip(0)], -1).contiguous()
    x = torch.randn(1, 2, 5, 128, generator=_gen(scaling), device="cuda")
    y = torch.empty_like(x)
    hb.hack_rope(plan, x, y, pos)
    # (the reference takes the plan's own frequencies: at 2^31 the last digit of a frequency is 5e-7 of a turn)
    f = torch.tensor(list(plan.freq)[:pairs], dtype=torch.float64)
    _close(y, *ref.rotate(x, pos, rotary, 0, axes, f, plan.gain))


def test_strides_in_place_and_shared_input(hb):
    g = _gen(5)
    plan = hb.hack_rope_plan(64, 64)
    f, gain = ref.frequencies(64, 1)
    pos = torch.arange(20, dtype=torch.int32, device="cuda")
    wide = torch.randn(2, 20, 7, 3 * 64, generator=g, device="cuda").to(torch.bfloat16)
    before = wide.clone()
    x = wide[..., 64:128].transpose(1, 2)                    # rows of 64 out of 192, tokens outside heads
    want, size = ref.rotate(before[..., 64:128].transpose(1, 2), pos, 64, 0, 1, f, gain)
    y = torch.empty(2, 7, 20, 64, dtype=torch.bfloat16, device="cuda")
    hb.hack_rope(plan, x, y, pos)
    _close(y, want, size)
    hb.hack_rope(plan, x, x, pos)                            # in place
    assert torch.equal(x.contiguous(), y)
    assert torch.equal(wide[..., :64], before[..., :64]) and torch.equal(wide[..., 128:], before[..., 128:])
    one = before[:1, ..., :64].transpose(1, 2).expand(3, -1, -1, -1)   # one batch element read three times
    out = torch.empty(3, 7, 20, 64, dtype=torch.bfloat16, device="cuda")
    hb.hack_rope(plan, one, out, pos)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    with pytest.raises(hb.HackError) as e:
        hb.hack_rope(plan, out, one, pos)                    # an output whose rows share memory
    assert e.value.status == 1


def test_what_does_not_turn_passes_bit_for_bit_beside_infinities(hb):
    plan = hb.hack_rope_plan(128, 32)
    x = torch.randn(1, 1, 4, 128, generator=_gen(6), device="cuda")
    x[..., 40] = float("inf")
    x[..., 41] = float("nan")
    y = torch.empty_like(x)
    hb.hack_rope(plan, x, y, torch.arange(4, dtype=torch.int32, device="cuda"))
    assert torch.equal(y[..., 32:].view(torch.int32), x[..., 32:].view(torch.int32))
    assert torch.isfinite(y[..., :32]).all()


def test_gradient_is_the_transpose(hb):
    """Against differences: sum(g * rope(x)) changes by sum(rope_transposed(g) * dx)."""
    gen = _gen(7)
    plan = hb.hack_rope_plan(64, 48, layout=1, scaling=3, factor=4.0, trained_length=1024)
    pos = torch.randint(0, 5000, (2, 11), generator=gen, device="cuda", dtype=torch.int32)
    x, dx, go = (torch.randn(2, 3, 11, 64, generator=gen, device="cuda") for _ in range(3))
    y0, y1, gx = (torch.empty_like(x) for _ in range(3))
    h = 0.5                                                  # (the rotation is linear: any step will do)
    hb.hack_rope(plan, x - h * dx, y0, pos)
    hb.hack_rope(plan, x + h * dx, y1, pos)
    hb.hack_rope(plan, go, gx, pos, transpose=True)
    left = (go.double() * (y1.double() - y0.double())).sum()
    right = (gx.double() * dx.double()).sum()
    # some thirty roundings of 2^-24 per element, of terms of size 4 |go| (|x| + |dx|)
    assert abs(left - right) <= 32 * 2.0 ** -24 * 4 * (go.abs() * (x.abs() + dx.abs())).sum().item()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("dim,rotary,layout,axes,tokens,heads,kv,batch", [
    (128, 128, 0, 2, 1, 16, 16, 2), (64, 64, 1, 2, 169, 30, 30, 3), (128, 64, 0, 1, 33, 8, 2, 1), (64, 20, 0, 1, 7, 5, 1, 2),
    (128, 0, 0, 1, 5, 3, 3, 2), (128, 96, 0, 1, 300, 12, 4, 1)])
def test_norm_rotation_and_layout(hb, dtype, norm, dim, rotary, layout, axes, tokens, heads, kv, batch):
    g = _gen(dim + tokens + norm)
    qkv = (torch.randn(batch, tokens, heads + 2 * kv, dim, generator=g, device="cuda") * 3).to(dtype)
    qkv[0, 0, 0] = 0                                         # a row without length
    q, k, v = (qkv[:, :, a:b].transpose(1, 2) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    outs = [torch.full((batch, n, tokens, dim), float("nan"), dtype=dtype, device="cuda") for n in (heads, kv, kv)]
    qw, kw = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda") for _ in range(2))
    qg = torch.rand(heads, generator=g, device="cuda") * 8 if norm == 2 else None
    kg = torch.rand(kv, generator=g, device="cuda") if norm == 1 else None
    pos = torch.rand(batch, tokens, 2, generator=g, device="cuda") * 64 if axes == 2 else torch.arange(tokens, dtype=torch.int32, device="cuda") + 90000
    plan = hb.hack_rope_plan(dim, rotary, layout=layout, axes=axes) if rotary else None
    hb.hack_qk_norm_rope(plan, q, k, v, *outs, pos if rotary else None, norm=norm, eps=1e-6, q_weight=qw, k_weight=kw, q_gain=qg, k_gain=kg)
    for x, out, w, gain in ((q, outs[0], qw, qg), (k, outs[1], kw, kg)):
        y = ref.normalise(x, norm, 1e-6, w, gain)
        if rotary:
            f, cs = ref.frequencies(rotary, axes)
            _close(out, *ref.rotate(y, pos, rotary, layout, axes, f, cs))
        else:
            _close(out, y, y.abs())
    assert torch.equal(outs[2], v)


def test_parts_may_be_left_out_and_bits_do_not_depend_on_the_batch(hb):
    g = _gen(9)
    plan = hb.hack_rope_plan(128)
    q = torch.randn(3, 6, 21, 128, generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.arange(21, dtype=torch.int32, device="cuda")
    both, alone = torch.empty_like(q), torch.empty_like(q)
    hb.hack_qk_norm_rope(plan, q, q, None, both, torch.empty_like(q), None, pos, norm=hb.HACK_NORM_L2)
    for b in range(3):
        hb.hack_qk_norm_rope(plan, q[b:b + 1], None, None, alone[b:b + 1], None, None, pos, norm=hb.HACK_NORM_L2)
    assert torch.equal(both, alone)
    hb.hack_rope(plan, q[:, :, :0], alone[:, :, :0], pos[:0])          # nothing to do
    assert torch.equal(both, alone)


def test_stream_and_graph(hb):
    plan = hb.hack_rope_plan(64, layout=1)
    x = torch.randn(2, 4, 9, 64, generator=_gen(11), device="cuda")
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    want, y = torch.empty_like(x), torch.zeros_like(x)
    hb.hack_rope(plan, x, want, pos)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hb.hack_rope(plan, x, y, pos, stream=torch.cuda.current_stream().cuda_stream)
    assert not torch.equal(want, y)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(want, y)
    x.mul_(2)                                                          # other values, other positions, the same graph
    pos.add_(100)
    graph.replay()
    hb.hack_rope(plan, x, want, pos, stream=torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(want, y)
