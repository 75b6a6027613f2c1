"""Caches of 4 bits: rows into them and back, and the attention over them, against the definitions in 64 bits."""
import math

import pytest
import torch

from tests import kv4_reference as ref

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


class Planes:
    """Planes of `rows` rows, filled with a pattern."""

    def __init__(self, rows, dim, fill=0x5a):
        self.k_codes, self.v_codes = (torch.full((rows, dim // 2), fill, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.k_scales, self.v_scales = (torch.full((rows, dim // 16), fill, dtype=torch.uint8, device="cuda") for _ in range(2))

    def all(self):
        return self.k_codes, self.k_scales, self.v_codes, self.v_scales

    def handle(self, hb, batch, heads, cap, row_off=None):
        return hb.HackKv4(*self.all(), batch=batch, n_kv_heads=heads, cap=cap, row_off=row_off)

    def randomise(self, g, spread=4):
        """Any codes from -7 to 7, scales around 1 / 4: stored rows of all sizes."""
        for c in (self.k_codes, self.v_codes):
            x = torch.randint(1, 16, c.shape + (2,), generator=g, device="cuda", dtype=torch.uint8)
            c.copy_(x[..., 0] | (x[..., 1] << 4))
        for s in (self.k_scales, self.v_scales):
            s.copy_(torch.randint(8 * 18 - spread, 8 * 18 + spread, s.shape, generator=g, device="cuda"))


# ------------------------------------------------------------------ rows in and out
def _rows_with_edges(g, dtype, *shape):
    x = torch.randn(*shape, generator=g, device="cuda") * torch.exp(torch.randn(*shape[:-1], 1, generator=g, device="cuda") * 3)
    flat = x.view(-1, 16)
    n = flat.shape[0]
    flat[0] = 0
    flat[1 % n] = torch.arange(16, device="cuda") - 7.5                       # halves: ties for a scale of 1
    flat[1 % n][0] = 7.0
    flat[2 % n] = 1e-30
    flat[3 % n] = 3e4
    flat[4 % n, 3], flat[4 % n, 5] = float("inf"), float("-inf")
    flat[5 % n, 0] = float("nan")
    flat[6 % n] = 7 * 0.171875 * torch.sign(flat[6 % n])                      # the largest of a block is 7 scales exactly
    if n > 7:
        flat[7] = 7 * 0.171875 * (1 + 2.0 ** -7)                              # and one bf16 step above
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim,batch,heads,tokens,cap", [(64, 1, 1, 1, 1), (128, 2, 3, 5, 20), (64, 3, 7, 169, 400), (128, 1, 2, 1025, 1300)])
def test_append_and_read(hb, dtype, dim, batch, heads, tokens, cap):
    g = _gen(dim + tokens)
    k, v = (_rows_with_edges(g, dtype, batch, heads, tokens, dim) for _ in range(2))
    lens = (torch.arange(batch * heads, device="cuda") * 13 % (cap - tokens + 1)).to(torch.int32)
    planes = Planes(batch * heads * cap, dim)
    kv4 = planes.handle(hb, batch, heads, cap)
    kv4.hack_kv4_append(k, v, lens)
    back = [torch.full_like(k, float("nan")) for _ in range(2)]
    kv4.hack_kv4_read(*back, lens)
    where = torch.arange(batch * heads, device="cuda")[:, None] * cap + lens[:, None] + torch.arange(tokens, device="cuda")
    untouched = torch.ones(batch * heads * cap, dtype=torch.bool, device="cuda")
    untouched[where.flatten()] = False
    for x, codes, scales, out in ((k, planes.k_codes, planes.k_scales, back[0]), (v, planes.v_codes, planes.v_scales, back[1])):
        c, byte, value = ref.quantise(x)
        assert torch.equal(codes[where].view(batch, heads, tokens, -1), ref.pack(c))
        assert torch.equal(scales[where].view(batch, heads, tokens, -1).long(), byte)
        assert torch.equal(out.double(), value)
        assert (codes[untouched] == 0x5a).all() and (scales[untouched] == 0x5a).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values_between_codes(hb, dtype):
    """Multiples of half a scale and their neighbours, for every mantissa of a scale: nearest code, ties to the even one."""
    m = torch.arange(8, dtype=torch.float64)
    s = ((8 + m) / 8)[:, None] * 2.0 ** torch.tensor([-12.0, -3, 0, 5])[None, :].double()
    half = torch.arange(-15, 17, dtype=torch.float64) / 2
    x = (s.flatten()[:, None] * half).to(torch.float32)
    x = torch.cat([x, torch.nextafter(x, torch.full_like(x, math.inf)), torch.nextafter(x, torch.full_like(x, -math.inf))]).to(dtype)
    x = torch.where(x.abs() > (7 * s.flatten().repeat(3))[:, None], torch.zeros_like(x), x)
    x[:, 0], x[:, 16] = (7 * s.flatten().repeat(3)).to(dtype), (7 * s.flatten().repeat(3)).to(dtype)
    x = torch.cat([x, x], 1)[None, None].cuda().contiguous()                  # rows of 64
    kv4 = Planes(x.shape[2], 64).handle(hb, 1, 1, x.shape[2])
    kv4.hack_kv4_append(x, -x, _ints(0))
    k, v = torch.empty_like(x), torch.empty_like(x)
    kv4.hack_kv4_read(k, v, _ints(0))
    assert torch.equal(k.double(), ref.quantise(x)[2])
    assert torch.equal(v.double(), ref.quantise(-x)[2])


def test_append_strided_padded_and_full(hb):
    g = _gen(3)
    batch, heads, tokens, dim, cap = 3, 2, 6, 64, 10
    wide = torch.randn(batch, tokens, heads, 4 * dim, generator=g, device="cuda").to(torch.bfloat16)
    k, v = wide[..., dim:2 * dim].transpose(1, 2), wide[..., 3 * dim:].transpose(1, 2)
    # heads in another order, with rows between them that belong to nobody
    row_off = torch.tensor([70, 1, 23, 35, 47, 59], dtype=torch.int64, device="cuda")
    lens = _ints(0, 7, -5, 10, 2 ** 31 - 1, 3)
    planes = Planes(82, dim)
    kv4 = planes.handle(hb, batch, heads, cap, row_off)
    kv4.hack_kv4_append(k, v, lens, new_lens=_ints(6, 4, 0))
    written = torch.zeros(82, dtype=torch.bool)
    for i, (start, n) in enumerate(((0, 6), (7, 3), (0, 4), (10, 0), (10, 0), (3, 0))):   # what fits of what each batch element has
        b, h = divmod(i, heads)
        for x, codes in ((k, planes.k_codes), (v, planes.v_codes)):
            assert torch.equal(codes[row_off[i] + start:row_off[i] + start + n], ref.pack(ref.quantise(x[b, h, :n])[0]))
        written[int(row_off[i]) + start:int(row_off[i]) + start + n] = True
    for p in planes.all():
        assert (p[~written] == 0x5a).all()
    # rows outside a head's own read as zeros
    out = [torch.full((batch, heads, 4, dim), float("nan"), device="cuda") for _ in range(2)]
    kv4.hack_kv4_read(*out, _ints(-2, 8, 100, -2 ** 31, 2 ** 31 - 1, 0))
    assert (out[0][0, 0, :2] == 0).all() and torch.equal(out[0][0, 0, 2:].double(), ref.quantise(k[0, 0, :2])[2])
    assert (out[0][0, 1, 2:] == 0).all() and torch.equal(out[1][0, 1, :2].double(), ref.quantise(v[0, 1, 1:3])[2])
    assert (out[0][1] == 0).all() and (out[1][2, 0] == 0).all() and torch.isfinite(out[0]).all()


def test_heads_outside_the_planes_have_no_rows(hb):
    g = _gen(33)
    heads, dim, cap, rows = 4, 64, 20, 60
    planes = Planes(rows, dim)
    planes.randomise(g)
    before = [p.clone() for p in planes.all()]
    row_off = torch.tensor([40, 41, -1, 2 ** 62], dtype=torch.int64, device="cuda")
    kv4 = planes.handle(hb, 1, heads, cap, row_off)
    k = torch.randn(1, heads, 3, dim, generator=g, device="cuda")
    kv4.hack_kv4_append(k, k, _ints(0, 0, 0, 0))
    back = [torch.full_like(k, 9.0) for _ in range(2)]
    kv4.hack_kv4_read(*back, _ints(0, 0, 0, 0))
    assert torch.equal(back[0][0, 0].double(), ref.quantise(k[0, 0])[2]) and (back[0][0, 1:] == 0).all() and (back[1][0, 1:] == 0).all()
    for p, b in zip(planes.all(), before):
        assert torch.equal(p[:40], b[:40]) and torch.equal(p[43:], b[43:])
    for dtype, form in ((torch.float32, 1), (torch.bfloat16, 1), (torch.bfloat16, 2)):
        q = torch.randn(1, heads, 5, dim, generator=g, device="cuda").to(dtype)
        out = torch.full_like(q, 9.0)
        kv4.hack_kv4_attend(q, out, _ints(3, 20, 20, 20), cap, workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"), form=form)
        want = ref.attend(q[0, :1], ref.quantise(k[0, 0])[2], ref.quantise(k[0, 0])[2], 3, 5, dim ** -0.5)
        assert ((out[0, :1].double() - want[0]).abs() <= ref.bound(*want, dtype, dim, 3)).all() and (out[0, 1:] == 0).all()


# ------------------------------------------------------------------ attention
def _check(hb, g, dtype, dim, batch, kv_heads, group, tokens, cap, lens, max_len=None, causal=False, window=0, n_sink=0, new_lens=None,
           appended=False, sm_scale=0.0, row_off=None, rows=None, q_layout="token", q_size=1.0, planes=None, form=0):
    rows = rows or batch * kv_heads * cap
    if planes is None:
        planes = Planes(rows, dim)
        planes.randomise(g)
    kv4 = planes.handle(hb, batch, kv_heads, cap, row_off)
    heads = kv_heads * group
    q = (torch.randn(batch, tokens, heads, dim, generator=g, device="cuda") * q_size).to(dtype)
    out = torch.full((batch, tokens, heads, dim), 77.0, dtype=dtype, device="cuda")
    q, out = (x.transpose(1, 2) if q_layout == "token" else x.transpose(1, 2).contiguous() for x in (q, out))
    max_len = cap if max_len is None else max_len
    lens_dev = _ints(*lens)
    new_dev = None if new_lens is None else _ints(*new_lens)
    need = kv4.hack_kv4_workspace(q, max_len, causal=causal, n_sink=n_sink, window=window, appended=appended, form=form)
    work = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")          # NaN for whoever reads what nobody wrote
    call = lambda: kv4.hack_kv4_attend(q, out, lens_dev, max_len, workspace=work[:need], new_lens=new_dev, appended=appended,   # noqa: E731
                                       causal=causal, n_sink=n_sink, window=window, sm_scale=sm_scale, form=form)
    call()
    first = out.clone()
    call()
    assert torch.equal(first, out)                                                    # the same bits every time
    assert (work[need:] == 0xff).all()
    scale = sm_scale or dim ** -0.5
    for i in range(batch * kv_heads):
        b, h = divmod(i, kv_heads)
        nq = tokens if new_lens is None else min(max(new_lens[b], 0), tokens)
        length = min(max(lens[i], 0) + (nq if appended else 0), max_len, cap)
        start = i * cap if row_off is None else int(row_off[i])
        k, v = (ref.values(c[start:start + cap], s[start:start + cap]) for c, s in ((planes.k_codes, planes.k_scales), (planes.v_codes, planes.v_scales)))
        want = ref.attend(q[b, h * group:(h + 1) * group], k, v, length, nq, scale, causal, window, n_sink)
        got = out[b, h * group:(h + 1) * group]
        assert torch.isfinite(got).all()
        over = (got[:, :nq].double() - want[0]).abs() - ref.bound(*want, dtype, dim, length)
        assert nq == 0 or over.max() <= 0, (i, length, over.max().item(), (got[:, :nq].double() - want[0]).abs().max().item())
        assert (got[:, nq:] == 77.0).all()
    return out


SHAPES = [  # dim, batch, kv_heads, group, tokens, cap
    (64, 1, 1, 1, 1, 1), (128, 1, 1, 1, 1, 33), (128, 2, 3, 1, 1, 700), (64, 1, 2, 4, 1, 3000), (128, 1, 2, 8, 1, 5000),
    (64, 3, 5, 3, 13, 300), (128, 1, 2, 1, 16, 257), (128, 1, 1, 2, 17, 128), (64, 2, 2, 1, 31, 95), (128, 1, 1, 1, 9, 20000),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim,batch,kv_heads,group,tokens,cap", SHAPES)
def test_attend_few_queries(hb, dtype, causal, dim, batch, kv_heads, group, tokens, cap):
    n = batch * kv_heads
    lens = [cap] + [(i * 101) % (cap + 1) for i in range(1, n)]
    _check(hb, _gen(cap), dtype, dim, batch, kv_heads, group, tokens, cap, lens, causal=causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("length", [0, 1, 2, 15, 16, 31, 32, 33, 64, 65, 127, 128, 129, 255, 257])
def test_attend_lengths(hb, dtype, length):
    _check(hb, _gen(length), dtype, 128, 1, 2, 2, 3, 300, [length, 300 - length], causal=True)
    _check(hb, _gen(length + 1), dtype, 64, 1, 2, 1, 40, 300, [length, 300 - length], causal=True)   # more queries than rows


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 5, 50])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (7, 4), (32, 0), (33, 40), (100, 3), (1000, 5)])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_window_and_first_rows(hb, dtype, tokens, window, n_sink, causal):
    _check(hb, _gen(window), dtype, 64, 1, 3, 2, tokens, 400, [400, 190, 12], causal=causal, window=window, n_sink=n_sink)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attend_padded_batch_and_limits(hb, dtype):
    g = _gen(21)
    # lengths before the append, queries that a batch element does not have, lengths out of range
    _check(hb, g, dtype, 128, 3, 2, 2, 6, 100, [10, 94, 50, 99, 0, 7], new_lens=[6, 3, 0], appended=True, causal=True)
    _check(hb, g, dtype, 64, 2, 2, 1, 4, 50, [-3, 2 ** 31 - 1, 50, 0], new_lens=[-1, 9], appended=True, causal=True)
    _check(hb, g, dtype, 64, 2, 2, 1, 4, 50, [2 ** 31 - 1, -2 ** 31, 49, 1], max_len=30)
    _check(hb, g, dtype, 64, 1, 1, 1, 4, 50, [20], max_len=0)
    _check(hb, g, dtype, 128, 1, 3, 1, 2, 40, [40, 3, 21], row_off=torch.tensor([81, 0, 40], dtype=torch.int64, device="cuda"), rows=122, q_layout="head")
    _check(hb, g, dtype, 128, 1, 3, 1, 2, 40, [40, 3, 21], sm_scale=2.5, q_size=3.0)


@pytest.mark.parametrize("dtype,form", [(torch.float32, 0), (torch.bfloat16, 1), (torch.bfloat16, 2)])
def test_attend_windows_past_every_position(hb, dtype, form):
    for window, n_sink in ((2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1)):
        _check(hb, _gen(30), dtype, 64, 1, 2, 1, 60, 200, [200, 30], causal=True, window=window, n_sink=n_sink, form=form)


def test_attend_equal_and_dominant_logits(hb):
    """All logits equal: the mean of the values.  One far above the others: that value, although the maximum comes last."""
    dim, cap = 64, 500
    planes = Planes(cap, dim)
    planes.randomise(_gen(4))
    planes.k_codes.fill_(0x88)                                    # zeros
    _check(hb, _gen(5), torch.bfloat16, dim, 1, 1, 1, 2, cap, [cap], planes=planes)
    planes.k_codes[cap - 1] = 0xff
    planes.k_scales[cap - 1] = 8 * 24
    _check(hb, _gen(6), torch.bfloat16, dim, 1, 1, 1, 5, cap, [cap], planes=planes, q_size=4.0)
    _check(hb, _gen(7), torch.float32, dim, 1, 1, 1, 5, cap, [cap], planes=planes, q_size=4.0)


def test_long_cache_past_32_bits_of_bytes(hb):
    """The last head's rows lie more than 2^32 bytes into the code planes."""
    dim, cap, heads = 128, 17_000_000, 4
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 12 GB")
    planes = Planes(1, dim)
    rows = heads * cap
    planes.k_codes, planes.v_codes = (torch.empty((rows, dim // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    planes.k_scales, planes.v_scales = (torch.empty((rows, dim // 16), dtype=torch.uint8, device="cuda") for _ in range(2))
    g = _gen(8)
    kv4 = planes.handle(hb, 1, heads, cap)
    k, v = (torch.randn(1, heads, 70, dim, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lens = _ints(0, 5, cap - 70, cap - 70)
    kv4.hack_kv4_append(k, v, lens)
    back = [torch.empty_like(k) for _ in range(2)]
    kv4.hack_kv4_read(*back, lens)
    assert torch.equal(back[0].double(), ref.quantise(k)[2]) and torch.equal(back[1].double(), ref.quantise(v)[2])
    # the last 70 rows of the last two heads, through a window that ends at their length
    q = torch.randn(1, heads, 1, dim, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    need = kv4.hack_kv4_workspace(q, cap, causal=True, window=70)
    kv4.hack_kv4_attend(q, out, lens + 70, cap, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), causal=True, window=70)
    for h in (2, 3):
        want = ref.attend(q[0, h:h + 1], *(ref.quantise(x[0, h])[2] for x in (k, v)), 70, 1, dim ** -0.5)
        assert ((out[0, h].double() - want[0][0]).abs() <= ref.bound(*want, torch.bfloat16, dim, 70)[0]).all()


def test_graph_replayed_with_other_lengths(hb):
    g = _gen(12)
    dim, cap = 128, 600
    planes = Planes(2 * cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, 2, cap)
    q = torch.randn(1, 4, 1, dim, generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(1, 2, 1, dim, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    out = torch.empty_like(q)
    lens = _ints(100, 37)
    need = kv4.hack_kv4_workspace(q, cap, causal=True, appended=True)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step(out, stream):
        kv4.hack_kv4_append(k, v, lens, stream=stream)
        kv4.hack_kv4_attend(q, out, lens, cap, workspace=work, causal=True, appended=True, stream=stream)

    step(out, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, torch.cuda.current_stream().cuda_stream)
        lens.add_(1)
    for _ in range(3):
        before = lens.clone()
        graph.replay()
        torch.cuda.synchronize()
        for h in range(2):
            n = int(before[h]) + 1
            kd, vd = (ref.values(c[h * cap:h * cap + n], s[h * cap:h * cap + n]) for c, s in ((planes.k_codes, planes.k_scales), (planes.v_codes, planes.v_scales)))
            want = ref.attend(q[0, 2 * h:2 * h + 2], kd, vd, n, 1, dim ** -0.5)
            assert ((out[0, 2 * h:2 * h + 2].double() - want[0]).abs() <= ref.bound(*want, torch.bfloat16, dim, n)).all()
        q.add_(0.125)
        k.mul_(-1)


def test_two_streams_with_workspaces_of_their_own(hb):
    g = _gen(13)
    dim, cap = 64, 60000
    planes = Planes(2 * cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, 2, cap)
    q = torch.randn(1, 2, 1, dim, generator=g, device="cuda").to(torch.bfloat16)
    need = kv4.hack_kv4_workspace(q, cap)
    assert need > 0                                               # (several CTAs share a head)
    lens = _ints(cap, cap - 1)
    alone = torch.empty_like(q)
    kv4.hack_kv4_attend(q, alone, lens, cap, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    works = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, w in zip(streams, outs, works):
            kv4.hack_kv4_attend(q, o, lens, cap, workspace=w, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], alone) and torch.equal(outs[1], alone)


# ------------------------------------------------------------------ many queries: tiles of 128 rows on the tensor cores
MANY = [  # dim, batch, kv_heads, group, tokens, cap
    (128, 1, 1, 1, 48, 100), (64, 1, 1, 1, 128, 128), (128, 1, 2, 1, 129, 300), (64, 2, 3, 3, 43, 257), (128, 1, 1, 4, 100, 1000),
    (64, 1, 2, 1, 513, 640), (128, 3, 2, 2, 65, 40), (64, 1, 1, 1, 300, 5000), (128, 1, 1, 8, 60, 9000), (128, 2, 80, 1, 130, 200),
    (64, 2, 80, 1, 257, 131),
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim,batch,kv_heads,group,tokens,cap", MANY)
@pytest.mark.parametrize("form", [1, 2])
def test_attend_many_queries(hb, form, causal, dim, batch, kv_heads, group, tokens, cap):
    n = batch * kv_heads
    lens = [cap] + [(i * 101) % (cap + 1) for i in range(1, n)]
    _check(hb, _gen(cap), torch.bfloat16, dim, batch, kv_heads, group, tokens, cap, lens, causal=causal, form=form)


@pytest.mark.parametrize("length", [0, 1, 31, 32, 33, 127, 128, 129, 255, 256, 257, 384, 511])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_many_queries_lengths(hb, dim, length):
    _check(hb, _gen(length), torch.bfloat16, dim, 1, 2, 1, 140, 512, [length, 512 - length], causal=dim == 64, form=2)
    _check(hb, _gen(length), torch.bfloat16, dim, 1, 2, 3, 100, 512, [length, 512 - length], causal=dim == 128, form=2)


@pytest.mark.parametrize("tokens", [60, 200])
@pytest.mark.parametrize("window,n_sink", [(1, 0), (1, 1), (7, 4), (128, 0), (100, 140), (300, 3), (1000, 5)])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_many_queries_window(hb, tokens, window, n_sink, causal):
    _check(hb, _gen(window), torch.bfloat16, 64, 1, 3, 2, tokens, 700, [700, 190, 12], causal=causal, window=window, n_sink=n_sink, form=2)
    _check(hb, _gen(window), torch.bfloat16, 128, 1, 1, 1, tokens, 700, [611], causal=causal, window=window, n_sink=n_sink, form=2)


def test_attend_many_queries_padded_and_limits(hb):
    g, dt = _gen(22), torch.bfloat16
    kw = dict(form=2)
    _check(hb, g, dt, 128, 3, 2, 2, 150, 400, [10, 94, 50, 99, 0, 7], new_lens=[150, 70, 0], appended=True, causal=True, **kw)
    _check(hb, g, dt, 64, 2, 2, 1, 300, 500, [-3, 2 ** 31 - 1, 50, 0], new_lens=[-1, 900], appended=True, causal=True, **kw)
    _check(hb, g, dt, 64, 2, 2, 1, 64, 500, [2 ** 31 - 1, -2 ** 31, 49, 1], max_len=300, **kw)
    _check(hb, g, dt, 64, 1, 1, 1, 64, 50, [20], max_len=0, **kw)
    _check(hb, g, dt, 128, 1, 3, 1, 70, 140, [140, 3, 121], row_off=torch.tensor([281, 0, 140], dtype=torch.int64, device="cuda"), rows=422, q_layout="head", **kw)
    _check(hb, g, dt, 128, 1, 3, 1, 70, 140, [140, 3, 21], sm_scale=2.5, q_size=3.0, **kw)


def test_the_library_chooses(hb):
    """Both forms' workspaces are those of the library's own choice, one way or the other, at sizes timed in both."""
    for dim, heads, tokens, cap, many in ((128, 16, 32, 10521, False), (128, 16, 64, 10521, True), (128, 64, 64, 2240, True),
                                          (64, 4, 64, 700, False), (128, 16, 1024, 64, True), (64, 256, 256, 680, True)):
        kv4 = Planes(heads * cap, dim).handle(hb, 1, heads, cap)
        q = torch.empty(1, heads, tokens, dim, dtype=torch.bfloat16, device="cuda")
        need = [kv4.hack_kv4_workspace(q, cap, form=f) for f in range(3)]
        assert need[0] == need[2 if many else 1], (dim, heads, tokens, cap, need)


def test_rows_whose_output_starts_on_16_bytes_only(hb):
    """bf16 rows 16 but not 32 bytes apart from a sector's start."""
    g, dim, cap, n = _gen(23), 64, 300, 130
    planes = Planes(cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, 1, cap)
    wide = torch.full((1, 1, n, dim + 8), 5.0, dtype=torch.bfloat16, device="cuda")
    q = torch.randn(1, 1, n, dim + 8, generator=g, device="cuda").to(torch.bfloat16)[..., 8:]
    for form in (1, 2):
        wide.fill_(5.0)
        kv4.hack_kv4_attend(q, wide[..., 8:], _ints(cap), cap, workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"), form=form)
        _rows_on_16_bytes(planes, q, wide, cap, n, dim)


def _rows_on_16_bytes(planes, q, wide, cap, n, dim):
    want = ref.attend(q[0], ref.values(planes.k_codes, planes.k_scales), ref.values(planes.v_codes, planes.v_scales), cap, n, dim ** -0.5)
    assert ((wide[0, ..., 8:].double() - want[0]).abs() <= ref.bound(*want, torch.bfloat16, dim, cap)).all()
    assert (wide[..., :8] == 5.0).all()


@pytest.mark.parametrize("dim", [64, 128])
def test_a_wait_that_runs_out_is_reported(hb, dim):
    from paper_2504_09261_b200 import binding as bd
    import ctypes as C
    g, cap, n = _gen(24), 2000, 300
    planes = Planes(2 * cap, dim)
    planes.randomise(g)
    kv4 = planes.handle(hb, 1, 2, cap)
    q = torch.randn(1, 2, n, dim, generator=g, device="cuda").to(torch.bfloat16)
    out, good = torch.empty_like(q), torch.empty_like(q)
    lens = _ints(cap, cap)
    need = kv4.hack_kv4_workspace(q, cap, form=hb.HACK_KV4_MANY)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    kv4.hack_kv4_attend(q, good, lens, cap, workspace=work, form=hb.HACK_KV4_MANY)
    kv4.hack_kv4_poll_status()
    args = kv4._attend(q, out, lens, cap, None, False, False, 0, 0, 0.0, work.numel(), hb.HACK_KV4_MANY)
    args.wait_polls = 1
    assert bd.lib.hack_kv4_attend(kv4._address, C.addressof(args), q.data_ptr(), out.data_ptr(), lens.data_ptr(), None, work.data_ptr(), None) == 0
    with pytest.raises(hb.HackError) as e:
        kv4.hack_kv4_poll_status()
    assert e.value.status == 6
    kv4.hack_kv4_poll_status()                                    # reported once
    kv4.hack_kv4_attend(q, out, lens, cap, workspace=work, form=hb.HACK_KV4_MANY)        # and the next call is right
    assert torch.equal(out, good)
    kv4.hack_kv4_poll_status()


# ------------------------------------------------------------------ together with the cache's steps
@pytest.mark.parametrize("config", [0, 1])
def test_from_projections_to_a_stored_cache(hb, config):
    """A decode that starts from projections (hack_scale_step_qkv) equals one that prepares q, k and v by hack_qk_norm_rope and
    steps by itself; the compressed rows of a layer then go to a 4-bit cache, tokens are appended and attended over."""
    from tests.parity_util import make_cache
    from workloads import SyntheticQKV, get_config
    cfg = get_config(config, n_layers=1)
    dt = torch.float32 if cfg.dtype == "f32" else torch.bfloat16
    mask = SyntheticQKV(cfg).head_is_contextual.numpy()
    one, two = make_cache(cfg, mask), make_cache(cfg, mask)
    b, h, d = cfg.batch, cfg.n_heads, cfg.head_dim
    g = _gen(31)
    plan = hb.hack_rope_plan(d, axes=2)
    gain = torch.full((h,), 6.0, device="cuda")
    for scale, side in enumerate(cfg.sides):
        n = side * side
        qkv = torch.randn(b, n, 3 * h, d, generator=g, device="cuda").to(dt)
        q, k, v = (qkv[:, :, i * h:(i + 1) * h].transpose(1, 2) for i in range(3))
        t = torch.arange(n, device="cuda")
        pos = torch.stack([t // side, t % side], -1).float() * (cfg.sides[-1] / side)
        outs = [torch.empty(b, h, n, d, dtype=dt, device="cuda") for _ in range(2)]
        one.hack_scale_step_qkv(0, scale, plan, q, k, v, outs[0], pos, norm=hb.HACK_NORM_L2, q_gain=gain)
        dense = [torch.empty(b, h, n, d, dtype=dt, device="cuda") for _ in range(3)]
        hb.hack_qk_norm_rope(plan, q, k, v, *dense, pos, norm=hb.HACK_NORM_L2, q_gain=gain)
        two.hack_scale_step(0, scale, *dense, outs[1])
        assert torch.equal(outs[0], outs[1])
    kept = one.hack_get_lengths(0)
    cap = max(kept) + 8
    planes = Planes(b * h * cap, d)
    kv4 = planes.handle(hb, b, h, cap)
    lens = _ints(*([2] * (b * h)))                                # behind two rows that are there already
    planes.randomise(g)
    one.hack_store_kv4(0, kv4, lens)
    for i in range(0, b * h, 7):
        for which, codes, scales in ((0, planes.k_codes, planes.k_scales), (1, planes.v_codes, planes.v_scales)):
            rows = torch.frombuffer(bytearray(one.hack_read_head(0, i // h, i % h, which)), dtype=dt).view(kept[i], d)
            c, byte, _ = ref.quantise(rows)
            assert torch.equal(codes[i * cap + 2:i * cap + 2 + kept[i]].cpu(), ref.pack(c))
            assert torch.equal(scales[i * cap + 2:i * cap + 2 + kept[i]].cpu().long(), byte)
    # five more tokens, causal among themselves, over everything stored
    x = torch.randn(3, b, h, 5, d, generator=g, device="cuda").to(dt)
    lens = lens + _ints(*kept)
    kv4.hack_kv4_append(x[1], x[2], lens)
    out = torch.empty_like(x[0])
    need = kv4.hack_kv4_workspace(x[0], cap, causal=True, appended=True)
    kv4.hack_kv4_attend(x[0], out, lens, cap, workspace=torch.empty(need, dtype=torch.uint8, device="cuda"), causal=True, appended=True)
    for i in range(0, b * h, 5):
        n = 2 + kept[i] + 5
        kd, vd = (ref.values(c[i * cap:i * cap + n], s[i * cap:i * cap + n]) for c, s in ((planes.k_codes, planes.k_scales), (planes.v_codes, planes.v_scales)))
        want = ref.attend(x[0][i // h, i % h][None], kd, vd, n, 5, d ** -0.5, causal=True)
        assert ((out[i // h, i % h].double() - want[0][0]).abs() <= ref.bound(*want, dt, d, n)[0]).all()
    one.close()
    two.close()


def test_decode_from_projections_in_a_graph(hb):
    """A whole decode that starts from projections, captured after the call that makes the buffers, replayed with other inputs."""
    from tests.parity_util import make_cache
    from workloads import SyntheticQKV, get_config
    cfg = get_config(1, n_layers=2)
    cache = make_cache(cfg, SyntheticQKV(cfg).head_is_contextual.numpy())
    b, h, d = cfg.batch, cfg.n_heads, cfg.head_dim
    g = _gen(41)
    plan = hb.hack_rope_plan(d, d // 2, layout=hb.HACK_ROPE_PAIRS)
    data = []
    for side in cfg.sides:
        n = side * side
        qkv = [torch.randn(b, n, 3, h, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
        data.append((qkv, [torch.empty(b, h, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                     torch.arange(n, dtype=torch.int32, device="cuda")))

    def loop(stream):
        cache.hack_reset()
        for scale, (qkv, outs, pos) in enumerate(data):
            for layer in range(2):
                cache.hack_scale_step_qkv(layer, scale, plan, *(qkv[layer][:, :, i].transpose(1, 2) for i in range(3)), outs[layer], pos,
                                          stream=stream)

    loop(None)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop(torch.cuda.current_stream().cuda_stream)
    for qkv, _, _ in data:
        for x in qkv:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    loop(None)
    torch.cuda.synchronize()
    want = [[o.clone() for o in outs] for _, outs, _ in data]
    for _, outs, _ in data:
        for o in outs:
            o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for w, (_, outs, _) in zip(want, data):
        assert torch.equal(w[0], outs[0]) and torch.equal(w[1], outs[1])
    cache.hack_poll_status()
    cache.close()


def test_step_from_projections_refuses(hb):
    from tests.parity_util import make_cache
    from workloads import SyntheticQKV, get_config
    cfg = get_config(1, n_layers=1)
    cache = make_cache(cfg, SyntheticQKV(cfg).head_is_contextual.numpy())
    b, h, d = cfg.batch, cfg.n_heads, cfg.head_dim
    q = torch.randn(b, h, 1, d, device="cuda").to(torch.bfloat16)
    plan, pos, out = hb.hack_rope_plan(d), _ints(0), torch.empty_like(q)
    for change in (dict(q=q[:, :4]), dict(k=q[:, :4]), dict(q=q.float(), k=q.float(), v=q.float())):
        kw = {**dict(q=q, k=q, v=q), **change}
        with pytest.raises((hb.HackError, ValueError)):
            cache.hack_scale_step_qkv(0, 0, plan, out=out, positions=pos, **kw)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):                                 # the first call allocates: not inside a capture
        with pytest.raises(hb.HackError) as e:
            cache.hack_scale_step_qkv(0, 0, plan, q, q, q, out, pos, stream=torch.cuda.current_stream().cuda_stream)
    assert e.value.status == 5
    cache.hack_scale_step_qkv(0, 0, plan, q, q, q, out, pos)      # nothing had changed
    kv4 = Planes(b * h * 4, d).handle(hb, b, h, 4)
    with pytest.raises(hb.HackError):
        cache.hack_store_kv4(1, kv4, _ints(*([0] * b * h)))
    with pytest.raises(hb.HackError):
        cache.hack_store_kv4(0, Planes(b * h * 4, 128).handle(hb, b, h, 4), _ints(*([0] * b * h)))
    cache.hack_poll_status()
    cache.close()
