"""Refusals of the operators around the cache: on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def hb():
    import __graft_entry__ as ge
    ge.build()
    import paper_2504_09261_b200 as pkg
    return pkg


GOOD = dict(head_dim=128, rotary_dim=64, layout=0, axes=1, base=10000.0, scaling=0, factor=1.0, trained_length=0)


@pytest.mark.parametrize("change,status", [
    (dict(head_dim=96), 2), (dict(rotary_dim=0), 1), (dict(rotary_dim=130), 1), (dict(rotary_dim=63), 1), (dict(rotary_dim=62, axes=2), 1),
    (dict(axes=3), 1), (dict(layout=2), 1), (dict(base=1.0), 1), (dict(base=float("nan")), 1), (dict(scaling=4), 1),
    (dict(scaling=1, factor=0.5), 1), (dict(scaling=2, factor=float("inf")), 1), (dict(scaling=3, factor=2.0), 1),
    (dict(scaling=3, factor=2.0, trained_length=4096, turns_fast=1.0, turns_slow=2.0), 1)])
def test_rope_plan_refuses(hb, change, status):
    hb.hack_rope_plan(**GOOD)
    with pytest.raises(hb.HackError) as e:
        hb.hack_rope_plan(**{**GOOD, **change})
    assert e.value.status == status and str(e.value)


def _rope_args(**change):
    from paper_2504_09261_b200 import binding as bd
    a = dict(device=0, dtype=1, batch=2, n_heads=3, n_tokens=4, positions_stride=0)
    a.update({k: v for k, v in change.items() if k in a})
    args = bd.HackRopeArgs(**a)
    args.x = args.y = bd.HackStrides(3 * 4 * 128, 4 * 128, 128)
    for k, v in change.items():
        if k in ("x", "y"):
            setattr(args, k, bd.HackStrides(*v))
    return args


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), 2), (dict(batch=0), 1), (dict(n_heads=0), 1), (dict(n_tokens=-1), 1), (dict(device=-1), 1),
    (dict(x=(1536, 512, 124)), 1), (dict(y=(1536, 512, 64)), 1), (dict(y=(0, 512, 128)), 1), (dict(y=(1536, 256, 128)), 1),
    (dict(y=(-1536, 512, 128)), 1)])
def test_rope_refuses(hb, change, status):
    from paper_2504_09261_b200 import binding as bd
    plan = hb.hack_rope_plan(128)
    args = _rope_args(**change)
    assert bd.lib.hack_rope(C.addressof(plan), C.addressof(args), 4096, 8192, 16384, None) == status
    assert hb.hack_last_error()


def test_rope_refuses_pointers(hb):
    from paper_2504_09261_b200 import binding as bd
    plan, args = hb.hack_rope_plan(128), _rope_args()
    p, a = C.addressof(plan), C.addressof(args)
    for call in ((None, a, 4096, 8192, 16384), (p, None, 4096, 8192, 16384), (p, a, None, 8192, 16384), (p, a, 4096, None, 16384),
                 (p, a, 4096, 8192, None), (p, a, 4104, 8192, 16384), (p, a, 4096, 8194, 16384)):
        assert bd.lib.hack_rope(*call, None) == 1, call
    blank = bd.HackRopePlan()
    blank.head_dim = 128
    assert bd.lib.hack_rope(C.addressof(blank), a, 4096, 8192, 16384, None) == 1
    nothing = _rope_args(n_tokens=0)
    assert bd.lib.hack_rope(p, C.addressof(nothing), None, None, None, None) == 0


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), 2), (dict(head_dim=80), 2), (dict(norm=3), 1), (dict(eps=0.0), 1), (dict(eps=float("nan")), 1), (dict(n_kv_heads=0), 1),
    (dict(v_out=None), 1), (dict(k=None), 1), (dict(positions=None), 1), (dict(plan=None), 1), (dict(q=None), 1), (dict(plan="other"), 1)])
def test_qk_norm_rope_refuses(hb, change, status):
    from paper_2504_09261_b200 import binding as bd
    plan = hb.hack_rope_plan(64 if change.get("plan") == "other" else 128)
    f = dict(device=0, dtype=0, batch=1, n_heads=2, n_kv_heads=2, n_tokens=3, head_dim=128, norm=1, eps=1e-6)
    f.update({k: v for k, v in change.items() if k in f})
    args = bd.HackQkvArgs(**f)
    for name in ("q", "k", "v", "q_out", "k_out", "v_out"):
        setattr(args, name, bd.HackStrides(768, 384, 128))
    ptr = dict(q=4096, k=8192, v=12288, q_out=16384, k_out=20480, v_out=24576, positions=28672)
    ptr.update({k: v for k, v in change.items() if k in ptr})
    p = None if "plan" in change and change["plan"] is None else C.addressof(plan)
    assert bd.lib.hack_qk_norm_rope(p, C.addressof(args), *ptr.values(), None, None, None, None, None) == status
    assert hb.hack_last_error()


def _kv4(**change):
    from paper_2504_09261_b200 import binding as bd
    f = dict(device=0, batch=2, n_kv_heads=3, head_dim=128, cap=50, reserved=0, rows=300, row_off=None, k_codes=4096, v_codes=8192, k_scales=12288,
             v_scales=16384)
    f.update(change)
    return bd.HackKv4Planes(*f.values())


@pytest.mark.parametrize("change,status", [(dict(head_dim=32), 2), (dict(batch=0), 1), (dict(n_kv_heads=-1), 1), (dict(cap=0), 1), (dict(device=-2), 1),
                                           (dict(k_codes=None), 1), (dict(rows=299), 1), (dict(rows=49, row_off=4096), 1), (dict(v_scales=16392), 1), (dict(batch=1 << 20, n_kv_heads=1 << 12), 1)])
def test_kv4_planes_refused(hb, change, status):
    from paper_2504_09261_b200 import binding as bd
    kv, rows = _kv4(**change), bd.HackKv4Rows(1, 4, bd.HackStrides(1536, 512, 128), bd.HackStrides(1536, 512, 128))
    at = bd.HackKv4Attend(1, 3, 1, 10, 0, 0, 0, 0, 0.0, 0, 0, bd.HackStrides(384, 128, 128), bd.HackStrides(384, 128, 128))
    k, r, a = C.addressof(kv), C.addressof(rows), C.addressof(at)
    need = C.c_size_t()
    assert bd.lib.hack_kv4_append(k, r, 4096, 4096, 4096, None, None) == status
    assert bd.lib.hack_kv4_read(k, r, 4096, 4096, 4096, None) == status
    assert bd.lib.hack_kv4_workspace(k, a, C.byref(need)) == status
    assert bd.lib.hack_kv4_attend(k, a, 4096, 8192, 4096, None, None, None) == status
    assert bd.lib.hack_kv4_append(None, r, 4096, 4096, 4096, None, None) == 1


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), 2), (dict(n_tokens=-1), 1), (dict(k=(1536, 512, 100)), 1), (dict(v=(1536, 512, 64)), 1)])
def test_kv4_rows_refused(hb, change, status):
    from paper_2504_09261_b200 import binding as bd
    kv = _kv4()
    rows = bd.HackKv4Rows(change.get("dtype", 1), change.get("n_tokens", 4), bd.HackStrides(*change.get("k", (1536, 512, 128))),
                          bd.HackStrides(*change.get("v", (1536, 512, 128))))
    k, r = C.addressof(kv), C.addressof(rows)
    assert bd.lib.hack_kv4_read(k, r, 4096, 8192, 4096, None) == status           # (64 apart: rows of an output would overlap)
    for call in ((k, r, None, 4096, 4096), (k, r, 4096, None, 4096), (k, r, 4096, 4096, None), (k, None, 4096, 4096, 4096), (k, r, 4100, 4096, 4096)):
        assert bd.lib.hack_kv4_append(*call, None, None) == (1 if change.get("dtype", 1) == 1 or call[1] is None else 2)
    none = bd.HackKv4Rows(1, 0)
    assert bd.lib.hack_kv4_append(k, C.addressof(none), None, None, None, None, None) == 0


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), 2), (dict(n_heads=4), 1), (dict(n_heads=0), 1), (dict(n_queries=-1), 1), (dict(max_len=-1), 1), (dict(window=-1), 1),
    (dict(n_sink=-1), 1), (dict(sm_scale=-1.0), 1), (dict(sm_scale=float("nan")), 1), (dict(n_queries=1 << 30), 1), (dict(wait_polls=-1), 1), (dict(form=3), 1),
    (dict(form=2, dtype=0), 2)])
def test_kv4_attend_refused(hb, change, status):
    from paper_2504_09261_b200 import binding as bd
    f = dict(dtype=1, n_heads=6, n_queries=1, max_len=10, appended=0, causal=0, window=0, n_sink=0, sm_scale=0.0, wait_polls=0, workspace_bytes=0)
    f.update({k: v for k, v in change.items() if k in f})
    args = bd.HackKv4Attend(*f.values(), bd.HackStrides(768, 128, 128), bd.HackStrides(768, 128, 128), change.get("form", 0), 0)
    kv = _kv4()
    k, a, need = C.addressof(kv), C.addressof(args), C.c_size_t()
    assert bd.lib.hack_kv4_workspace(k, a, C.byref(need)) == status
    assert bd.lib.hack_kv4_attend(k, a, 4096, 8192, 4096, None, None, None) == status
    assert hb.hack_last_error()


def test_kv4_attend_refuses_tensors(hb):
    from paper_2504_09261_b200 import binding as bd
    kv = _kv4()
    good = dict(dtype=1, n_heads=6, n_queries=1, max_len=10, appended=0, causal=0, window=0, n_sink=0, sm_scale=0.0, wait_polls=0, workspace_bytes=0)

    def call(q=4096, out=8192, lens=4096, strides=(768, 128, 128), out_strides=(768, 128, 128), n=1):
        args = bd.HackKv4Attend(*{**good, "n_queries": n}.values(), bd.HackStrides(*strides), bd.HackStrides(*out_strides))
        return bd.lib.hack_kv4_attend(C.addressof(kv), C.addressof(args), q, out, lens, None, None, None)

    assert call(q=None) == call(out=None) == call(lens=None) == call(q=4104) == call(strides=(768, 129, 128)) == 1
    assert call(out_strides=(0, 128, 128)) == call(out_strides=(768, 64, 128)) == 1
    assert call(n=0, q=None, out=None, lens=None) == 0
    assert bd.lib.hack_kv4_attend(C.addressof(kv), None, 4096, 8192, 4096, None, None, None) == 1
    assert bd.lib.hack_store_kv4(None, 0, C.addressof(kv), 4096, None) == 1
    assert bd.lib.hack_scale_step_qkv(None, 0, 0, *([None] * 12)) == 1
