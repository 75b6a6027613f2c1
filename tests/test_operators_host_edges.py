"""Arguments at the edges of the operators around the cache: answered or refused on the host (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def hb():
    import __graft_entry__ as ge
    ge.build()
    import paper_2504_09261_b200 as pkg
    return pkg


@pytest.mark.parametrize("norm,eps,refused", [(2, 1e-40, True), (2, 2.0 ** -149, True), (2, 2.0 ** -126, False), (1, 1e-40, False)])
def test_an_eps_without_a_reciprocal_is_refused(hb, norm, eps, refused):
    from paper_2504_09261_b200 import binding as bd
    none = bd.HackStrides()
    args = bd.HackQkvArgs(0, 0, 1, 2, 0, 0, 64, norm, eps, 0, 0, *([none] * 6))       # (no tokens: nothing else is looked at)
    assert bd.lib.hack_qk_norm_rope(None, C.addressof(args), *([None] * 12)) == (1 if refused else 0)
    assert not refused or "reciprocal" in hb.hack_last_error()


def _kv4(**change):
    from paper_2504_09261_b200 import binding as bd
    f = dict(device=0, batch=2, n_kv_heads=3, head_dim=128, cap=50, reserved=0, rows=300, row_off=None, k_codes=4096, v_codes=8192, k_scales=12288,
             v_scales=16384)
    f.update(change)
    return bd.HackKv4Planes(*f.values())


def _attend(**change):
    from paper_2504_09261_b200 import binding as bd
    f = dict(dtype=1, n_heads=6, n_queries=1, max_len=10, appended=0, causal=0, window=0, n_sink=0, sm_scale=0.0, wait_polls=0, workspace_bytes=0)
    form = change.pop("form", 0)
    f.update(change)
    return bd.HackKv4Attend(*f.values(), bd.HackStrides(768, 128, 128), bd.HackStrides(768, 128, 128), form, 0)


@pytest.mark.parametrize("form", [0, 1, 2])
def test_no_queries_need_no_workspace(hb, form):
    """(A launch of no tiles cannot be planned: the share of the multiprocessors for each would be a division by zero.)"""
    from paper_2504_09261_b200 import binding as bd
    need, kv, at = C.c_size_t(77), _kv4(), _attend(n_queries=0, form=form)
    assert bd.lib.hack_kv4_workspace(C.addressof(kv), C.addressof(at), C.byref(need)) == 0
    assert need.value == 0


@pytest.mark.parametrize("cap,refused", [(2 ** 31 - 1, True), (2 ** 31 - 511, True), (2 ** 31 - 512, False)])
def test_a_cap_next_to_the_end_of_32_bits_is_refused(hb, cap, refused):
    """A run of rows that starts in front of such a length would end past 32 bits and be taken for one that lies within it."""
    from paper_2504_09261_b200 import binding as bd
    kv, at, need = _kv4(cap=cap, rows=6 * 2 ** 31), _attend(n_queries=0), C.c_size_t()
    k = C.addressof(kv)
    rows = bd.HackKv4Rows(1, 0)
    want = 1 if refused else 0
    assert bd.lib.hack_kv4_workspace(k, C.addressof(at), C.byref(need)) == want
    assert bd.lib.hack_kv4_attend(k, C.addressof(at), None, None, None, None, None, None) == want
    assert bd.lib.hack_kv4_append(k, C.addressof(rows), None, None, None, None, None) == want
    assert bd.lib.hack_kv4_read(k, C.addressof(rows), None, None, None, None) == want


@pytest.fixture
def store(monkeypatch):
    """The binding's argument structs, empty.  (Calls on CPU tensors are marshalled as any other and refused by the library.)"""
    from paper_2504_09261_b200 import binding as bd
    held = {}
    monkeypatch.setattr(bd, "_args_of", held)
    return held


def _cpu_cache(hb):
    import torch
    return hb.HackKv4(*(torch.zeros(50, n, dtype=torch.uint8) for n in (32, 4, 32, 4)), batch=1, n_kv_heads=1, cap=50)


def test_arguments_are_held_by_value(hb, store):
    """A number that lives in a tensor and changes there: the call sees what is in it, not what was."""
    import torch
    x, lens = torch.zeros(1, 1, 1, 64), torch.zeros(1, dtype=torch.int32)
    kv4 = _cpu_cache(hb)
    numbers = dict(max_len=torch.tensor(10), n_sink=torch.tensor(1), window=torch.tensor(4), form=torch.tensor(0), causal=torch.tensor(False),
                   appended=torch.tensor(False), sm_scale=torch.tensor(0.5))
    eps, norm, transpose = torch.tensor(0.5), torch.tensor(1), torch.tensor(False)
    plan = hb.hack_rope_plan(64)

    def newest(call):
        with pytest.raises(hb.HackError) as e:
            call()
        assert e.value.status == 1
        return list(store.values())[-1][0]

    def calls():
        a = newest(lambda: kv4.hack_kv4_attend(x, x.clone(), lens, **numbers))
        n = newest(lambda: hb.hack_qk_norm_rope(None, x, None, None, x, None, None, None, norm=norm, eps=eps))
        r = newest(lambda: hb.hack_rope(plan, x, x, lens, transpose=transpose))
        return a.max_len, a.n_sink, a.window, a.form, a.causal, a.appended, a.sm_scale, n.eps, n.norm, r.transpose

    assert calls() == (10, 1, 4, 0, 0, 0, 0.5, 0.5, 1, 0)
    for t in (*numbers.values(), eps, norm, transpose):
        t.add_(1) if t.dtype != torch.bool else t.fill_(True)
    assert calls() == (11, 2, 5, 1, 1, 1, 1.5, 1.5, 2, 1)
    held = len(store)
    with pytest.raises(hb.HackError):
        kv4.hack_kv4_attend(x, x.clone(), lens, **numbers)
    assert held == 6 and len(store) == held                              # a value that was seen before needs no other struct
    for key in store:
        assert all(isinstance(v, (str, int, float, bool, tuple, type(None))) for v in key[0]), key[0]


def test_a_store_that_is_emptied_meanwhile(hb, store, monkeypatch):
    """Another thread's call empties the full store between this one's struct and its use: the struct is made again."""
    import torch
    from paper_2504_09261_b200 import binding as bd
    keep, made = bd._keep, []

    def meanwhile(key, args):
        keep(key, args)
        made.append(key)
        if len(made) % 2:
            store.clear()

    monkeypatch.setattr(bd, "_keep", meanwhile)
    x, ints = torch.zeros(1, 1, 1, 64), torch.zeros(1, dtype=torch.int32)
    kv4 = _cpu_cache(hb)
    plan = hb.hack_rope_plan(64)
    calls = (lambda: hb.hack_rope(plan, x, x, ints), lambda: hb.hack_qk_norm_rope(None, x, None, None, x, None, None, None),
             lambda: kv4.hack_kv4_append(x, x, ints), lambda: kv4.hack_kv4_read(x, x.clone(), ints[:1]),
             lambda: kv4.hack_kv4_attend(x, x, ints, 10))
    for i, call in enumerate(calls):
        store.clear()
        with pytest.raises(hb.HackError) as e:
            call()
        assert e.value.status == 1                                       # (the library's answer to tensors on the host)
        assert len(made) == 2 * (i + 1)


@pytest.mark.parametrize("dim,axes,trained,fast,slow", [
    (64, 1, 512, 200.0, 100.0),          # every pair turns less than turns_slow times
    (64, 1, 4, 32.0, 1.0), (128, 2, 6, 0.0, 0.0), (128, 1, 512, 81.0, 80.0), (64, 2, 1, 2.0, 1.0),
    (64, 1, 4096, 32.0, 1.0), (128, 1, 10 ** 9, 32.0, 1.0), (128, 2, 8192, 1000.0, 0.5), (64, 1, 512, 80.0, 20.0)])
def test_bands_stretch_what_turns_too_little(hb, dim, axes, trained, fast, slow):
    """Pairs that turn at least turns_fast times keep their frequency, pairs that turn turns_slow times or less have it divided."""
    import math
    factor = 8.0
    plan = hb.hack_rope_plan(dim, axes=axes, scaling=hb.HACK_ROPE_BANDS, factor=factor, trained_length=trained, turns_fast=fast, turns_slow=slow)
    plain = hb.hack_rope_plan(dim, axes=axes)
    fast, slow = fast or 32.0, slow or 1.0
    last = 1.0
    for i in range(dim // 2 // axes):
        part, turns = plan.freq[i] / plain.freq[i], trained * plain.freq[i] / (2 * math.pi)
        if turns < slow * (1 - 1e-9):
            assert abs(part * factor - 1) < 1e-12, (i, turns)
        if turns > fast * (1 + 1e-9):
            assert part == 1, (i, turns)
        assert 1 / factor * (1 - 1e-12) <= part <= last                # and a ramp downwards between them
        last = part


def test_arrays_off_their_size_are_refused(hb):
    """The kernels read these one number at a time: one that straddles its own size would be a misaligned address on the GPU."""
    from paper_2504_09261_b200 import binding as bd
    held = hb.hack_rope_plan(128)
    plan, strides = C.addressof(held), bd.HackStrides(768, 384, 128)
    rope = bd.HackRopeArgs(0, 0, 1, 2, 3, 0, 0, 0, 0, strides, strides)
    assert bd.lib.hack_rope(plan, C.addressof(rope), 4096, 8192, 16386, None) == 1 and "4 bytes" in hb.hack_last_error()
    qkv = bd.HackQkvArgs(0, 0, 1, 2, 2, 3, 128, 1, 1e-6, 0, 0, *([strides] * 6))
    for off in range(5):                     # positions, q_weight, k_weight, q_gain, k_gain
        arrays = [8192 + (2 if i == off else 0) for i in range(5)]
        assert bd.lib.hack_qk_norm_rope(plan, C.addressof(qkv), *([4096] * 6), *arrays, None) == 1
        assert "4 bytes" in hb.hack_last_error()
    kv, kv_off, at = _kv4(), _kv4(row_off=4100), _attend()
    rows = bd.HackKv4Rows(1, 4, bd.HackStrides(1536, 512, 128), bd.HackStrides(1536, 512, 128))
    k, r, a = C.addressof(kv), C.addressof(rows), C.addressof(at)
    for call in (lambda: bd.lib.hack_kv4_append(k, r, 4096, 4096, 4098, None, None), lambda: bd.lib.hack_kv4_append(k, r, 4096, 4096, 4096, 4097, None),
                 lambda: bd.lib.hack_kv4_read(k, r, 4096, 4096, 4099, None), lambda: bd.lib.hack_kv4_attend(k, a, 4096, 8192, 4097, None, None, None),
                 lambda: bd.lib.hack_kv4_attend(k, a, 4096, 8192, 4096, 4098, None, None)):
        assert call() == 1 and "4 bytes" in hb.hack_last_error()
    assert bd.lib.hack_kv4_append(C.addressof(kv_off), r, 4096, 4096, 4096, None, None) == 1 and "8 bytes" in hb.hack_last_error()


def test_marshalling_without_the_compiled_module(hb, monkeypatch):
    """Where the module of csrc/pycall.c is not built, ctypes makes the same calls: the same keys, the same arguments in the same
    places, the same answers."""
    import os
    import torch
    from paper_2504_09261_b200 import binding as bd
    exists = os.path.exists
    monkeypatch.setattr(bd.os.path, "exists", lambda p: "_hackcall" not in str(p) and exists(p))
    call, run = bd._load_call()
    monkeypatch.undo()
    assert run is not bd._run and bd._run.__class__.__name__ == "builtin_function_or_method"
    assert call(bd._SCORE, 0, 0, 0, None, None, None, None) == bd._call(bd._SCORE, 0, 0, 0, None, None, None, None) == 1
    x, ints = torch.zeros(2, 3, 4, 128), torch.zeros(4, dtype=torch.int32)
    seen = []
    # struct by struct as the entry points want them, with the sizes that each refuses by another text or serves without a launch
    kv, plan = _kv4(), hb.hack_rope_plan(128)
    strides = bd.HackStrides(1536, 512, 128)
    for address, lead, tensors, structs in (
            (bd._ROPE, plan, (x, x, ints), [bd.HackRopeArgs(0, 0, 2, 3, n, 0, 0, 0, 0, strides, bd.HackStrides(s, 512, 128)) for n, s in ((0, 1536), (4, 0), (-1, 0))]),
            (bd._QK_NORM_ROPE, plan, (x, x, None, x, None, None, ints, None, None, None, None), [bd.HackQkvArgs(0, 0, 2, 3, 3, 4, 128, 1, 1e-6)]),
            (bd._QK_NORM_ROPE, None, (x, None, None, x, None, None, ints, None, None, None, None), [bd.HackQkvArgs(0, 0, 2, 3, 3, 4, 128, 1, 1e-6)]),
            (bd._KV4_APPEND, kv, (x, None, ints, None), [bd.HackKv4Rows(0, 4, strides, strides), bd.HackKv4Rows(0, 0)]),
            (bd._KV4_APPEND, kv, (x, x, None, ints), [bd.HackKv4Rows(0, 4, strides, strides)]),
            (bd._KV4_READ, kv, (x, x, None), [bd.HackKv4Rows(0, 4, strides, strides), bd.HackKv4Rows(0, 0)]),
            (bd._KV4_ATTEND, kv, (x, x, None, None, None), [_attend(), _attend(n_queries=0)]),
            (bd._KV4_ATTEND, kv, (x, None, ints, None, None), [_attend()])):
        for args in structs:
            store, lead_at = {}, None if lead is None else C.addressof(lead)
            key = run(store, "head", address, lead_at, None, *tensors)
            assert key == bd._run(store, "head", address, lead_at, None, *tensors) and key.__class__ is tuple and not store
            store[key] = (args, C.addressof(args))
            answers = []
            for f in (run, bd._run):
                status = f(store, "head", address, lead_at, None, *tensors)
                answers.append((status, hb.hack_last_error() if status else ""))
            assert answers[0] == answers[1] and answers[0][0].__class__ is int, answers
            seen.append(answers[0])
    assert {s for s, _ in seen} == {0, 1} and len({t for _, t in seen}) >= 6, seen
