"""CPU checks of the operators on quantized layers: argument validation of the C entry points (fake pointers, never
dereferenced: every call fails before anything is enqueued), argument structs, and the plan of a batch's requests."""
import ctypes as C

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def adapt():
    from paper_2605_11222_b200 import adapt, build
    build.build()
    adapt._library()
    return adapt


FAKE = 0x10000


def _layer(adapt, d_in=128, d_out=64, group=64, packed=FAKE, grid=FAKE):
    return adapt.PackedLayer(C.sizeof(adapt.PackedLayer), d_in, d_out, group, packed, grid)


def _bank(adapt, n=2, rank=8, down=FAKE, up=FAKE, scale=FAKE):
    return adapt.Adapters(C.sizeof(adapt.Adapters), n, rank, down, up, scale)


def test_sizes_of_a_packed_layer(adapt):
    lib = adapt._library()
    assert lib.admmq_packed_bytes(4096, 1024) == 4096 * 1024 // 2
    assert lib.admmq_packed_bytes(72, 8) == 2 * 8 * 32                     # 72 channels: two blocks of 64
    assert lib.admmq_grid_bytes(4096, 1024, 128) == 32 * 1024 * 8
    assert lib.admmq_grid_bytes(4096, 1024, 0) == lib.admmq_grid_bytes(4096, 1024, 4096) == 1024 * 8
    for bad in [(60, 64), (64, 60), (0, 64), (64, 0), (14344, 64), (-8, 8)]:
        assert lib.admmq_packed_bytes(*bad) == 0
    for bad in [(128, 64, 32), (128, 64, 48), (128, 64, 256), (128, 64, -64), (192, 64, 128)]:
        assert lib.admmq_grid_bytes(*bad) == 0


def test_pack_layer_refuses_bad_arguments(adapt):
    from paper_2605_11222_b200 import binding as B
    f = adapt._library().admmq_pack_layer
    ok = [FAKE, FAKE, FAKE, 128, 64, 4, 64, FAKE, FAKE, FAKE, None]

    def with_(i, v):
        a = list(ok)
        a[i] = v
        return f(*a)

    for i in (0, 1, 2, 7, 8, 9):
        assert with_(i, None) == B.ERR_INVALID_ARG
    assert with_(7, FAKE + 8) == B.ERR_INVALID_ARG
    assert with_(5, 5) == B.ERR_UNSUPPORTED and with_(5, 8) == B.ERR_UNSUPPORTED
    assert with_(5, 1) == B.ERR_SHAPE and with_(5, 9) == B.ERR_SHAPE
    assert with_(6, 32) == B.ERR_SHAPE and with_(3, 124) == B.ERR_SHAPE and with_(4, 63) == B.ERR_SHAPE


@pytest.mark.parametrize("name", ["admmq_linear_forward", "admmq_linear_grad_input"])
def test_linear_refuses_bad_arguments(adapt, name):
    from paper_2605_11222_b200 import binding as B
    f = getattr(adapt._library(), name)
    grad = name.endswith("input")
    ldi, ldo = (64, 128) if grad else (128, 64)
    layer, bank = _layer(adapt), _bank(adapt)
    ok = [C.byref(layer), C.byref(bank), 5, FAKE, FAKE, ldi, FAKE, ldo, FAKE, FAKE, None]

    def with_(i, v):
        a = list(ok)
        a[i] = v
        return f(*a)

    assert with_(0, None) == B.ERR_INVALID_ARG
    for i in (3, 4, 6, 8, 9):
        assert with_(i, None) == B.ERR_INVALID_ARG
    for i in (4, 6, 8):
        assert with_(i, FAKE + 8) == B.ERR_INVALID_ARG
    for i, ld in ((5, ldi), (7, ldo)):
        assert with_(i, ld - 8) == B.ERR_SHAPE and with_(i, ld + 4) == B.ERR_SHAPE
    assert with_(2, -1) == B.ERR_SHAPE and with_(2, 2 ** 31) == B.ERR_SHAPE
    for bad in (_layer(adapt, 124), _layer(adapt, 128, 60), _layer(adapt, 128, 64, 96)):
        assert with_(0, C.byref(bad)) == B.ERR_SHAPE
    for bad in (_layer(adapt, packed=None), _layer(adapt, grid=FAKE + 4)):
        assert with_(0, C.byref(bad)) == B.ERR_INVALID_ARG
    layer2 = _layer(adapt)
    layer2.struct_size -= 4
    assert with_(0, C.byref(layer2)) == B.ERR_INVALID_ARG
    for bad in (_bank(adapt, 0), _bank(adapt, 70000), _bank(adapt, 2, 12), _bank(adapt, 2, 136), _bank(adapt, 2, 0)):
        assert with_(1, C.byref(bad)) == B.ERR_SHAPE
    for bad in (_bank(adapt, down=None), _bank(adapt, up=FAKE + 2), _bank(adapt, scale=None)):
        assert with_(1, C.byref(bad)) == B.ERR_INVALID_ARG
    assert with_(2, 0) == B.OK                                             # no rows: nothing to do


def test_argument_structs_have_the_c_sizes(adapt):
    """A struct of another size is refused before anything else; with the right one the next check speaks."""
    from paper_2605_11222_b200 import binding as B
    lib = adapt._library()
    n = adapt._GRAD_ARGS.size
    good = adapt._GRAD_ARGS.pack(n, 124, 64, 1, 8, 1, *[FAKE] * 5, 128, *[FAKE] * 3, 64, FAKE, FAKE)
    assert lib.admmq_adapter_grad(good, None) == B.ERR_SHAPE               # d_in 124
    bad = adapt._GRAD_ARGS.pack(n + 8, 124, 64, 1, 8, 1, *[FAKE] * 5, 128, *[FAKE] * 3, 64, FAKE, FAKE)
    assert lib.admmq_adapter_grad(bad, None) == B.ERR_INVALID_ARG
    n = adapt._QK_ARGS.size

    def qk(size=n, dtype=1, hq=2, hk=1, d=64, rot=64, rows=3, eps=1e-6, q=FAKE, row=128, pos=FAKE, npos=10,
           status=FAKE, back=(0,) * 10):
        return adapt._QK_ARGS.pack(size, dtype, hq, hk, d, rot, rows, eps, q, FAKE, row, 64, 64, 64, FAKE, FAKE, FAKE,
                                   FAKE, npos, pos, FAKE, FAKE, 128, 64, 64, 64, *back, status)

    fwd, bwd = lib.admmq_qk_norm_rope, lib.admmq_qk_norm_rope_backward
    assert fwd(qk(size=n - 8), None) == B.ERR_INVALID_ARG
    assert fwd(qk(rows=0), None) == B.OK
    for kw in (dict(d=40), dict(d=272), dict(rot=24), dict(rot=80), dict(hq=0), dict(hk=-1), dict(row=132), dict(rows=-1),
               dict(npos=0)):
        assert fwd(qk(**kw), None) == B.ERR_SHAPE, kw
    for kw in (dict(dtype=2), dict(eps=-1.0), dict(eps=float("nan")), dict(q=0), dict(q=FAKE + 8), dict(pos=0),
               dict(status=0)):
        assert fwd(qk(**kw), None) == B.ERR_INVALID_ARG, kw
    assert bwd(qk(), None) == B.ERR_INVALID_ARG                            # no dy, no workspace
    ws = lib.admmq_qk_workspace_bytes(64)
    assert ws > 0 and lib.admmq_qk_workspace_bytes(40) == 0
    assert bwd(qk(back=(FAKE, FAKE, 128, 64, 64, 64, FAKE, FAKE, FAKE, ws - 1)), None) == B.ERR_WORKSPACE


def test_adapter_grad_refuses_bad_arguments(adapt):
    from paper_2605_11222_b200 import binding as B
    f, S = adapt._library().admmq_adapter_grad, adapt._GRAD_ARGS

    def call(d_in=128, d_out=64, n=2, rank=8, rows=5, order=FAKE, offsets=FAKE, h=FAKE, u=FAKE, x=FAKE, ldx=128, codes=0,
             scale=0, dy=FAKE, lddy=64, gd=FAKE, gu=FAKE):
        return f(S.pack(S.size, d_in, d_out, n, rank, rows, order, offsets, h, u, x, ldx, codes, scale, dy, lddy, gd, gu),
                 None)

    assert f(None, None) == B.ERR_INVALID_ARG
    for kw in (dict(d_out=60), dict(n=0), dict(n=65536), dict(rank=12), dict(rank=136), dict(rows=-1), dict(ldx=120),
               dict(ldx=132), dict(lddy=56), dict(lddy=68)):
        assert call(**kw) == B.ERR_SHAPE, kw
    for kw in (dict(order=0), dict(offsets=0), dict(h=0), dict(u=FAKE + 4), dict(x=0), dict(x=FAKE + 2), dict(dy=0),
               dict(gd=0), dict(gu=FAKE + 8), dict(x=0, codes=FAKE), dict(x=0, codes=FAKE + 8, scale=FAKE)):
        assert call(**kw) == B.ERR_INVALID_ARG, kw


def test_checkpoint_refuses_bad_arguments(adapt):
    from paper_2605_11222_b200 import binding as B
    lib = adapt._library()
    for f, ok in ((lib.admmq_checkpoint_save, [FAKE, 1, 4, 64, 64, FAKE, FAKE, None]),
                  (lib.admmq_checkpoint_restore, [FAKE, FAKE, 4, 64, FAKE, 1, 64, None])):
        save = f is lib.admmq_checkpoint_save
        dt, ld, ptrs = (1, 4, (0, 5, 6)) if save else (5, 6, (0, 1, 4))
        width = 3

        def with_(i, v):
            a = list(ok)
            a[i] = v
            return f(*a)

        assert with_(dt, 2) == B.ERR_INVALID_ARG
        for i in ptrs:
            assert with_(i, None) == B.ERR_INVALID_ARG
        assert with_(width, 60) == B.ERR_SHAPE and with_(width, 0) == B.ERR_SHAPE
        assert with_(ld, 56) == B.ERR_SHAPE and with_(ld, 68) == B.ERR_SHAPE
        assert with_(2, -1) == B.ERR_SHAPE and with_(2, 0) == B.OK


def test_request_plan(adapt):
    from paper_2605_11222_b200 import binding as B
    plan = adapt.RequestPlan([2, 0, 3, 1, 2], [1, 0, -1, 3, 1], 4, device="cpu")
    assert plan.n_rows == 8
    assert plan.row_adapter.tolist() == [1, 1, -1, -1, -1, 3, 1, 1]
    off = plan.offsets.tolist()
    assert off == [0, 0, 4, 4, 5]
    assert plan.order.tolist()[:5] == [0, 1, 6, 7, 5]                      # rows of adapter 1 in order, then of 3
    assert all(t.dtype == torch.int32 for t in (plan.row_adapter, plan.order, plan.offsets))
    empty = adapt.RequestPlan([], [], 2, device="cpu")
    assert empty.n_rows == 0 and empty.offsets.tolist() == [0, 0, 0]
    rng = np.random.default_rng(0)
    lengths, ids = rng.integers(0, 9, 50), rng.integers(-1, 7, 50)
    plan = adapt.RequestPlan(lengths, ids, 7, device="cpu")
    rows = np.repeat(ids, lengths)
    for a in range(7):
        o = plan.offsets.tolist()
        assert plan.order.tolist()[o[a]: o[a + 1]] == np.flatnonzero(rows == a).tolist()
    for bad in (([1, 2], [0]), ([-1], [0])):
        with pytest.raises(adapt.AdmmqError) as e:
            adapt.RequestPlan(*bad, 2, device="cpu")
        assert e.value.status == B.ERR_SHAPE
    for a in (-2, 2):
        with pytest.raises(adapt.AdmmqError):
            adapt.RequestPlan([1], [a], 2, device="cpu")


def test_waits_by_parity_of_the_pair_form_know_the_phase_before(adapt):
    """The projection on CTA pairs shares its K steps out to groups of warps by step number, adapter steps counted, and its
    codes to slots and barriers by code step, adapter steps not counted.  A group waits on a barrier by parity, which is
    sound only if it knows the phase before to be over: it took those codes itself, or they belong to a step that a wait
    of its own has seen done (steps are done in order, and a step's codes have landed before it is done)."""
    out = [C.c_int() for _ in range(5)]
    adapt._library().admmq_test_pair_rings(*[C.byref(o) for o in out])
    groups, stages, row_stages, slots, barriers = [o.value for o in out]
    assert row_stages <= stages and barriers % slots == 0
    rng = np.random.default_rng(1)
    cases = [(kb, [e] * 12) for kb in (1, 2, 3, 4, 7, 64) for e in range(9)]
    cases += [(kb, rng.integers(0, 6, 60).tolist()) for kb in (1, 2, 3, 5, 8, 64) for _ in range(20)]
    for num_kb, extras in cases:
        done = [-1] * groups                       # last step that the group's waits have seen done
        taken = [set() for _ in range(groups)]     # code steps that it took
        step_of = []                               # of every code step
        it = 0
        for extra in extras:                       # the tiles of a pair
            for k in range(num_kb + extra):
                g = it % groups
                if k < num_kb:
                    ct = len(step_of)
                    step_of.append(it)
                    before = ct - barriers
                    assert before < 0 or before in taken[g] or step_of[before] <= done[g], (num_kb, extras, it)
                    taken[g].add(ct)
                depths = (stages,) if k < num_kb else (stages, row_stages)
                for depth in depths:               # the stage is free: step it - depth is done
                    last = it - depth
                    assert last < stages or last - stages <= done[g], (num_kb, extras, it)
                    done[g] = max(done[g], last)
                it += 1


def test_threads_share_one_status_word(adapt, monkeypatch):
    """Two threads at a device's first call: one word, since kernels keep the pointer that the call was given."""
    import threading
    import time
    index, made, got = 77, [], []
    zeros, start = torch.zeros, threading.Barrier(8)

    def slow_zeros(*size, **kw):
        made.append(zeros(*size, dtype=kw["dtype"]))
        time.sleep(0.02)
        return made[-1]

    def first_call():
        start.wait()
        got.append(adapt._status(index))

    monkeypatch.setattr(torch, "zeros", slow_zeros)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    threads = [threading.Thread(target=first_call) for _ in range(8)]
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        assert len(made) == 1 and got == [made[0].data_ptr()] * 8
    finally:
        adapt._status_words.pop(index, None)


def test_queries_in_a_graph_are_refused_before_anything_else(adapt):
    from paper_2605_11222_b200 import binding as B
    q, w = torch.ones(1, 1, 16), torch.ones(16)
    args = (w, w, torch.ones(2, 8), torch.ones(2, 8), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(adapt.AdmmqError, match="requires grad") as e:
        adapt.qk_norm_rope(q.clone().requires_grad_(), q, *args)
    assert e.value.status == B.ERR_INVALID_ARG
    with torch.no_grad(), pytest.raises(adapt.AdmmqError, match="on a GPU"):
        adapt.qk_norm_rope(q.clone().requires_grad_(), q, *args)


def test_a_checkpoint_of_more_blocks_than_a_device_holds_is_refused(adapt):
    from paper_2605_11222_b200 import binding as B
    lib = adapt._library()
    for rows, width in ((2 ** 30, 136), (2 ** 30, 256), (2 ** 24, 16384), (2 ** 18, 2 ** 20)):      # 2^31 blocks and more
        assert lib.admmq_checkpoint_save(FAKE, 1, rows, width, width, FAKE, FAKE, None) == B.ERR_SHAPE
        assert lib.admmq_checkpoint_restore(FAKE, FAKE, rows, width, FAKE, 1, width, None) == B.ERR_SHAPE


def test_the_extension_is_rebuilt_for_another_torch_or_python(adapt, monkeypatch, tmp_path):
    """It is compiled against their internals: a change of either makes it stale, whatever the sources' dates."""
    import os
    import subprocess
    from paper_2605_11222_b200 import build
    so, runs = tmp_path / "_adapt.so", []

    def compiler(cmd, **kw):
        runs.append(cmd)
        so.write_bytes(b"")
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build, "BIND", os.fspath(so))
    monkeypatch.setattr(build, "BIND_FOR", os.fspath(tmp_path / "_adapt.for"), raising=False)
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build._build_bind(False, [])
    build._build_bind(False, [])
    assert len(runs) == 1
    with monkeypatch.context() as m:
        m.setattr(torch, "__version__", "0.0.0")
        build._build_bind(False, [])
        assert len(runs) == 2
    build._build_bind(False, [])                 # and back
    assert len(runs) == 3
    with monkeypatch.context() as m:
        m.setattr("sys.version", "0.0.0 of another build")
        build._build_bind(False, [])
        assert len(runs) == 4
