"""The optimiser step at the ends of its numbers: zeros, gradients next to both ends of float32, and factors that float32 does not hold.  Tolerances: muon_bounds.py."""
import ctypes as C

import pytest
import torch

import paper_2111_10672_amd as spb
from muon_bounds import U, check_matrices
from paper_2111_10672_amd.binding import _check
from test_host_streams import run, runtime  # noqa: F401
from test_muon import HYPER, _numpy, _step, _tensor

# on the Gram matrix, in two launches a step, in three
SHAPES = [(20, 24), (24, 20), (70, 90), (300, 320)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_gradient_of_zeros_leaves_only_the_decay(shape, dtype):
    """Whatever ns_eps: 0 / (0 + eps) is 0."""
    for eps in (5e-324, 1e-300, 1e-50, 1e-40, 1e-35, 1e-7, 1e300):
        t = _tensor(shape, 1, dtype, 1, seed=5)
        t["m"].zero_()
        t["grads"][0].zero_()
        before = t["w"].double()
        _step([t], {**HYPER, "ns_eps": eps})
        want = before * (1.0 - HYPER["lr"] * HYPER["weight_decay"])
        half = 2.0 ** -8 if dtype == torch.bfloat16 else U
        assert bool(((t["w"].double() - want).abs() <= (half + 4 * U) * before.abs()).all()), eps
        assert not t["m"].any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradients_next_to_the_ends_of_float32(shape, dtype):
    """1 / |u| or the scale that follows from it leaves float32, u does not: the update is that of any other size.  (Without momentum, so that u is the gradient itself.)"""
    for scale, eps in ((1e-42, 1e-300), (1e-39, 5e-324), (1e-36, 1e-45), (3e37, 1e-7)):
        hyper = {**HYPER, "momentum": 0.0, "nesterov": False, "ns_eps": eps}
        t = _tensor(shape, 1, dtype, 1, seed=6, w=0.0, scale=scale)
        t["m"].zero_()
        before = _numpy(t)
        _step([t], hyper)
        check_matrices(before, _numpy(t), dtype, hyper)


@pytest.mark.gpu
def test_moments_of_zero_under_the_smallest_adam_eps():
    for dtype in (torch.bfloat16, torch.float32):
        t = _tensor((515,), 0, dtype, 1, seed=7)
        for x in (t["m"], t["v"], t["grads"][0]):
            x[::2] = 0.0
        before = t["w"].double()
        _step([t], {**HYPER, "adam_eps": 1.2e-38})
        assert bool(t["w"].isfinite().all())
        half = 2.0 ** -8 if dtype == torch.bfloat16 else U
        want = before * (1.0 - HYPER["lr"] * HYPER["weight_decay"])
        assert bool(((t["w"].double() - want).abs() <= (half + 4 * U) * before.abs())[::2].all())


# ---- refusals: all found on the host ----------------------------------------------------------------------------------

def _call(config=None, **patch):
    grads = (C.c_void_p * 1)(1 << 20)
    t = (spb.binding.spb_muon_tensor * 1)()
    t[0].w, t[0].m, t[0].v, t[0].grads = 1 << 12, 1 << 13, 1 << 14, C.cast(grads, C.POINTER(C.c_void_p))
    t[0].rows, t[0].cols, t[0].rate_scale, t[0].count, t[0].dtype, t[0].blocks = 6, 5, 1.0, 1, 1, 1
    for k, v in patch.items():
        setattr(t[0], k, v)
    _check(spb.lib().spb_muon_step(t, 1, C.byref(spb.muon_config(**{**HYPER, **(config or {})})), 1 << 21, 1 << 20, None))


@pytest.mark.parametrize("config,patch", [(dict(lr=1e39), {}), (dict(rms=1e39), {}), (dict(momentum=-1e39), {}), (dict(weight_decay=1e39), {}), (dict(lr=1e20, rms=1e20), {}),
                                          (dict(lr=1e20, weight_decay=1e20), {}), (dict(lr=1e20, weight_decay=1e20), dict(blocks=0)), ({}, dict(rate_scale=1e300)),
                                          (dict(rms=2e38), dict(rate_scale=100.0)), (dict(adam_eps=1e-39), dict(blocks=0)), (dict(adam_eps=1e-50), dict(blocks=0)),
                                          (dict(adam_eps=1e-39), {})])
def test_factors_that_float32_does_not_hold_are_refused(config, patch):
    with pytest.raises(spb.SpbError) as e:
        _call(config, **patch)
    assert e.value.code == -1 and "spb_muon_step" in str(e.value)


def test_the_server_step_refuses_them_too():
    import workloads as wl
    m = spb.spb_model_create(spb.desc_from_config(wl.get_config("ragged_mlp_bf16")))
    try:
        n = spb.spb_param_count(m)
        spb.spb_bind_params(m, [(i + 1) << 32 for i in range(n)])
        blocks = [int(len(spb.spb_param_info(m, i)["shape"]) > 1) for i in range(n)]
        size = spb.spb_aggregate_muon_workspace_size(m, blocks)
        at = lambda k: [(k << 44) + (i << 32) for i in range(n)]
        for config in (dict(lr=1e39), dict(lr=1e20, rms=1e20), dict(adam_eps=1e-40)):
            with pytest.raises(spb.SpbError) as e:
                spb.spb_aggregate_muon(m, [4], [at(1)], blocks, at(2), at(3), spb.muon_config(**{**HYPER, **config}), True, 1 << 60, size, 0)
            assert e.value.code == -1, config
    finally:
        spb.spb_model_destroy(m)


def test_factors_at_the_ends_of_float32_are_taken(run):  # noqa: F811
    run("""
    def call(config, blocks=1):
        grads, t = (C.c_void_p * 1)(1 << 20), (spb.binding.spb_muon_tensor * 1)()
        t[0].w, t[0].m, t[0].v, t[0].grads = 1 << 12, 1 << 13, 1 << 14, C.cast(grads, C.POINTER(C.c_void_p))
        t[0].rows, t[0].cols, t[0].rate_scale, t[0].count, t[0].dtype, t[0].blocks = 6, 5, 1.0, 1, 1, blocks
        spb.binding._check(spb.lib().spb_muon_step(t, 1, C.byref(spb.muon_config(**config)), 1 << 21, 1 << 20, None))
    for config in (dict(lr=1e30), dict(lr=0.0), dict(lr=1e-300), dict(lr=0.1, ns_eps=5e-324), dict(lr=0.1, ns_eps=1e300), dict(lr=0.1, adam_eps=1.2e-38), dict(lr=0.1, beta1=1 - 1e-9)):
        call(config)
        call(config, 0)
    """)


def test_more_matrices_than_a_step_takes_have_no_workspace_size():
    """2^31 of them and more would not be counted right."""
    t = (spb.binding.spb_muon_tensor * 2)()
    size = C.c_size_t(77)
    for x in t:
        x.rows, x.cols, x.dtype, x.blocks = 1 << 30, 1, 1, 1 << 30
    for n in (1, 2):
        with pytest.raises(spb.SpbError) as e:
            _check(spb.lib().spb_muon_workspace_size(t, n, C.byref(size)))
        assert e.value.code == -1 and size.value == 77
    t[0].rows = t[0].blocks = 1 << 17                                   # 2^17 of 256 x 256, padded: as many as a step takes
    _check(spb.lib().spb_muon_workspace_size(t, 1, C.byref(size)))
    assert size.value > (1 << 17) * 4
    with pytest.raises(spb.SpbError) as e:
        _call(rows=1 << 18, cols=1, blocks=1 << 18)
    assert e.value.code == -1 and "too many" in str(e.value)


def test_the_server_step_of_more_matrices_than_it_takes_has_no_workspace_size():
    import workloads as wl
    cfg = dict(wl.get_config("ragged_mlp_bf16"), dims=[8, 1 << 16, 1 << 16])
    m = spb.spb_model_create(spb.desc_from_config(cfg))
    try:
        blocks = [1 << 16 if len(spb.spb_param_info(m, i)["shape"]) > 1 else 0 for i in range(spb.spb_param_count(m))]
        with pytest.raises(spb.SpbError) as e:
            spb.spb_aggregate_muon_workspace_size(m, blocks)
        assert e.value.code == -1
    finally:
        spb.spb_model_destroy(m)


# Two float32 tensors of 6 x 5 and 40 entries: a matrix and one that AdamW takes.
PLACES = dict(w0=1 << 16, m0=2 << 16, g0=3 << 16, w1=4 << 16, m1=5 << 16, v1=6 << 16, g1=7 << 16, ws=8 << 16)


def _places(lib, **patch):
    p = {**PLACES, **patch}
    t, keep = (spb.binding.spb_muon_tensor * 2)(), []
    for x, g, fields in ((t[0], "g0", dict(w=p["w0"], m=p["m0"], rows=6, cols=5, blocks=1)), (t[1], "g1", dict(w=p["w1"], m=p["m1"], v=p["v1"], rows=40, cols=1, blocks=0))):
        keep.append((C.c_void_p * 1)(p[g]))
        for k, v in dict(fields, rate_scale=1.0, count=1, dtype=0, grads=C.cast(keep[-1], C.POINTER(C.c_void_p))).items():
            setattr(x, k, v)
    size = C.c_size_t()
    _check(lib.spb_muon_workspace_size(t, 2, C.byref(size)))
    _check(lib.spb_muon_step(t, 2, C.byref(spb.muon_config(**HYPER)), p["ws"], size.value, None))


@pytest.mark.parametrize("patch", [dict(m0=PLACES["w0"]), dict(m0=PLACES["w0"] + 116), dict(w1=PLACES["m0"] + 4), dict(v1=PLACES["w1"] + 156), dict(w1=PLACES["w0"] - 156),
                                   dict(ws=PLACES["w0"] - 256), dict(w0=PLACES["ws"] + 256), dict(g0=PLACES["m1"]), dict(g0=PLACES["v1"] + 156), dict(g1=PLACES["w0"] - 156),
                                   dict(g0=PLACES["m0"]), dict(g1=PLACES["ws"] + 64)])
def test_tensors_that_lie_in_one_another_are_refused(patch):
    with pytest.raises(spb.SpbError) as e:
        _places(spb.lib(), **patch)
    assert e.value.code == -1 and "lies in" in str(e.value), patch


def test_tensors_side_by_side_and_gradients_of_one_place_are_taken(run):  # noqa: F811
    import inspect
    run(f"PLACES, HYPER = {PLACES!r}, {HYPER!r}\nfrom paper_2111_10672_amd.binding import _check\n" + inspect.getsource(_places) + """
for patch in (dict(), dict(m0=PLACES["w0"] + 120), dict(w1=PLACES["w0"] - 160), dict(g1=PLACES["w0"] - 160), dict(g0=PLACES["g1"]), dict(g0=PLACES["v1"] + 160)):
    _places(spb.lib(), **patch)
""")


# ---- tensors as Python hands them over --------------------------------------------------------------------------------

def test_tensors_in_host_memory_are_refused():
    with pytest.raises(ValueError, match="GPU"):
        spb.spb_muon_step([_tensor((300,), 0, torch.float32, 1, 0, device="cpu")], spb.muon_config(**HYPER), None, 0, 0)
    spb.spb_muon_step([], spb.muon_config(**HYPER), None, 0, 0)


@pytest.mark.gpu
def test_what_lies_elsewhere_or_is_too_small_is_refused_beside_tensors_on_the_gpu():
    a, b = _tensor((30, 40), 1, torch.bfloat16, 2, 0), _tensor((300,), 0, torch.float32, 1, 1)
    size = spb.spb_muon_workspace_size([a, b])
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for tensors in ([{**a, "w": a["w"].cpu()}, b], [a, {**b, "w": b["w"].cpu()}], [{**a, "m": a["m"].cpu()}, b], [a, {**b, "v": b["v"].cpu()}],
                    [{**a, "grads": [a["grads"][0], a["grads"][1].cpu()]}, b]):
        with pytest.raises(ValueError, match="GPU"):
            spb.spb_muon_step(tensors, spb.muon_config(**HYPER), ws, size, 0)
    for workspace in (ws.cpu(), ws[:size - 1]):
        with pytest.raises(ValueError, match="workspace"):
            spb.spb_muon_step([a, b], spb.muon_config(**HYPER), workspace, size, 0)


def test_lists_of_the_server_step_have_an_entry_per_parameter():
    """Shorter ones were read behind their end, on the host."""
    import workloads as wl
    m = spb.spb_model_create(spb.desc_from_config(wl.get_config("ragged_mlp_bf16")))
    try:
        n = spb.spb_param_count(m)
        spb.spb_bind_params(m, [(i + 1) << 32 for i in range(n)])
        blocks = [int(len(spb.spb_param_info(m, i)["shape"]) > 1) for i in range(n)]
        size = spb.spb_aggregate_muon_workspace_size(m, blocks)
        at = lambda k: [(k << 44) + (i << 32) for i in range(n)]
        good = dict(depths=[4, 2], worker_grads=[at(1), at(1)], blocks=blocks, first=at(2), second=at(3), workspace=1 << 60)
        for bad in (dict(worker_grads=[at(1)]), dict(worker_grads=[at(1), at(1)[1:]]), dict(blocks=blocks[1:]), dict(blocks=blocks + [1]), dict(first=at(2)[:-1]), dict(second=[]),
                    dict(workspace=torch.empty(size - 1, dtype=torch.uint8)), dict(workspace=torch.empty(size, dtype=torch.uint8))):
            with pytest.raises(ValueError):
                spb.spb_aggregate_muon(m, **{**good, **bad}, config=spb.muon_config(**HYPER), scale_lr=True, workspace_bytes=size, stream=0)
        with pytest.raises(ValueError):
            spb.spb_aggregate_muon_workspace_size(m, blocks[1:])
    finally:
        spb.spb_model_destroy(m)
