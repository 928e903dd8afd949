"""Calls of the heads' entries that share memory or bring tensors other than those described.  Values: the bits of the plain call, which test_heads.py holds to the oracle."""
import ctypes as C

import pytest
import torch

import paper_2111_10672_amd as spb
from paper_2111_10672_amd.binding import _check
from test_heads import CASES, Case
from test_host_streams import run, runtime  # noqa: F401


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n, c in CASES.items() if c.get("norm", True)])
def test_backward_in_place_of_x(name):
    print("case", name, flush=True)
    case = Case(**CASES[name])
    dx = torch.empty(case.x.shape, dtype=case.x.dtype, device="cuda")
    grads = case.backward(dx)
    x, spare = case.x, case.x.clone()
    again = case.backward(case.x)                                       # the kernel reads a row of x and writes dx in its place
    assert torch.equal(x, dx) and not torch.equal(x, spare)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)


def _place(entry, **patch):
    x = torch.empty(2, 3, 4, 16, dtype=torch.bfloat16)
    d = spb.heads_desc(x, 3, norm=True, rotary=spb.spb_rotary_sections([3, 5]))
    for k, v in patch.items():
        setattr(d, k, (C.c_int64 * 3)(*v))
    size = spb.spb_heads_workspace_size(d)
    if entry == "forward":
        _check(spb.lib().spb_heads_forward(C.byref(d), 4096, 4096, 1 << 20, 3, 0, 1 << 21, 0, None))
    elif entry == "of_dy":
        _check(spb.lib().spb_heads_backward(C.byref(d), 1 << 22, 4096, 4096, 1 << 20, 3, 0, 1 << 21, 1 << 23, 1 << 24, 1 << 25, size, None))
    else:
        _check(spb.lib().spb_heads_backward(C.byref(d), 4096, 1 << 22, 4096, 1 << 20, 3, 0, 1 << 21, 1 << 23, 1 << 24, 1 << 25, size, None))


@pytest.mark.parametrize("entry,patch", [("forward", dict(y_stride=[384, 64, 16])), ("forward", dict(x_stride=[0, 64, 16])), ("forward", dict(y_stride=[192, 16, 48])),
                                         ("of_dy", dict(dx_stride=[384, 64, 16])), ("of_dy", dict(y_stride=[192, 128, 32])), ("of_x", dict(dx_stride=[384, 64, 16])),
                                         ("of_x", dict(x_stride=[192, 0, 16]))])
def test_in_place_with_other_strides_is_refused(entry, patch):
    with pytest.raises(spb.SpbError) as e:
        _place(entry, **patch)
    assert e.value.code == -1 and "in place" in str(e.value)


def test_in_place_with_the_same_strides_is_taken(run):  # noqa: F811
    run("""
    def place(batch, back, **patch):
        d = spb.binding.spb_heads_desc()
        d.dtype, d.batch, d.seq, d.heads_q, d.heads_k, d.head_dim, d.norm, d.eps = 1, batch, 3, 3, 1, 16, 1, 1e-5
        d.x_stride, d.y_stride, d.dx_stride = [(C.c_int64 * 3)(*patch.get(n, (192, 64, 16))) for n in ("x", "y", "dx")]
        n = spb.spb_heads_workspace_size(d)
        if back:
            spb.binding._check(spb.lib().spb_heads_backward(d, 4096, 1 << 22, 4096, None, 0, 0, 1 << 21, 1 << 23, 1 << 24, 1 << 25, n, None))
        else:
            spb.binding._check(spb.lib().spb_heads_forward(d, 4096, 4096, None, 0, 0, 1 << 21, None, None))
    place(2, False)
    place(2, True, y=(256, 64, 16))
    place(1, False, y=(999, 64, 16))              # a stride that nothing steps by
    place(1, True, dx=(999, 64, 16))
    """)


def _refused(words, call):
    with pytest.raises(ValueError) as e:
        call()
    assert words in str(e.value), str(e.value)


X = torch.empty(2, 3, 7, 16, dtype=torch.bfloat16)[:, :, :4]
DENSE = torch.empty(2, 3, 4, 16, dtype=torch.bfloat16)
OTHERS = [torch.empty(2, 3, 4, 16, dtype=torch.bfloat16), torch.empty(2, 3, 4, 16), torch.empty(1, 3, 4, 16, dtype=torch.bfloat16), torch.empty(2, 3, 8, 8, dtype=torch.bfloat16),
          torch.empty(2, 4, 3, 16, dtype=torch.bfloat16).transpose(1, 2), torch.empty(2, 3, 4, 32, dtype=torch.bfloat16)[..., ::2], torch.empty(2, 3, 64, dtype=torch.bfloat16),
          torch.empty(0, 3, 4, 16, dtype=torch.bfloat16)]


@pytest.mark.parametrize("other", range(len(OTHERS)))
def test_tensors_other_than_described_are_refused(other):
    """y and dx default to x's strides: a dense y behind a description of a slice would be written out of range."""
    bad, rotary, pos = OTHERS[other], spb.spb_rotary_sections([8]), torch.zeros(1, 1, 3, dtype=torch.int32)
    of_slice, of_dense = spb.heads_desc(X, 3, rotary=rotary), spb.heads_desc(DENSE, 3, norm=True)
    if other:                                                           # (the first is as the dense description says)
        for call in (lambda: spb.spb_heads_forward(of_dense, bad, DENSE, None, torch.ones(2, 16, dtype=torch.bfloat16), None, 0),
                     lambda: spb.spb_heads_backward(of_dense, bad, DENSE, DENSE, None, None, None, None, None, 0, 0)):
            _refused("x: ", call)
    for call, name in ((lambda: spb.spb_heads_forward(of_slice, X, bad, pos, None, None, 0), "y"),
                       (lambda: spb.spb_heads_backward(of_slice, None, bad, X, pos, None, None, None, None, 0, 0), "dy"),
                       (lambda: spb.spb_heads_backward(of_slice, None, X, bad, pos, None, None, None, None, 0, 0), "dx")):
        _refused("described are", call)
        with pytest.raises(ValueError, match=f"^{name}: "):
            call()


def test_a_description_changed_by_hand_is_what_counts():
    d = spb.heads_desc(DENSE, 3, rotary=spb.spb_rotary_sections([8]))
    d.y_stride[1] = 128
    _refused("y: ", lambda: spb.spb_heads_forward(d, DENSE, DENSE, torch.zeros(1, 1, 3, dtype=torch.int32), None, None, 0))
    d.y_stride[1], d.seq = 64, 6
    _refused("x: ", lambda: spb.spb_heads_forward(d, DENSE, DENSE, torch.zeros(1, 1, 6, dtype=torch.int32), None, None, 0))


def test_tensors_in_host_memory_are_refused():
    d = spb.heads_desc(DENSE, 3, norm=True)
    gamma = torch.ones(2, 16, dtype=torch.bfloat16)
    _refused("on cpu", lambda: spb.spb_heads_forward(d, DENSE, DENSE, None, gamma, None, 0))
    _refused("on cpu", lambda: spb.spb_heads_backward(d, DENSE, DENSE, DENSE, None, gamma, gamma.float(), gamma.float(), None, 0, 0))


@pytest.mark.gpu
def test_what_lies_elsewhere_or_is_too_small_is_refused_beside_tensors_on_the_gpu():
    case = Case(2, 3, 3, 1, 16, sections=(8,))
    y = torch.empty_like(case.x)
    d = spb.heads_desc(case.x, 3, y=y, norm=True, rotary=case.rotary)
    size = spb.spb_heads_workspace_size(d)
    ws, grads = torch.empty(size, dtype=torch.uint8, device="cuda"), [torch.empty(2, 16, device="cuda") for _ in range(2)]
    forward = dict(x=case.x, y=y, pos=case.pos, gamma=case.gamma, beta=case.beta)
    backward = dict(x=case.x, dy=case.dy, dx=y, pos=case.pos, gamma=case.gamma, dgamma=grads[0], dbeta=grads[1], workspace=ws)
    for name in forward:
        _refused("on cpu", lambda: spb.spb_heads_forward(d, **{**forward, name: forward[name].cpu()}, stream=0))
    for name in backward:
        _refused("on cpu", lambda: spb.spb_heads_backward(d, **{**backward, name: backward[name].cpu()}, workspace_bytes=size, stream=0))
    _refused("bytes", lambda: spb.spb_heads_backward(d, **{**backward, "workspace": ws[:size - 1]}, workspace_bytes=size, stream=0))
    # a stride that nothing steps by may be any
    one = Case(1, 1, 3, 1, 16, sections=(8,))
    want, got = torch.empty_like(one.x), torch.empty_like(one.x)
    one.forward(want)
    odd = one.x.as_strided((1, 1, 4, 16), (7, 5, 16, 1))
    spb.spb_heads_forward(spb.heads_desc(one.x, 3, norm=True, rotary=one.rotary), odd, got, one.pos, one.gamma, one.beta, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(got, want)


def test_workspaces_smaller_than_said_are_refused():
    from paper_2111_10672_amd.binding import _workspace
    _refused("bytes", lambda: _workspace(torch.empty(99, dtype=torch.uint8), 100, -1))
    assert _workspace(None, 0, 0) is None and _workspace(1 << 20, 100, 0) == 1 << 20


def test_an_encoders_positions_are_those_of_its_tokens():
    """They are read by every later pass: fewer than the model's tokens would be read out of range."""
    import workloads as wl
    cfg = wl.get_config("small_encoder_bf16")
    b, s, rotary = cfg["batch"], cfg["seq"], spb.spb_rotary_sections([4, 4])
    m = spb.spb_model_create(spb.desc_from_config(cfg))
    try:
        for shape in ((2, 1, s - 1), (2, 1, s + 1), (2, b + 1, s), (1, b, s), (2, s), (2, b, s, 1)):
            _refused("positions", lambda: spb.spb_encoder_heads(m, rotary, torch.zeros(shape, dtype=torch.int32)))
        _refused("positions", lambda: spb.spb_encoder_heads(m, rotary, torch.zeros(2, b, s)))
        for shape in ((2, 1, s), (2, b, s), (3, b, s)):
            spb.spb_encoder_heads(m, rotary, torch.zeros(shape, dtype=torch.int32))
    finally:
        spb.spb_model_destroy(m)
