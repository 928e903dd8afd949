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
