"""Every kernel behind the orthogonalised update against float64: which shapes reach which is asked of the library on a stand-in for the HIP runtime, and what each
makes of them is held entry by entry where the storage allows, and in the Frobenius norm over many steps.  The tolerances (muon_bounds.py) are a few per cent of
the update at most, and tests without a GPU show that they refuse a parameter left as it was and products with a part missing."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2111_10672_amd as spb
from muon_bounds import A, B, check_matrices, entry_room, frobenius_room, with_unit_columns
from muon_bounds import C as C5
from test_host_streams import run, runtime  # noqa: F401
from test_muon import HYPER, MATRICES, _numpy, _step, _tensor

BF16, F32 = torch.bfloat16, torch.float32

# (type, matrices, rows, columns) -> tile of the symmetric products, tile of the updates (32: its k shared by four wavefronts) and the stages of their rings
STACKS = {
    "bf16_32": ((BF16, 1, 290, 600), (32, 2), (32, 2)),
    "bf16_32_tall": ((BF16, 1, 600, 290), (32, 2), (32, 2)),
    "bf16_64": ((BF16, 8, 400, 420), (64, 6), (64, 6)),
    "bf16_64_tall": ((BF16, 8, 420, 400), (64, 6), (64, 6)),
    "bf16_128_alone": ((BF16, 4, 841, 1000), (128, 4), (128, 4)),
    "bf16_128_alone_tall": ((BF16, 4, 1000, 841), (128, 4), (128, 4)),
    "bf16_128_256": ((BF16, 16, 700, 760), (128, 2), (256, 2)),
    "bf16_128_256_tall": ((BF16, 16, 760, 700), (128, 2), (256, 2)),
    "bf16_256_128": ((BF16, 25, 651, 801), (256, 2), (128, 2)),
    "bf16_256_128_tall": ((BF16, 25, 801, 651), (256, 2), (128, 2)),
    "bf16_long": ((BF16, 4, 4096, 1024), (128, 4), (256, 2)),
    "f32_32": ((F32, 1, 300, 500), (32, 2), (32, 2)),
    "f32_32_tall": ((F32, 1, 500, 300), (32, 2), (32, 2)),
    "f32_64": ((F32, 6, 290, 330), (64, 4), (64, 4)),
    "f32_64_tall": ((F32, 6, 330, 290), (64, 4), (64, 4)),
    "f32_128": ((F32, 11, 590, 650), (128, 2), (128, 2)),
    "f32_128_tall": ((F32, 12, 770, 520), (128, 2), (128, 2)),
}
# the same for matrices of two launches a step: (threads' rows of the strips, tile of X X^T)
PAIRS = {
    "bf16_pair_64": ((BF16, 1, 36, 54), 64, 16),
    "bf16_pair_128": ((BF16, 2, 100, 300), 128, 16),
    "bf16_pair_128_many": ((BF16, 21, 73, 71), 128, 32),
    "bf16_pair_256": ((BF16, 1, 287, 160), 256, 16),
    "f32_pair_64": ((F32, 1, 54, 62), 64, 16),
    "f32_pair_128_many": ((F32, 15, 95, 72), 128, 32),
    "f32_pair_192": ((F32, 1, 158, 149), 256, 16),
    "f32_pair_256": ((F32, 1, 250, 600), 256, 16),
}

LAUNCHED = """
import re
from paper_2111_10672_amd.binding import spb_muon_tensor

def launched(bf16, blocks, rows, cols, steps=2):
    '''Kernels of a step, each with its template's numbers.'''
    t, g = (spb_muon_tensor * 1)(), (C.c_void_p * 1)(1 << 40)
    t[0].w, t[0].m, t[0].grads = 1 << 41, 1 << 42, C.cast(g, C.POINTER(C.c_void_p))
    t[0].rows, t[0].cols, t[0].rate_scale, t[0].count, t[0].dtype, t[0].blocks = blocks * rows, cols, 1.0, 1, bf16, blocks
    size = C.c_size_t()
    spb.binding._check(spb.lib().spb_muon_workspace_size(t, 1, C.byref(size)))
    hip.fake_clear()
    spb.binding._check(spb.lib().spb_muon_step(t, 1, C.byref(spb.muon_config(lr=0.1, ns_steps=steps)), 1 << 43, size.value, None))
    out = []
    for line in log():
        if line.startswith("launch"):
            name, numbers = re.search(r"\\d+([a-z_]+_kernel)(?:I(.*?)EEv)?", line).groups()
            out.append((name,) + tuple(int(n) for n in re.findall(r"L[ib](\\d+)E", (numbers or "") + "E")))
    return out
"""


def test_shapes_reach_every_product_kernel(run):  # noqa: F811
    wanted = {n: (s[0] == BF16, *s[1:], sym, upd) for n, (s, sym, upd) in STACKS.items()}
    run(LAUNCHED + f"""
wanted, seen = {wanted!r}, set()
for name, (bf16, blocks, rows, cols, sym, upd) in wanted.items():
    planes, got = 1 if bf16 else 2, launched(bf16, blocks, rows, cols)
    def product(mode, tile, stages):
        waves = (2, 4) if tile == 256 else (2, 2)
        return ("small_product_kernel", mode, planes, stages) if tile == 32 else ("product_kernel", mode, planes, tile, stages, *waves)
    steps = [product(0, *sym), product(1, *sym), product(2, *upd), product(0, *sym), product(1, *sym), product(3, *upd)]
    assert got == [("update_kernel",), ("normalise_kernel", planes, 0)] + steps, (name, got)
    seen |= set(steps)
rings = [(1, 64, 6, 2, 2), (1, 128, 4, 2, 2), (1, 128, 2, 2, 2), (1, 256, 2, 2, 4), (2, 64, 4, 2, 2), (2, 128, 2, 2, 2)]
every = {{("product_kernel", mode) + r for mode in range(4) for r in rings}} | {{("small_product_kernel", mode, p, 2) for mode in range(4) for p in (1, 2)}}
assert seen == every, every ^ seen
""")


def test_shapes_reach_every_kernel_of_two_launches_a_step(run):  # noqa: F811
    wanted = {n: (s[0] == BF16, *s[1:], rows, tile) for n, (s, rows, tile) in PAIRS.items()}
    run(LAUNCHED + f"""
seen = set()
for name, (bf16, blocks, rows, cols, most, tile) in {wanted!r}.items():
    planes, got = 1 if bf16 else 2, launched(bf16, blocks, rows, cols)
    gram, strips = [k for k in got if k[0] == "share_gram_kernel"], [k for k in got if k[0] == "pair_kernel"]
    assert [k[1:3] for k in gram] == [(planes, tile)] * 2 and strips == [("pair_kernel", 0, planes, most), ("pair_kernel", 1, planes, most)], (name, got)
    seen |= {{k[:3] for k in gram}} | set(strips)
assert len(seen) == 4 + 2 * 2 * 3, seen
""")


ALL = {**{n: s for n, (s, _a, _b) in STACKS.items()}, **{n: s for n, (s, _a, _b) in PAIRS.items()}}


def _one_step(name, steps, u):
    """The parameter after a step of `steps` products from zero, without momentum: minus the orthogonalised u, rounded once."""
    dtype, blocks, rows, cols = ALL[name]
    hyper = dict(HYPER, lr=1.0, rms=1.0 / math.sqrt(max(rows, cols)), momentum=0.0, nesterov=False, ns_steps=steps, weight_decay=0.0)
    t = dict(w=torch.zeros(blocks, rows, cols, dtype=dtype, device="cuda"), m=torch.zeros(blocks, rows, cols, device="cuda"), grads=[u.cuda()], blocks=blocks)
    _step([t], hyper)
    return hyper, t["w"]


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [1, 2])
@pytest.mark.parametrize("name", ALL)
def test_every_entry(name, steps):
    print("case", name, steps, flush=True)
    dtype, blocks, rows, cols = ALL[name]
    gen = torch.Generator().manual_seed(blocks + rows)
    u = torch.stack([with_unit_columns(rows, cols, gen) for _ in range(blocks)])
    hyper, w = _one_step(name, steps, u)
    again = _one_step(name, steps, u)[1]
    assert torch.equal(w, again)                                        # the same bits on every run
    half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    for k in range(blocks):
        want, room = entry_room(u[k].cuda().double(), dtype == BF16, hyper)
        got = -w[k].double()
        got = got if rows <= cols else got.T
        room = room + (half + 4 * 2.0 ** -24) * want.abs()
        assert bool(((got - want).abs() <= room).all()), (k, float(((got - want).abs() / room).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ALL)
def test_five_steps(name):
    print("case", name, flush=True)
    dtype, blocks, rows, cols = ALL[name]
    for rank in (0, 3):
        t = _tensor((blocks * rows, cols), blocks, dtype, 2, seed=rows, rank=rank)
        before = _numpy(t)
        _step([t])
        after = _numpy(t)
        for k in sorted({0, blocks // 2, blocks - 1}):                   # (a singular value decomposition each)
            cut = lambda x: x[k * rows:(k + 1) * rows]
            one = dict(w=cut(before["w"]), m=cut(before["m"]), grads=[cut(g) for g in before["grads"]], blocks=1)
            check_matrices(one, dict(w=cut(after["w"]), m=cut(after["m"])), dtype, HYPER, count=blocks)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", MATRICES)
def test_small_matrices(name, dtype):
    print("case", name, dtype, flush=True)
    for w in (0.0, 0.03):
        t = _tensor(dtype=dtype, seed=1, w=w, **MATRICES[name])
        before = _numpy(t)
        _step([t])
        check_matrices(before, _numpy(t), dtype, HYPER)


# Up to 8 steps on the Gram matrix in float64, more in products of the whole: the switch between them, and each against the formula.
STEPS = [(shape, steps) for shape in [(48, 150), (150, 33), (17, 17), (20, 300), (1, 9)] for steps in (3, 8, 9, 16)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,steps", STEPS)
def test_few_and_many_steps(shape, steps, dtype):
    print("case", shape, steps, dtype, flush=True)
    hyper = {**HYPER, "ns_steps": steps}
    t = _tensor(shape, 1, dtype, 2, seed=12, w=0.0)
    before = _numpy(t)
    _step([t], hyper)
    check_matrices(before, _numpy(t), dtype, hyper)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("patch", [dict(nesterov=False, momentum=0.0), dict(ns_steps=1), dict(ns_steps=2, weight_decay=0.0), dict(ns_steps=7, lr=0.5), dict(ns_eps=1.0)])
def test_settings(patch, dtype):
    hyper = {**HYPER, **patch}
    for shape in ((100, 140), (20, 30), (300, 320)):
        t = _tensor(shape, 1, dtype, 2, seed=2, w=0.0)
        before = _numpy(t)
        _step([{**t, "rate_scale": 0.75}], hyper)
        check_matrices(before, _numpy(t), dtype, hyper, 0.75)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_replayed_graphs(dtype):
    """Every way of forming the steps in one graph, replayed with the program's own work between."""
    shapes = [(1, 20, 300), (2, 100, 300), (1, 300, 310), (8, 420, 400), (16, 600, 640)]
    tensors = [_tensor((b * r, c), b, dtype, 2, seed=r) for b, r, c in shapes]
    start = [(t["w"].clone(), t["m"].clone()) for t in tensors]
    _step(tensors)                                                        # (company may change tiles, and with them the order of sums)
    want = [(t["w"].clone(), t["m"].clone()) for t in tensors]
    size = spb.spb_muon_workspace_size(tensors)
    ws, side = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            spb.spb_muon_step(tensors, spb.muon_config(**HYPER), ws, size, side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t, (w, m) in zip(tensors, start):
            t["w"].copy_(w)
            t["m"].copy_(m)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, (w, m) in zip(tensors, want):
            assert torch.equal(t["w"], w) and torch.equal(t["m"], m), t["w"].shape


# ---- what the tolerances refuse, without a GPU ------------------------------------------------------------------------

@pytest.mark.parametrize("steps,most", [(1, {BF16: 0.02, F32: 1e-4}), (2, {BF16: 0.15, F32: 1e-3})])
def test_the_bounds_of_entries_are_a_small_part_of_them(steps, most):
    for name, (dtype, _blocks, rows, cols) in ALL.items():
        if max(rows, cols) <= 1000:
            want, room = entry_room(with_unit_columns(rows, cols, torch.Generator().manual_seed(1)).double(), dtype == BF16, dict(HYPER, ns_steps=steps))
            room = room + 2.0 ** (-8 if dtype == BF16 else -24) * want.abs()
            assert float(room.norm() / want.norm()) <= most[dtype], name


def _refused(before, after, dtype, hyper):
    with pytest.raises(AssertionError) as e:
        check_matrices(before, after, dtype, hyper)
    return bool(e.value.args) and len(e.value.args[0]) == 4             # (too far off, not too much room)


def _momentum(before, hyper):
    return hyper["momentum"] * before["m"] + sum(before["grads"]) / len(before["grads"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", MATRICES)
def test_a_parameter_left_as_it_was_is_refused(name, dtype):
    case = dict(MATRICES[name])
    if case["blocks"] > 16:                                              # a few of them say as much
        per = case["shape"][0] // case["blocks"] if len(case["shape"]) == 2 else None
        case.update(blocks=4, shape=(4 * per, *case["shape"][1:]) if per else (4, *case["shape"][1:]))
    for w in (0.0, 0.03):
        before = _numpy(_tensor(dtype=dtype, seed=1, w=w, device="cpu", **case))
        assert _refused(before, dict(w=before["w"], m=_momentum(before, HYPER)), dtype, HYPER)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,steps", STEPS)
def test_a_parameter_left_as_it_was_is_refused_after_any_number_of_steps(shape, steps, dtype):
    hyper = {**HYPER, "ns_steps": steps}
    before = _numpy(_tensor(shape, 1, dtype, 2, seed=12, w=0.0, device="cpu"))
    assert _refused(before, dict(w=before["w"], m=_momentum(before, hyper)), dtype, hyper)
    if steps == 9:                                                       # and so is one step more or less
        for other in (8, 10):
            wrong = oracle.muon_step(before["w"], before["m"], None, before["grads"], 1, hyper["lr"], {**hyper, "ns_steps": other})
            assert _refused(before, dict(w=wrong[0], m=wrong[1]), dtype, hyper), other


def _steps_with(u, steps, spoil):
    """The orthogonalised u where spoil changes each A that a step forms, and each X."""
    x = u / np.linalg.norm(u)
    for k in range(steps):
        a = spoil("a", x @ x.T, k)
        x = spoil("x", (A * np.eye(len(a)) + B * a + C5 * a @ a) @ x, k)
    return x


def _no_mirror(what, v, k):
    """The mirror image of one 32 x 32 tile is not written."""
    if what == "a" and k == 0:
        v = v.copy()
        v[:32, 64:96] = 0.0
    return v


def _no_edge(what, v, k):
    """The rows behind the last whole tile of 64 are not formed."""
    if what == "x" and k == 0 and len(v) % 64:
        v = v.copy()
        v[len(v) // 64 * 64:] = 0.0
    return v


def _wrong_tile(what, v, k):
    """One tile of A holds another's values."""
    if what == "a" and k == 0:
        v = v.copy()
        v[96:128, :32] = v[128:160, :32]
        v[:32, 96:128] = v[96:128, :32].T
    return v


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("spoil", [_no_mirror, _no_edge, _wrong_tile])
@pytest.mark.parametrize("shape", [(290, 600), (300, 310)])
def test_products_with_a_part_missing_are_refused(shape, spoil, bf16):
    u = with_unit_columns(*shape, torch.Generator().manual_seed(3)).double()
    for steps in (1, 2):
        want, room = entry_room(u, bf16, dict(HYPER, ns_steps=steps))
        good = _steps_with(u.numpy(), steps, lambda what, v, k: v)
        assert np.allclose(good, want.numpy(), atol=1e-7)                # (ns_eps aside)
        room = room.numpy() + 2.0 ** (-8 if bf16 else -24) * np.abs(good)
        assert (np.abs(_steps_with(u.numpy(), steps, spoil) - want.numpy()) > room).any()


@pytest.mark.parametrize("bf16", [True, False])
def test_values_as_the_kernels_store_them_are_taken(bf16):
    """Steps in float64 whose X, A and B are rounded as the kernels' storage rounds them stay inside both bounds."""
    def stored(v, by):
        hi = (v * by).astype(np.float16).astype(np.float64)
        return (hi if bf16 else hi + ((v * by - hi) * 2048).astype(np.float16).astype(np.float64) / 2048) / by

    gen = torch.Generator().manual_seed(4)
    for u in (with_unit_columns(290, 300, gen).double().numpy(), 1e-3 * torch.randn(130, 520, generator=gen).double().numpy(), 1e-3 * torch.randn(66, 66, generator=gen).double().numpy()):
        sigma = 2.0 ** round(0.5 * math.log2(u.size))
        for steps in (1, 2, 5, 9):
            hyper = dict(HYPER, ns_steps=steps)
            x = stored(u / (np.linalg.norm(u) + hyper["ns_eps"]), sigma)
            for _ in range(steps):
                a = stored(x @ x.T, 1024.0)
                b = stored(A * np.eye(len(a)) + B * a + C5 * a @ a, 1024.0)
                x = stored(b @ x, sigma)
            want = oracle.orthogonalise(u, steps, hyper["ns_eps"])
            assert np.linalg.norm(x - want) <= frobenius_room(u, bf16, hyper)
            if steps <= 2:
                exact, room = entry_room(torch.from_numpy(u), bf16, hyper)
                assert np.allclose(exact.numpy(), want, atol=1e-12) and (np.abs(x - want) <= room.numpy()).all()
