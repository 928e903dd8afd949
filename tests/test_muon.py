"""The optimiser step with orthogonalised matrices through the C ABI: refusals on the host, values on the GPU against the oracle in float64.

Tolerances, with u = 2^-24.  Moments: two roundings an addition, (contributors + 4) u of the magnitudes.  AdamW: 16 u of rate |step| and 4 u of |w|, then half a
step of the storage type.  The orthogonalised matrix, in the Frobenius norm: the Newton-Schulz step's divided differences (p(s) - p(t)) / (s - t) and
(p(s) + p(t)) / (s + t) are at most L = 3.4445 in magnitude where singular values stay below 1.3, so an error grows at most L-fold a step; a step adds the
rounding of X, A and B to h relative (h = 2^-11 for bfloat16 parameters, 2^-21 for float32 ones: value and remainder, each product's remainder x remainder
left out) and that of its three sums (k / 16 + 16) u of |P| |Q| each.  A step of two launches rounds Z = b X + c A X in the place of B, and multiplies it by A:
h |Z| |A| where the other has h |B| |X|, of which `bound` takes the larger; its sums b X + A (c X) and A Z stay below those of B and B X.  `bound` adds these up along
the exact iterates.  Applied to w = 0, what is left is the storage type's half step."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2111_10672_amd as spb
import workloads as wl

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
HYPER = dict(lr=0.02, rms=0.2, momentum=0.9, nesterov=True, ns_steps=5, ns_eps=1e-7, beta1=0.9, beta2=0.95, adam_eps=1e-8, weight_decay=0.1, step=3)
GROWTH = 3.4445


def bound(u, dtype, hyper):
    """Frobenius bound of the error of the orthogonalised u."""
    h = 2.0 ** -11 if dtype == torch.bfloat16 else 2.0 ** -21
    x = np.asarray(u, dtype=np.float64)
    x = x if x.shape[0] <= x.shape[1] else x.T
    x = x / (np.linalg.norm(x) + hyper["ns_eps"])
    fro, two = np.linalg.norm, lambda a: np.linalg.norm(a, 2)
    chain = lambda k: (k / 16 + 16) * U
    err = (h + 64 * U) * fro(x)
    for _ in range(hyper["ns_steps"]):
        a = x @ x.T
        b = -4.7750 * a + 2.0315 * a @ a
        new = GROWTH * x + b @ x
        off_a = h * fro(a) + chain(x.shape[1]) * fro(x) ** 2
        off_b = (4.7750 + 2 * 2.0315 * two(a)) * off_a + 2.0315 * chain(len(a)) * fro(a) ** 2
        stored = h * max(fro(b) * two(x), two(a) * fro(-4.7750 * x + 2.0315 * a @ x))
        err = GROWTH * err + stored + off_b * two(x) + chain(len(a)) * fro(b) * fro(x) + (h + 4 * U) * fro(new)
        x = new
    return err


def _tensor(shape, blocks, dtype, workers, seed, w=0.03, rank=0, scale=1e-3, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)
    t = dict(w=(w * randn(*shape)).to(dtype), m=scale * randn(*shape), grads=[scale * randn(*shape) for _ in range(workers)], blocks=blocks)
    if rank:                                         # strong directions over a floor of noise
        strong = 5 * scale * randn(shape[0], rank) @ randn(rank, math.prod(shape[1:])).reshape(rank, -1)
        t["grads"] = [g + strong.reshape(shape) for g in t["grads"]]
    if blocks == 0:
        t["v"] = (scale * randn(*shape)) ** 2
    return {k: v.to(device) if torch.is_tensor(v) else [g.to(device) for g in v] if k == "grads" else v for k, v in t.items()}


def _numpy(t):
    return {k: v.double().cpu().numpy() if torch.is_tensor(v) else [g.double().cpu().numpy() for g in v] if k == "grads" else v for k, v in t.items()}


def _step(tensors, hyper=HYPER, stream=None):
    size = spb.spb_muon_workspace_size(tensors)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if size else None     # nothing may need to start at zero
    spb.spb_muon_step(tensors, spb.muon_config(**hyper), ws, size, torch.cuda.current_stream().cuda_stream if stream is None else stream)
    return ws


def _check(before, after, dtype, hyper=HYPER, rate_scale=1.0):
    blocks = before["blocks"]
    rate = hyper["lr"] * rate_scale
    flat = before["w"].reshape(before["w"].shape[0], -1) if not (blocks and before["w"].ndim == 3 and before["w"].shape[0] == blocks) else before["w"].reshape(-1, before["w"].shape[-1])
    shape = flat.shape
    old = {k: v.reshape(shape) if isinstance(v, np.ndarray) else [g.reshape(shape) for g in v] if k == "grads" else v for k, v in before.items()}
    new = {k: v.reshape(shape) if isinstance(v, np.ndarray) else v for k, v in after.items()}
    w, m, v = oracle.muon_step(old["w"], old["m"], old.get("v"), old["grads"], blocks, rate, hyper)
    n = len(old["grads"])
    size = np.abs(old["m"]) + sum(np.abs(g) for g in old["grads"]) / n
    assert (np.abs(new["m"] - m) <= (n + 4) * U * size + 1e-44).all()
    if blocks == 0:
        assert (np.abs(new["v"] - v) <= (2 * n + 10) * U * (v + (sum(np.abs(g) for g in old["grads"]) / n) ** 2) + 1e-44).all()
        # the root halves v's relative error; where gradients cancel, m's error is relative to their magnitudes
        root = np.sqrt(v / (1 - hyper["beta2"] ** hyper["step"])) + hyper["adam_eps"]
        step = size / (1 - hyper["beta1"] ** hyper["step"]) / root
        off_v = (2 * n + 10) * U * (1 + (sum(np.abs(g) for g in old["grads"]) / n) ** 2 / np.maximum(v, 1e-300))
        tol = HALF[dtype] * np.abs(w) + 4 * U * np.abs(old["w"]) + rate * step * ((n + 16) * U + off_v)
        assert (np.abs(new["w"] - w) <= tol).all()
        return
    r, c = shape[0] // blocks, shape[1]
    u = (sum(old["grads"]) / n + hyper["momentum"] * m if hyper["nesterov"] else m).reshape(blocks, r, c)
    for k in range(blocks):
        rows = slice(k * r, (k + 1) * r)
        step = rate * hyper["rms"] * math.sqrt(max(r, c))
        far = np.linalg.norm(new["w"][rows] - w[rows])
        room = step * bound(u[k], dtype, hyper) + HALF[dtype] * np.linalg.norm(w[rows]) + 4 * U * np.linalg.norm(old["w"][rows])
        assert far <= room, (k, far, room)


MATRICES = {
    "one_entry": dict(shape=(1, 1), blocks=1, workers=1),
    "one_row": dict(shape=(1, 70), blocks=1, workers=2),
    "one_column": dict(shape=(70, 1), blocks=1, workers=2),
    "rows_apart": dict(shape=(5, 33), blocks=5, workers=1),
    "small": dict(shape=(17, 23), blocks=1, workers=3),
    "small_tall": dict(shape=(61, 40), blocks=1, workers=8),
    "tile": dict(shape=(64, 64), blocks=1, workers=1, rank=2),
    "beyond_tile": dict(shape=(65, 129), blocks=1, workers=2, rank=3),
    "qkv": dict(shape=(3 * 72, 72), blocks=3, workers=2),
    "stack": dict(shape=(4, 130, 100), blocks=4, workers=1),
    "tall_stack": dict(shape=(3, 200, 136), blocks=3, workers=2, rank=2),
    "wide": dict(shape=(130, 520), blocks=1, workers=4, rank=4),
    "tall": dict(shape=(700, 256), blocks=1, workers=1),
    "square": dict(shape=(384, 384), blocks=1, workers=2, rank=8),
    "stem": dict(shape=(64, 7, 7, 3), blocks=1, workers=2),
    "conv": dict(shape=(96, 3, 3, 24), blocks=1, workers=1),
    "narrow_33_wide": dict(shape=(33, 8192), blocks=1, workers=1, rank=2),
    "vector": dict(shape=(150,), blocks=1, workers=1),
    "stack_64": dict(shape=(70 * 60, 90), blocks=70, workers=1),
    "stack_192": dict(shape=(3, 190, 300), blocks=3, workers=2, rank=2),
    "stack_128": dict(shape=(24, 140, 120), blocks=24, workers=1),
    "stack_256": dict(shape=(16, 250, 600), blocks=16, workers=1, rank=2),
    "long_64": dict(shape=(2, 5000, 57), blocks=2, workers=1, rank=1),
    "narrow_16": dict(shape=(16, 1000), blocks=1, workers=2, rank=3),
    "narrow_33": dict(shape=(5 * 33, 130), blocks=5, workers=1),
    "narrow_48_long": dict(shape=(48, 8192), blocks=1, workers=1, rank=2),
    "narrow_48_longer": dict(shape=(8200, 48), blocks=1, workers=1, rank=2),
    "beyond_narrow": dict(shape=(300, 49), blocks=1, workers=1, rank=2),
    "narrow_48_tall": dict(shape=(2, 777, 48), blocks=2, workers=3),
    "many_narrow": dict(shape=(257, 8, 24), blocks=257, workers=1),
    "most_narrow": dict(shape=(256, 20, 24), blocks=256, workers=1),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", MATRICES)
def test_matrices(name, dtype):
    print("case", name, dtype, flush=True)
    for w in (0.0, 0.03):
        t = _tensor(dtype=dtype, seed=1, w=w, **MATRICES[name])
        before = _numpy(t)
        _step([t])
        _check(before, _numpy(t), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("patch", [dict(nesterov=False, momentum=0.0), dict(ns_steps=1), dict(ns_steps=2, weight_decay=0.0), dict(ns_steps=7, lr=0.5), dict(ns_eps=1.0)])
def test_settings(patch, dtype):
    hyper = {**HYPER, **patch}
    t = _tensor((100, 140), 1, dtype, 2, seed=2, w=0.0)
    t["rate_scale"] = 0.75
    before = _numpy({k: v for k, v in t.items() if k != "rate_scale"})
    _step([t], hyper)
    _check(before, _numpy({k: v for k, v in t.items() if k != "rate_scale"}), dtype, hyper, 0.75)


# Entry by entry, for the two float16 of a float32 parameter: err bounds |error of X| and grows with every product P Q by |dP| |Q| + |P| |dQ| + chain |P| |Q|, with
# every matrix stored by 2^-21 of each entry (the remainder x remainder that its products leave out among it) and 2^-40 for entries so small that the remainder,
# in steps of 2^-35 at sigma or tau times the entry, is short of bits.  A remainder taken from another rounding than that of
# the stored value is off by a step of float16, 2^-11 of the entry at least, which no later product takes back.
@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(64, 4000), (128, 512), (512, 96), (130, 1031)])
@pytest.mark.parametrize("steps", [1, 2])
def test_every_entry_of_a_float32_matrix(shape, steps):
    hyper = dict(HYPER, lr=1.0, rms=1.0 / math.sqrt(max(shape)), momentum=0.0, nesterov=False, ns_steps=steps, weight_decay=0.0)
    t = _tensor(shape, 1, torch.float32, 1, 77)
    t["w"].zero_()
    u = t["grads"][0].double().cpu().numpy()
    _step([t], hyper)
    got = -t["w"].double().cpu().numpy()
    if shape[0] > shape[1]:
        u, got = u.T, got.T
    h, tiny = 2.0 ** -21, 2.0 ** -40
    chain = lambda k: (k / 16 + 16) * U
    x = u / (np.linalg.norm(u) + hyper["ns_eps"])
    err = (h + 4 * U) * np.abs(x) + tiny
    for _ in range(steps):
        a = x @ x.T
        off_a = err @ np.abs(x.T) + np.abs(x) @ err.T + chain(x.shape[1]) * np.abs(x) @ np.abs(x.T)
        stored_a = off_a + h * np.abs(a) + tiny
        b = -4.7750 * a + 2.0315 * a @ a
        off_b = 4.7750 * stored_a + 2.0315 * (stored_a @ np.abs(a) + np.abs(a) @ stored_a + chain(len(a)) * np.abs(a) @ np.abs(a)) + 8 * U * np.abs(b)
        b = b + GROWTH * np.eye(len(a))
        off_b += h * np.abs(b) + tiny
        err = off_b @ np.abs(x) + np.abs(b) @ err + chain(len(a)) * np.abs(b) @ np.abs(x)
        x = b @ x
        err += (h + 4 * U) * np.abs(x) + tiny
    assert (np.abs(got - x) <= err).all(), float((np.abs(got - x) / err).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape", [(48, 150), (150, 33), (17, 17), (1, 9)])
def test_a_short_side_in_one_and_in_many_products(shape, dtype):
    """Up to 8 steps may run on the small Gram matrix, more as products of the whole: both against the formula, whose 8 and 9 steps differ."""
    for steps in (1, 2, 3, 8, 9, 16):
        hyper = {**HYPER, "ns_steps": steps}
        t = _tensor(shape, 1, dtype, 2, seed=12, w=0.0)
        before = _numpy(t)
        _step([t], hyper)
        _check(before, _numpy(t), dtype, hyper)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("numel,workers", [(1, 1), (3, 8), (1000, 2), (2049, 4), (100003, 3)])
def test_adamw(numel, workers, dtype):
    t = _tensor((numel,), 0, dtype, workers, seed=3)
    before = _numpy(t)
    _step([t])
    _check(before, _numpy(t), dtype)


@pytest.mark.gpu
def test_many_tensors_of_all_kinds_at_once():
    """More tensors than a launch's table holds, of one shape and of many, both types, matrices and others in turn."""
    tensors = []
    for i in range(40):
        shape, blocks = [((40 + i, 70), 1), ((33, 2 * i + 1), 0), ((3 * 64, 64), 3), ((150, 130), 1), ((7 + i,), 0)][i % 5]
        tensors.append(_tensor(shape, blocks, torch.float32 if i % 3 == 0 else torch.bfloat16, 1 + i % 8, seed=10 + i))
    before = [_numpy(t) for t in tensors]
    alone = []
    for t in tensors:
        one = {k: v.clone() if torch.is_tensor(v) else v for k, v in t.items()}
        _step([one])
        alone.append(one)
    _step(tensors)
    for b, t, one in zip(before, tensors, alone):
        _check(b, _numpy(t), t["w"].dtype)
        assert torch.equal(t["w"], one["w"]) and torch.equal(t["m"], one["m"])     # company changes no bits


@pytest.mark.gpu
@pytest.mark.parametrize("sides", [(3, 40), (60, 90), (260, 300)])
def test_more_shapes_than_a_launch_holds(sides):
    tensors = [_tensor((sides[0] + i, sides[1]), 1, torch.bfloat16 if i % 2 else torch.float32, 1 + i % 3, seed=40 + i, w=0.0) for i in range(56)]
    before = [_numpy(t) for t in tensors]
    _step(tensors)
    for b, t in zip(before, tensors):
        _check(b, _numpy(t), t["w"].dtype)


@pytest.mark.gpu
def test_tensors_at_odd_addresses():
    for dtype in (torch.bfloat16, torch.float32):
        for blocks, shape in ((1, (30, 41)), (0, (1229,))):
            t = _tensor(shape, blocks, dtype, 2, seed=4)
            want = {k: v.clone() if torch.is_tensor(v) else v for k, v in t.items()}
            _step([want])
            n = math.prod(shape)
            shift = lambda x: torch.cat([x.new_zeros(1), x.reshape(-1)])[1:1 + n].reshape(shape)
            t = {k: shift(v) if torch.is_tensor(v) else [shift(g) for g in v] if k == "grads" else v for k, v in t.items()}
            _step([t])
            assert torch.equal(t["w"], want["w"]) and torch.equal(t["m"], want["m"])


@pytest.mark.gpu
def test_gradients_of_zeros_of_extreme_size_and_not_numbers():
    for dtype in (torch.bfloat16, torch.float32):
        t = _tensor((70, 90), 1, dtype, 1, seed=5)
        t["m"].zero_()
        t["grads"][0].zero_()
        before = _numpy(t)
        _step([t])
        _check(before, _numpy(t), dtype)                      # only the decay
        for scale in (1e-28, 1e30):                           # squares leave float32's range; ns_eps matters for the first
            t = _tensor((70, 90), 1, dtype, 2, seed=6, w=0.0, scale=scale)
            hyper = {**HYPER, "ns_eps": 1e-35}
            before = _numpy(t)
            _step([t], hyper)
            _check(before, _numpy(t), dtype, hyper)
        a, b = _tensor((70, 90), 1, dtype, 1, seed=7), _tensor((70, 90), 1, dtype, 1, seed=8)
        a["grads"][0][3, 4] = float("nan")
        before = _numpy(b)
        _step([a, b])
        assert a["w"].isnan().all()
        _check(before, _numpy(b), dtype)                      # the other matrix of the launch does not see it


@pytest.mark.gpu
def test_replayed_graph_and_other_stream():
    tensors = [_tensor((200, 130), 1, torch.bfloat16, 2, seed=9), _tensor((300,), 0, torch.bfloat16, 2, seed=10), _tensor((60, 60), 1, torch.float32, 1, seed=11)]
    start = [{k: v.clone() for k, v in t.items() if k in ("w", "m", "v")} for t in tensors]
    reset = lambda: [t[k].copy_(v) for t, s in zip(tensors, start) for k, v in s.items()]
    _step(tensors)
    want = [{k: t[k].clone() for k in s} for t, s in zip(tensors, start)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        reset()
        ws = _step(tensors, stream=side.cuda_stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            spb.spb_muon_step(tensors, spb.muon_config(**HYPER), ws, ws.numel(), side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        reset()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip(tensors, want):
            assert all(torch.equal(t[k], w[k]) for k in w)


def _blocks(infos):
    """Matrices of the hidden layers by Newton-Schulz, queries, keys and values apart; embeddings, the head, norms and biases by AdamW."""
    return [0 if len(i["shape"]) < 2 or "embed" in i["name"] or "head" in i["name"] or "qknorm" in i["name"] else 3 if "qkv" in i["name"] else 1 for i in infos]


@pytest.mark.gpu
@pytest.mark.parametrize("name,depths,scale_lr", [("ragged_mlp_f32", [1, 2, 4], True), ("ragged_mlp_bf16", [4, 4], False), ("qk_encoder_bf16", [0, 1, 2, 3], True),
                                                  ("small_resnet_basic_bf16", [2, 3, 5], True)])
def test_server_step_of_a_model(name, depths, scale_lr):
    cfg = wl.get_config(name)
    params = wl.make_params(cfg, 0, perturbed=True)
    model = spb.SpbModel(cfg, params, positions=wl.make_batch(cfg, 0).get("positions"))
    names, units = [i["name"] for i in model.infos], {i["name"]: i["unit"] for i in model.infos}
    blocks = _blocks(model.infos)
    first, second = wl.make_velocity(cfg, 0), {n: t ** 2 for n, t in wl.make_velocity(cfg, 1).items()}
    grads = wl.make_worker_grads(cfg, 0, len(depths))
    dev_m = [first[n].cuda() for n in names]
    dev_v = [None if b else second[n].cuda() for n, b in zip(names, blocks)]
    # below a worker's cut its buffers are poisoned: they must never be read
    dev_g = [[g[n].cuda() if units[n] >= model.n_units - k else torch.full(g[n].shape, float("nan"), device="cuda") for n in names] for g, k in zip(grads, depths)]
    size = spb.spb_aggregate_muon_workspace_size(model.handle, blocks)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    spb.spb_aggregate_muon(model.handle, depths, dev_g, blocks, dev_m, dev_v, spb.muon_config(**HYPER), scale_lr, ws, size, model.stream())
    torch.cuda.synchronize()
    for i, n in enumerate(names):
        who = oracle.contributors(units[n], model.n_units, depths)
        if not who:
            assert torch.equal(model.params[i].cpu(), params[n]) and torch.equal(dev_m[i].cpu(), first[n])
            continue
        before = dict(w=params[n].double().numpy(), m=first[n].double().numpy(), grads=[grads[j][n].double().numpy() for j in who], blocks=blocks[i])
        after = dict(w=model.params[i].double().cpu().numpy(), m=dev_m[i].double().cpu().numpy())
        if not blocks[i]:
            before["v"], after["v"] = second[n].double().numpy(), dev_v[i].double().cpu().numpy()
        _check(before, after, params[n].dtype, rate_scale=len(who) / len(depths) if scale_lr else 1.0)
    model.close()


@pytest.mark.gpu
def test_iterations_of_an_encoder_with_heads_and_muon():
    """The operators as a training job uses them: three workers' truncated steps of an encoder whose heads are normed and turned, the server's orthogonalised
    step, twice over, each server step against the oracle's on the gradients the GPU formed."""
    cfg = wl.get_config("qk_encoder_bf16")
    params, batches = wl.make_params(cfg, 0, perturbed=True), [wl.make_batch(cfg, j) for j in range(3)]
    model = spb.SpbModel(cfg, params, positions=batches[0]["positions"])
    names, blocks = [i["name"] for i in model.infos], _blocks(model.infos)
    units = {i["name"]: i["unit"] for i in model.infos}
    depths = [spb.spb_worker_depth(model.handle, j, 3) for j in (1, 2, 3)]
    bufs = [[torch.full_like(g, float("nan")) for g in model.grads] for _ in depths]
    first = [torch.zeros_like(g) for g in model.grads]
    second = [torch.zeros_like(g) for g in model.grads]
    size = spb.spb_aggregate_muon_workspace_size(model.handle, blocks)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for it in (1, 2):
        hyper = {**HYPER, "step": it}
        for j, k in enumerate(depths):
            spb.spb_bind_grads(model.handle, bufs[j])
            model.step({n: t.cuda() for n, t in batches[j].items() if n != "positions"}, k)
        before = [(p.double().cpu().numpy(), a.double().cpu().numpy(), b.double().cpu().numpy()) for p, a, b in zip(model.params, first, second)]
        spb.spb_aggregate_muon(model.handle, depths, bufs, blocks, first, second, spb.muon_config(**hyper), True, ws, size, model.stream())
        torch.cuda.synchronize()
        for i, n in enumerate(names):
            who = oracle.contributors(units[n], model.n_units, depths)
            g = [bufs[j][i].double().cpu().numpy() for j in who]
            assert all(np.isfinite(x).all() for x in g), n
            after = dict(w=model.params[i].double().cpu().numpy(), m=first[i].double().cpu().numpy(), v=second[i].double().cpu().numpy())
            _check(dict(w=before[i][0], m=before[i][1], v=before[i][2], grads=g, blocks=blocks[i]), after, torch.bfloat16, hyper, len(who) / 3)
    model.close()


# ---- refusals: all found on the host --------------------------------------------------------------------------------

def test_tensors_and_settings_that_are_refused():
    from paper_2111_10672_amd.binding import _check as check
    lib = spb.lib()
    grads = (C.c_void_p * 2)(256, 512)

    def call(n=1, ws=256, size=1 << 20, config=None, twice=False, **patch):
        arr = (spb.binding.spb_muon_tensor * 2)()
        for a, w in zip(arr, (1024, 1024 if twice else 2048)):
            a.w, a.m, a.v, a.grads, a.rows, a.cols, a.rate_scale, a.count, a.dtype, a.blocks = w, 256, 256, C.cast(grads, C.POINTER(C.c_void_p)), 6, 5, 1.0, 2, 1, 1
            for k, v in patch.items():
                setattr(a, k, v)
        check(lib.spb_muon_step(arr, n, C.byref(spb.muon_config(**{**HYPER, **(config or {})})), ws, size, 0))

    for patch in (dict(rows=0), dict(cols=0), dict(rows=1 << 31), dict(rows=1 << 62), dict(rows=131073 * 4, blocks=131073, n=1), dict(blocks=-1), dict(blocks=4), dict(rows=65537, blocks=1), dict(cols=65537), dict(dtype=2), dict(count=0), dict(count=9),
                  dict(grads=None), dict(w=0), dict(w=1025), dict(m=0), dict(m=258), dict(v=0, blocks=0), dict(v=257, blocks=0), dict(rate_scale=-1.0), dict(rate_scale=float("nan")),
                  dict(n=-1), dict(n=2, twice=True), dict(n=2), dict(blocks=0)):      # (m and v are at one address)
        with pytest.raises(spb.SpbError) as e:
            call(**patch)
        assert e.value.code == -1, patch
    for config in (dict(lr=float("nan")), dict(rms=float("inf")), dict(momentum=float("nan")), dict(beta1=1.0), dict(beta2=-0.1), dict(ns_eps=0.0), dict(adam_eps=0.0), dict(step=0),
                   dict(ns_steps=0), dict(ns_steps=17), dict(weight_decay=float("inf"))):
        with pytest.raises(spb.SpbError) as e:
            call(config=config)
        assert e.value.code == -1, config
    for patch in (dict(ws=0), dict(ws=128), dict(size=100)):
        with pytest.raises(spb.SpbError) as e:
            call(**patch)
        assert e.value.code == -4, patch
    grads[1] = 0
    with pytest.raises(spb.SpbError) as e:
        call()
    assert e.value.code == -1 and "gradient 1" in str(e.value)
    check(lib.spb_muon_step(None, 0, C.byref(spb.muon_config(**HYPER)), 0, 0, 0))             # nothing to do
    with pytest.raises(spb.SpbError):
        check(lib.spb_muon_step(None, 0, None, 0, 0, 0))


def test_workspace_sizes():
    t = _tensor((96, 3, 3, 24), 1, torch.bfloat16, 1, 0, device="cpu")
    flat = _tensor((96, 216), 1, torch.bfloat16, 1, 0, device="cpu")
    assert spb.spb_muon_workspace_size([t]) == spb.spb_muon_workspace_size([flat]) > 96 * 216 * 4
    assert spb.spb_muon_workspace_size([_tensor((50,), 0, torch.float32, 1, 0, device="cpu")]) == 0 == spb.spb_muon_workspace_size([])
    wide = _tensor((96, 216), 1, torch.float32, 1, 0, device="cpu")
    assert spb.spb_muon_workspace_size([wide]) > spb.spb_muon_workspace_size([flat])
    for bad in (dict(m=flat["m"].T), dict(m=flat["m"].reshape(216, 96)), dict(grads=[flat["grads"][0].double()]), dict(w=flat["w"].T)):
        with pytest.raises(ValueError):
            spb.spb_muon_step([{**flat, **bad}], spb.muon_config(**HYPER), None, 0, 0)


def test_server_step_arguments():
    cfg = wl.get_config("ragged_mlp_bf16")
    m = spb.spb_model_create(spb.desc_from_config(cfg))
    try:
        n = spb.spb_param_count(m)
        blocks, ptr = [1] * n, [256] * n
        size = spb.spb_aggregate_muon_workspace_size(m, blocks)
        config = spb.muon_config(**HYPER)
        with pytest.raises(spb.SpbError) as e:                     # 200 rows in 3 blocks
            spb.spb_aggregate_muon_workspace_size(m, [3] + blocks[1:])
        assert e.value.code == -1
        with pytest.raises(spb.SpbError) as e:
            spb.spb_aggregate_muon(m, [4], [ptr], blocks, ptr, ptr, config, True, 256, size, 0)
        assert e.value.code == -3                                  # not bound
        spb.spb_bind_params(m, [256 * (i + 1) for i in range(n)])
        for depths, g, first, second, ws, bytes_, code in (([5], ptr, ptr, ptr, 256, size, -2), ([-1], ptr, ptr, ptr, 256, size, -2), ([4] * 9, ptr, ptr, ptr, 256, size, -1),
                                                           ([4], [None] * n, ptr, ptr, 256, size, -1), ([4], ptr, [None] * n, ptr, 256, size, -1),
                                                           ([4], ptr, ptr, ptr, 256, size - 1, -4), ([4], ptr, ptr, ptr, None, size, -4)):
            with pytest.raises(spb.SpbError) as e:
                spb.spb_aggregate_muon(m, depths, [g] * len(depths), blocks, first, second, config, True, ws, bytes_, 0)
            assert e.value.code == code, (depths, code)
        with pytest.raises(spb.SpbError) as e:
            spb.spb_aggregate_muon(m, [4], [ptr], [0] * n, ptr, [None] * n, config, True, None, 0, 0)
        assert e.value.code == -1
    finally:
        spb.spb_model_destroy(m)

@pytest.mark.parametrize("dtype,dims", [("bf16", [56, 64, 8, 1192, 8]), ("bf16", [64, 104, 24, 2400, 8, 48]), ("f32", [232, 160, 2712, 568, 8])])
def test_the_server_steps_workspace_covers_every_depth(dtype, dims):
    """Few tensors can need more than many: their matrices are padded for themselves."""
    cfg = dict(family="mlp", dtype=dtype, batch=4, dims=dims)
    m = spb.spb_model_create(spb.desc_from_config(cfg))
    try:
        infos = [spb.spb_param_info(m, i) for i in range(spb.spb_param_count(m))]
        blocks = [int(len(p["shape"]) > 1) for p in infos]
        size = spb.spb_aggregate_muon_workspace_size(m, blocks)
        stored = torch.bfloat16 if dtype == "bf16" else torch.float32
        for unit in range(len(dims) - 1):
            some = [dict(w=torch.empty(p["shape"], dtype=stored), blocks=b) for p, b in zip(infos, blocks) if p["unit"] >= unit]
            assert spb.spb_muon_workspace_size(some) <= size, unit
    finally:
        spb.spb_model_destroy(m)
