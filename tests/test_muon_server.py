"""The oracle's server step with orthogonalised matrices: pinned on the CPU, and the library's held to it on the GPU."""
import math

import numpy as np
import pytest
import torch

import oracle
import paper_2111_10672_amd as spb
import workloads as wl
from muon_bounds import U, frobenius_room
from test_muon import HYPER, _blocks

UNITS, N_UNITS = {"a.weight": 0, "a.bias": 0, "b.weight": 1, "b.bias": 1, "c.weight": 2}, 3
BLOCKS = {"a.weight": 1, "a.bias": 0, "b.weight": 2, "b.bias": 0, "c.weight": 0}
SHAPES = {"a.weight": (6, 5), "a.bias": (6,), "b.weight": (8, 6), "b.bias": (8,), "c.weight": (3, 8)}


def _server(seed, workers):
    rng = np.random.default_rng(seed)
    make = lambda: {n: rng.standard_normal(s) for n, s in SHAPES.items()}
    return make(), make(), {n: v ** 2 for n, v in make().items()}, [make() for _ in range(workers)]


def test_parameters_that_nobody_reached_keep_everything():
    w, m, v, grads = _server(0, 2)
    new = oracle.aggregate_muon(UNITS, N_UNITS, w, m, v, grads, [1, 2], BLOCKS, HYPER, True)
    for n in ("a.weight", "a.bias"):
        assert all(np.array_equal(x[n], y[n]) for x, y in zip(new, (w, m, v)))
    assert not any(np.array_equal(new[0][n], w[n]) for n in ("b.weight", "b.bias", "c.weight"))


def test_gradients_of_workers_that_did_not_reach_a_parameter_are_not_read():
    w, m, v, grads = _server(1, 3)
    poisoned = [{n: np.full_like(g, np.nan) if UNITS[n] < N_UNITS - k else g for n, g in per.items()} for per, k in zip(grads, [1, 2, 3])]
    for scale in (True, False):
        a = oracle.aggregate_muon(UNITS, N_UNITS, w, m, v, grads, [1, 2, 3], BLOCKS, HYPER, scale)
        b = oracle.aggregate_muon(UNITS, N_UNITS, w, m, v, poisoned, [1, 2, 3], BLOCKS, HYPER, scale)
        assert all(np.array_equal(x[n], y[n]) for x, y in zip(a[:2], b[:2]) for n in SHAPES)


def test_the_rate_goes_by_the_share_of_workers_and_the_gradient_by_their_mean():
    """Matrices against their singular values, the rest against torch's AdamW, both for the one gradient that the contributors' mean is."""
    w, m, v, grads = _server(2, 4)
    zero = {n: np.zeros(s) for n, s in SHAPES.items()}
    depths, hyper = [0, 2, 3, 2], {**HYPER, "step": 1}
    for scale in (True, False):
        new, first, second = oracle.aggregate_muon(UNITS, N_UNITS, w, zero, zero, grads, depths, BLOCKS, hyper, scale)
        for n, unit in UNITS.items():
            who = [j for j, k in enumerate(depths) if unit >= N_UNITS - k]
            g = sum(grads[j][n] for j in who) / len(who)
            rate = hyper["lr"] * (len(who) / 4 if scale else 1.0)
            if BLOCKS[n] == 0:
                t = torch.tensor(w[n], requires_grad=True)
                t.grad = torch.tensor(g)
                torch.optim.AdamW([t], lr=rate, betas=(hyper["beta1"], hyper["beta2"]), eps=hyper["adam_eps"], weight_decay=hyper["weight_decay"]).step()
                assert np.allclose(new[n], t.detach().numpy(), atol=1e-13)
                continue
            assert np.array_equal(first[n], g) and second[n] is None
            for rows in np.split(np.arange(len(g)), BLOCKS[n]):
                left, s, right = np.linalg.svd((1 + hyper["momentum"]) * g[rows], full_matrices=False)
                s = s / (np.sqrt((s * s).sum()) + hyper["ns_eps"])
                for _ in range(5):
                    s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
                step = rate * hyper["rms"] * math.sqrt(max(len(rows), g.shape[1]))
                assert np.allclose(new[n][rows], (1 - rate * hyper["weight_decay"]) * w[n][rows] - step * (left * s @ right), atol=1e-12)


@pytest.mark.gpu
@pytest.mark.parametrize("name,depths,scale_lr", [("ragged_mlp_f32", [1, 2, 4], True), ("ragged_mlp_bf16", [2, 0, 4, 3], True), ("qk_encoder_bf16", [0, 1, 2, 3], False),
                                                  ("small_resnet_basic_bf16", [2, 3, 5], True)])
def test_server_step_against_the_oracles(name, depths, scale_lr):
    cfg = wl.get_config(name)
    params = wl.make_params(cfg, 0, perturbed=True)
    model = spb.SpbModel(cfg, params, positions=wl.make_batch(cfg, 0).get("positions"))
    names, units = [i["name"] for i in model.infos], {i["name"]: i["unit"] for i in model.infos}
    blocks = dict(zip(names, _blocks(model.infos)))
    first, second = wl.make_velocity(cfg, 0), {n: t ** 2 for n, t in wl.make_velocity(cfg, 1).items()}
    grads = wl.make_worker_grads(cfg, 0, len(depths))
    wide = lambda d: {n: t.double().numpy() for n, t in d.items()}
    want = oracle.aggregate_muon(units, model.n_units, wide(params), wide(first), wide(second), [wide(g) for g in grads], depths, blocks, HYPER, scale_lr)
    dev_m, dev_v = [first[n].cuda() for n in names], [second[n].cuda() for n in names]
    size = spb.spb_aggregate_muon_workspace_size(model.handle, list(blocks.values()))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    spb.spb_aggregate_muon(model.handle, depths, [[g[n].cuda() for n in names] for g in grads], list(blocks.values()), dev_m, dev_v, spb.muon_config(**HYPER), scale_lr, ws, size,
                           model.stream())
    torch.cuda.synchronize()
    for i, n in enumerate(names):
        w, m, v = (x.double().cpu().numpy() for x in (model.params[i], dev_m[i], dev_v[i]))
        who = [j for j, k in enumerate(depths) if units[n] >= model.n_units - k]
        if not who:
            assert np.array_equal(w, want[0][n]) and np.array_equal(m, want[1][n]) and np.array_equal(v, want[2][n]), n
            continue
        c, half = len(who), 2.0 ** (-8 if params[n].dtype == torch.bfloat16 else -24)
        rate = HYPER["lr"] * (c / len(depths) if scale_lr else 1.0)
        mean = sum(np.abs(grads[j][n].double().numpy()) for j in who) / c
        size_m = np.abs(first[n].double().numpy()) + mean
        assert (np.abs(m - want[1][n]) <= (c + 4) * U * size_m + 1e-44).all(), n
        if not blocks[n]:
            # as for AdamW's parameters alone: relative errors of m (of its magnitudes) and v carried into the quotient
            assert (np.abs(v - want[2][n]) <= (2 * c + 10) * U * (want[2][n] + mean ** 2) + 1e-44).all(), n
            root = np.sqrt(want[2][n] / (1 - HYPER["beta2"] ** HYPER["step"])) + HYPER["adam_eps"]
            off_v = (2 * c + 10) * U * (1 + mean ** 2 / np.maximum(want[2][n], 1e-300))
            room = half * np.abs(want[0][n]) + 4 * U * np.abs(params[n].double().numpy()) + rate * size_m / (1 - HYPER["beta1"] ** HYPER["step"]) / root * ((c + 16) * U + off_v)
            assert (np.abs(w - want[0][n]) <= room).all(), n
            continue
        assert torch.equal(dev_v[i].cpu(), second[n]), n                # not a matrix's
        g = sum(grads[j][n].double().numpy() for j in who) / c
        u = (g + HYPER["momentum"] * want[1][n]).reshape(len(g), -1)
        flat = lambda t: np.asarray(t).reshape(len(g), -1)
        for rows in np.split(np.arange(len(g)), blocks[n]):
            step = rate * HYPER["rms"] * math.sqrt(max(len(rows), u.shape[1]))
            room = step * frobenius_room(u[rows], params[n].dtype == torch.bfloat16, HYPER, blocks[n])
            room += half * np.linalg.norm(flat(want[0][n])[rows]) + 4 * U * np.linalg.norm(flat(params[n].double().numpy())[rows])
            assert np.linalg.norm(flat(w)[rows] - flat(want[0][n])[rows]) <= room, n
    model.close()
