"""Pins for the oracle's head norm, rotary positions and orthogonalised update: finite differences, invariants, an independent singular value
decomposition, torch's AdamW."""
import numpy as np
import pytest
import torch

import oracle
import workloads as wl
from oracle import ops


def test_rotation_depends_on_differences_of_positions_and_keeps_lengths():
    rng = np.random.default_rng(0)
    for inter in (False, True):
        q, k = rng.standard_normal((2, 6, 1, 16))
        pos = rng.integers(-50, 50, (2, 6))
        both = [ops.rotate(t, ops.rotary_angles(p, [5, 2]), inter) for t, p in ((q, pos), (k, pos[:, ::-1]))]
        moved = [ops.rotate(t, ops.rotary_angles(p + 1000, [5, 2]), inter) for t, p in ((q, pos), (k, pos[:, ::-1]))]
        assert np.allclose((both[0] * both[1]).sum(-1), (moved[0] * moved[1]).sum(-1), atol=1e-9)
        assert np.allclose(np.linalg.norm(both[0], axis=-1), np.linalg.norm(q, axis=-1))
        assert np.array_equal(both[0][..., 14:], q[..., 14:])            # behind the last pair
        back = ops.rotate(both[0], -ops.rotary_angles(pos, [5, 2]), inter)
        assert np.allclose(back, q)
    a = ops.rotary_angles([[3], [7]], [2, 2], base=16.0)
    assert np.allclose(a, [[3, 3 / 2, 7 / 4, 7 / 8]])
    assert np.allclose(ops.rotary_angles([[3], [7]], [2, 2], base=16.0, own_ladder=True), [[3, 3 / 4, 7, 7 / 4]])


def test_finite_differences_of_an_encoder_with_norm_and_rotation():
    cfg = dict(wl.get_config("tiny_encoder"), hidden=16, qk_norm=1e-3, rotary=dict(sections=[1, 2], base=10.0, own_ladder=False, interleaved=False))
    p = {k: v.double().numpy().copy() for k, v in wl.make_params(cfg, seed=4, perturbed=True).items()}
    for name in p:
        if name.endswith("weight") and p[name].ndim == 2 and "qknorm" not in name:
            p[name] *= 12.0
    batch = wl.make_batch(cfg, seed=4)
    _, grads = oracle.spb_step(cfg, p, batch, wl.unit_count(cfg))
    assert set(grads) == set(p)
    for name in [n for n in p if "attn" in n or "ln1" in n]:
        arr, fd = p[name], np.zeros_like(p[name])
        for idx in np.ndindex(arr.shape):
            h, keep = 1e-6 * max(1.0, abs(arr[idx])), arr[idx]
            arr[idx] = keep + h
            up = oracle.spb_step(cfg, p, batch, 0)[0]
            arr[idx] = keep - h
            fd[idx] = (up - oracle.spb_step(cfg, p, batch, 0)[0]) / (2 * h)
            arr[idx] = keep
        assert np.abs(fd - grads[name]).max() / max(np.abs(fd).max(), 1e-12) < 2e-6, name


@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (7, 7), (1, 6), (6, 1)])
def test_orthogonalise_applies_the_quintic_to_singular_values(shape):
    u = np.random.default_rng(1).standard_normal(shape)
    left, s, right = np.linalg.svd(u, full_matrices=False)
    s = s / (np.linalg.norm(u) + 1e-7)
    for _ in range(5):
        s = 3.4445 * s - 4.7750 * s ** 3 + 2.0315 * s ** 5
    assert np.allclose(oracle.orthogonalise(u), left * s @ right, atol=1e-12)
    assert np.array_equal(oracle.orthogonalise(np.zeros(shape)), np.zeros(shape))


def test_adamw_is_torchs():
    rng = np.random.default_rng(2)
    w = torch.tensor(rng.standard_normal(11), dtype=torch.float64, requires_grad=True)
    opt = torch.optim.AdamW([w], lr=0.03, betas=(0.8, 0.9), eps=1e-6, weight_decay=0.1)
    mine, m, v = w.detach().numpy().copy(), np.zeros(11), np.zeros(11)
    for step in range(1, 5):
        g = rng.standard_normal((3, 11))
        w.grad = torch.tensor(g.mean(0))
        opt.step()
        mine, m, v = oracle.muon_step(mine, m, v, list(g), 0, 0.03, dict(beta1=0.8, beta2=0.9, adam_eps=1e-6, weight_decay=0.1, step=step))
        assert np.allclose(mine, w.detach().numpy(), atol=1e-13)
