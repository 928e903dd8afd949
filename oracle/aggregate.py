"""Parameter-server side of one SPB iteration on the CPU (oracle side, test infrastructure).

Sec. 2 of the paper: every worker sends the gradients of the suffix it backpropagated; the server averages each
layer's gradient over the workers that contributed to it, scales the learning rate with that number, and updates
its copy of the model.  Sec. 4.1 names the optimizer: SGD with momentum and weight decay.  Everything is float64;
`q` rounds a parameter to its storage type after the update (identity, or round_to_bf16).

Readings where the paper is silent: worker j of K backpropagates ceil(j L / K) units (rounded up, so that worker K
is always complete); the learning rate of a parameter with c contributors is lr * c / K; the update is
v <- mu v + (g + wd w), w <- w - rate v (no dampening, no Nesterov term); a parameter without contributors is left
as it is, velocity included.
"""
from __future__ import annotations

import math

import numpy as np


def worker_depths(n_units: int, n_workers: int) -> list:
    """Depth (units from the output end) of workers 1..K: ceil(j L / K)."""
    return [math.ceil(j * n_units / n_workers) for j in range(1, n_workers + 1)]


def contributors(unit: int, n_units: int, depths) -> list:
    """Indices of the workers whose suffix reaches down to `unit`."""
    return [j for j, k in enumerate(depths) if unit >= n_units - k]


def aggregate_update(param_units: dict, n_units: int, params: dict, velocity: dict, worker_grads: list, depths,
                     lr: float, momentum: float, weight_decay: float, scale_lr: bool, q=lambda a: a):
    """One server step.  param_units: name -> owning unit.  Returns (new params, new velocity) as float64 arrays."""
    new_w, new_v = {}, {}
    n_workers = len(depths)
    for name, unit in param_units.items():
        w = np.asarray(params[name], dtype=np.float64)
        v = np.asarray(velocity[name], dtype=np.float64)
        who = contributors(unit, n_units, depths)
        if not who:
            new_w[name], new_v[name] = w.copy(), v.copy()
            continue
        g = np.zeros_like(w)
        for j in who:
            g = g + np.asarray(worker_grads[j][name], dtype=np.float64)
        g = g / len(who)
        rate = lr * len(who) / n_workers if scale_lr else lr
        v = momentum * v + (g + weight_decay * w)
        new_v[name] = v
        new_w[name] = q(w - rate * v)
    return new_w, new_v


def orthogonalise(u, steps: int = 5, eps: float = 1e-7):
    """Newton-Schulz: X = u / (|u|_F + eps), then `steps` times X <- p(X), the odd quintic p(s) = 3.4445 s - 4.7750 s^3 + 2.0315 s^5 applied to the
    singular values, which lets those of a full-rank matrix end near 1."""
    x = np.asarray(u, dtype=np.float64)
    x = x / (np.sqrt((x * x).sum()) + eps)
    for _ in range(steps):
        gram = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
        poly = 3.4445 * np.eye(len(gram)) - 4.7750 * gram + 2.0315 * gram @ gram
        x = poly @ x if x.shape[0] <= x.shape[1] else x @ poly
    return x


def muon_step(w, m, v, grads, blocks: int, rate: float, hyper: dict):
    """One optimiser step of one parameter from its contributors' gradients: (w, m, v), all float64.  blocks >= 1: that many equal groups of rows
    are matrices, whose momentum is orthogonalised; 0: AdamW."""
    w, m = np.asarray(w, dtype=np.float64), np.asarray(m, dtype=np.float64)
    g = sum(np.asarray(x, dtype=np.float64) for x in grads) / len(grads)
    keep = 1.0 - rate * hyper["weight_decay"]
    if blocks == 0:
        m = hyper["beta1"] * m + (1.0 - hyper["beta1"]) * g
        v = hyper["beta2"] * np.asarray(v, dtype=np.float64) + (1.0 - hyper["beta2"]) * g * g
        step = (m / (1.0 - hyper["beta1"] ** hyper["step"])) / (np.sqrt(v / (1.0 - hyper["beta2"] ** hyper["step"])) + hyper["adam_eps"])
        return keep * w - rate * step, m, v
    m = hyper["momentum"] * m + g
    u = (g + hyper["momentum"] * m if hyper["nesterov"] else m).reshape(blocks, w.shape[0] // blocks, -1)
    x = np.stack([orthogonalise(b, hyper["ns_steps"], hyper["ns_eps"]) for b in u])
    return keep * w - rate * hyper["rms"] * math.sqrt(max(u.shape[1:])) * x.reshape(w.shape), m, None


def aggregate_muon(param_units: dict, n_units: int, params: dict, first: dict, second: dict, worker_grads: list, depths, blocks: dict, hyper: dict,
                   scale_lr: bool, q=lambda a: a):
    """aggregate_update with muon_step in place of SGD.  Returns (new params, new first moments, new second moments)."""
    out = {}, {}, {}
    for name, unit in param_units.items():
        who = contributors(unit, n_units, depths)
        if not who:
            new = tuple(None if t is None else np.asarray(t, dtype=np.float64) for t in (params[name], first[name], second.get(name)))
        else:
            rate = hyper["lr"] * len(who) / len(depths) if scale_lr else hyper["lr"]
            new = muon_step(params[name], first[name], second.get(name), [worker_grads[j][name] for j in who], blocks[name], rate, hyper)
            new = (q(new[0]),) + new[1:]
        for d, t in zip(out, new):
            d[name] = t
    return out
