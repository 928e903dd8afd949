"""Encoder steps whose query and key rows are normed and turned by positions, on the GPU against the oracle: every depth end to end, each layer
by itself, a replayed graph, and the plain encoder's bits where nothing is asked for."""
import numpy as np
import pytest
import torch

import oracle
import paper_2111_10672_amd as spb
import workloads as wl
from parity import TOL, check_gradients, rel_fro, rel_max

pytestmark = pytest.mark.gpu

NAMES = ["qk_encoder_bf16", "qk_long_encoder_bf16", "qk_norm_encoder_bf16", "rotary_encoder_bf16"]


def _setup(name, seed=0):
    cfg = wl.get_config(name)
    params, batch = wl.make_params(cfg, seed, True), wl.make_batch(cfg, seed)
    model = spb.SpbModel(cfg, params, positions=batch.get("positions"))
    dev = {n: t.cuda() for n, t in batch.items() if n != "positions"}
    return cfg, params, batch, model, dev


@pytest.mark.parametrize("name", NAMES)
def test_every_depth(name):
    cfg, params, batch, model, dev = _setup(name)
    n_units = wl.unit_count(cfg)
    _, exact = oracle.spb_step(cfg, params, batch, n_units)
    ref_loss, ref = oracle.spb_step(cfg, params, batch, n_units, oracle.round_to_bf16)
    unit_of = {n: u for n, _s, u, _i in wl.tensor_specs(cfg)}
    for k in range(n_units + 1):
        print(f"case {name} k={k}", flush=True)
        for g in model.grads:
            g.fill_(float("nan"))
        model.step(dev, k)
        torch.cuda.synchronize()
        assert abs(model.loss.item() - ref_loss) <= 5e-3 * abs(ref_loss)
        gpu = {n: g.double().cpu().numpy() for n, g in model.grad_dict(k).items()}
        want = {n for n, u in unit_of.items() if u >= n_units - k}
        assert set(gpu) == want
        check_gradients(gpu, {n: ref[n] for n in want}, "bf16", {n: exact[n] for n in want}, label=f"{name} k={k}")
        for info, g in zip(model.infos, model.grads):
            if info["unit"] < n_units - k:
                assert torch.isnan(g).all(), f"{info['name']} was written below the cut"
    model.close()


@pytest.mark.parametrize("name", NAMES)
def test_each_layer_by_itself(name):
    """A layer's parameter gradients from the input and the incoming gradient that the GPU stored, at the flat tolerance."""
    cfg, params, batch, model, dev = _setup(name, 3)
    n_units = wl.unit_count(cfg)
    units = oracle.build_units(cfg)
    p = {n: t.double().numpy() for n, t in params.items()}
    b = {n: t.numpy() for n, t in batch.items()}
    for u in range(1, n_units - 1):
        k = n_units - u
        model.step(dev, k)
        torch.cuda.synchronize()
        vin, vout = spb.spb_unit_io(model.handle, k, u)
        x, dout = model.read_view(vin).numpy(), model.read_view(vout).numpy()
        units[u].forward(x, p, oracle.round_to_bf16, b)
        g, _ = units[u].backward(dout, p, oracle.round_to_bf16, False)
        got = model.grad_dict(k)
        for n, r in g.items():
            # q, k and v biases meet only in differences: a key bias without the norm has no gradient but rounding, held to its neighbours' scale
            a = got[n].double().cpu().numpy()
            assert rel_max(a, r) <= TOL["bf16"] and rel_fro(a, r) <= TOL["bf16"], (name, u, n, rel_max(a, r))
    model.close()


def test_replays_from_a_graph():
    cfg, params, batch, model, dev = _setup("qk_encoder_bf16", 1)
    k = 4
    model.step(dev, k)
    torch.cuda.synchronize()
    eager, loss = {n: g.clone() for n, g in model.grad_dict(k).items()}, model.loss.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        model.step(dev, k)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            model.step(dev, k)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for g in model.grads:
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(model.loss, loss)
        for n, g in model.grad_dict(k).items():
            assert torch.equal(g, eager[n]), n
    model.close()


def test_positions_of_zero_and_no_norm_leave_the_plain_encoder():
    """Angles of zero turn nothing: the same bits as an encoder without positions."""
    cfg = wl.get_config("small_encoder_bf16")
    params, batch = wl.make_params(cfg, 2, True), wl.make_batch(cfg, 2)
    dev = {n: t.cuda() for n, t in batch.items()}
    plain = spb.SpbModel(cfg, params)
    turned = spb.SpbModel(dict(cfg, rotary=dict(sections=[8])), params, positions=torch.zeros(1, 1, cfg["seq"], dtype=torch.int32))
    for m in (plain, turned):
        m.step(dev, 4)
    torch.cuda.synchronize()
    assert torch.equal(plain.loss, turned.loss)
    for (n, a), b in zip(plain.grad_dict(4).items(), turned.grad_dict(4).values()):
        assert torch.equal(a, b), n
    plain.close()
    turned.close()
