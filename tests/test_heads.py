"""Norm and rotation of query and key heads through the C ABI: refusals on the host, values and gradients on the GPU against the oracle in float64.

Tolerances, with u = 2^-24: a stored result is off by half a step of its type, eps / 2 = 2^-8 (bfloat16) or 2^-24 (float32) of its value, plus
what float32 arithmetic leaves.  With G lanes a row and at most 8 + log2 G + 8 additions in a chain, a mean is off by 25 u max|x|, so is every x - mean;
the root of the variance by 30 u relative; a turned value adds its partner's error and 8 u of both (products, sum, cosine and sine 2 u each, the
fraction of a turn pi 2^-24).  In all at most (2 * 55 + 16) u <= 128 u times the row's largest |gamma| max|x| / sigma + |beta| (without norm: max|x|).
Backward: the same for the turned gradient, the two means and xh: 256 u max|h| / sigma (1 + max|x| / sigma)^2.  A sum over rows: chains of at most
256 additions, 256 u of the sum of the magnitudes, and what the terms are off by."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2111_10672_amd as spb
from oracle import ops

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _strided(b, s, h, d, dtype, layout, device, gen=None, scale=1.0):
    """[b, s, h, d] in a layout: dense tokens, tokens inside wider rows, heads before tokens, or rows that start at an odd element."""
    make = lambda *shape: (scale * torch.randn(*shape, generator=gen)).to(dtype).to(device)
    if layout == "heads":
        return make(b, h, s, d).transpose(1, 2)
    if layout == "wide":
        return make(b, s, h + 3, d)[:, :, 1:h + 1]
    if layout == "odd":
        return make(b, s, h, d + 3)[..., 1:d + 1]
    return make(b, s, h, d)


class Case:
    def __init__(self, b, s, hq, hk, d, dtype=torch.bfloat16, layout="tokens", sections=(), interleaved=False, own_ladder=False, norm=True, beta=True, eps=1e-5,
                 shared_pos=False, far=1000, seed=0, device="cuda", loud=1.0):
        gen = torch.Generator().manual_seed(seed)
        h = hq + hk
        self.x = _strided(b, s, h, d, dtype, layout, device, gen)
        self.x.mul_(loud)
        self.dy = _strided(b, s, h, d, dtype, layout, device, gen, 0.1)
        self.hq, self.norm, self.eps = hq, norm, eps
        rows = 2 if hk else 1
        self.gamma = (1 + 0.3 * torch.randn(rows, d, generator=gen)).to(dtype).to(device) if norm else None
        self.beta = (0.3 * torch.randn(rows, d, generator=gen)).to(dtype).to(device) if norm and beta else None
        self.sections, self.kind = list(sections), dict(interleaved=interleaved, own_ladder=own_ladder)
        self.rotary = spb.spb_rotary_sections(self.sections, 10000.0, **self.kind) if sections else None
        self.pos = torch.randint(-far, far + 1, (max(1, len(sections)), 1 if shared_pos else b, s), generator=gen, dtype=torch.int32).to(device) if sections else None

    def angles(self):
        b, s = self.x.shape[:2]
        pos = self.pos.cpu().numpy()
        return ops.rotary_angles(np.broadcast_to(pos, (pos.shape[0], b, s)).reshape(pos.shape[0], -1), self.sections, **self.kind)

    def rows(self, t):
        """Weights per head."""
        t = t.double().cpu().numpy()
        hk = self.x.shape[2] - self.hq
        return np.concatenate([np.repeat(t[:1], self.hq, 0), np.repeat(t[-1:], hk, 0)]) if hk else np.repeat(t, self.hq, 0)

    def check_forward(self, y):
        b, s, h, d = self.x.shape
        x = self.x.double().cpu().numpy().reshape(b * s, h, d)
        amp = np.abs(x).max(-1, keepdims=True)
        if self.norm:
            gamma = self.rows(self.gamma)
            beta = self.rows(self.beta) if self.beta is not None else np.zeros_like(gamma)
            x, (_xh, rstd) = ops.head_norm_fwd(x, gamma, beta, self.eps)
            amp = np.abs(gamma).max(-1)[None, :, None] * amp * rstd + np.abs(beta).max(-1)[None, :, None]
        if self.sections:
            x = ops.rotate(x, self.angles(), self.kind["interleaved"])
        got = y.double().cpu().numpy().reshape(b * s, h, d)
        tol = HALF[y.dtype] * np.abs(x) + 128 * U * amp
        assert (np.abs(got - x) <= tol).all(), float((np.abs(got - x) / tol).max())

    def check_backward(self, dx, dgamma, dbeta):
        b, s, h, d = self.x.shape
        x, g = (t.double().cpu().numpy().reshape(b * s, h, d) for t in (self.x, self.dy))
        if self.sections:
            g = ops.rotate(g, -self.angles(), self.kind["interleaved"])
        tol = 128 * U * np.abs(g).max(-1, keepdims=True) * np.ones_like(g)
        if self.norm:
            gamma = self.rows(self.gamma)
            _, (xh, rstd) = ops.head_norm_fwd(x, gamma, 0 * gamma, self.eps)
            big = 1 + np.abs(x).max(-1, keepdims=True) * rstd
            hmax = np.abs(gamma).max(-1)[None, :, None] * np.abs(g).max(-1, keepdims=True)
            tol = 256 * U * rstd * hmax * big ** 2 * np.ones_like(g)
            want, scale, shift = ops.head_norm_bwd(g, gamma, (xh, rstd))
            fold = (lambda t: np.stack([t[:self.hq].sum(0), t[self.hq:].sum(0)])) if h > self.hq else (lambda t: t.sum(0, keepdims=True))
            off = 128 * U * np.abs(g).max(-1, keepdims=True)
            for got, ref, size in ((dgamma, scale, np.abs(g * xh) * 256 * U + np.abs(g) * 64 * U * big + off * np.abs(xh)), (dbeta, shift, np.abs(g) * 256 * U + off)):
                far = np.abs(got.double().cpu().numpy() - fold(ref))
                assert (far <= fold(size.sum(0)) + 1e-30).all(), float((far / (fold(size.sum(0)) + 1e-30)).max())
            g = want
        got = dx.double().cpu().numpy().reshape(b * s, h, d)
        tol = tol + HALF[dx.dtype] * np.abs(g)
        assert (np.abs(got - g) <= tol).all(), float((np.abs(got - g) / tol).max())

    def forward(self, y, stream=None):
        desc = spb.heads_desc(self.x, self.hq, y=y, norm=self.norm, eps=self.eps, rotary=self.rotary)
        spb.spb_heads_forward(desc, self.x, y, self.pos, self.gamma, self.beta, torch.cuda.current_stream().cuda_stream if stream is None else stream)

    def backward(self, dx):
        desc = spb.heads_desc(self.x, self.hq, y=self.dy, dx=dx, norm=self.norm, eps=self.eps, rotary=self.rotary)
        size = spb.spb_heads_workspace_size(desc)
        ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
        grads = [torch.full(self.gamma.shape, float("nan"), device="cuda") for _ in range(2)] if self.norm else [None, None]
        spb.spb_heads_backward(desc, self.x if self.norm else None, self.dy, dx, self.pos, self.gamma, *grads, ws, size, torch.cuda.current_stream().cuda_stream)
        return grads


CASES = {
    "one_token": dict(b=1, s=1, hq=12, hk=12, d=64, sections=(10, 11, 11)),
    "one_element": dict(b=2, s=3, hq=1, hk=0, d=1),
    "smallest_pair": dict(b=1, s=5, hq=1, hk=1, d=2, sections=(1,), norm=False),
    "encoder_rows": dict(b=3, s=37, hq=12, hk=12, d=64, layout="wide", sections=(16, 16)),
    "rotation_alone": dict(b=2, s=65, hq=8, hk=2, d=128, sections=(20, 22, 22), norm=False, far=2 ** 31 - 1),
    "rotation_interleaved": dict(b=2, s=33, hq=4, hk=4, d=128, sections=(32, 32), interleaved=True, own_ladder=True),
    "part_of_head": dict(b=1, s=70, hq=5, hk=3, d=128, sections=(16,), shared_pos=True),
    "part_of_head_interleaved": dict(b=2, s=17, hq=3, hk=1, d=96, sections=(4, 4, 4, 4), interleaved=True),
    "norm_alone": dict(b=5, s=51, hq=7, hk=0, d=64),
    "norm_80": dict(b=2, s=77, hq=16, hk=16, d=80, beta=False),
    "norm_256": dict(b=1, s=40, hq=2, hk=2, d=256, sections=(64, 64)),
    "norm_8": dict(b=2, s=40, hq=3, hk=5, d=8),
    "heads_first": dict(b=3, s=29, hq=4, hk=4, d=64, layout="heads", sections=(32,), shared_pos=True),
    "odd_size": dict(b=2, s=31, hq=3, hk=2, d=100, sections=(25, 25)),
    "odd_size_norm": dict(b=2, s=31, hq=3, hk=2, d=37, sections=(5, 4)),
    "eight_byte_chunks": dict(b=2, s=33, hq=5, hk=3, d=72, sections=(18, 18)),
    "eight_byte_chunks_256": dict(b=1, s=23, hq=2, hk=2, d=252, sections=(60, 60)),
    "four_byte_chunks": dict(b=2, s=33, hq=5, hk=3, d=106, sections=(20, 14, 14), interleaved=True),
    "four_byte_chunks_small": dict(b=2, s=33, hq=5, hk=0, d=6, sections=(2,)),
    "four_byte_chunks_254": dict(b=1, s=23, hq=2, hk=2, d=254, sections=(64, 62)),
    "f32_eight_byte_chunks": dict(b=2, s=21, hq=2, hk=1, d=38, dtype=torch.float32, sections=(10, 8)),
    "odd_pairs": dict(b=2, s=31, hq=3, hk=2, d=100, sections=(25,)),
    "odd_start": dict(b=2, s=19, hq=4, hk=4, d=64, layout="odd", sections=(16, 16), interleaved=True),
    "whole_255": dict(b=1, s=13, hq=1, hk=1, d=255, sections=(127,)),
    "f32": dict(b=2, s=45, hq=6, hk=6, d=64, dtype=torch.float32, sections=(16, 8, 8), far=10 ** 6),
    "f32_256": dict(b=1, s=21, hq=2, hk=1, d=256, dtype=torch.float32, sections=(32, 32, 32, 32), interleaved=True),
    "f32_20": dict(b=2, s=21, hq=2, hk=1, d=20, dtype=torch.float32, sections=(4,)),
    "f32_odd": dict(b=2, s=21, hq=2, hk=1, d=27, dtype=torch.float32, layout="odd", sections=(6, 7)),
    "f32_turn": dict(b=2, s=9, hq=3, hk=0, d=12, dtype=torch.float32, sections=(6,), norm=False, interleaved=True),
    "many_tokens": dict(b=4, s=1200, hq=3, hk=1, d=32, sections=(8, 8)),
    "few_heads": dict(b=3, s=22001, hq=1, hk=0, d=16),
    "few_heads_turned": dict(b=2, s=9001, hq=2, hk=1, d=40, sections=(10, 10)),
    "few_heads_general": dict(b=1, s=17001, hq=1, hk=1, d=9, dtype=torch.float32, sections=(3,)),
    "few_heads_128_pairs": dict(b=1, s=4999, hq=1, hk=0, d=256, sections=(43, 43, 42), far=2 ** 31 - 1),
    "large_values": dict(b=1, s=33, hq=4, hk=4, d=64, loud=1e15, sections=(32,)),
    "small_values": dict(b=1, s=33, hq=4, hk=4, d=64, loud=1e-12, dtype=torch.float32),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_forward(name):
    print("case", name, flush=True)
    case = Case(**CASES[name])
    y = torch.empty(case.x.shape, dtype=case.x.dtype, device="cuda")
    case.forward(y)
    case.check_forward(y)
    again = case.x.clone().as_strided(case.x.shape, case.x.stride()) if case.x.is_contiguous() else case.x
    kept = case.x.clone()
    desc = spb.heads_desc(again, case.hq, norm=case.norm, eps=case.eps, rotary=case.rotary)      # in place: the same bits
    spb.spb_heads_forward(desc, again, again, case.pos, case.gamma, case.beta, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(again, y)
    case.x = kept


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
def test_backward(name):
    print("case", name, flush=True)
    case = Case(**CASES[name])
    dx = torch.empty(case.x.shape, dtype=case.x.dtype, device="cuda")
    grads = case.backward(dx)
    case.check_backward(dx, *grads)
    again = case.backward(case.dy)                                                              # in place of dy: the same bits
    assert torch.equal(case.dy, dx)
    for a, b in zip(grads, again):
        assert a is None or torch.equal(a, b)


@pytest.mark.gpu
def test_rows_behind_the_last_head_and_between_rows_stay():
    wide = torch.randn(2, 9, 7, 64, device="cuda").to(torch.bfloat16)
    before = wide.clone()
    case = Case(2, 9, 2, 1, 64, sections=(16, 16))
    x = wide[:, :, 2:5]
    case.x = x.clone()
    desc = spb.heads_desc(x, 2, norm=True, rotary=case.rotary)
    spb.spb_heads_forward(desc, x, x, case.pos, case.gamma, case.beta, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(wide[:, :, :2], before[:, :, :2]) and torch.equal(wide[:, :, 5:], before[:, :, 5:])
    case.check_forward(x)


@pytest.mark.gpu
def test_broadcast_input_constant_rows_and_values_that_are_not_numbers():
    case = Case(4, 11, 2, 2, 64, sections=(32,))
    case.x = case.x[:1].expand(4, -1, -1, -1)                      # one sequence for all
    y = torch.empty(4, 11, 4, 64, dtype=torch.bfloat16, device="cuda")
    case.forward(y)
    case.check_forward(y)
    dx = torch.empty_like(y)
    case.check_backward(dx, *case.backward(dx))
    case = Case(1, 5, 2, 1, 64)
    case.x = case.x.contiguous()
    case.x[0, 1] = 3.0                                             # no variance: beta comes out
    case.x[0, 2, 0, 7] = float("nan")
    case.x[0, 3, 1, 5] = float("inf")
    y = torch.empty_like(case.x)
    case.forward(y)
    assert torch.equal(y[0, 1, :2], case.beta[:1].expand(2, -1)) and torch.equal(y[0, 1, 2], case.beta[1])
    assert y[0, 2, 0].isnan().all() and y[0, 3, 1].isnan().any()
    bad = torch.zeros(5, 3, dtype=torch.bool)
    bad[2, 0] = bad[3, 1] = True
    assert y[0].cpu()[~bad].isfinite().all()                       # other rows do not see it


@pytest.mark.gpu
def test_gradient_against_differences():
    """A directional derivative of a float32 forward pass: central differences of step h are off by h^2 and by rounding / h."""
    case = Case(2, 7, 3, 2, 24, dtype=torch.float32, sections=(4, 8))
    dx = torch.empty_like(case.x)
    dgamma, dbeta = case.backward(dx)
    gen = torch.Generator().manual_seed(5)
    h = 2.0 ** -8
    for tensor, grad in ((case.x, dx), (case.gamma, dgamma), (case.beta, dbeta)):
        way = torch.randn(tensor.shape, generator=gen).cuda()
        kept, ends = tensor.clone(), []
        for sign in (1, -1):
            tensor.copy_(kept + sign * h * way)
            y = torch.empty_like(case.x)
            case.forward(y)
            ends.append(y.double())
        tensor.copy_(kept)
        numeric = ((ends[0] - ends[1]) / (2 * h) * case.dy.double()).sum().item()
        exact = (grad.double() * way.double()).sum().item()
        # third derivatives of a normed row of order 1 along a direction of length sqrt(24): 24^1.5 h^2 / 6 a row of |dy| 0.1 * sqrt(24); rounding: 128 u * 4 / h a value
        room = case.x[..., 0].numel() * 0.5 * (24 ** 1.5 * h * h / 6 + 128 * U * 4 / h * 5)
        assert abs(numeric - exact) <= room, (numeric, exact, room)


@pytest.mark.gpu
def test_other_streams_and_replayed_graphs():
    case = Case(3, 50, 4, 4, 64, sections=(16, 16))
    want = torch.empty_like(case.x)
    case.forward(want)
    dx = torch.empty_like(case.x)
    grads = case.backward(dx)
    desc = spb.heads_desc(case.x, 4, y=case.dy, dx=dx, norm=True, rotary=case.rotary)
    size = spb.spb_heads_workspace_size(desc)
    y, dx2 = torch.empty_like(want), torch.empty_like(dx)
    outs = [torch.empty_like(g) for g in grads]
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def both(stream):
        case.forward(y, stream)
        spb.spb_heads_backward(desc, case.x, case.dy, dx2, case.pos, case.gamma, *outs, ws, size, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(side.cuda_stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both(side.cuda_stream)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in (y, dx2, *outs):
            t.fill_(float("nan"))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx2, dx) and all(torch.equal(a, b) for a, b in zip(outs, grads))


@pytest.mark.gpu
@pytest.mark.parametrize("b,s", [(0, 5), (5, 0)])
def test_no_tokens(b, s):
    x = torch.empty(b, s, 3, 16, dtype=torch.bfloat16, device="cuda")
    gamma = torch.ones(2, 16, dtype=torch.bfloat16, device="cuda")
    desc = spb.heads_desc(x, 2, norm=True)
    spb.spb_heads_forward(desc, x, x, None, gamma, None, 0)
    grads = [torch.full((2, 16), float("nan"), device="cuda") for _ in range(2)]
    size = spb.spb_heads_workspace_size(desc)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    spb.spb_heads_backward(desc, x, x, x, None, gamma, *grads, ws, size, 0)
    assert all((g == 0).all() for g in grads)


@pytest.mark.gpu
@pytest.mark.parametrize("dim,layout", [(2, "tokens"), (3, "tokens")])
def test_more_tokens_than_workgroups(dim, layout):
    """2^24 + 5 tokens of one head, past the 2^20 workgroups of 16 tokens: the last ones as the first."""
    n, tail = 2 ** 24 + 5, 1000
    x = torch.randn(1, n, 1, dim, device="cuda").to(torch.bfloat16)
    rotary = spb.spb_rotary_sections([1])
    pos = (torch.arange(n, device="cuda", dtype=torch.int32) % 1000).view(1, 1, n)
    y = torch.zeros_like(x)
    desc = spb.heads_desc(x, 1, y=y, rotary=rotary)
    spb.spb_heads_forward(desc, x, y, pos, None, None, torch.cuda.current_stream().cuda_stream)
    for at in (0, n - tail):
        part = x[:, at:at + tail].contiguous()
        want = torch.zeros_like(part)
        spb.spb_heads_forward(spb.heads_desc(part, 1, rotary=rotary), part, want, pos[:, :, at:at + tail].contiguous(), None, None, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(y[:, at:at + tail], want)
    assert (y != 0).any(-1).sum() >= n - 100


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Two sequences 2^31 + 64 elements apart."""
    gap = 2 ** 31 + 64
    flat = torch.zeros(gap + 4 * 64, dtype=torch.bfloat16, device="cuda")
    case = Case(2, 2, 1, 1, 64, sections=(32,))
    x = flat.as_strided((2, 2, 2, 64), (gap, 128, 64, 1))
    x.copy_(case.x)
    case.x = x
    y = torch.empty(2, 2, 2, 64, dtype=torch.bfloat16, device="cuda")
    case.forward(y)
    case.check_forward(y)
    case.dy = case.dy.contiguous()
    want = torch.empty_like(y)
    case.backward(want)
    out = torch.zeros(gap + 4 * 64, dtype=torch.bfloat16, device="cuda").as_strided((2, 2, 2, 64), (gap, 128, 64, 1))
    case.backward(out)
    assert torch.equal(out, want)


# ---- refusals: all found on the host --------------------------------------------------------------------------------

def _desc(**patch):
    x = torch.empty(2, 3, 4, 16, dtype=torch.bfloat16)
    d = spb.heads_desc(x, 3, norm=True, rotary=spb.spb_rotary_sections([3, 5]))
    for k, v in patch.items():
        if k.startswith("r_"):
            if isinstance(v, tuple):
                getattr(d.rotary, k[2:])[v[0]] = v[1]
            else:
                setattr(d.rotary, k[2:], v)
        else:
            setattr(d, k, (C.c_int64 * 3)(*v) if isinstance(v, list) else v)
    return d


@pytest.mark.parametrize("patch", [dict(dtype=2), dict(batch=-1), dict(batch=65536, seq=32768), dict(heads_q=0), dict(heads_k=-1), dict(head_dim=0), dict(head_dim=257),
                                   dict(eps=0.0), dict(eps=float("nan")), dict(norm=0, r_pairs=0), dict(r_pairs=9), dict(r_pairs=-1), dict(r_axes=0), dict(r_axes=5),
                                   dict(r_axis=(2, 2)), dict(r_axis=(0, -1)), dict(r_freq=(1, float("inf"))), dict(x_stride=[-64, 64, 16]), dict(x_stride=[1 << 60, 64, 16]), dict(y_stride=[192, 64, 15]),
                                   dict(y_stride=[192, 48, 16]), dict(y_stride=[0, 64, 16]), dict(y_stride=[128, 64, 16])])
def test_descriptions_that_are_refused(patch):
    with pytest.raises(spb.SpbError) as e:
        d = _desc(**patch)
        spb.lib()
        from paper_2111_10672_amd.binding import _check
        _check(spb.lib().spb_heads_forward(C.byref(d), 256, 512, 256, 3, 0, 256, 256, 0))
    assert e.value.code == -1 and "spb_heads_forward" in str(e.value)


def test_pointers_and_workspaces_that_are_refused():
    from paper_2111_10672_amd.binding import _check
    lib, d = spb.lib(), _desc()
    size = spb.spb_heads_workspace_size(d)
    assert size >= 4 * 2 * 2 * 16 and spb.spb_heads_workspace_size(_desc(norm=0)) == 0
    forward = dict(x=256, y=512, pos=256, a=6, b=3, gamma=256, beta=0)
    for patch in (dict(x=0), dict(y=0), dict(x=257), dict(pos=0), dict(pos=258), dict(gamma=0), dict(gamma=257), dict(beta=257)):
        with pytest.raises(spb.SpbError) as e:
            _check(lib.spb_heads_forward(C.byref(d), *{**forward, **patch}.values(), 0))
        assert e.value.code == -1
    backward = dict(x=256, dy=256, dx=512, pos=256, a=6, b=3, gamma=256, dgamma=256, dbeta=256, ws=256, bytes=size)
    for patch, code in ((dict(x=0), -1), (dict(dy=0), -1), (dict(dx=0), -1), (dict(dx=513), -1), (dict(pos=0), -1), (dict(gamma=0), -1), (dict(dgamma=0), -1),
                        (dict(dbeta=258), -1), (dict(ws=0), -4), (dict(ws=128), -4), (dict(bytes=size - 1), -4)):
        with pytest.raises(spb.SpbError) as e:
            _check(lib.spb_heads_backward(C.byref(d), *{**backward, **patch}.values(), 0))
        assert e.value.code == code, patch
    with pytest.raises(spb.SpbError):
        _check(lib.spb_heads_backward(C.byref(_desc(dx_stride=[192, 64, 0])), *backward.values(), 0))


def test_binding_refuses_tensors_of_other_shapes():
    x = torch.empty(2, 3, 4, 16)
    for bad in (dict(y=torch.empty(2, 3, 4, 8)), dict(y=torch.empty(2, 3, 4, 16).bfloat16()), dict(dx=torch.empty(2, 3, 16, 4).transpose(2, 3))):
        with pytest.raises(ValueError):
            spb.heads_desc(x, 2, **bad)
    with pytest.raises(ValueError):
        spb.heads_desc(x.half(), 2)
    d = spb.heads_desc(x, 2, norm=True, rotary=spb.spb_rotary_sections([4, 4]))
    pos, gamma = torch.zeros(2, 1, 3, dtype=torch.int32), torch.ones(2, 16)
    for p, g in ((pos.long(), gamma), (pos[:1], gamma), (pos[:, :, :2], gamma), (torch.zeros(2, 3, 3, dtype=torch.int32), gamma), (pos, gamma[:1]), (pos, gamma.bfloat16())):
        with pytest.raises(ValueError):
            spb.spb_heads_forward(d, x, x, p, g, None, 0)


@pytest.mark.parametrize("args", [dict(sections=[]), dict(sections=[1] * 5), dict(sections=[-1, 3]), dict(sections=[0, 0]), dict(sections=[100, 29]), dict(sections=[4], base=0.0),
                                  dict(sections=[4], base=float("inf"))])
def test_sections_that_are_refused(args):
    with pytest.raises(spb.SpbError) as e:
        spb.spb_rotary_sections(**args)
    assert e.value.code == -1


def test_sections_fill_axes_and_frequencies():
    r = spb.spb_rotary_sections([2, 0, 3], base=16.0)
    assert (r.pairs, r.axes, list(r.axis[:5])) == (5, 3, [0, 0, 2, 2, 2])
    assert np.allclose(list(r.freq[:5]), 16.0 ** (-np.arange(5) / 5))
    r = spb.spb_rotary_sections([2, 0, 3], base=16.0, own_ladder=True, interleaved=True)
    assert r.interleaved == 1 and np.allclose(list(r.freq[:5]), [1, 1 / 4, 1, 16 ** (-1 / 3), 16 ** (-2 / 3)])


def test_encoders_take_norm_and_rotation_before_their_parameters_are_bound():
    import workloads as wl
    cfg = wl.get_config("small_encoder_bf16")
    m = spb.spb_model_create(spb.desc_from_config(cfg))
    other = spb.spb_model_create(spb.desc_from_config(wl.get_config("cfg1")))
    try:
        plain = [spb.spb_workspace_size(m, k) for k in range(5)]
        names = [spb.spb_param_info(m, i)["name"] for i in range(spb.spb_param_count(m))]
        rotary = spb.spb_rotary_sections([8])
        pos = torch.zeros(1, 1, 40, dtype=torch.int32)
        with pytest.raises(spb.SpbError) as e:
            spb.spb_encoder_heads(other, rotary, pos)
        assert e.value.code == -6
        for bad in (dict(rotary=spb.spb_rotary_sections([9]), pos=pos), dict(rotary=rotary, pos=None), dict(rotary=None, pos=None, norm=True, eps=0.0)):
            with pytest.raises(spb.SpbError) as e:
                spb.spb_encoder_heads(m, **bad)
            assert e.value.code == -1
        spb.spb_encoder_heads(m, rotary, pos)
        assert [spb.spb_workspace_size(m, k) for k in range(5)] == plain and spb.spb_param_count(m) == len(names)
        spb.spb_encoder_heads(m, rotary, pos, norm=True)
        infos = [spb.spb_param_info(m, i) for i in range(spb.spb_param_count(m))]
        new = [i for i in infos if "qknorm" in i["name"]]
        assert [i["name"] for i in infos if "qknorm" not in i["name"]] == names
        assert [(i["name"], i["shape"], i["unit"]) for i in new[:2]] == [("layer0.attn.qknorm.weight", (2, 16), 1), ("layer0.attn.qknorm.bias", (2, 16), 1)]
        sizes = [spb.spb_workspace_size(m, k) for k in range(5)]
        assert sizes[0] == plain[0] and sizes[4] > plain[4] and all(b >= a for a, b in zip(sizes, sizes[1:]))
        spb.spb_encoder_heads(m, None, None)                       # as created
        assert [spb.spb_workspace_size(m, k) for k in range(5)] == plain and spb.spb_param_count(m) == len(names)
        spb.spb_bind_params(m, [256] * len(names))
        with pytest.raises(spb.SpbError) as e:
            spb.spb_encoder_heads(m, rotary, pos)
        assert e.value.code == -3
    finally:
        spb.spb_model_destroy(m)
        spb.spb_model_destroy(other)
