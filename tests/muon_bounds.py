"""How far an orthogonalised update may be from the one in float64, from the number formats alone; used by the tests of the optimiser step.

With u = 2^-24.  X, A and B (or Z) are stored to h relative: 2^-11 for bfloat16 parameters (half a step of float16), 2^-21 for float32 ones (value and remainder,
each product's remainder x remainder left out), and to half a step of float16's subnormal numbers where they are small.  A float32 sum over k products in the matrix
cores is off by (k / 16 + 16) u of the sum of magnitudes.  Matrices with a short side of at most 32 (bfloat16) or 48 (float32), 8192 long, 256 of a kind, run up to 8
steps on the Gram matrix in float64 instead."""
import math

import numpy as np

U, D = 2.0 ** -24, 2.0 ** -53
A, B, C = 3.4445, -4.7750, 2.0315


def chain(k):
    return (k / 16 + 16) * U


def storage(bf16):
    """(relative error, error of small entries of X times sigma, and of A and B) of what lies between two products."""
    return (2.0 ** -11, 2.0 ** -25, 2.0 ** -35) if bf16 else (2.0 ** -21, 2.0 ** -36, 2.0 ** -46)


def on_the_gram_matrix(shape, count, bf16, steps):
    return min(shape) <= (32 if bf16 else 48) and max(shape) <= 8192 and count <= 256 and steps <= 8


def _divided(a, b):
    """(p(a) - p(b)) / (a - b) of the step's polynomial."""
    return A + B * (a * a + a * b + b * b) + C * (a ** 4 + a ** 3 * b + a * a * b * b + a * b ** 3 + b ** 4)


def _values(u, eps):
    """Singular values of the start, and whether the long side has other directions."""
    u = np.asarray(u, dtype=np.float64)
    u = u if u.shape[0] <= u.shape[1] else u.T
    x = u / (np.linalg.norm(u) + eps)
    if len(x) <= 256:
        return np.linalg.svd(x, compute_uv=False), u.shape[0] != u.shape[1]
    return np.sqrt(np.maximum(np.linalg.eigvalsh(x @ x.T), 0.0)), u.shape[0] != u.shape[1]      # (small ones to 1e-8, which no growth notices)


def frobenius_room(u, bf16, hyper, count=1):
    """Bound of the Frobenius norm of the error of the orthogonalised matrix u.

    An error of X between the directions of the singular values s and t grows over a step by the polynomial's divided differences (p(s) - p(t)) / (s - t) and
    (p(s) + p(t)) / (s + t), and over several by their products along the iterates of s and t.  Rounding errors of the entries of a large matrix know nothing of its directions:
    each pair of them gets its share of the sum of squares, and what comes out by the end is that sum over the pairs, each times its own growth.  A rounding error
    is spread evenly over a step, whose root mean square is 1 / sqrt(3) of the half step, and the errors of different roundings add up in squares; A and B hold each twice.  Twice
    the root covers chance and terms of second order.  For a short side below 16 there are too few to go by: every entry off by its half step, all
    errors of one sign and with the largest growth."""
    steps = hyper["ns_steps"]
    s, wide = _values(u, hyper["ns_eps"])
    if on_the_gram_matrix(np.shape(u), count, bf16, steps):
        return _gram_room(s, hyper, np.shape(u))
    h, small_x, small_a = storage(bf16)
    n, m = sorted(np.shape(u))
    # half steps of subnormals add up to sqrt(n m) / sigma of them, sigma the power of two next to the root of the padded size
    small_x *= 1.5 * (min(1.0, math.sqrt(n * m) / 32.0))
    path = [s]
    for _ in range(steps):
        path.append(A * path[-1] + B * path[-1] ** 3 + C * path[-1] ** 5)
    # growth[k][i, j] from after k steps to the end, and that into the long side's other directions
    growth, rest = [np.ones((n, n))], [np.ones(n)]
    even, odd, none = np.ones((n, n)), np.ones((n, n)), np.ones(n)
    for t in reversed(path[:-1]):
        even = even * np.abs(_divided(t[:, None], t[None, :]))
        odd = odd * np.abs(_divided(t[:, None], -t[None, :]))
        none = none * np.abs(_divided(t, 0.0 * t))
        growth.append(np.maximum(even, odd))
        rest.append(none)
    growth, rest = growth[::-1], rest[::-1]
    fro = lambda v: math.sqrt(float((v * v).sum()))

    few = n < 16
    part = 1.0 if few else 3.0 ** -0.5

    def anywhere(k, err):
        """An error of X_k of Frobenius norm err, spread over all its entries."""
        if few:
            return err * max(float(growth[k].max()), float(rest[k].max()) if wide else 0.0)
        return err * math.sqrt(float((growth[k] ** 2).sum() + (m - n) * (rest[k] ** 2).sum()) / (n * m))

    def through(k, err, by):
        """A symmetric n x n error of Frobenius norm err whose entry i, j is multiplied by by[i, j] in the directions of X_{k+1}."""
        if few:
            return err * float(by.max()) * float(growth[k + 1].max())
        return math.sqrt(2.0) * err / n * fro(np.sqrt((by ** 2 + by.T ** 2) / 2) * growth[k + 1])

    errors = [anywhere(0, part * h * fro(s) + small_x), anywhere(0, 64 * U * fro(s))]
    for k in range(steps):
        x, a = path[k], path[k] ** 2
        b = B * a + C * a * a
        side = np.ones((n, 1)) * x[None, :]
        in_a = np.abs(B + C * (a[:, None] + a[None, :])) * side
        errors += [through(k, part * h * fro(a) + n * small_a, in_a), through(k, chain(m) * fro(x) ** 2, in_a), through(k, C * chain(n) * fro(a) ** 2 + 8 * U * fro(b), side)]
        in_b = math.hypot(through(k, part * h * fro(b) + n * small_a, side), anywhere(k + 1, part * h * A * fro(x)))          # (on B's diagonal is A)
        in_z = anywhere(k + 1, (part * h * fro(B * x + C * a * x) + small_x) * float(a.max()))
        errors += [max(in_b, in_z), anywhere(k + 1, 8 * U * A * fro(x)), anywhere(k + 1, chain(n) * (fro(b) + A) * fro(x) + 4 * U * fro(path[k + 1])),
                   anywhere(k + 1, part * h * fro(path[k + 1]) + small_x)]
    return sum(errors) if few else 2.0 * math.sqrt(sum(e * e for e in errors))


def _gram_room(s, hyper, shape):
    """The chain on A in float64 and one float32 product: Q = q(A), X = Q X_0.

    An error of A_k between the directions of a and b changes what is left of the chain, q_k(A_k) = p(A_{k+n-1}) ... p(A_k) with p(a) = a I + b a + c a a, by
    the divided difference q_k[a, b], and X by that times the singular value of X_k; A_{k+1} = f(A_k), f(a) = a p(a)^2, carries errors on.  The products of float64 are off
    by 16 n of their rounding (n / 4 additions each, three products, a norm of at most 17)."""
    n, steps = min(shape), hyper["ns_steps"]
    p = lambda a: A + B * a + C * a * a
    pd = lambda a, b: B + C * (a + b)
    c5 = (A * A, 2 * A * B, B * B + 2 * A * C, 2 * B * C, C * C)                 # f's coefficients of a .. a^5
    fd = lambda a, b: sum(c * sum(a ** i * b ** (k - i) for i in range(k + 1)) for k, c in enumerate(c5))
    path = [s * s]
    for _ in range(steps):
        path.append(path[-1] * p(path[-1]) ** 2)
    total = 0.0
    for k in range(steps):
        left, spread, whole = np.ones_like(s)[:, None], np.ones((len(s), len(s))), 0.0
        for j in range(k, steps):
            a, b = path[j][:, None], path[j][None, :]
            right = np.ones_like(s)
            for i in range(j + 1, steps):
                right = right * p(path[i])
            whole = whole + np.abs(left * pd(a, b) * spread * right[None, :])
            left, spread = left * np.abs(p(a)), spread * np.abs(fd(a, b))
        made = 16 * n * D * 17 * math.sqrt(n) if k else 16 * n * D
        total += made * float(np.max(whole * np.sqrt(np.abs(path[k]))[None, :]))
    q = np.ones_like(s)
    for j in range(steps):
        q = q * p(path[j])
    fro = math.sqrt(float((q * q).sum()))
    return 2.0 * total + 2 * (n + 16) * U * fro * math.sqrt(float((s * s).sum())) + 2.0 ** -60


def entry_room(u, bf16, hyper):
    """(orthogonalised u with the shorter side first, bound of each entry's error) after a step or two of products over the whole matrix; u: float64, on any device.

    Entry by entry: a product P Q is off by |dP| |Q| + |P| |dQ| + chain |P| |Q|, what is stored by h of each entry more.  (Products of absolute values
    grow too fast for more steps.)"""
    import torch
    u = u if u.shape[0] <= u.shape[1] else u.T.contiguous()
    n, m = u.shape
    h, small_x, small_a = storage(bf16)
    small_x /= 2.0 ** min(14, round(0.5 * math.log2(n * m)))              # (a padded matrix has a larger sigma)
    x = u / (u.square().sum().sqrt() + hyper["ns_eps"])
    err = (h + 4 * U) * x.abs() + small_x
    for _ in range(hyper["ns_steps"]):
        size, xt, et = x.abs(), x.T.contiguous().abs(), err.T.contiguous()
        a = x @ x.T.contiguous()
        off_a = err @ xt + size @ et + err @ et + chain(m) * (size @ xt) + h * a.abs() + small_a
        flat = a.abs()
        b = B * a + C * (a @ a)
        off_b = -B * off_a + C * (off_a @ flat + flat @ off_a + off_a @ off_a + chain(n) * (flat @ flat)) + 8 * U * b.abs()
        z = b @ x
        b = b + A * torch.eye(n, dtype=b.dtype, device=b.device)
        off_b = off_b + h * b.abs() + small_a
        new = b @ x
        off = off_b @ size + b.abs() @ err + off_b @ err + chain(n) * (b.abs() @ size)
        if n <= 256:                                                     # Z = b X + c A X is rounded where B is above
            z = B * x + C * (a @ x)
            off = off + flat @ (h * z.abs() + small_x)
        x, err = new, off + (h + 4 * U) * new.abs() + small_x
    return x, err


def with_unit_columns(n, m, generator, scale=1e-3):
    """[a I | M] (its transpose if n > m): the first product of a step shows every entry of B in a column of its own.  M's entries are of one sign, so that the entries of A
    are of the size of the sums that bound their errors."""
    import torch
    short, long = sorted((n, m))
    units = min(short, long - short) or short // 2
    part = torch.randn(short, long, generator=generator).abs()
    size = math.sqrt(max(long - units, 1))
    part[:, :units] = 0.0
    part[torch.arange(units), torch.arange(units)] = size
    part = scale * part
    return part if n <= m else part.T.contiguous()


def check_matrices(before, after, dtype, hyper, rate_scale=1.0, count=None, most=0.1):
    """A parameter of `blocks` matrices after a step against the oracle's, in the Frobenius norm of each; the room may be no more than `most` of the update."""
    import torch

    import oracle
    blocks, rate = before["blocks"], hyper["lr"] * rate_scale
    stacked = before["w"].ndim == 3 and before["w"].shape[0] == blocks
    shape = (-1, before["w"].shape[-1]) if stacked else (before["w"].shape[0], -1)
    flat = lambda t: np.asarray(t).reshape(shape)
    bf16 = dtype == torch.bfloat16
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    w, m, _ = oracle.muon_step(flat(before["w"]), flat(before["m"]), None, [flat(g) for g in before["grads"]], blocks, rate, hyper)
    n = len(before["grads"])
    size = np.abs(flat(before["m"])) + sum(np.abs(flat(g)) for g in before["grads"]) / n
    assert (np.abs(flat(after["m"]) - m) <= (n + 4) * U * size + 2.0 ** -149).all()
    r, c = m.shape[0] // blocks, m.shape[1]
    u = sum(flat(g) for g in before["grads"]) / n + hyper["momentum"] * m if hyper["nesterov"] else m
    step = rate * hyper["rms"] * math.sqrt(max(r, c))
    keep = 1.0 - rate * hyper["weight_decay"]
    for k in range(blocks):
        rows = slice(k * r, (k + 1) * r)
        update = np.linalg.norm(w[rows] - keep * flat(before["w"])[rows])
        room = step * frobenius_room(u[rows], bf16, hyper, count or blocks)
        assert room <= most * update, (k, room, update)                  # else the test would say nothing
        room += half * np.linalg.norm(w[rows]) + 4 * U * np.linalg.norm(flat(before["w"])[rows])
        far = np.linalg.norm(flat(after["w"])[rows] - w[rows])
        assert far <= room, (k, far, room, update)
