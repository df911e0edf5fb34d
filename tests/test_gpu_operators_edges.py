"""The ends of what the adapters and the vocabulary losses take: values and slopes beyond fp32, the smallest factors, sums over very long
axes, sums of so few products that every piece of a value shows.  Against plain forms in 64 bits, element by element."""
import numpy as np
import pytest

import operators_reference as ref
from test_gpu_operators import DTYPES, OPS, Loss, Projection, close, dev, handle, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# ------------------------------------------------------------------------------------------ losses
@pytest.mark.parametrize("kind", list(DTYPES))
@pytest.mark.parametrize("vocab", [300, 517, 3000, 40003])
@pytest.mark.parametrize("more", [{}, dict(shift=(1, 2), gap=3), dict(in_place=True)])
def test_policy_slopes_beyond_fp32(kind, vocab, more):
    """A ratio, or a KL term, of e^120: the slope is infinite, and so is the gradient of a logit of q > 0; one of q = 0 (a logit of -inf) has
    none; the action's has the slope's sign, and at q = 1 it is NaN.  (No power here underflows: logits of a spread of three.)"""
    q = Loss([4, 5], vocab, kind, seed=4, **more)
    z = q.z
    for t in (0, 1, 2, 5):
        dead = torch.arange(vocab, device="cuda") % 7 == t % 7
        dead[int(q.action[t])] = False
        z[t, dead] = float("-inf")
    z[4], z[4, int(q.action[4])] = float("-inf"), 1.0     # a single token left
    keep = z.clone()
    logp = torch.log_softmax(z.double(), dim=1).gather(1, dev(q.action).long()[:, None])[:, 0].cpu().numpy()
    q.old[:], q.ref[:], q.adv[:] = logp, logp, 0.0
    q.old[[0, 4]], q.adv[[0, 4]] = logp[[0, 4]] - 120.0, -1.0   # the ratio, not clipped for a negative advantage: a positive slope
    q.ref[[1, 5]] = logp[[1, 5]] + 120.0                  # the KL term: a negative slope
    q.old[2], q.adv[2] = logp[2] - 120.0, 1.0             # clipped: no slope from it
    q.call("policy")
    d = q.d
    for t, sign in ((0, 1.0), (1, -1.0), (5, -1.0)):
        want = torch.where(keep[t] == float("-inf"), 0.0, -sign * float("inf"))
        want[int(q.action[t])] = sign * float("inf")
        assert torch.equal(d[t].float(), want), t
    assert torch.isnan(d[4, int(q.action[4])]) and (d[4] == 0).sum() == vocab - 1
    assert torch.isfinite(d[2]).all() and (d[2][keep[2] == float("-inf")] == 0).all()
    rest = [3, 6, 7, 8]
    assert torch.isfinite(d[rest]).all() and torch.isfinite(q.row_loss[rest]).all()
    assert torch.isposinf(q.row_loss[[0, 1, 4, 5]]).all() and torch.isfinite(q.row_loss[2])
    assert q.h.status() == 0


@pytest.mark.parametrize("bad", [[0, 0, 1], [-1, 0, 0], [1, 0, 0], [5, 5, 5]])
def test_bad_ranges_of_a_batch_without_rows_are_reported(bad):
    import paper_2102_06280_b200 as p
    q, z = Projection([0, 0], 64, 32, 4), Loss([0, 0], 100)
    rs = dev(np.array(bad, dtype=np.int32))

    def policy(loss):
        none = torch.zeros(0, device="cuda")
        z.h.policy_loss(z.z, none.int(), none, none, z.rs, none, loss=loss)

    def distill(loss):
        z.h.distill(z.z, torch.zeros(0, 5, device="cuda", dtype=torch.int32), torch.zeros(0, 5, device="cuda"), z.rs, torch.zeros(0, device="cuda"), loss=loss)

    for h, call in ((q.h, q.forward), (q.h, q.backward), (z.h, lambda: policy(None)), (z.h, lambda: policy(z.loss)), (z.h, lambda: distill(None)), (z.h, lambda: distill(z.loss))):
        q.rs, z.rs = dev(q.rowstart), dev(z.rowstart)
        call()
        assert h.status() == 0
        q.rs = z.rs = rs
        call()
        torch.cuda.synchronize()
        assert h.status() == p.STATUS_BAD_INDEX
    assert (q.G[:, q.ad.a_off: q.ad.a_off + 256] == 0).all() and (z.loss == 0).all()


# ------------------------------------------------------------------------------------------ adapters
# Sums over very long axes.  All values are positive, so truncated sums would fall short of the result by a part that grows with the axis: 2^-24 and more
# of the partial sum at every MMA.  The bounds: a run of at most 32 MMAs, each off by at most a step (2^-23) of the partial sum, whose mean over a run of positive
# terms is not above its end: 2^-18.  The runs' sums, n of them, are added with rounding, 2^-24 each of a partial sum: n 2^-24 at most for an element; over
# many elements the roundings cancel, and the mean keeps the truncation's 2^-18.  (Pieces of h, m, l: 2^-26 and less.)
def _long_sum_close(got, want, runs, what):
    rel = ((got.double() - want) / want).flatten()
    assert rel.abs().max().item() <= 2.0 ** -18 + runs * 2.0 ** -24, what
    assert abs(rel.mean().item()) <= 2.0 ** -18, what


def _ramp(shape, seed, dtype=torch.float32):
    return (0.5 + torch.rand(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))).to(dtype)


@pytest.mark.parametrize("workers,rank,rows,inp,out", [(1, 64, 9728, 131072, 8), (1, 16, 19200, 131072, 8), (2, 48, 9728, 40000, 8), (160, 8, 160, 131072, 8), (1, 64, 9728, 8, 100000)])
def test_adapters_sum_over_very_wide_rows(workers, rank, rows, inp, out):
    """hidden (and, for a wide output, d_hidden) of rows that are one of 128, again and again; too many tiles for the width to be shared by blocks."""
    import paper_2102_06280_b200 as p
    wide, down = max(inp, out), out > inp
    lay = p.lowrank_layout([(inp, out, rank)])
    ad, h = lay.adapters[0], handle(workers, lay.ld)
    X = _ramp((workers, lay.ld), 1)
    few = _ramp((128, wide), 2, torch.bfloat16)
    v = few.repeat(-(-rows // 128), 1)[:rows]
    W, other = torch.zeros(out, inp, device="cuda", dtype=torch.bfloat16), torch.zeros(rows, 8, device="cuda", dtype=torch.bfloat16)
    rs = torch.tensor([rows * w // workers for w in range(workers + 1)], dtype=torch.int32, device="cuda")
    c, hidden = torch.zeros(rows, rank, device="cuda"), torch.zeros(rows, rank, device="cuda")
    if down:
        h.lowrank_backward(ad, X, W, other, hidden, v, rs, torch.zeros_like(X), c)
    else:
        h.lowrank_forward(ad, X, W, v, rs, other, c)
    off = ad.b_off if down else ad.a_off
    want = torch.empty(rows, rank, device="cuda", dtype=torch.float64)
    for w in range(workers):
        F = X[w, off: off + rank * wide].double().view(rank, wide)
        a, b = int(rs[w]), int(rs[w + 1])
        want[a:b] = (v[a: min(b, a + 128)].double() @ F.t()).repeat(-(-(b - a) // 128), 1)[: b - a]
    _long_sum_close(c, want, wide / 512, "hidden")
    assert h.status() == 0


@pytest.mark.parametrize("rank,rows", [(64, 40000), (20, 30000), (48, 33000)])
def test_adapters_sum_over_very_many_rows(rank, rows):
    """Gradients of one worker's factors; so many columns that its rows are not shared by blocks."""
    import paper_2102_06280_b200 as p
    inp, out = 9600, 9728
    lay = p.lowrank_layout([(inp, out, rank)])
    ad, h = lay.adapters[0], handle(1, lay.ld)
    X, G = torch.zeros(1, lay.ld, device="cuda"), torch.zeros(1, lay.ld, device="cuda")
    X[:, ad.b_off: ad.b_off + rank * out] = _ramp((1, rank * out), 3) / out
    x, dy, hidden = _ramp((rows, inp), 4, torch.bfloat16), _ramp((rows, out), 5, torch.bfloat16), _ramp((rows, rank), 6)
    W, u = torch.zeros(out, inp, device="cuda", dtype=torch.bfloat16), torch.zeros(rows, rank, device="cuda")
    rs = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    h.lowrank_backward(ad, X, W, x, hidden, dy, rs, G, u)
    _long_sum_close(G[0, ad.a_off: ad.a_off + rank * inp].view(rank, inp), u.double().t() @ x.double(), rows / 512, "dA")
    _long_sum_close(G[0, ad.b_off: ad.b_off + rank * out].view(rank, out), hidden.double().t() @ dy.double(), rows / 512, "dB")
    assert h.status() == 0


# The ends of the fp32 range.  Inputs are taken as they are (fp32 or bf16 numbers); a result is off by what its sum of products may be (2 (n + 4) 2^-24 of their
# magnitudes, as everywhere), and, where it is subnormal, by three roundings to multiples of 2^-149: 2^-148 with the factor 1.5 that multiplies one.
SMALLEST = 2.0 ** -148
SHAPES = [([1, 2, 1], 136, 264, 5), ([3, 0, 9, 2], 520, 72, 16), ([1, 2, 4], 264, 200, 33), ([1, 5], 72, 136, 64),      # a few rows to a worker
          ([40, 130, 7], 136, 264, 5), ([300, 0, 280], 520, 200, 16), ([90, 60], 264, 520, 33), ([200, 70], 72, 136, 64), ([33, 65, 20], 136, 136, 48)]


def _put(q, A=None, B=None):
    for v, off in ((A, q.ad.a_off), (B, q.ad.b_off)):
        if v is not None:
            v = v.astype(np.float32)
            q.X[:, off: off + v[0].size] = dev(v.reshape(q.n, -1))
            if off == q.ad.a_off:
                q.A = v
            else:
                q.B = v


def _check_fp32(q, hidden):
    """hidden of the forward call; d_hidden, dA and dB of the backward call that is given `hidden`."""
    f64 = lambda a: np.asarray(a, dtype=np.float64)  # noqa: E731
    A, B, x, dy, c = f64(q.A), f64(q.B), host(q.x), host(q.dy), f64(hidden)
    q.forward()
    got = host(q.hidden)
    q.backward(hidden=dev(hidden))
    u, G = host(q.u), host(q.G)
    with np.errstate(all="ignore"):
        for w, a, b in ref.ranges(q.rowstart):
            def one(got, first, second, k, what):
                want, size = k * (first @ second), abs(k) * (np.abs(first) @ np.abs(second))
                close(got, want, 2 * (first.shape[1] + 4) * ref.U32 * size + SMALLEST, what)
            one(got[a:b], x[a:b], A[w].T, 1.0, "hidden")
            one(u[a:b], dy[a:b], B[w].T, q.scale, "d_hidden")
            one(G[w, q.ad.a_off: q.ad.a_off + A[w].size].reshape(A[w].shape), u[a:b].T, x[a:b], 1.0, "dA")
            one(G[w, q.ad.b_off: q.ad.b_off + B[w].size].reshape(B[w].shape), c[a:b].T, dy[a:b], q.scale, "dB")
    assert q.h.status() == 0


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("size", [1e-32, 1e-36, 1e-38, 3e-42])
def test_adapters_of_the_smallest_values(shape, size):
    q = Projection(*shape, seed=1)
    _put(q, q.A * size, q.B * size)
    _check_fp32(q, (size * np.random.default_rng(5).standard_normal((q.rows, shape[3]))).astype(np.float32))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("size", [2e31, 1e37, 2e38])
def test_adapters_of_the_largest_values(shape, size):
    """Up to the largest fp32 number; x and dy are so small that no sum passes it."""
    q, rng, most = Projection(*shape, seed=2), np.random.default_rng(6), np.finfo(np.float32).max
    q.x *= 2.0 ** -12
    q.dy *= 2.0 ** -12

    def large(like):
        v = np.clip(size * rng.standard_normal(like), -float(most), float(most)).astype(np.float32)
        v.reshape(-1)[:: 17] = most if size > 1e38 else size
        return v
    _put(q, large(q.A.shape), large(q.B.shape))
    _check_fp32(q, large((q.rows, shape[3])))


@pytest.mark.parametrize("shape", SHAPES)
def test_adapters_of_infinite_values(shape):
    """An infinite value gives what the formula gives: an infinity of its sign where the other factor has one, NaN where two disagree."""
    q, rng = Projection(*shape, seed=3), np.random.default_rng(7)
    rank, (w, a, b) = shape[3], max(ref.ranges(q.rowstart), key=lambda r: r[2] - r[1])
    A, B, hidden = q.A.copy(), q.B.copy(), rng.standard_normal((q.rows, rank)).astype(np.float32)
    A[w, rank - 1, 7], A[w, 0, 0], B[w, rank // 2, 70], hidden[a, rank - 1] = np.inf, np.nan, -np.inf, np.inf
    _put(q, A, B)
    _check_fp32(q, hidden)
    _put(q, np.ones_like(A), -2 * np.ones_like(B))        # (bf16 numbers: two of their three pieces are 0, and 0 x inf is NaN)
    q.x[a, 3], q.dy[b - 1, 11] = float("inf"), float("-inf")
    _check_fp32(q, np.ones_like(hidden))


def _check_bf16(q):
    """y and dx, each from the hidden and d_hidden that the library has for it.  The bound is the plain forms' (operators_reference.py), without what the hidden
    values are off by.  scale x hidden is an fp32 number: half a step of the smallest ones, 2^-150, times B; where two bf16 pieces hold it, or a factor, that
    is 2^-134, times the other.  Products and sums below 2^-126 may be taken as 0 (an adapter's, and W's), and y as a multiple of 2^-133.  From 2^128 (1 - 2^-9) on a
    value rounds to a bf16 infinity (the largest number is 2^128 (1 - 2^-8)); none lies so near that border that its bound reaches over it.  Where
    terms of both signs come to 2^126, beside larger ones, their fp32 sum may be an infinity of either sign, NaN or a number, by its order: such an element is not compared."""
    f64 = lambda a: np.asarray(a, dtype=np.float64)  # noqa: E731
    A, B, W, x, dy = f64(q.A), f64(q.B), host(q.W), host(q.x), host(q.dy)
    rank = A.shape[1]
    q.forward()
    q.backward()
    y, hid, dx, u = host(q.y), host(q.hidden), host(q.dx), host(q.u)
    bias = 0.0 if q.bias is None else host(q.bias)
    with np.errstate(all="ignore"):
        for w, a, b in ref.ranges(q.rowstart):
            def one(got, v, M, c, F, k, more, what):
                want, low = v @ M + k * (c @ F) + more, abs(k) * (np.abs(c) @ np.abs(F))
                off = 2 * (len(M) + 3 * rank + 4) * ref.U32 * (np.abs(v) @ np.abs(M) + low + np.abs(more)) + 2.0 ** -16 * low + (abs(k) * rank + len(M)) * 2.0 ** -126
                off = off + 2.0 ** -134 * ((1 + 2.0 ** -16) * np.abs(F).sum(axis=0) + np.abs(k * c).sum(axis=1, keepdims=True))
                border = 2.0 ** 128 * (1 - 2.0 ** -9)
                anything = np.isfinite(want) & (low >= 2.0 ** 127) & (low - np.abs(k * (c @ F)) >= 2.0 ** 126)
                got, want = np.where(anything, 0.0, got), np.where(anything, 0.0, want)
                assert not (np.abs(np.abs(want) - border) <= off)[np.isfinite(want) & ~anything].any()
                want = np.where(np.isfinite(want) & (np.abs(want) >= border), np.copysign(np.inf, want), want)
                close(got, want, off + ref.U16["bf16"] * (np.abs(want) + off) + 2.0 ** -134, what)
            one(y[a:b], x[a:b], W.T, hid[a:b], B[w], q.scale, bias, "y")
            one(dx[a:b], dy[a:b], W, u[a:b], A[w], 1.0, 0.0, "dx")
    assert q.h.status() == 0


# (few rows to a worker; little work; pairs of blocks, tiles of 128 and of 256 columns, workers of several tiles and several workers in one)
PRODUCTS = [([1, 2, 1], 136, 264, 5), ([40, 130, 7], 136, 264, 5), ([90, 60], 264, 520, 33), ([300, 0, 280, 90], 520, 2000, 16), ([700, 655], 1304, 2600, 33),
            ([200, 900], 2600, 1000, 64)]


@pytest.mark.parametrize("shape", PRODUCTS)
@pytest.mark.parametrize("a,b", [(1e30, 1e-38), (1e30, 3e-42), (1e-38, 1e30), (3e-42, 1e31), (1e-34, 1.0), (1.0, 1e-34)])
def test_adapters_share_of_small_and_large_values(shape, a, b):
    """The adapter's share alone (W is 0): factors of very different sizes, whose products are ordinary numbers."""
    q = Projection(*shape, seed=4, bias=False)
    q.W.zero_()
    _put(q, q.A * a, q.B * b)
    _check_bf16(q)


@pytest.mark.parametrize("shape", PRODUCTS)
def test_adapters_share_of_a_few_small_large_and_infinite_values(shape):
    q, rng = Projection(*shape, seed=5), np.random.default_rng(8)
    A, B = q.A.copy(), q.B.copy()
    for v in (A, B):                                      # a few values of a factor lie at the ends, most do not
        n = v.size // 50
        v.reshape(-1)[rng.choice(v.size, n, replace=False)] = rng.choice([1e-38, 1e-41, 1e-37, 1e25], size=n) * rng.standard_normal(n)
    _put(q, A, B)
    _check_bf16(q)
    most = np.finfo(np.float32).max
    A, B = q.A.copy() * 0 + 1, q.B.copy() * 0 + 2
    w = max(ref.ranges(q.rowstart), key=lambda r: r[2] - r[1])[0]
    A[w, 1, :], B[w, 2, 9], A[w, 3, 60] = 0.0, most, most
    A[w, 1, 5] = most                                     # of one value of x: hidden = x times it, large but finite for |x| < 1
    q.x[:, 5] = torch.clamp(q.x[:, 5], -0.99, 0.99)
    q.x[:, 60] = torch.clamp(q.x[:, 60], -0.25, 0.25)
    q.dy[:, 9] = torch.clamp(q.dy[:, 9], -0.25, 0.25)
    B[w, 1, :], B[w, 3, :] = 2.0 ** -20, 2.0 ** -20
    q.scale = 2.0 ** -4
    _put(q, A, B)
    _check_bf16(q)


@pytest.mark.parametrize("shape", PRODUCTS)
def test_adapters_share_of_infinite_hidden_values(shape):
    """hidden of a row that has overflowed: its y is an infinity of B's sign, not NaN, and only in its row."""
    q = Projection(*shape, seed=6, bias=False)
    w, a, b = max(ref.ranges(q.rowstart), key=lambda r: r[2] - r[1])
    A, B = q.A.copy(), q.B.copy()
    A[w, 1, 7], B[w, 0, 9] = np.inf, -np.inf              # rows of worker w: hidden[:, 1] is infinite, d_hidden[:, 0] too
    _put(q, A, B)
    _check_bf16(q)
    _put(q, np.ones_like(A), np.ones_like(B))
    q.x[a, 3], q.dy[b - 1, 11] = float("inf"), float("-inf")
    q.W.abs_()                                            # of one sign: no infinities that disagree
    _check_bf16(q)


# ------------------------------------------------------------------------------------------ together, as they are used
def test_a_policy_step_and_its_round():
    """A projection with adapters, two policy losses of its logits (the first's log-probabilities are the second's old ones), the gradient into G and the round
    that mixes the adapters; from the launches and from a graph."""
    import paper_2102_06280_b200 as p
    from oracle import dbw_oracle as orc
    from workloads import configs as wl
    rng, rank, inp, vocab = np.random.default_rng(12), 8, 136, 1000
    rowptr, col = wl.ring(5)
    lay = p.lowrank_layout([(inp, vocab, rank)])
    ad, h = lay.adapters[0], p.Dbw(rowptr, col, d=lay.ld)
    rowstart = np.concatenate([[0], np.cumsum([30, 4, 0, 170, 60])]).astype(np.int32)
    rows, rs = int(rowstart[-1]), dev(rowstart)
    X = torch.zeros(5, lay.ld, device="cuda")
    X[:, ad.a_off: ad.a_off + rank * inp] = dev(rng.standard_normal((5, rank * inp)).astype(np.float32)) / inp ** 0.5
    X[:, ad.b_off: ad.b_off + rank * vocab] = dev(rng.standard_normal((5, rank * vocab)).astype(np.float32)) * 0.3
    W, x = (dev(rng.standard_normal((vocab, inp))) / inp ** 0.5).bfloat16(), dev(rng.standard_normal((rows, inp))).bfloat16()
    action, adv, weight = rng.integers(0, vocab, size=rows).astype(np.int32), rng.standard_normal(rows).astype(np.float32), (rng.random(rows) > 0.2).astype(np.float32)
    action_d, adv_d, weight_d = dev(action), dev(adv), dev(weight)
    f32 = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    z, d, dx = (torch.zeros(rows, n, device="cuda", dtype=torch.bfloat16) for n in (vocab, vocab, inp))
    hidden, u, G, out, old, logp, row, loss = f32(rows, rank), f32(rows, rank), torch.zeros_like(X), torch.zeros_like(X), f32(rows), f32(rows), f32(rows), f32(5)
    times, b = 1.0 + rng.exponential(size=5), np.ones(5, dtype=np.int32)
    td, bd, kept, lr = dev(times), dev(b), torch.zeros(len(col), dtype=torch.uint8, device="cuda"), 0.25
    first_old = torch.full((rows,), -6.0, device="cuda")

    def step():
        h.lowrank_forward(ad, X, W, x, rs, z, hidden, scale=2.0)
        h.policy_loss(z, action_d, first_old, adv_d, rs, row, logp=old, row_weight=weight_d)
        h.policy_loss(z, action_d, old, adv_d, rs, row, loss=loss, logp=logp, d_logits=d, ref_logp=first_old, kl_coef=0.05, temperature=1.25, row_weight=weight_d)
        h.lowrank_backward(ad, X, W, x, hidden, d, rs, G, u, d_in=dx, scale=2.0)
        h.round(X, td, bd, lr, out, kept, G_ext=G)

    step()
    f = lambda v: np.float64(np.float32(v))  # noqa: E731
    args = (rowstart, weight.astype(np.float64), "bf16")
    a64, six = adv.astype(np.float64), np.full(rows, -6.0)
    was = ref.policy(host(z), action, six, None, a64, 1.0, f(0.2), f(0.2), 0.0, *args)
    close(host(old), was[6], was[7], "log-probabilities of the first loss")
    want = ref.policy(host(z), action, host(old), six, a64, 1.25, f(0.2), f(0.2), f(0.05), *args)
    close(host(loss), want[2], want[3], "loss")
    close(host(d), want[4], want[5], "d_logits")
    A, B = host(X[:, ad.a_off: ad.a_off + rank * inp]).reshape(5, rank, inp), host(X[:, ad.b_off: ad.b_off + rank * vocab]).reshape(5, rank, vocab)
    dA, eA, dB, eB, *_ = ref.lowrank_backward(A, B, host(W), host(x), host(hidden), host(d), rowstart, 2.0)
    close(host(G[:, ad.a_off: ad.a_off + rank * inp]), dA.reshape(5, -1), eA.reshape(5, -1), "dA")
    close(host(G[:, ad.b_off: ad.b_off + rank * vocab]), dB.reshape(5, -1), eB.reshape(5, -1), "dB")
    r = orc.dbw_round(rowptr, col, host(X), times, b, lr, G=host(G))
    assert np.array_equal(kept.cpu().numpy(), r["kept"])
    assert (np.abs(host(out) - r["X"]).max(axis=1) / np.abs(r["X"]).max(axis=1)).max() <= 1e-5   # the bar of the mix kernels' own tests
    first = [v.clone() for v in (z, old, logp, loss, d, G, dx, out)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for v in (z, old, logp, loss, d, G, dx, out):
        v.zero_()
    for _ in range(3):
        graph.replay()
        for v, w in zip((z, old, logp, loss, d, G, dx, out), first):
            assert torch.equal(v, w)
    assert h.status() == 0
