"""hidden, d_hidden and the gradients of the adapters' factors are fp32 results: an fp32 value enters a product with a bf16 one as three bf16 pieces, and
every one of them counts.  In a long sum a lost piece would hide behind the bound of the sum; here every result has one or two products.

A sum of n products of the two is off by at most 2 (n + 2) 2^-24 of their magnitudes: the pieces' rest (2^-27), sums of the first pieces, which are truncated to
fp32, n - 1 of 2^-23, the additions of the three sums and the multiplication by the scale, 2^-24 each.  Two pieces leave 2^-18 of a value, 64 2^-24, so no more
than a few of many values stay within that; the CPU test shows it of these very inputs."""
import numpy as np
import pytest

U32 = 2.0 ** -24

# (a few rows to a worker; more, in every size of the tensor-core kernels; gradients shared by several blocks and not)
SHAPES = [([1, 3, 2, 5], 520, 264, 8), ([4, 9, 1], 136, 1000, 16), ([2, 7], 264, 520, 31), ([6, 6], 1304, 72, 64),
          ([150, 40], 520, 264, 16), ([90, 0, 130], 264, 1000, 32), ([100, 70, 33], 520, 520, 47), ([300, 33], 1000, 520, 64), ([17] * 40, 520, 264, 12),
          ([700], 2600, 2600, 10), ([260, 250], 1304, 1304, 64)]


def inputs(shape, seed=11):
    """x and dy with two values to a row, in columns that hardly repeat; bf16 numbers.  Factors and hidden values of all magnitudes around 1."""
    lengths, inp, out, rank = shape
    rng, rows = np.random.default_rng(seed), sum(lengths)

    def sparse(width):
        m = np.zeros((rows, width))
        for t in range(rows):
            m[t, [(2 * t) % width, (2 * t + 1) % width]] = np.round(128 * (1 + rng.random(2))) / 128 * rng.choice([-1.0, 1.0], 2)
        return m
    wide = lambda *s: (rng.standard_normal(s) * 2.0 ** rng.integers(-6, 7, s)).astype(np.float32)  # noqa: E731
    return sparse(inp), sparse(out), wide(len(lengths), rank, inp), wide(len(lengths), rank, out), wide(rows, rank)


def bf16(v):
    """The nearest bf16 numbers, ties to even."""
    u = np.asarray(v, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def pieces(v, n):
    """The sum of the first n."""
    rest, total = np.asarray(v, np.float32), np.zeros(np.shape(v))
    for _ in range(n):
        p = bf16(rest)
        total, rest = total + p, rest - p
    return total


def products(shape):
    """(what, first operand, fp32 operand) of every sum, worker by worker: first @ second, or for gradients second.T @ first."""
    lengths = shape[0]
    x, dy, A, B, hidden = inputs(shape)
    cuts = np.concatenate([[0], np.cumsum(lengths)])
    for w, (a, b) in enumerate(zip(cuts, cuts[1:])):
        yield "hidden", x[a:b], A[w].T
        yield "d_hidden", dy[a:b], B[w].T
        yield "dB", dy[a:b].T, hidden[a:b]


def bound(first, second):
    n = (first != 0).sum(axis=1, keepdims=True)
    return 2 * (n + 2) * U32 * (np.abs(first) @ np.abs(second))


@pytest.mark.parametrize("shape", SHAPES)
def test_the_bound_needs_three_pieces(shape):
    beyond, of = {}, {}                                   # of each kind of sum, by the number of pieces
    for what, first, second in products(shape):
        want, allowed = first @ second.astype(np.float64), bound(first, second.astype(np.float64))
        assert (np.abs(first @ pieces(second, 3) - want) <= allowed).all(), what
        for n in (1, 2):
            key = (what, n)
            beyond[key] = beyond.get(key, 0) + (np.abs(first @ pieces(second, n) - want) > allowed).sum()
            of[key] = of.get(key, 0) + (allowed > 0).sum()
    assert all(beyond[k] > 0.5 * of[k] for k in of), (beyond, of)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
def test_every_piece_counts(shape):
    torch = pytest.importorskip("torch")
    import operators_reference as ref
    from test_gpu_operators import Projection, close, dev, host
    lengths, inp, out, rank = shape
    x, dy, A, B, hidden = inputs(shape)
    q = Projection(lengths, inp, out, rank, scale=-0.75)
    q.x.copy_(dev(x))
    q.dy.copy_(dev(dy))
    assert np.array_equal(host(q.x), x) and np.array_equal(host(q.dy), dy)
    q.X[:, q.ad.a_off: q.ad.a_off + rank * inp] = dev(A.reshape(q.n, -1))
    q.X[:, q.ad.b_off: q.ad.b_off + rank * out] = dev(B.reshape(q.n, -1))
    q.forward()
    got = host(q.hidden)
    q.backward(hidden=dev(hidden))
    u, G = host(q.u), host(q.G)
    for w, a, b in ref.ranges(q.rowstart):
        def one(got, first, second, k, what):
            second = second.astype(np.float64)
            close(got, k * (first @ second), abs(k) * bound(first, second), what)
        one(got[a:b], x[a:b], A[w].T, 1.0, "hidden")
        one(u[a:b], dy[a:b], B[w].T, q.scale, "d_hidden")
        one(G[w, q.ad.a_off: q.ad.a_off + rank * inp].reshape(rank, inp).T, x[a:b].T, u[a:b], 1.0, "dA")
        one(G[w, q.ad.b_off: q.ad.b_off + rank * out].reshape(rank, out).T, dy[a:b].T, hidden[a:b], q.scale, "dB")
    assert q.h.status() == 0 and torch.isfinite(q.y).all()
