"""GPU parity of the digital operators beside the crossbar layers (group norm with an activation, low-rank adapters, global gradient norm and
clipped step) against their float64 definitions, at the sizes, orders and values where they can go wrong."""
import numpy as np
import pytest
import torch

from oracle import digital

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                       # half a step of a float, relative


@pytest.fixture(scope="module")
def xb():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2002_11151_amd import xbar
    xbar.lib()
    return xbar


def dev(a, dtype=np.float32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def within(got, want, bound, what=""):
    got = host(got)
    assert got.shape == want.shape, what
    off = np.abs(got - want) - bound
    assert np.isfinite(got).all() and (off <= 0).all(), "%s: %g over the bound, at %s" % (what, off.max(), np.unravel_index(off.argmax(), off.shape))


# ---- group norm ------------------------------------------------------------------------------------
KINDS = ("none", "relu", "silu")


def gn_case(shape, seed, skip):
    rng = np.random.default_rng(seed)
    x = (rng.normal(size=shape) * 2 + rng.normal(size=shape[-1])).astype(np.float32)
    dy = rng.normal(size=shape).astype(np.float32)
    gamma, beta = rng.uniform(0.5, 1.5, size=shape[-1]).astype(np.float32), rng.normal(size=shape[-1]).astype(np.float32)
    gamma[::3] *= -1
    return x, dy, gamma, beta, rng.normal(size=shape).astype(np.float32) if skip else None


def gn_check(xb, shape, groups, kind, skip, seed=0):
    x, dy, gamma, beta, s = gn_case(shape, seed, skip)
    act = KINDS.index(kind)
    sd = None if s is None else dev(s)
    y, mean, invstd = xb.gn_fwd(dev(x), dev(gamma), dev(beta), groups, 1e-5, act, sd)
    m64, i64 = digital.gn_stats(x, groups, 1e-5)
    within(mean, m64, 2 * U * np.abs(m64) + 1e-12, "mean")
    within(invstd, i64, 2.1 * U * i64, "invstd")
    m, i = host(mean), host(invstd)                                     # rounded statistics are what is used, in both directions
    xhat, z = digital.gn_z(x, gamma, beta, m, i, s)
    want = digital.act(z, kind)
    # one rounding of z; the smooth activation adds its exponential (2 U, and U |z| from its argument), a sum and a division
    slack = 1.01 * U * np.abs(want) + 1e-13 if kind != "silu" else U * (8 * np.abs(want) + 1.2 * np.abs(z)) + 1e-36
    within(y, want, slack, "y")
    got = xb.gn_bwd(dev(x), dev(dy), dev(gamma), dev(beta), mean, invstd, act, sd)
    dx, dgamma, dbeta, dskip = digital.gn_bwd(x, dy, gamma, beta, m, i, kind, s)
    e = np.abs(dy) * U * (16 + 8 * np.abs(z)) if kind == "silu" else np.zeros_like(z)      # error of the error behind the activation
    if skip:
        within(got[3], dskip, e + 1.01 * U * np.abs(dskip), "dskip")
    n, c = shape[0], shape[-1]
    mean_of = lambda t: digital._spread(t.reshape(n, -1, groups, c // groups).mean((1, 3)), x, groups)
    ge = np.abs(gamma) * e
    far = digital._spread(i, x, groups) * (ge + mean_of(ge) + np.abs(xhat) * mean_of(ge * np.abs(xhat)))
    size = digital._spread(i, x, groups) * np.abs(gamma) * np.abs(dy).max()                # of the terms, in double precision
    within(got[0], dx, far + 1.01 * U * np.abs(dx) + 1e-12 * size * (1 + np.abs(xhat)), "dx")
    axes = tuple(range(x.ndim - 1))
    within(got[1], dgamma, (e * np.abs(xhat)).sum(axes) + 1.01 * U * np.abs(dgamma) + 1e-12 * (np.abs(dy * xhat)).sum(axes), "dgamma")
    within(got[2], dbeta, e.sum(axes) + 1.01 * U * np.abs(dbeta) + 1e-12 * np.abs(dy).sum(axes), "dbeta")


# one value a group; channels that are no quads; groups across and inside a quad; one position; positions that end inside a block's share; many
# channels; many samples of next to nothing; the networks' own layers
@pytest.mark.parametrize("shape,groups", [
    ((1, 1), 1), ((3, 7), 7), ((1, 64), 4), ((2, 5, 3, 6), 3), ((2, 4, 4, 64), 32), ((3, 7, 5, 30), 5), ((2, 9, 9, 12), 1), ((1, 8, 8, 64), 16),
    ((5, 33, 31, 20), 5), ((2, 56, 56, 64), 32), ((1, 7, 7, 2048), 32), ((700, 3, 40), 8), ((1, 257, 129, 3), 3), ((4, 13, 11, 1030), 103),
    ((2, 28, 28, 512), 32), ((1, 64, 64, 128), 2), ((3, 20, 20, 96), 4), ((16, 1, 1, 4096), 64), ((2, 600, 68), 17)])
@pytest.mark.parametrize("kind,skip", [("none", False), ("relu", True), ("silu", False)])
def test_group_norm(xb, shape, groups, kind, skip):
    gn_check(xb, shape, groups, kind, skip)


@pytest.mark.parametrize("kind,skip", [("none", True), ("relu", False), ("silu", True)])
def test_group_norm_other_branches(xb, kind, skip):
    gn_check(xb, (3, 11, 9, 48), 6, kind, skip, 1)
    gn_check(xb, (2, 70, 61, 50), 10, kind, skip, 2)


def test_group_norm_of_a_constant_and_of_a_large_mean(xb):
    """A group without spread has xhat = 0 and 1 / sqrt(eps); one whose mean is 2^20 times its spread keeps the digits of the spread."""
    x = np.full((2, 6, 6, 8), 3.25, dtype=np.float32)
    one, zero = np.ones(8, np.float32), np.zeros(8, np.float32)
    y, mean, invstd = xb.gn_fwd(dev(x), dev(one), dev(zero), 2, 1e-5)
    assert not host(y).any() and (host(mean) == 3.25).all() and np.abs(host(invstd) * np.sqrt(1e-5) - 1).max() < 2.1 * U
    rng = np.random.default_rng(7)
    for shape in ((1, 40, 40, 32), (2, 130, 130, 64)):
        x = (1024.0 + rng.integers(0, 16, size=shape) * 2.0 ** -13).astype(np.float32)      # exact in float
        _, mean, invstd = xb.gn_fwd(dev(x), dev(np.ones(shape[-1])), dev(np.zeros(shape[-1])), 4, 0.0)
        m64, i64 = digital.gn_stats(x, 4, 0.0)
        within(mean, m64, 2 * U * np.abs(m64))
        within(invstd, i64, 2.1 * U * i64)


def test_group_norm_keeps_nan_to_its_group(xb):
    x, dy, gamma, beta, _ = gn_case((2, 6, 5, 16), 3, False)
    x[1, 2, 3, 5] = np.nan
    y, mean, invstd = xb.gn_fwd(dev(x), dev(gamma), dev(beta), 4)
    bad = np.zeros((2, 4), bool)
    bad[1, 1] = True
    assert np.array_equal(np.isnan(mean.cpu().numpy()), bad) and np.array_equal(np.isnan(invstd.cpu().numpy()), bad)
    lost = np.zeros(x.shape, bool)
    lost[1, :, :, 4:8] = True
    assert np.array_equal(np.isnan(y.cpu().numpy()), lost)
    dx, dgamma, _ = xb.gn_bwd(dev(x), dev(dy), dev(gamma), dev(beta), mean, invstd)
    assert np.array_equal(np.isnan(dx.cpu().numpy()), lost) and np.isnan(dgamma.cpu().numpy()).sum() == 4
    r = xb.gn_fwd(dev(x), dev(gamma), dev(beta), 4, 1e-5, xb.ACT_RELU)[0]
    assert not r.cpu().numpy()[lost].any()                                                  # as relu_fwd


# ---- adapters --------------------------------------------------------------------------------------
def adapter_case(rows, K, N, rank, n, seed, bf16=False):
    rng = np.random.default_rng(seed)
    M = len(rows)
    f = lambda *s: rng.normal(size=s).astype(np.float32)
    A, B = dev(f(n, rank, K) / np.sqrt(K)), dev(f(n, rank, N) / np.sqrt(rank))
    if bf16:
        A, B = A.bfloat16(), B.bfloat16()
    return dict(rows=np.asarray(rows, dtype=np.int32), X=f(M, K), base=f(M, N), back=f(M, K), dY=f(M, N), A=A, B=B,
                scale=rng.uniform(0.5, 2, n).astype(np.float32))


def adapter_check(xb, c, in_place=False):
    A, B, rows = c["A"], c["B"], c["rows"]
    n, rank, K = A.shape
    N, M = B.shape[2], len(rows)
    A64, B64 = host(A), host(B)
    plan = xb.adapter_plan(dev(rows, np.int32), n)
    base, X, scale, dY, back = (dev(c[k]) for k in ("base", "X", "scale", "dY", "back"))
    Y, T = xb.adapter_fwd(plan, base, X, A, B, scale, out=base if in_place else None)
    want, T64 = digital.adapter_fwd(rows, c["base"], c["X"], A64, B64, c["scale"])
    # sums of n products in single precision, whatever their order: n U times the sum of their sizes; a quarter of the terms at most is added one
    # after another (four of them meet in an instruction), then shares and waves
    aX, aA, aB, s64 = np.abs(c["X"]).astype(np.float64), np.abs(A64), np.abs(B64), np.abs(c["scale"]).astype(np.float64)
    chain = lambda k: (k / 4 + 48) * U
    sizes, aT = digital.adapter_fwd(rows, np.zeros_like(want), aX, aA, aB, s64)
    within(T, T64, chain(K) * aT + 1e-30, "T")
    within(Y, want, (chain(K) + chain(rank) + 4 * U) * sizes + 2 * U * (np.abs(c["base"]) + np.abs(want)), "Y")
    out = (rows < 0) | (rows >= n)
    assert np.array_equal(host(Y)[out], c["base"][out].astype(np.float64)) and not host(T)[out].any()
    T32 = host(T)
    dX, dA, dB = xb.adapter_bwd(plan, back, dY, X, T, A, B, scale, out=back if in_place else None)
    dXw, dAw, dBw, dT = digital.adapter_bwd(rows, c["back"], c["dY"], c["X"], T32, A64, B64, c["scale"])
    aY = np.abs(c["dY"]).astype(np.float64)
    sx, sa, sb, _ = digital.adapter_bwd(rows, np.zeros_like(dXw), aY, aX, np.abs(T32), aA, aB, s64)
    within(dX, dXw, (chain(N) + chain(rank) + 4 * U) * sx + 2 * U * (np.abs(c["back"]) + np.abs(dXw)), "dX")
    within(dA, dAw, (chain(N) + chain(M) + 4 * U) * sa + 1e-30, "dA")
    within(dB, dBw, (chain(M) + 4 * U) * sb + 1e-30, "dB")
    assert np.array_equal(host(dX)[out], c["back"][out].astype(np.float64))
    none, dA2, dB2 = xb.adapter_bwd(plan, None, dY, X, T, A, B, scale)
    assert none is None and torch.equal(dA, dA2) and torch.equal(dB, dB2)                   # without dX, and in a fixed order


def mixed(M, n, seed, share=0.15):
    rng = np.random.default_rng(seed)
    rows = rng.integers(0, n, size=M)
    rows[rng.random(M) < share] = -1
    return rows


@pytest.mark.parametrize("M,K,N,rank,n", [
    (1, 1, 1, 1, 1), (1, 2048, 1000, 8, 4), (3, 17, 5, 3, 2), (16, 64, 64, 16, 1), (17, 100, 36, 17, 3), (33, 63, 65, 5, 40), (64, 784, 500, 8, 3),
    (70, 36, 300, 33, 5), (130, 500, 10, 64, 2), (40, 129, 257, 100, 2), (50, 260, 130, 128, 7), (300, 48, 52, 4, 1), (700, 31, 70, 7, 3),
    (1500, 20, 24, 12, 900)])
@pytest.mark.parametrize("bf16", [False, True])
def test_adapters(xb, M, K, N, rank, n, bf16):
    adapter_check(xb, adapter_case(mixed(M, n, M + n), K, N, rank, n, M, bf16))


def test_adapters_without_rows_and_rows_without_adapters(xb):
    adapter_check(xb, adapter_case([-1] * 40, 20, 28, 4, 2, 1))                              # no row has one
    adapter_check(xb, adapter_case([5, -7, 2 ** 31 - 1, 0, -2 ** 31, 0], 20, 28, 4, 2, 2))    # numbers outside the range
    adapter_check(xb, adapter_case([2] * 33, 20, 28, 4, 6, 3), in_place=True)                # all rows one adapter, the others none
    adapter_check(xb, adapter_case(np.arange(130) % 65 - 1, 40, 44, 9, 64, 4), in_place=True)


@pytest.mark.parametrize("M", [31, 32, 33, 64, 65, 255, 256, 257, 512, 513, 1023, 1024, 1025])
def test_adapter_tiles_and_chunks_end_everywhere(xb, M):
    adapter_check(xb, adapter_case(np.minimum(np.arange(M) // 256, 1), 24, 20, 4, 2, M))


def test_adapters_with_many_rows_in_any_order(xb):
    rng = np.random.default_rng(9)
    rows = rng.permutation(np.repeat([0, 1, 2, -1], [8000, 37, 1, 1200]))
    adapter_check(xb, adapter_case(rows, 12, 8, 3, 4, 5))


def test_adapters_keep_infinities_to_their_rows(xb):
    """A row, an adapter or a rank that holds an infinity or a NaN spoils nothing else; what lies behind the last rank or column is not read."""
    c = adapter_case([0, 1, 0, -1, 2, 1], 22, 26, 5, 3, 6)
    clean = {k: (v.clone() if torch.is_tensor(v) else v.copy()) for k, v in c.items()}
    c["X"][1, 4], c["X"][3, 0], c["dY"][1, 2], c["dY"][3, 1] = np.inf, np.nan, np.nan, np.inf
    c["A"][2, 3, 7] = float("nan")
    c["B"][2, 4, 9] = float("inf")

    def run(c):
        plan = xb.adapter_plan(dev(c["rows"], np.int32), 3)
        X, scale = dev(c["X"]), dev(c["scale"])
        Y, T = xb.adapter_fwd(plan, dev(c["base"]), X, c["A"], c["B"], scale)
        return (Y, T) + xb.adapter_bwd(plan, dev(c["back"]), dev(c["dY"]), X, T, c["A"], c["B"], scale)
    got, want = run(c), run(clean)
    for g, w in zip(got[:3], want[:3]):
        assert torch.equal(g[[0, 2, 3, 5]], w[[0, 2, 3, 5]])
        assert torch.isfinite(w).all()
    for g, w in zip(got[3:], want[3:]):
        assert torch.equal(g[0], w[0])


def test_plan_of_another_batch_writes_nothing(xb):
    c = adapter_case([0, 1, 0, 1], 20, 24, 4, 2, 8)
    plan = xb.adapter_plan(dev(c["rows"], np.int32), 2)
    other = xb.adapter_plan(dev([0, 1, 0, 1, 1], np.int32), 2)
    other.rows = 4                                                                           # (the binding itself refuses it)
    with pytest.raises(AssertionError):
        xb.adapter_fwd(xb.adapter_plan(dev([0, 1, 0], np.int32), 2), dev(c["base"]), dev(c["X"]), c["A"], c["B"], dev(c["scale"]))
    out = torch.full((4, 24), 7.0, device="cuda")
    xb.adapter_fwd(other, dev(c["base"]), dev(c["X"]), c["A"], c["B"], dev(c["scale"]), out=out)
    assert (out == 7.0).all()
    xb.adapter_fwd(plan, dev(c["base"]), dev(c["X"]), c["A"], c["B"], dev(c["scale"]), out=out)
    assert (out != 7.0).any()


# ---- gradients of many tensors ---------------------------------------------------------------------
def grads_of(sizes, seed):
    rng = np.random.default_rng(seed)
    return [(rng.normal(size=n) * 10.0 ** rng.integers(-3, 2)).astype(np.float32) for n in sizes]


SIZES = [[1], [4], [3, 0, 5], [16384], [16385, 1, 16383], [64] * 40, [100003, 7, 65536, 2], list(range(1, 260)), [5] * 130 + [0] * 20 + [70000]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
def test_gradient_norm_and_clipping(xb, sizes):
    grads = grads_of(sizes, len(sizes))
    params = grads_of(sizes, 1000 + len(sizes))
    want = digital.grad_norm(grads)
    g = [dev(t) for t in grads]
    got = float(xb.grad_norm(g).cpu()[0])
    assert abs(got - want) <= 1.01 * U * want
    for most in (want / 3, want * 3):
        c = digital.clip_factor(want, most)
        p = [dev(t) for t in params]
        norm = xb.clip_sgd(p, g, 0.125, most)
        assert float(norm.cpu()[0]) == got
        for a, b, q in zip(p, grads, params):                         # max_norm is a float; lr c rounded, its product with g, the sum
            step = 0.125 * c * b.astype(np.float64)
            within(a, q - step, U * (np.abs(q - step) + 4 * np.abs(step)), "p")
        assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(g, grads))              # the step leaves the gradients alone
        h = [t.clone() for t in g]
        assert float(xb.grad_clip(h, most).cpu()[0]) == got
        assert all(torch.equal(xb.sgd(dev(q), b, 0.125), a) for q, b, a in zip(params, h, p) if b.numel())
        for a, b in zip(h, grads):
            if c == 1.0:
                assert np.array_equal(a.cpu().numpy(), b)
            else:
                within(a, c * b.astype(np.float64), 4 * U * np.abs(c * b.astype(np.float64)) + 1e-45, "g")


def test_step_without_a_limit_is_the_plain_one(xb):
    g, p = [dev(t) for t in grads_of([1000, 33], 5)], [dev(t) for t in grads_of([1000, 33], 6)]
    want = [xb.sgd(t.clone(), u, 0.03) for t, u in zip(p, g)]
    xb.clip_sgd(p, g, 0.03)
    assert all(torch.equal(a, b) for a, b in zip(p, want))


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_no_numbers_move_nothing(xb, bad):
    grads, params = grads_of([700, 20000], 7), grads_of([700, 20000], 8)
    grads[1][12345] = bad
    g, p = [dev(t) for t in grads], [dev(t) for t in params]
    for norm in (xb.grad_norm(g), xb.grad_clip(g, 1.0), xb.clip_sgd(p, g, 0.1, 1.0)):
        assert not np.isfinite(float(norm.cpu()[0]))
    assert all(np.array_equal(a.cpu().numpy(), b, equal_nan=True) for a, b in zip(g + p, grads + params))


def test_gradients_beyond_the_range_of_their_squares(xb):
    for size in (1e30, 1e-30):
        g = [torch.full((5000,), size, device="cuda"), torch.full((3,), size, device="cuda")]
        want = float(np.float32(size)) * np.sqrt(5003)
        assert abs(float(xb.grad_clip(g, 1e-33).cpu()[0]) - want) <= 1.01 * U * want
        assert np.abs(host(g[0]) * np.sqrt(5003) / float(np.float32(1e-33)) - 1).max() < 1e-5    # (results near the smallest normal numbers)


def test_empty_lists_of_elements(xb):
    e = torch.empty(0, device="cuda")
    assert float(xb.grad_norm([e]).cpu()[0]) == 0.0 and float(xb.clip_sgd([e, e], [e, e], 0.1, 1.0).cpu()[0]) == 0.0


# ---- how programs call them ------------------------------------------------------------------------
def test_another_stream_and_a_captured_graph(xb):
    """Every operator on a side stream, captured and replayed with new inputs in the same tensors, eager work between the replays: each replay
    gives the eager result bit for bit.  Two graphs have workspaces of their own."""
    def state(seed):
        x, dy, gamma, beta, s = gn_case((3, 9, 10, 24), seed, True)
        c = adapter_case(mixed(70, 5, seed), 240, 36, 6, 5, seed)
        return dict(x=dev(x), dy=dev(dy), gamma=dev(gamma), beta=dev(beta), skip=dev(s), rows=dev(c["rows"], np.int32), X=dev(c["X"]),
                    base=dev(c["base"]), back=dev(c["back"]), dY=dev(c["dY"]), A=c["A"], B=c["B"], scale=dev(c["scale"]),
                    p=dev(grads_of([1000], seed)[0]), q=dev(grads_of([37], seed)[0]))

    def work(s):
        y, mean, invstd = xb.gn_fwd(s["x"], s["gamma"], s["beta"], 6, 1e-5, xb.ACT_SILU, s["skip"])
        grads = xb.gn_bwd(s["x"], s["dy"], s["gamma"], s["beta"], mean, invstd, xb.ACT_SILU, s["skip"])
        plan = xb.adapter_plan(s["rows"], 5)
        Y, T = xb.adapter_fwd(plan, s["base"], s["X"], s["A"], s["B"], s["scale"])
        back = xb.adapter_bwd(plan, s["back"], s["dY"], s["X"], T, s["A"], s["B"], s["scale"])
        p = [s["p"].clone(), s["q"].clone()]
        norm = xb.clip_sgd(p, [s["p"], s["q"]], 0.1, 0.5)
        clipped = [s["p"].clone(), s["q"].clone()]
        xb.grad_clip(clipped, 0.25)
        return [y, mean, invstd, *grads, Y, T, *back, *p, norm, *clipped, xb.grad_norm([s["dY"], s["X"]])]
    fixed = [state(0), state(1)]
    graphs, outs, side = [], [], torch.cuda.Stream()
    for s in fixed:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work(s)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs.append(work(s))
        graphs.append(graph)
    for turn in range(3):
        for k in (0, 1):
            new = state(10 + 2 * turn + k)
            for name, t in fixed[k].items():
                t.copy_(new[name])
        want = [work(s) for s in fixed]
        torch.cuda.synchronize()
        for k in (1, 0):
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(outs[k], want[k]))


# ---- networks --------------------------------------------------------------------------------------
class Recorder:
    """The binding, keeping what the digital operators were given and gave."""
    joins_passes = True

    def __init__(self, xb):
        self.xb, self.calls = xb, []

    def __getattr__(self, name):
        real = getattr(self.xb, name)
        if name not in ("adapter_fwd", "adapter_bwd", "gn_fwd", "gn_bwd", "clip_sgd", "update", "fwd", "bwd"):
            return real

        def call(*args, **kw):
            copy = lambda v: v.clone() if torch.is_tensor(v) else [copy(t) for t in v] if isinstance(v, list) else v
            given = [copy(a) for a in args]
            got = real(*args, **kw)
            self.calls.append((name, given, copy(got) if torch.is_tensor(got) else tuple(copy(t) for t in got)))
            return got
        return call


def perceptron(xb, seed=2):
    import workloads
    from paper_2002_11151_amd import sequential
    spec = [("flatten",), ("fc", 60), ("groupnorm", 6, "silu"), ("fc", 10)]
    net = sequential.Sequential(workloads.config_kwargs("mlp"), spec, batch=24, in_shape=(50,), signed_input=False, seed=seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.rand((24, 50), generator=gen, device="cuda")
    labels = (torch.arange(24, device="cuda") % 10).to(torch.int32)
    net.calibrate(x, labels)
    net.frozen, net.max_grad_norm = True, 0.05
    net.add_adapters(3, 4)
    for L in net.layers:
        L.adapters.B.normal_(generator=gen).mul_(0.1)
    net.set_requests(dev([0, 1, 2, -1] * 6, np.int32))
    return net, x, labels


def test_step_of_a_frozen_network(xb):
    """One step of adapters and normalisation beside fixed crossbars, all operators together: the parameters move by the clipped gradients, which
    are those of the definitions on what went through the crossbars."""
    net, x, labels = perceptron(xb)
    net.ops = Recorder(xb)
    layers, norm = net.layers, net.stack[2][1][0]
    digital_params = [layers[1].adapters.A, layers[1].adapters.B, norm.gamma, norm.beta, layers[0].adapters.A, layers[0].adapters.B]
    before, weights = [p.clone() for p in digital_params], [L.W.clone() for L in layers]
    net.train_step(x, labels, 0.5)
    calls = net.ops.calls
    assert [c[0] for c in calls] == ["fwd", "adapter_fwd", "gn_fwd", "fwd", "adapter_fwd", "bwd", "adapter_bwd", "gn_bwd", "adapter_bwd", "clip_sgd"]
    assert all(torch.equal(L.W, w) for L, w in zip(layers, weights))
    (_, given, (y, T)), (_, gn_given, (z, mean, invstd)) = calls[1], calls[2]
    assert torch.equal(given[1], calls[0][2]) and torch.equal(gn_given[0], y) and torch.equal(calls[3][1][2], z)
    assert torch.equal(calls[6][1][1], calls[5][2]) and torch.equal(calls[7][1][1], calls[6][2][0])   # dX in place on the crossbar's error
    rows = np.array([0, 1, 2, -1] * 6)
    for k in (6, 8):
        _, (plan, base, dY, X, T, A, B, scale), (dX, dA, dB) = calls[k]
        want = digital.adapter_bwd(rows, np.zeros(X.shape), host(dY), host(X), host(T), host(A), host(B), host(scale))
        for got, w in ((dA, want[1]), (dB, want[2])):
            assert np.abs(host(got) - w).max() <= 1e-5 * np.abs(w).max()              # (60-term sums: some 2^-20 of their size)
    params, grads, lr, most = calls[9][1]
    assert [g.shape for g in grads] == [p.shape for p in digital_params] and torch.equal(grads[2], calls[7][2][1])
    size = digital.grad_norm([host(g) for g in grads])
    assert size > most and abs(float(net.grad_norm.cpu()[0]) - size) <= 1.01 * U * size
    for p, b, g in zip(digital_params, before, grads):
        step = lr * most / size * host(g)
        within(p, host(b) - step, U * (np.abs(host(b)) + 6 * np.abs(step)), "parameter")


def test_serving_with_compact_adapters(xb):
    """bfloat16 adapters give what their rounded values give, and a row without an adapter what the crossbars give."""
    net, x, labels = perceptron(xb)
    for L in net.layers:
        L.adapters.compact()
    got = net.forward(x, 0)
    for L in net.layers:
        L.adapters.A, L.adapters.B = L.adapters.A.float(), L.adapters.B.float()
    assert torch.equal(got, net.forward(x, 0))
    net.set_requests(None)
    plain = net.forward(x, 0)
    assert torch.equal(got[3::4], plain[3::4]) and not torch.equal(got, plain)


@pytest.mark.parametrize("kind", ["perceptron", "residual"])
def test_frozen_steps_from_a_hip_graph(xb, kind):
    def make():
        if kind == "perceptron":
            return perceptron(xb)
        import workloads
        from paper_2002_11151_amd import resnet_cifar
        net = resnet_cifar.ResNetCifar(workloads.config_kwargs("resnet20"), batch=4, n_blocks=1, image=8, classes=10, widths=(16, 32, 64), seed=1,
                                       norm="group", groups=4)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(5)
        x, labels = torch.randn((4, 8, 8, 3), generator=gen, device="cuda"), torch.arange(4, device="cuda").to(torch.int32)
        net.calibrate(x, labels)
        net.frozen, net.max_grad_norm = True, 0.5
        net.add_adapters(2, 5)
        net.set_requests(dev([1, 0, -1, 1], np.int32))
        return net, x, labels
    (eager, x, labels), (graphed, _, _) = make(), make()
    batches = [x, x * 0.5, x * 0.75, x * 0.25]
    want = [eager.train_step(b, labels, 0.02).clone() for b in batches]
    norms = float(eager.grad_norm.cpu()[0])
    got = [graphed.capture(batches[0], labels, 0.02).clone()]
    for b in batches[1:]:
        torch.cuda.synchronize()
        got.append(graphed.replay(b, labels).clone())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and float(graphed.grad_norm.cpu()[0]) == norms > 0
    for a, b in zip(eager.layers, graphed.layers):
        assert torch.equal(a.W, b.W)
        if a.adapters is not None:
            assert torch.equal(a.adapters.A, b.adapters.A) and torch.equal(a.adapters.B, b.adapters.B) and b.adapters.B.any()


# ---- beyond 32 bits --------------------------------------------------------------------------------
def test_elements_beyond_32_bits(xb):
    """Tensors of more than 2^31 elements: what lies at their end is right (compared there, in float64, with the same chains' bounds)."""
    for shape, groups in (((3, 12_000_000, 64), 4), ((2_200_000, 1, 1024), 1)):    # sums in three launches; groups in registers
        C = shape[-1]
        ones, zeros = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
        x = torch.empty(shape, device="cuda").normal_()
        assert x.numel() > 2 ** 31
        y, mean, invstd = xb.gn_fwd(x, ones, zeros, groups)
        part = x[-1:, -1000:].cpu().numpy()
        want = torch.stack([x[-1].reshape(-1, groups, C // groups)[:, g].double().mean() for g in range(groups)]).cpu().numpy()
        assert np.abs(host(mean[-1]) - want).max() <= 2 * U * np.abs(want).max() + 1e-12
        z = digital.gn_z(part, np.ones(C), np.zeros(C), host(mean[-1:]), host(invstd[-1:]))[1]
        within(y[-1:, -1000:], z, 1.01 * U * np.abs(z) + 1e-13)
        dx = xb.gn_bwd(x, y, ones, zeros, mean, invstd)[0]
        assert float(dx[-1, -1000:].abs().max()) < 1e-2                              # the error along y itself is taken out of dx (eps is left)
        del x, y, dx
    M, K = 40_000, 60_000
    X = torch.empty((M, K), device="cuda").normal_()
    assert X.numel() > 2 ** 31
    rows = (torch.arange(M, device="cuda") % 3 - 1).to(torch.int32)
    A, B, scale = torch.randn((2, 2, K), device="cuda"), torch.randn((2, 2, 8), device="cuda"), torch.ones(2, device="cuda")
    base = torch.randn((M, 8), device="cuda")
    plan = xb.adapter_plan(rows, 2)
    Y, T = xb.adapter_fwd(plan, base, X, A, B, scale)
    tail = slice(M - 6, M)
    c = [t.cpu().numpy() for t in (rows[tail], base[tail], X[tail], A, B, scale)]
    want, T64 = digital.adapter_fwd(*c)
    sizes, aT = digital.adapter_fwd(c[0], np.zeros_like(want), *[np.abs(t) for t in c[2:]])
    within(T[tail], T64, (K / 4 + 48) * U * aT + 1e-30)
    within(Y[tail], want, (K / 4 + 60) * U * sizes + 2 * U * (np.abs(c[1]) + np.abs(want)))
    dX = xb.adapter_bwd(plan, X, Y, X[:, :].clone(), T, A, B, scale)[0]
    dXw = digital.adapter_bwd(c[0], c[2], host(Y[tail]), c[2], host(T[tail]), c[3], c[4], c[5])[0]
    size = digital.adapter_bwd(c[0], np.zeros_like(dXw), np.abs(host(Y[tail])), c[2], host(T[tail]), np.abs(c[3]), np.abs(c[4]), c[5])[0]
    within(dX[tail], dXw, 60 * U * size + 2 * U * (np.abs(c[2]) + np.abs(dXw)))
    flat = X.reshape(-1)
    flat.zero_()
    flat[-1], flat[2 ** 31 + 5], flat[3] = 3.0, 4.0, 12.0
    assert float(xb.grad_clip([flat], 6.5).cpu()[0]) == 13.0 and float(flat[-1]) == 1.5 and float(flat[2 ** 31 + 5]) == 2.0


# ---- captured steps of networks --------------------------------------------------------------------
def test_replays_follow_the_requests(xb):
    """Other requests before every replay, memory of the plan's size taken in between: each replay is the eager step with those requests."""
    (eager, x, labels), (graphed, _, _) = perceptron(xb), perceptron(xb)
    rng = np.random.default_rng(11)
    turns = [dev(rng.integers(-1, 3, size=24), np.int32) for _ in range(4)]
    want = []
    for rows in turns:
        eager.set_requests(rows)
        want.append(eager.train_step(x, labels, 0.2).clone())
    graphed.set_requests(turns[0])
    got, taken = [graphed.capture(x, labels, 0.2).clone()], []
    for rows in turns[1:]:
        graphed.set_requests(rows)
        taken += [torch.full((n,), 1, dtype=torch.uint8, device="cuda") for n in (graphed.requests.buffer.numel(), 64, 4096)]
        torch.cuda.synchronize()
        got.append(graphed.replay(x, labels).clone())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and not torch.equal(want[0], want[1])
    for a, b in zip(eager.layers, graphed.layers):
        assert torch.equal(a.adapters.A, b.adapters.A) and torch.equal(a.adapters.B, b.adapters.B)
    graphed.set_requests(None)
    with pytest.raises(ValueError):
        graphed.replay(x, labels)


def test_norms_of_captured_steps(xb):
    """net.grad_norm after the capture, after replays and after an eager step between them: that of the eager network's step."""
    (eager, x, labels), (graphed, _, _) = perceptron(xb), perceptron(xb)
    want, got = [], []
    for step in (graphed.capture, None, None):
        eager.train_step(x, labels, 0.2)
        want.append(float(eager.grad_norm.cpu()[0]))
        graphed.replay(x, labels) if step is None else step(x, labels, 0.2)
        torch.cuda.synchronize()
        got.append(float(graphed.grad_norm.cpu()[0]))
    assert got == want and want[0] > 0


def test_weights_loaded_into_a_frozen_network(xb):
    """Weights written after the planes were programmed are what the next eager pass and the next replay run on."""
    (eager, x, labels), (graphed, _, _) = perceptron(xb), perceptron(xb)
    want, got = [eager.train_step(x, labels, 0.1).clone()], [graphed.capture(x, labels, 0.1).clone()]
    for turn in range(2):
        for net in (eager, graphed):
            net.layers[turn].W.mul_(-0.75)
        want.append(eager.train_step(x, labels, 0.1).clone())
        torch.cuda.synchronize()
        got.append(graphed.replay(x, labels).clone())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for a, b in zip(eager.layers, graphed.layers):
        fresh = xb.tile(a.cfg, a.W, a.w_max, 1 + a.index)                       # layer 0 written before step 1, layer 1 before step 2
        dy = torch.randn((3, a.N), device="cuda")                               # (the planes' own bytes have gaps that nothing writes)
        errors = [xb.bwd(a.cfg, planes, dy, a.K, a.w_max, 4.0) for planes in (fresh, a.planes, b.planes)]
        assert torch.equal(errors[0], errors[1]) and torch.equal(errors[0], errors[2])


def test_normalisation_in_front_of_the_first_convolution(xb):
    """Its parameters move by the gradients of the definition on the error that comes back through the convolution's crossbars."""
    import workloads
    from paper_2002_11151_amd import sequential
    spec = [("groupnorm", 2, "silu"), ("conv", 8, 3, 1, 1), ("relu",), ("flatten",), ("fc", 10)]
    net = sequential.Sequential(workloads.config_kwargs("resnet20"), spec, batch=5, in_shape=(7, 6, 4), seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x, labels = torch.randn((5, 7, 6, 4), generator=gen, device="cuda"), torch.arange(5, device="cuda").to(torch.int32)
    net.calibrate(x, labels)
    net.ops, norm = Recorder(xb), net.stack[0][1][0]
    net.train_step(x, labels, 0.5)
    (given, got), = [c[1:] for c in net.ops.calls if c[0] == "gn_bwd"]
    _, dgamma, dbeta, _ = digital.gn_bwd(*(host(t) for t in given[:6]), "silu")
    assert given[1].any()
    for p, g, start in ((norm.gamma, dgamma, 1.0), (norm.beta, dbeta, 0.0)):
        assert np.abs(host(p) - (start - 0.5 * g)).max() <= 1e-5 * np.abs(g).max() + 2 * U      # smooth activation: some 30 U of each term


def test_group_norm_of_the_most_positions(xb):
    """2^31 - 512 positions of one channel: what lies at their end, the statistics, and (sums of blocks up to the last) dgamma and dbeta."""
    n = 2 ** 31 - 512
    x = torch.empty((1, n, 1), device="cuda").normal_()
    one, half = torch.ones(1, device="cuda"), torch.full((1,), 0.5, device="cuda")
    y, mean, invstd = xb.gn_fwd(x, one, half, 1)
    total = [0.0, 0.0]
    for part in x.reshape(-1).split(2 ** 28):
        total = [total[0] + float(part.double().sum()), total[1] + float(part.double().square().sum())]
    m = total[0] / n
    within(mean, np.array([[m]]), 2 * U * abs(m) + 1e-12)
    within(invstd, np.array([[(total[1] / n - m * m + 1e-5) ** -0.5]]), np.array([[2.2 * U]]))
    m, i = host(mean)[0, 0], host(invstd)[0, 0]
    want = lambda t: (host(t) - m) * i
    for at in (slice(0, 1000), slice(n - 1000, n)):
        z = want(x[0, at]) + 0.5
        within(y[0, at], z, 1.01 * U * np.abs(z) + 1e-13)
    del y
    dy = torch.empty((1, n, 1), device="cuda").normal_()
    dx, dgamma, dbeta = xb.gn_bwd(x, dy, one, half, mean, invstd)
    s0 = s1 = size = 0.0
    for g, part in zip(dy.reshape(-1).split(2 ** 28), x.reshape(-1).split(2 ** 28)):
        g, xhat = g.double(), (part.double() - m) * i
        s0, s1, size = s0 + float(g.sum()), s1 + float((g * xhat).sum()), size + float((g * xhat).abs().sum())
    within(dbeta, np.array([s0]), np.array([1.01 * U * abs(s0) + 1e-12 * size]))
    within(dgamma, np.array([s1]), np.array([1.01 * U * abs(s1) + 1e-12 * size]))
    for at in (slice(0, 1000), slice(n - 1000, n)):
        z = i * (host(dy[0, at]) - s0 / n - want(x[0, at]) * s1 / n)
        within(dx[0, at], z, 1.01 * U * np.abs(z) + 1e-12)


# ---- plans of many adapters; gradients beyond 32 bits ----------------------------------------------
@pytest.mark.parametrize("M,n", [(200, 257), (256, 1100), (1, 65536), (257, 1023), (257, 1024), (600, 1025), (3000, 1500), (5000, 4100), (2500, 65536)])
def test_adapters_with_plans_of_many(xb, M, n):
    """Prefix sums over several thousand adapters, most of them without rows; batches of one launch with more adapters than threads."""
    rows = mixed(M, n, M + n)
    rows[0], rows[-1] = n - 1, 0
    adapter_check(xb, adapter_case(rows, 5, 6, 2, n, M))


def sums_of(t, *more, axes, step):
    """Sums over `axes` of a product of device tensors in float64, `step` of the longest axis at a time (all of them broadcast along it)."""
    at = int(np.argmax(t.shape))
    total = 0.0
    for part in zip(*[u.split(step, at) if u.shape[at] == t.shape[at] else [u] * -(-t.shape[at] // step) for u in (t, *more)]):
        product = part[0].double()
        for u in part[1:]:
            product = product * u.double()
        total = total + product.sum(axes)
    return total


@pytest.mark.parametrize("shape,groups", [((3, 12_000_000, 64), 4), ((2_200_000, 1, 1024), 4)], ids=["three_launches", "in_registers"])
def test_group_norm_gradients_beyond_32_bits(xb, shape, groups):
    """More than 2^31 elements, errors that have nothing to do with x: dx at both ends, all of dgamma and dbeta."""
    B, C = shape[0], shape[-1]
    gamma, beta = torch.linspace(0.5, 1.5, C, device="cuda"), torch.zeros(C, device="cuda")
    x, dy = torch.empty(shape, device="cuda").normal_(), torch.empty(shape, device="cuda").normal_()
    assert x.numel() > 2 ** 31
    _, mean, invstd = xb.gn_fwd(x, gamma, beta, groups)
    dx, dgamma, dbeta = xb.gn_bwd(x, dy, gamma, beta, mean, invstd)
    of = lambda t: t.double().repeat_interleave(C // groups, dim=1)[:, None, :]           # [batch][groups] to [batch][1][channels]
    m, i, step = of(mean), of(invstd), 400_000 if B == 3 else 60_000
    s0 = sums_of(dy, axes=(0, 1), step=step)
    s1 = sums_of(dy, x, i, axes=(0, 1), step=step) - sums_of(dy, m, i, axes=(0, 1), step=step)
    size = x.numel() / C * 4.0                                                            # of the terms: normal numbers
    within(dbeta, s0.cpu().numpy(), 1.01 * U * np.abs(s0.cpu().numpy()) + 1e-12 * size)
    within(dgamma, s1.cpu().numpy(), 1.01 * U * np.abs(s1.cpu().numpy()) + 1e-12 * size)
    for b in (0, B - 1):
        g, xhat = gamma.double(), lambda t: (t.double() - m[b]) * i[b]
        a0 = a1 = 0.0
        for d, t in zip(dy[b].split(1_000_000), x[b].split(1_000_000)):
            a0, a1 = a0 + (g * d.double()).sum(0), a1 + (g * d.double() * xhat(t)).sum(0)
        mean_of = lambda a: (a.reshape(groups, -1).sum(1) / (shape[1] * C // groups)).repeat_interleave(C // groups)
        for part in (slice(0, 500), slice(-500, None)):
            want = i[b] * (g * dy[b, part].double() - mean_of(a0) - xhat(x[b, part]) * mean_of(a1))
            want = want.cpu().numpy()
            within(dx[b, part], want, 1.01 * U * np.abs(want) + 1e-11)


def test_adapter_gradients_beyond_32_bits(xb):
    """Adapters, gradients and partial gradients of more than 2^31 elements each: the last columns of adapters with one chunk of rows and with several,
    at both ends; T and dX of the last rows."""
    M, K, N, rank, n = 8192, 600_000, 8, 128, 40
    at = torch.arange(M, device="cuda")
    rows = torch.where(at % 6 < 5, at % 6, 5 + (at // 6) % (n - 5)).to(torch.int32)
    rows[-1] = n - 1
    counts = torch.bincount(rows.long(), minlength=n).tolist()
    slots = sum(-(-c // 256) for c in counts if c > 256)                                  # chunks of 256 rows
    assert n * rank * K > 2 ** 31 and slots * rank * K > 2 ** 31 and min(counts) > 0 and counts[n - 1] <= 256 < counts[4]
    X, A = torch.empty((M, K), device="cuda").normal_(), torch.empty((n, rank, K), device="cuda").normal_()
    B, scale = torch.randn((n, rank, N), device="cuda"), 0.5 + torch.rand(n, device="cuda")
    base, dY, back = torch.randn((M, N), device="cuda"), torch.randn((M, N), device="cuda"), X.clone()
    plan = xb.adapter_plan(rows, n)
    Y, T = xb.adapter_fwd(plan, base, X, A, B, scale)
    dX, dA, dB = xb.adapter_bwd(plan, back, dY, X, T, A, B, scale, out=back)
    chain = lambda k: (k / 4 + 48) * U
    for m in (M - 1, M - 2):
        a = int(rows[m])
        x, w = X[m].double(), A[a].double()
        within(T[m], torch.mv(w, x).cpu().numpy(), chain(K) * torch.mv(w.abs(), x.abs()).cpu().numpy())
        t = T[m].double() * scale[a].double()
        want, size = torch.mv(B[a].double().t().contiguous(), t), torch.mv(B[a].double().abs().t().contiguous(), t.abs())
        within(Y[m], (base[m].double() + want).cpu().numpy(), ((chain(rank) + 4 * U) * size + 2 * U * (size + base[m].abs())).cpu().numpy())
        dT = torch.mv(B[a].double(), dY[m].double()) * scale[a].double()
        aT = torch.mv(B[a].double().abs(), dY[m].double().abs()) * scale[a].double()
        want, size = x + torch.mv(w.t().contiguous(), dT), torch.mv(w.abs().t().contiguous(), aT)
        within(dX[m], want.cpu().numpy(), ((chain(N) + chain(rank) + 4 * U) * size + 2 * U * (x.abs() + want.abs())).cpu().numpy())
    for a in (0, 4, 5, n - 1):
        mine = (rows == a).nonzero().flatten()
        y, f = dY[mine].double(), scale[a].double()
        dT, aT = (torch.matmul(u, v.t().contiguous()) * f for u, v in ((y, B[a].double()), (y.abs(), B[a].double().abs())))
        for cols in (slice(0, 64), slice(K - 64, K)):
            x = X[mine, cols].double()
            want, size = torch.matmul(dT.t().contiguous(), x), torch.matmul(aT.t().contiguous(), x.abs())
            within(dA[a][:, cols], want.cpu().numpy(), (chain(N) + chain(M) + 4 * U) * size.cpu().numpy())
        t = T[mine].double()
        want, size = (torch.matmul(u.t().contiguous(), v) * f for u, v in ((t, y), (t.abs(), y.abs())))
        within(dB[a], want.cpu().numpy(), (chain(M) + 4 * U) * size.cpu().numpy())


@pytest.mark.parametrize("frozen", [False, True])
def test_captured_steps_with_batch_norm_and_changing_requests(xb, frozen):
    """A residual network whose batch norms and adapters step together, clipped, its devices written or not: replays are the eager steps."""
    import workloads
    from paper_2002_11151_amd import resnet_cifar

    def make():
        net = resnet_cifar.ResNetCifar(workloads.config_kwargs("resnet20"), batch=4, n_blocks=1, image=8, classes=10, widths=(16, 32, 64), seed=4)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(6)
        x, labels = torch.randn((4, 8, 8, 3), generator=gen, device="cuda"), torch.arange(4, device="cuda").to(torch.int32)
        net.calibrate(x, labels)
        net.frozen, net.max_grad_norm = frozen, 0.5
        net.add_adapters(3, 5)
        return net, x, labels
    (eager, x, labels), (graphed, _, _) = make(), make()
    turns = [dev(t, np.int32) for t in ([1, 0, -1, 2], [2, 2, 2, 2], [-1, -1, -1, -1], [0, 1, 2, 0])]
    want, got = [], []
    for k, rows in enumerate(turns):
        for net, out in ((eager, want), (graphed, got)):
            net.set_requests(rows)
            step = net.train_step if net is eager else net.replay if k else net.capture
            out.append((step(x, labels).clone() if step == net.replay else step(x, labels, 0.02).clone(), net.grad_norm.clone()))
            torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(c, d) for (a, c), (b, d) in zip(got, want))
    for a, b in zip(eager.layers, graphed.layers):
        assert torch.equal(a.W, b.W)
    a, b = eager.fc.adapters, graphed.fc.adapters
    assert torch.equal(a.A, b.A) and torch.equal(a.B, b.B) and b.B.any() and torch.equal(eager.stem_bn.gamma, graphed.stem_bn.gamma)


def test_eager_steps_between_replays(xb):
    """The captured step keys its write noise by the step that it is, whatever steps ran before it."""
    (eager, x, labels), (mixed_, _, _) = perceptron(xb), perceptron(xb)
    assert all(L.cfg.flags & xb.NI_UPD_NOISE and L.cfg.upd_noise_gamma > 0 for L in eager.layers)
    eager.frozen = mixed_.frozen = False
    want = [eager.train_step(x, labels, 0.1).clone() for _ in range(5)]
    got = [mixed_.capture(x, labels, 0.1).clone(), mixed_.train_step(x, labels, 0.1).clone()]
    got += [mixed_.replay(x, labels).clone(), mixed_.train_step(x, labels, 0.1).clone(), mixed_.replay(x, labels).clone()]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a.W, b.W) for a, b in zip(eager.layers, mixed_.layers))


@pytest.mark.parametrize("shape,groups", [((1, 112, 112, 64), 1), ((2, 70, 61, 50), 1), ((1, 40, 40, 1500), 1), ((3, 50, 51, 96), 2), ((1, 6000, 3), 1), ((1, 90, 91, 5), 1)])
@pytest.mark.parametrize("kind,skip", [("none", False), ("silu", True)])
def test_group_norm_of_few_large_groups(xb, shape, groups, kind, skip):
    """Thousands of partial sums per group, more channels of a group than threads that add them up, and fewer."""
    gn_check(xb, shape, groups, kind, skip, 3)
