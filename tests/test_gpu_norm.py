"""Layer norm on the GPU, through the C ABI, against its formulas in 64 bits: every type and
optional argument, one column to rows that do not fit in registers, odd widths, rows of equal
values, values that are not finite, streams, graphs."""
import pytest
import torch

import layer_ref as R
from gpu_util import need_gpu, say
from test_gpu_dense import Guarded, dev, rnd

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (3, 2), (1, 1024), (5, 7), (70, 8), (300, 33), (64, 64), (129, 100), (33, 128), (1000, 255), (41, 256), (77, 500),
         (2100, 512), (18, 831), (600, 1024), (37, 1500), (5, 2048), (19, 2050), (1027, 4096), (9, 5001), (6, 8192), (3, 8200),
         (5, 11008), (4, 16384), (3, 16390), (66, 33000)]


def inputs(N, D, dt, seed):
    X = rnd(seed, N, D) * torch.exp(rnd(seed + 1, N, 1)) + 2.0 * rnd(seed + 2, N, 1)
    X[:, ::37] *= 10.0
    return dev(X, dt), dev(1 + 0.2 * rnd(seed + 3, D), dt), dev(0.3 * rnd(seed + 4, D), dt)


def stats(X, eps):
    X = X.double()
    m = X.mean(1)
    return m.float(), ((X - m[:, None]).square().mean(1) + eps).rsqrt().float()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, dt):
    H = need_gpu()
    say(f"norm forward {shape} {dt}")
    N, D = shape
    i = SIZES.index(shape)
    X, gamma, beta = inputs(N, D, dt, 5 * i)
    gamma, beta = gamma if i % 4 != 1 else None, beta if i % 4 not in (1, 2) else None
    Y, mean, rstd = Guarded(N, D, dt=dt), Guarded(N), Guarded(N)
    H.layer_norm_fwd(X, gamma, beta, Y.t, mean.t, rstd.t, 1e-5)
    torch.cuda.synchronize()
    want = R.norm_fwd(X, gamma, beta, 1e-5, dt)
    for name, g in (("Y", Y), ("mean", mean), ("rstd", rstd)):
        R.check(name, g.t, want[name])
        g.fences()
    Y2 = Guarded(N, D, dt=dt)
    H.layer_norm_fwd(X, gamma, beta, Y2.t, eps=1e-5)  # without the statistics
    assert torch.equal(Y.t, Y2.t)
    Z = X.clone()
    H.layer_norm_fwd(Z, gamma, beta, Z, eps=1e-5)  # over its input
    assert torch.equal(Y.t, Z)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(shape, dt):
    H = need_gpu()
    say(f"norm backward {shape} {dt}")
    N, D = shape
    i = SIZES.index(shape)
    X, gamma, _ = inputs(N, D, dt, 5 * i)
    mean, rstd = stats(X, 1e-5)
    gamma = gamma if i % 4 != 1 else None
    dY, past = dev(rnd(5 * i + 7, N, D), dt), dev(rnd(5 * i + 8, N, D), dt) if i % 2 else None
    dX, dg, db = Guarded(N, D, dt=dt), Guarded(D, dt=dt), Guarded(D, dt=dt)
    n = H.norm_workspace_bytes(N, D)
    ws = torch.full((n // 4 + 4,), float("nan"), device="cuda").view(torch.uint8)[:n]
    H.layer_norm_bwd(dY, X, gamma, mean, rstd, dX.t, dg.t, db.t, past, ws)
    torch.cuda.synchronize()
    want = R.norm_bwd(dY, X, gamma, mean, rstd, past, dt)
    for name, g in (("dX", dX), ("dgamma", dg), ("dbeta", db)):
        R.check(name, g.t, want[name])
        g.fences()
    # each output by itself, and dX over an input
    only = Guarded(N, D, dt=dt)
    H.layer_norm_bwd(dY, X, gamma, mean, rstd, only.t, past=past)
    assert torch.equal(only.t, dX.t)
    for k, ref in ((0, dg), (1, db)):
        one = Guarded(D, dt=dt)
        H.layer_norm_bwd(dY, X, gamma, mean, rstd, None, one.t if k == 0 else None, one.t if k else None)
        assert torch.equal(one.t, ref.t)
    for over in (dY, past):
        if over is not None:
            t = over.clone()
            H.layer_norm_bwd(t if over is dY else dY, X, gamma, mean, rstd, t, past=t if over is past else past)
            assert torch.equal(t, dX.t)
            t, g, b = over.clone(), torch.empty_like(dg.t), torch.empty_like(db.t)
            H.layer_norm_bwd(t if over is dY else dY, X, gamma, mean, rstd, t, g, b, past=t if over is past else past)
            assert torch.equal(t, dX.t) and torch.equal(g, dg.t) and torch.equal(b, db.t)


def test_rows_of_equal_values():
    """No variance: rstd is 1 / sqrt(eps), Y is beta; with eps = 0 such a row, and no other, is NaN."""
    H = need_gpu()
    for D in (1, 48, 777, 9000):
        X = rnd(1, 6, D).float().cuda() if D > 1 else torch.ones(6, 1, device="cuda")
        X[2] = 3.0
        beta = rnd(2, D).float().cuda()
        Y, mean, rstd = torch.empty_like(X), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
        H.layer_norm_fwd(X, None, beta, Y, mean, rstd, 1e-6)
        assert torch.equal(Y[2], beta) and float(mean[2]) == 3.0 and abs(float(rstd[2]) - 1e3) < 1e-3
        H.layer_norm_fwd(X, None, beta, Y, mean, rstd, 0.0)
        assert torch.isnan(Y[2]).all()
        if D > 1:
            assert torch.isfinite(Y[[0, 1, 3, 4, 5]]).all()


def test_far_offset_rows():
    """A mean a thousand times the deviation: the variance is of the differences, not of squares."""
    H = need_gpu()
    for D in (40, 1000, 4096):
        X = (1000.0 + rnd(1, 33, D)).float().cuda()
        Y, mean, rstd = torch.empty_like(X), torch.empty(33, device="cuda"), torch.empty(33, device="cuda")
        H.layer_norm_fwd(X, None, None, Y, mean, rstd, 1e-5)
        want = R.norm_fwd(X, None, None, 1e-5, "f32")
        R.check("Y", Y, want["Y"])
        R.check("rstd", rstd, want["rstd"])
        assert (rstd.cpu().double() / want["rstd"][0] - 1).abs().max() < 1e-3


def test_rows_that_are_not_finite_stay_by_themselves():
    H = need_gpu()
    for N, D, dt in ((64, 24, "bf16"), (40, 1000, "f32"), (9, 8192, "f16"), (5, 40000, "bf16")):
        X, gamma, beta = inputs(N, D, dt, 3)
        bad = X.clone()
        bad[1, D // 2], bad[3] = float("inf"), float("nan")
        Y, Yb = torch.empty_like(X), torch.empty_like(X)
        H.layer_norm_fwd(X, gamma, beta, Y)
        H.layer_norm_fwd(bad, gamma, beta, Yb)
        keep = [i for i in range(N) if i not in (1, 3)]
        assert torch.equal(Y[keep], Yb[keep])
        assert torch.isnan(Yb[3]).all() and not torch.isfinite(Yb[1]).any()


def test_gradient_is_the_forward_s_difference():
    H = need_gpu()
    N, D = 30, 75
    X, gam, bet, G = (rnd(k, *s).float().double() for k, s in enumerate(((N, D), (D,), (D,), (N, D))))
    f = lambda t: t.float().cuda()  # noqa: E731
    Y, mean, rstd, dX = (torch.empty(*s, device="cuda") for s in ((N, D), (N,), (N,), (N, D)))
    dg, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    H.layer_norm_fwd(f(X), f(gam), f(bet), Y, mean, rstd)
    H.layer_norm_bwd(f(G), f(X), f(gam), mean, rstd, dX, dg, db)

    def loss(x, g, b):
        d = x - x.mean(1, keepdim=True)
        return ((d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * g + b) * G).sum()

    e, args = 2.0 ** -12, [X, gam, bet]
    for k, g in enumerate((dX, dg, db)):
        d = rnd(20 + k, *args[k].shape)
        up, dn = list(args), list(args)
        up[k], dn[k] = args[k] + e * d, args[k] - e * d
        want, along = float((loss(*up) - loss(*dn)) / (2 * e)), g.cpu().double() * d
        assert abs(float(along.sum()) - want) <= 1e-4 * float(along.norm()), k


def test_streams_and_graphs_give_the_same_bits():
    H = need_gpu()
    N, D, dt = 900, 640, "bf16"
    X, gamma, beta = inputs(N, D, dt, 1)
    dY, past = dev(rnd(7, N, D), dt), dev(rnd(8, N, D), dt)
    ws = H.norm_workspace(N, D)
    outs = [torch.empty_like(X), torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(X),
            torch.empty_like(gamma), torch.empty_like(gamma)]

    def call():
        H.layer_norm_fwd(X, gamma, beta, *outs[:3])
        H.layer_norm_bwd(dY, X, gamma, outs[1], outs[2], outs[3], outs[4], outs[5], past, ws)

    call()
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for rep in range(3):
        for t in outs:
            t.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref)), rep
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref)), rep
