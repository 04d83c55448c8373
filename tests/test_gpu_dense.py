"""Dense linear layer on the GPU, through the C ABI, against its formulas in 64 bits: every
type, activation and optional argument, sizes that fill no tile and no 16-byte line, one token
to many, values that are not finite, streams, graphs and shared workspaces."""
import pytest
import torch

import layer_ref as R
from gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu


def rnd(seed, *shape, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale


def dev(t, dt):
    return None if t is None else t.to(R.DT[dt]).cuda()


class Guarded:
    """An output between two fences, all NaN at first: what is left unwritten or written past
    its ends shows."""

    def __init__(self, *shape, dt="f32"):
        n = 1
        for k in shape:
            n *= k
        self.buf = torch.full((n + 512,), float("nan"), dtype=R.DT[dt], device="cuda")
        self.t = self.buf[256:256 + n].view(*shape)
        self.n = n

    def fences(self):
        assert torch.isnan(self.buf[:256]).all() and torch.isnan(self.buf[256 + self.n:]).all(), "written past its ends"


def workspace(H, which, N, D, C, dt):
    """A workspace full of NaN: nothing in it may be read before it is written."""
    n = H.dense_workspace_bytes(which, N, D, C, R.DT[dt])
    return torch.full(((n + 3) // 4 + 64,), float("nan"), dtype=torch.float32, device="cuda").view(torch.uint8)[:max(n, 16)]


def fwd(H, N, D, C, dt, act, bias=True, res=True, keep=True, seed=0):
    X, W = dev(rnd(seed, N, D), dt), dev(rnd(seed + 1, C, D, scale=D ** -0.5), dt)
    b = dev(rnd(seed + 2, C, scale=0.3), dt) if bias else None
    r = dev(rnd(seed + 3, N, C), dt) if res else None
    Y, Z = Guarded(N, C, dt=dt), Guarded(N, C, dt=dt)
    H.dense_linear_fwd(X, W, Y.t, b, r, Z.t if keep else None, H.ACT_CODES[act], workspace(H, H.WS_DENSE_FWD, N, D, C, dt))
    torch.cuda.synchronize()
    want = R.dense_fwd(X, W, b, r, act, dt)
    R.check("Y", Y.t, want["Y"])
    if keep:
        R.check("Z", Z.t, want["Z"])
    Y.fences(), Z.fences()


def bwd(H, N, D, C, dt, act, grads=("dX", "dW", "dbias"), seed=0):
    dY, X = dev(rnd(seed, N, C, scale=0.1), dt), dev(rnd(seed + 1, N, D), dt)
    W = dev(rnd(seed + 2, C, D, scale=D ** -0.5), dt)
    Z = dev(rnd(seed + 3, N, C, scale=1.5), dt) if act != "none" else None
    out = {"dX": Guarded(N, D, dt=dt), "dW": Guarded(C, D, dt=dt), "dbias": Guarded(C, dt=dt)}
    give = lambda k: out[k].t if k in grads else None  # noqa: E731
    H.dense_linear_bwd(dY, X if "dW" in grads else None, W if "dX" in grads else None, give("dX"), give("dW"),
                       give("dbias"), Z, H.ACT_CODES[act], workspace(H, H.WS_DENSE_BWD, N, D, C, dt))
    torch.cuda.synchronize()
    want = R.dense_bwd(dY, Z, X, W, act, dt)
    for k in out:
        if k in grads:
            R.check(k, out[k].t, want[k])
        else:
            assert torch.isnan(out[k].t).all(), k
        out[k].fences()


SIZES = [(1, 1, 1), (1, 768, 768), (1, 1024, 4096), (2, 4097, 3), (3, 5, 7), (5, 64, 30), (16, 1024, 512), (17, 129, 65),
         (31, 520, 1000), (33, 96, 136), (64, 1024, 256), (100, 2048, 48), (130, 200, 72), (257, 264, 520), (300, 72, 1000),
         (513, 1000, 328), (1000, 8, 2), (2048, 64, 64), (4100, 256, 192)]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, dt):
    H = need_gpu()
    say(f"dense forward {shape} {dt}")
    i = SIZES.index(shape)
    fwd(H, *shape, dt, R.ACTS[i % 6], bias=i % 3 != 1, res=i % 2 == 0, keep=i % 4 != 3, seed=10 * i)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_backward(shape, dt):
    H = need_gpu()
    say(f"dense backward {shape} {dt}")
    i = SIZES.index(shape)
    bwd(H, *shape, dt, R.ACTS[(i + 1) % 6], seed=10 * i)


# whole and partial tiles, K of one stage to many: the sizes around every limit of the launch rules
EDGES = [(128, 64, 128), (256, 128, 256), (255, 192, 257), (384, 1032, 640), (1024, 512, 1024), (1536, 2056, 520),
         (70, 8192, 136), (2050, 328, 2056), (8200, 136, 264)]


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("shape", EDGES, ids=lambda s: "x".join(map(str, s)))
def test_tile_edges(shape, dt):
    H = need_gpu()
    say(f"dense edges {shape} {dt}")
    i = EDGES.index(shape)
    fwd(H, *shape, dt, R.ACTS[(i + 2) % 6], seed=7 * i)
    bwd(H, *shape, dt, R.ACTS[(i + 3) % 6], seed=7 * i + 1)


# both gradients at once: K of either split or not, rows that need a copy, few tokens, few outputs
PAIRS = [(928, 128, 2048), (1647, 64, 904), (341, 1011, 376), (379, 1280, 640), (9, 600, 128), (3, 128, 2368), (20, 451, 192),
         (900, 128, 64), (1674, 369, 64), (345, 30, 257), (69, 1024, 70), (1, 204, 1456),
         (1860, 1480, 896), (2031, 1415, 944), (4035, 2088, 160), (1680, 2312, 1592), (6172, 808, 1600), (6299, 885, 1560)]


@pytest.mark.parametrize("dt", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("shape", PAIRS, ids=lambda s: "x".join(map(str, s)))
def test_both_gradients(shape, dt):
    H = need_gpu()
    say(f"dense both gradients {shape} {dt}")
    i = PAIRS.index(shape)
    bwd(H, *shape, dt, R.ACTS[i % 6], seed=5 * i)
    bwd(H, *shape, dt, R.ACTS[i % 6], grads=("dX", "dW"), seed=5 * i + 1)


@pytest.mark.parametrize("dt", ["f16", "f32"])
@pytest.mark.parametrize("N", [1, 6, 130, 1025, 5000])
def test_bias_gradient(N, dt):
    H = need_gpu()
    for i, C in enumerate((1, 3, 9, 17, 63, 134, 520, 1001)):
        say(f"dense bias gradient {N} x {C} {dt}")
        bwd(H, N, 8, C, dt, R.ACTS[(N + i) % 6], grads=("dbias",), seed=i)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2001, 40), (7, 333, 40), (16, 65, 16), (40, 4097, 33), (70, 31, 9)], ids=lambda s: "x".join(map(str, s)))
def test_rows_between_dwords(shape, dt):
    H = need_gpu()
    say(f"dense odd rows {shape} {dt}")
    fwd(H, *shape, dt, "gelu", seed=2)
    bwd(H, *shape, dt, "silu", seed=3)


@pytest.mark.parametrize("dt", ["f16", "f32"])
def test_nothing_is_written_past_the_workspace(dt):
    """A workspace of exactly the queried bytes, for every set of gradients."""
    H = need_gpu()
    t = R.DT[dt]
    for N, D, C in PAIRS[:9] + [(1860, 1480, 896), (1201, 333, 203), (300, 4096, 40), (2000, 24, 72)]:
        say(f"dense workspace {N} x {D} x {C} {dt}")
        X, W, g = dev(rnd(1, N, D), dt), dev(rnd(2, C, D, scale=0.03), dt), dev(rnd(3, N, C), dt)
        for which in (H.WS_DENSE_FWD, H.WS_DENSE_BWD):
            n = H.dense_workspace_bytes(which, N, D, C, t)
            buf = torch.full((n + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
            ws = buf[:n]
            if which == H.WS_DENSE_FWD:
                for res, Z in ((None, None), (g, None), (g, torch.empty_like(g))):
                    H.dense_linear_fwd(X, W, torch.empty_like(g), None, res, Z, H.ACT_SILU, ws if n else None)
            else:
                for a, b, c in ((1, 1, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1)):
                    o = [torch.empty_like(v) if k else None for v, k in ((X, a), (W, b), (W[:, 0].contiguous(), c))]
                    H.dense_linear_bwd(g, X, W, *o, g, H.ACT_SILU, ws)
            torch.cuda.synchronize()
            assert bool((buf[n:] == 0x5A).all()), which


def test_more_tokens_than_a_grid_s_side():
    H = need_gpu()
    N, D, C = 2200000, 8, 5
    say(f"dense {N} x {D} x {C} f16")
    fwd(H, N, D, C, "f16", "relu", seed=6)
    bwd(H, N, D, C, "f16", "none", seed=7)


@pytest.mark.parametrize("dt", ["f16", "f32"])
@pytest.mark.parametrize("shape", [(1024, 128, 1032), (300, 512, 320), (64, 2048, 128)], ids=lambda s: "x".join(map(str, s)))
def test_optional_tensors(shape, dt):
    H = need_gpu()
    for res in (False, True):
        for keep in (False, True):
            say(f"dense optional tensors {shape} {dt} residual {res} Z {keep}")
            fwd(H, *shape, dt, "tanh", res=res, keep=keep, seed=4)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", R.ACTS)
def test_activations(act, dt):
    """Z over the activation's whole range: X is z itself, W the identity."""
    H = need_gpu()
    z = torch.cat([torch.linspace(-12, 12, 4001, dtype=torch.float64), torch.tensor([0.0, -0.0, 1e-6, -1e-6, 60.0, -60.0, 300.0, -300.0])])
    n = z.numel()
    X = torch.zeros(n, 8, dtype=torch.float64)
    X[:, 0] = z
    X, W = dev(X, dt), dev(torch.eye(8, dtype=torch.float64), dt)
    Y, Z, ones = Guarded(n, 8, dt=dt), Guarded(n, 8, dt=dt), torch.ones(n, 8, device="cuda", dtype=R.DT[dt])
    H.dense_linear_fwd(X, W, Y.t, None, None, Z.t, H.ACT_CODES[act])
    assert torch.equal(Z.t, X)
    R.check("act", Y.t, R.dense_fwd(X, W, None, None, act, dt)["Y"])
    dX = Guarded(n, 8, dt=dt)
    H.dense_linear_bwd(ones, None, W, dX.t, None, None, Z.t, H.ACT_CODES[act])
    R.check("slope", dX.t, R.dense_bwd(ones, X, None, W, act, dt)["dX"])


@pytest.mark.parametrize("grads", [("dX",), ("dW",), ("dbias",), ("dX", "dbias"), ("dW", "dbias"), ("dX", "dW")], ids="+".join)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_some_gradients(grads, act):
    H = need_gpu()
    bwd(H, 77, 136, 200, "bf16", act, grads, seed=3)
    bwd(H, 77, 67, 35, "f16", act, grads, seed=4)


def test_gradient_is_the_forward_s_difference():
    """The gradients along random directions against central differences of the layer in 64
    bits (step 2^-12: their error is of the order of 2^-24 of the third derivative)."""
    H = need_gpu()
    N, D, C = 40, 72, 56
    for act in R.ACTS[2:]:
        X, W, b, G = rnd(1, N, D), rnd(2, C, D, scale=D ** -0.5), rnd(3, C), rnd(4, N, C)
        X, W, b, G = (t.float().double() for t in (X, W, b, G))
        Y, Z = torch.empty(N, C, device="cuda"), torch.empty(N, C, device="cuda")
        f = lambda t: t.float().cuda()  # noqa: E731
        H.dense_linear_fwd(f(X), f(W), Y, f(b), None, Z, H.ACT_CODES[act])
        dX, dW, db = torch.empty(N, D, device="cuda"), torch.empty(C, D, device="cuda"), torch.empty(C, device="cuda")
        H.dense_linear_bwd(f(G), f(X), f(W), dX, dW, db, Z, H.ACT_CODES[act])
        loss = lambda x, w, c: (R.act(x @ w.t() + c, act) * G).sum()  # noqa: E731
        e = 2.0 ** -12
        for k, (t, g) in enumerate(((X, dX), (W, dW), (b, db))):
            d = rnd(9 + k, *t.shape)
            args = [X, W, b]
            up, dn = list(args), list(args)
            up[k], dn[k] = t + e * d, t - e * d
            want = float((loss(*up) - loss(*dn)) / (2 * e))
            got = float((g.cpu().double() * d).sum())
            scale = float((g.cpu().double() * d).norm())
            assert abs(got - want) <= 1e-4 * scale, (act, k, got, want)


def test_rows_with_values_that_are_not_finite_stay_by_themselves():
    """A token of NaN or infinities makes its own row of Y and dX not finite and no other."""
    H = need_gpu()
    for N, D, C in ((9, 64, 128), (200, 192, 136), (300, 67, 35)):
        for dt in ("bf16", "f32"):
            X, W = rnd(1, N, D), dev(rnd(2, C, D, scale=0.1), dt)
            clean = dev(X, dt)
            X[3], X[5, 0] = float("nan"), float("inf")
            bad = dev(X, dt)
            outs = []
            for x in (clean, bad):
                Y, dX = torch.empty(N, C, device="cuda", dtype=R.DT[dt]), torch.empty(N, D, device="cuda", dtype=R.DT[dt])
                H.dense_linear_fwd(x, W, Y)
                g = dev(rnd(5, N, C), dt)
                if x is bad:
                    g[3] = float("nan")
                H.dense_linear_bwd(g, None, W, dX, None)
                outs.append((Y, dX))
            keep = [i for i in range(N) if i not in (3, 5)]
            for a, b in zip(*outs):
                assert torch.equal(a[keep], b[keep])
            assert torch.isnan(outs[1][0][3]).all() and not torch.isfinite(outs[1][0][5]).any()
            assert torch.isnan(outs[1][1][3]).all()


def test_relu_and_slope_keep_nan():
    H = need_gpu()
    X = torch.full((4, 8), float("nan"), device="cuda")
    W = torch.eye(8, device="cuda")
    for act in R.ACTS:
        Y = torch.zeros(4, 8, device="cuda")
        H.dense_linear_fwd(X, W, Y, act=H.ACT_CODES[act])
        assert torch.isnan(Y).all(), act


@pytest.mark.parametrize("shape", [(40, 64, 128), (300, 520, 264), (9, 4096, 72), (33, 35, 67)], ids=lambda s: "x".join(map(str, s)))
def test_residual_may_be_the_output(shape):
    H = need_gpu()
    N, D, C = shape
    for dt in ("f16", "f32"):
        X, W, r = dev(rnd(1, N, D), dt), dev(rnd(2, C, D, scale=D ** -0.5), dt), dev(rnd(3, N, C), dt)
        want = torch.empty_like(r)
        H.dense_linear_fwd(X, W, want, None, r, None, H.ACT_TANH)
        Y = r.clone()
        H.dense_linear_fwd(X, W, Y, None, Y, None, H.ACT_TANH)
        assert torch.equal(Y, want)


@pytest.mark.parametrize("shape", [(700, 1024, 264), (1860, 1480, 896), (901, 333, 200)], ids=lambda s: "x".join(map(str, s)))
def test_equal_inputs_give_equal_bits_on_any_stream(shape):
    """Twice in turn on the default stream, then on two other streams at once, each with its own
    workspace and outputs."""
    H = need_gpu()
    say(f"dense streams {shape}")
    N, D, C = shape
    for dt in ("bf16", "f32"):
        X, W, g, z = dev(rnd(1, N, D), dt), dev(rnd(2, C, D, scale=0.03), dt), dev(rnd(3, N, C), dt), dev(rnd(4, N, C), dt)

        def call():
            o = [torch.empty_like(t) for t in (g, X, W, W[:, 0].contiguous())]
            H.dense_linear_fwd(X, W, o[0], act=H.ACT_GELU)
            H.dense_linear_bwd(g, X, W, o[1], o[2], o[3], z, H.ACT_GELU)
            return o

        a, b = call(), call()
        torch.cuda.synchronize()
        s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
        with torch.cuda.stream(s1):
            c = call()
        with torch.cuda.stream(s2):
            d = call()
        torch.cuda.synchronize()
        for o in (b, c, d):
            assert all(torch.equal(p, q) for p, q in zip(a, o))
        only = torch.empty_like(a[3])  # the bias gradient's sums have one order, whatever adds them
        H.dense_linear_bwd(g, None, None, None, None, only, z, H.ACT_GELU)
        assert torch.equal(only, a[3])


def test_two_graphs_share_a_workspace():
    """Captured calls of different sizes on one workspace, replayed in turn with eager calls
    between them: every replay gives the eager bits."""
    H = need_gpu()
    shapes = [(33, 2048, 136), (300, 264, 520), (1860, 1480, 896), (1201, 333, 200)]
    dt = "f16"
    ws = torch.empty(max(H.dense_workspace_bytes(w, *s, R.DT[dt]) for s in shapes for w in (H.WS_DENSE_FWD, H.WS_DENSE_BWD)) + 16,
                     dtype=torch.uint8, device="cuda")
    calls, graphs = [], []
    for i, (N, D, C) in enumerate(shapes):
        X, W, g = dev(rnd(i, N, D), dt), dev(rnd(i + 2, C, D, scale=0.03), dt), dev(rnd(i + 4, N, C), dt)
        b, r = dev(rnd(i + 6, C), dt), dev(rnd(i + 8, N, C), dt)
        outs = [torch.empty_like(t) for t in (g, g, X, W, b)]

        def call(X=X, W=W, g=g, b=b, r=r, o=outs):
            H.dense_linear_fwd(X, W, o[0], b, r, o[1], H.ACT_SILU, ws)
            H.dense_linear_bwd(g, X, W, o[2], o[3], o[4], o[1], H.ACT_SILU, ws)

        call()
        torch.cuda.synchronize()
        calls.append((call, outs, [t.clone() for t in outs]))
    side = torch.cuda.Stream()
    for call, _, _ in calls:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    torch.cuda.synchronize()
    for rep in range(3):
        for graph, (call, outs, ref) in zip(graphs, calls):
            for t in outs:
                t.fill_(float("nan"))
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(outs, ref)), rep
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(outs, ref)), rep


def test_a_block_of_a_transformer():
    """h = x + W2 gelu(W1 norm(x) + b1) + b2 and its gradients, as a program strings the calls
    together, with the quantised product beside them on the same activations."""
    H = need_gpu()
    N, D, F, dt = 384, 128, 512, "f32"
    t = lambda x: x.float().double()  # noqa: E731
    x, gam, bet = t(rnd(1, N, D)), t(1 + 0.1 * rnd(2, D)), t(0.1 * rnd(3, D))
    w1, b1, w2, b2 = t(rnd(4, F, D, scale=D ** -0.5)), t(rnd(5, F)), t(rnd(6, D, F, scale=F ** -0.5)), t(rnd(7, D))
    dh = t(rnd(8, N, D))
    leaves = [v.clone().requires_grad_() for v in (x, gam, bet, w1, b1, w2, b2)]
    X, G, B, W1, B1, W2, B2 = leaves
    mu = X.mean(1, keepdim=True)
    n = (X - mu) / torch.sqrt(((X - mu) ** 2).mean(1, keepdim=True) + 1e-5) * G + B
    h = X + R.act(n @ W1.t() + B1, "gelu") @ W2.t() + B2
    want = [h, *torch.autograd.grad(h, leaves, dh)]
    X, G, B, W1, B1, W2, B2, dH = (dev(v, dt) for v in (x, gam, bet, w1, b1, w2, b2, dh))
    new = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    y, mean, rstd, z, a, out = new(N, D), new(N), new(N), new(N, F), new(N, F), new(N, D)
    H.layer_norm_fwd(X, G, B, y, mean, rstd, 1e-5)
    H.dense_linear_fwd(y, W1, a, B1, None, z, H.ACT_GELU)
    H.dense_linear_fwd(a, W2, out, B2, X)
    da, dW2, dB2, dy, dW1, dB1, dX, dG, dB = (new(*s) for s in ((N, F), (D, F), (D,), (N, D), (F, D), (F,), (N, D), (D,), (D,)))
    H.dense_linear_bwd(dH, a, W2, da, dW2, dB2)
    H.dense_linear_bwd(da, y, W1, dy, dW1, dB1, z, H.ACT_GELU)
    H.layer_norm_bwd(dy, X, G, mean, rstd, dX, dG, dB, dH)
    # fp32 throughout: chains of sums of at most 512 terms; 1e-5 of each result's size
    for name, got, ref in zip(("h", "dx", "dgamma", "dbeta", "dW1", "db1", "dW2", "db2"), (out, dX, dG, dB, dW1, dB1, dW2, dB2), want):
        e = (got.cpu().double() - ref.detach()).norm() / ref.detach().norm()
        assert e < 1e-5, (name, float(e))
    # the norm's output feeds the quantised product as it is
    yq, saved = new(N, F), H.Saved.empty(N, D, F)
    H.hq_linear_fwd(y, W1, yq, saved, 5)
    H.dense_linear_fwd(y, W1, a)
    assert (yq - a).norm() / a.norm() < 0.25
