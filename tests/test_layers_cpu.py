"""Host-side checks of the dense linear layer and the layer norm (no GPU needed, nothing is
launched): exports, refusals, workspace sizes, and the tests' own formulas against autograd."""
import ctypes
import math

import pytest
import torch

import layer_ref as R
from test_device_code import kernels, llvm, objects, resources  # noqa: F401 (fixtures)

H = pytest.importorskip("paper_2306_11987_amd", reason="libhqlss.so not built")
lib = H.lib

OK, NULL, SHAPE, BLOCK, ALIGN, DTYPE, WS, OVF, HIP, ARG, SCRATCH = range(11)
FAKE = 1 << 20
host_only = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-only ABI validation checks (fake pointers)")


def test_exports():
    raw = ctypes.CDLL(H._binding.LIB_PATH)
    for name in ("dense_linear_fwd", "dense_linear_bwd", "layer_norm_fwd", "layer_norm_bwd", "hqlss_dense_workspace_bytes",
                 "hqlss_norm_workspace_bytes"):
        assert hasattr(raw, name), name


def fwd(X=FAKE, W=FAKE, bias=None, res=None, Y=FAKE, Z=None, N=128, D=256, C=256, dt=0, act=0, ws=FAKE, nbytes=0):
    return lib.dense_linear_fwd(X, W, bias, res, Y, Z, N, D, C, dt, act, ws, nbytes, None)


@host_only
def test_dense_forward_refusals():
    for k in ("X", "W", "Y"):
        assert fwd(**{k: None}) == NULL
        assert fwd(**{k: FAKE + 8}) == ALIGN
    for k in ("bias", "res", "Z"):
        assert fwd(**{k: FAKE + 4}) == ALIGN
    for k in ("N", "D", "C"):
        assert fwd(**{k: 0}) == SHAPE
        assert fwd(**{k: -5}) == SHAPE
        assert fwd(**{k: (1 << 30) + 1}) == SHAPE
    assert fwd(D=(1 << 24) + 1) == SHAPE
    assert fwd(dt=3) == DTYPE and fwd(dt=-1) == DTYPE
    assert fwd(act=6) == ARG and fwd(act=-1) == ARG
    assert fwd(ws=FAKE + 4) == ALIGN


def bwd(dY=FAKE, Z=None, X=FAKE, W=FAKE, dX=FAKE, dW=FAKE, db=FAKE, N=128, D=256, C=256, dt=0, act=0, ws=FAKE, nbytes=0):
    return lib.dense_linear_bwd(dY, Z, X, W, dX, dW, db, N, D, C, dt, act, ws, nbytes, None)


@host_only
def test_dense_backward_refusals():
    assert bwd(dY=None) == NULL
    assert bwd(dX=None, dW=None, db=None) == NULL
    assert bwd(X=None) == NULL and bwd(W=None) == NULL  # each is read for a gradient that is asked for
    assert bwd(act=H.ACT_GELU) == NULL  # without Z
    for k in ("dY", "Z", "X", "W", "dX", "dW", "db", "ws"):
        assert bwd(**{k: FAKE + 8}) == ALIGN
    assert bwd(N=0) == SHAPE and bwd(C=(1 << 24) + 1) == SHAPE
    assert bwd(dt=7) == DTYPE
    assert bwd(act=6) == ARG
    assert bwd(ws=None) == WS
    need = H.dense_workspace_bytes(H.WS_DENSE_BWD, 128, 256, 256, torch.float32)
    assert need > 0 and bwd(Z=FAKE, act=H.ACT_GELU, nbytes=need - 1) == WS


def nfwd(X=FAKE, gamma=None, beta=None, Y=FAKE, mean=None, rstd=None, N=8, D=64, dt=0, eps=1e-5):
    return lib.layer_norm_fwd(X, gamma, beta, Y, mean, rstd, N, D, dt, eps, None)


def nbwd(dY=FAKE, X=FAKE, gamma=None, mean=FAKE, rstd=FAKE, past=None, dX=FAKE, dg=FAKE, db=FAKE, N=8, D=64, dt=0, ws=FAKE, nbytes=0):
    return lib.layer_norm_bwd(dY, X, gamma, mean, rstd, past, dX, dg, db, N, D, dt, ws, nbytes, None)


@host_only
def test_norm_refusals():
    for k in ("X", "Y"):
        assert nfwd(**{k: None}) == NULL
    for k in ("X", "gamma", "beta", "Y", "mean", "rstd"):
        assert nfwd(**{k: FAKE + 4}) == ALIGN
    assert nfwd(N=0) == SHAPE and nfwd(D=0) == SHAPE and nfwd(D=(1 << 24) + 1) == SHAPE and nfwd(N=(1 << 30) + 1) == SHAPE
    assert nfwd(dt=3) == DTYPE
    for eps in (-1e-5, math.nan, math.inf):
        assert nfwd(eps=eps) == ARG
    for k in ("dY", "X", "mean", "rstd"):
        assert nbwd(**{k: None}) == NULL
    assert nbwd(dX=None, dg=None, db=None) == NULL
    for k in ("dY", "X", "gamma", "mean", "rstd", "past", "dX", "dg", "db", "ws"):
        assert nbwd(**{k: FAKE + 4}) == ALIGN
    assert nbwd(N=0) == SHAPE and nbwd(dt=9) == DTYPE
    assert nbwd(ws=None) == WS
    assert nbwd(nbytes=H.norm_workspace_bytes(8, 64) - 1) == WS


def test_workspace_sizes():
    b = lambda *a: H.dense_workspace_bytes(*a)  # noqa: E731
    for dt in R.DT.values():
        for which in (H.WS_DENSE_FWD, H.WS_DENSE_BWD):
            assert b(which, 0, 8, 8, dt) == b(which, 8, 0, 8, dt) == b(which, 8, 8, (1 << 24) + 1, dt) == 0
        assert b(2, 8, 8, 8, dt) == 0
        assert b(H.WS_DENSE_BWD, 8, 8, 8, dt) > 0
    assert H.norm_workspace_bytes(0, 8) == H.norm_workspace_bytes(8, 0) == 0
    assert 0 < H.norm_workspace_bytes(1, 1) <= H.norm_workspace_bytes(16384, 8192)


def test_binding_refuses_what_the_library_cannot_see():
    X, W, Y = torch.zeros(4, 8), torch.zeros(3, 8), torch.zeros(4, 3)
    with pytest.raises(ValueError):  # not on the GPU
        H.dense_linear_fwd(X, W, Y)
    want = H._binding._want
    for bad in (torch.zeros(3, 9), torch.zeros(8, 3), torch.zeros(3, 8, dtype=torch.float16), torch.zeros(3, 8)):
        with pytest.raises(ValueError):
            want("W", bad, (3, 8), torch.float32, 0)
    with pytest.raises(ValueError):
        H.dense_linear_fwd(X.to(torch.int32), W, Y)


@pytest.mark.parametrize("a", R.ACTS)
def test_reference_gradients_are_autograd_s(a):
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    X, W, b, res, dY = r(5, 7).requires_grad_(), r(3, 7).requires_grad_(), r(3).requires_grad_(), r(5, 3), r(5, 3)
    z = X @ W.t() + b
    y = R.act(z, a) + res
    dX, dW, db = torch.autograd.grad(y, (X, W, b), dY)
    got = R.dense_bwd(dY, z, X, W, a, "f32")
    for k, w in (("dX", dX), ("dW", dW), ("dbias", db)):
        assert torch.allclose(got[k][0], w, rtol=1e-12, atol=1e-12)
    f = R.dense_fwd(X, W, b, res, a, "f32")
    assert torch.allclose(f["Y"][0], y) and torch.allclose(f["Z"][0], z)


def test_reference_norm_is_torch_s():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    X, gam, bet, dY, past = r(5, 7).requires_grad_(), r(7).requires_grad_(), r(7).requires_grad_(), r(5, 7), r(5, 7)
    y = torch.nn.functional.layer_norm(X, (7,), gam, bet, 1e-3)
    dX, dg, db = torch.autograd.grad(y, (X, gam, bet), dY)
    f = R.norm_fwd(X, gam, bet, 1e-3, "f32")
    assert torch.allclose(f["Y"][0], y)
    m, s = f["mean"][0], f["rstd"][0]
    got = R.norm_bwd(dY, X, gam, m, s, past, "f32")
    for k, w in (("dX", dX + past), ("dgamma", dg), ("dbeta", db)):
        assert torch.allclose(got[k][0], w, rtol=1e-12, atol=1e-12)


def test_no_kernel_keeps_data_in_private_memory(resources):
    """But for the 256 x 256 tiles, whose few spilled addresses stay out of the main loop (below), and
    the backward of 16-bit rows of 1025 to 1536 pieces (56 bytes, faster than reading rows again)."""
    names = ("dense_kernel", "dense_pair_kernel", "direct_kernel", "direct_grads_kernel", "dense_reduce_kernel", "pad_kernel",
             "act_grad_kernel", "norm_fwd_kernel", "norm_bwd_kernel", "norm_fwd_long", "norm_bwd_long", "norm_cols_long",
             "column_reduce_kernel")
    for name in names:
        for sym, _, private in kernels(resources, name):
            assert private <= (64 if "norm_bwd_kernel" in sym and "ILi0E" not in sym and "ELi512ELi3E" in sym else 0), sym
    for sym, _, private in kernels(resources, "dense_solo"):
        assert private <= 160, sym


def test_main_loops_hold_nothing_but_their_work(objects, resources):
    """The stages of the tiles that are alone on their CU, from barrier to barrier: no private memory, and
    no wait for every load but the one before the barrier of the last stages."""
    seen = 0
    symbols = {s[:-3] for s, _, _ in kernels(resources, "dense_solo")}
    for obj in objects:
        if "dense_solo" not in llvm("llvm-readelf", "--symbols", "--wide", obj):
            continue
        for sym in symbols:
            text = llvm("llvm-objdump", "-d", "--no-show-raw-insn", "--no-leading-addr", "--disassemble-symbols=" + sym, obj)
            part = []
            for line in text.splitlines():
                ins = line.split("//")[0].strip()
                if not ins.startswith("s_barrier"):
                    part.append(ins)
                    continue
                if any(i.startswith("v_mfma") for i in part):
                    seen += 1
                    assert not any(i.startswith("scratch_") for i in part), sym
                    assert sum("vmcnt(0)" in i for i in part) <= 1, sym
                part = []
    assert seen >= 6 * 3 * 2
