"""The dense steps around a decode layer's attention against 64 bits: residual
addition with RMSNorm and the 8-bit output, and products with 4-bit weights."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
TINY = 2.0 ** -100


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _np(t):
    return t.detach().to(torch.float64).cpu().numpy()


# ------------------------------------------------------------------ norm

def _norm(x, res, w, eps=1e-6, want=("sum", "y", "y8")):
    T, d = x.shape
    out = {"sum": torch.full_like(x, 7.0), "y": torch.full_like(x, 7.0),
           "y8": torch.zeros(T, d, dtype=E4M3, device=DEV), "scale": torch.full((T,), 7.0, device=DEV)}
    q8 = "y8" in want
    dm.decomoe_add_rmsnorm_q8(x, res, w, out["sum"] if "sum" in want else None, out["y"] if "y" in want else None,
                              out["y8"] if q8 else None, out["scale"] if q8 else None, eps=eps)
    torch.cuda.synchronize()
    return out


def _check_norm(x, res, w, eps=1e-6):
    out = _norm(x, res, w, eps)
    s = _np(x) + (0.0 if res is None else _np(res))
    v = O.rmsnorm(s, eps, None if w is None else _np(w))
    # storage rounding: half an ulp of 8 (bf16) or 24 bits, the fp32 addition's
    # rounding first
    u = 2.0 ** -8 if x.dtype == BF16 else 2.0 ** -23
    assert (np.abs(_np(out["sum"]) - s) <= u * np.abs(s)).all()
    # fp32 sum of d squares by lanes and a tree (d / 32 + 10 roundings, halved by
    # the root), rsqrt (2 ulp), two products: 2^-24 each
    f = (x.shape[1] / 64 + 16) * 2.0 ** -24 + 2.0 ** -22
    assert (np.abs(_np(out["y"]) - v) <= (u + f) * np.abs(v) + 1e-37).all()
    a = np.maximum(np.abs(v).max(1), TINY)
    scale = _np(out["scale"])
    assert (np.abs(scale - a / 448) <= (f + 2.0 ** -22) * a / 448).all()
    # e4m3: half an ulp of 4 bits, or half of its smallest step, 2^-9
    q = _np(out["y8"])
    assert np.isin(q, O.e4m3_values()).all() and np.abs(q).max() <= 448
    err = np.abs(q * scale[:, None] - v)
    assert (err <= (2.0 ** -4 + 4 * f) * np.abs(v) + scale[:, None] * 2.0 ** -10 * 1.01).all()
    # the largest value of a row maps onto the largest code
    assert (np.abs(q).max(1)[np.abs(v).max(1) > TINY] == 448).all()
    return out


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(1, 8), (1, 64), (3, 72), (1, 2048), (24, 2048), (5, 4096), (2, 8192), (1, 16384),
                                 (3, 20008), (2, 65536), (1300, 2048), (400, 200), (3000, 64), (700, 5120)])
def test_add_rmsnorm_parity(dtype, T, d):
    g = torch.Generator().manual_seed(T * 7 + d)
    x, r = torch.randn(T, d, generator=g).to(dtype).to(DEV), (3 * torch.randn(T, d, generator=g)).to(dtype).to(DEV)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(dtype).to(DEV)
    full = _check_norm(x, r, w)
    _check_norm(x, None, w)
    _check_norm(x, r, None, eps=0.0)
    # outputs that are not asked for change nothing in the others
    for want in (("sum",), ("y",), ("y8",), ("sum", "y8"), ("y", "y8")):
        out = _norm(x, r, w, want=want)
        for n in want + (("scale",) if "y8" in want else ()):
            assert torch.equal(out[n].view(torch.uint8) if n == "y8" else out[n],
                               full[n].view(torch.uint8) if n == "y8" else full[n]), (n, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_add_rmsnorm_in_place(dtype):
    for d in (2048, 40000):
        x, r = (torch.randn(9, d, device=DEV).to(dtype) for _ in range(2))
        ref = _norm(x, r, None)
        a, b = x.clone(), r.clone()
        dm.decomoe_add_rmsnorm_q8(a, b, None, b, a)  # the sum onto the residual, the norm onto x
        assert torch.equal(a, ref["y"]) and torch.equal(b, ref["sum"])
        a = x.clone()
        dm.decomoe_add_rmsnorm_q8(a, r, None, a)
        assert torch.equal(a, ref["sum"])


def test_add_rmsnorm_extreme_rows():
    d = 256
    x = torch.zeros(8, d, device=DEV)
    x[1] = 1e-30
    x[2, 3] = 1.0
    x[3] = 3e4
    x[4] = torch.linspace(-1, 1, d, device=DEV) * 1e-12
    _check_norm(x[:5].contiguous(), None, None)
    _check_norm(x[:4].to(BF16), None, None)
    # a row that is not finite: its outputs follow the formula, its neighbours are untouched
    x[5, 7], x[6, 0] = float("nan"), float("inf")
    x[7] = 1.0
    out = _norm(x, None, None)
    assert torch.isnan(out["y"][5]).all() and torch.isnan(out["scale"][5]) and torch.isnan(out["y8"][5].float()).all()
    assert torch.isnan(out["y"][6, 0]) and (out["y"][6, 1:] == 0).all() and torch.isnan(out["scale"][6])
    assert torch.equal(out["y"][7], torch.ones(d, device=DEV) * out["y"][7, 0]) and torch.isfinite(out["y"][7]).all()
    assert (out["y8"][0].float() == 0).all() and torch.isfinite(out["scale"][0])


def test_add_rmsnorm_refusals():
    x = torch.zeros(2, 64, dtype=BF16, device=DEV)
    y8, s = torch.zeros(2, 64, dtype=E4M3, device=DEV), torch.zeros(2, device=DEV)
    for args in ((x, x.float(), None, x), (x, x[:1], None, x), (x, None, x[0].float(), x), (x, None, x[0, :8], x),
                 (x, None, None, None, None, y8.view(torch.uint8), s), (x, None, None, None, None, y8, s[:1]),
                 (x.cpu(), None, None, x)):
        with pytest.raises(ValueError):
            dm.decomoe_add_rmsnorm_q8(*args)
    for args in ((x, None, None), (x, None, None, x, x), (x, None, None, None, None, y8), (x, None, None, x, None, None, s),
                 (x.view(-1)[:126].view(18, 7), None, None, x.view(-1)[:126].view(18, 7))):
        with pytest.raises(dm.DecomoeError) as e:
            dm.decomoe_add_rmsnorm_q8(*args)
        assert e.value.code == dm.DECOMOE_ERR_INVALID_ARG
    with pytest.raises(TypeError):
        dm.decomoe_add_rmsnorm_q8(x.half(), None, None, x.half())


# ------------------------------------------------------------------ 4-bit weights

def _w4(T, N, K, group, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    w = torch.randint(0, 256, (N, K // 2), generator=g).to(torch.uint8)
    ws = (torch.rand(N, K // group, generator=g) * 0.02 - 0.005).to(BF16)
    x = torch.randn(T, K, generator=g)
    xs = None
    if kind == E4M3:
        a = x.abs().amax(1, keepdim=True)
        xs = (a[:, 0] / 448).float()
        x = x * 448 / a
    return x.to(kind), w, ws, xs


def _check_w4(T, N, K, group, kind, out_dtype=BF16, seed=0, pad=0):
    x, w, ws, xs = _w4(T, N, K, group, kind, seed)
    xd = torch.zeros(T, K + pad, dtype=F32).to(kind)
    xd.view(torch.uint8 if kind == E4M3 else torch.int16)[:, :K] = x.view(torch.uint8 if kind == E4M3 else torch.int16)
    if pad:
        xd.view(torch.uint8 if kind == E4M3 else torch.int16)[:, K:] = -1  # NaN in either type: never read
    xd = xd.to(DEV)[:, :K]
    out = torch.full((T * N + 3,), 5.0, dtype=out_dtype, device=DEV)
    args = (xd, w.to(DEV), ws.to(DEV), out[:T * N].view(T, N))
    dm.decomoe_w4_linear(*args, x_scale=None if xs is None else xs.to(DEV))
    torch.cuda.synchronize()
    assert (out[T * N:] == 5).all()
    first = out.clone()
    dm.decomoe_w4_linear(*args, x_scale=None if xs is None else xs.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    x64 = _np(x) * (1.0 if xs is None else _np(xs)[:, None])
    ref = x64 @ O.w4_dequant(w.numpy(), _np(ws)).T
    # products are exact; a group's sum is accumulated in fp32 by at most eight
    # products of 16 terms with |q| up to 32 (an offset included) and corrected
    # once, then scaled and added up: 2^-18 of sum |x| 16 |scale| covers them
    # twice over; then the output's own rounding
    mag = np.abs(x64) @ np.repeat(np.abs(_np(ws)), group, axis=1).T * 16
    u = 2.0 ** -8 if out_dtype == BF16 else 2.0 ** -23
    err = np.abs(_np(out[:T * N].view(T, N)) - ref)
    assert (err <= u * np.abs(ref) + 2.0 ** -18 * mag).all(), float((err - u * np.abs(ref)).max())


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,N,K", [(1, 1, 128), (1, 17, 256), (2, 64, 384), (5, 100, 1152), (8, 512, 2048), (9, 33, 640),
                                   (16, 31, 128), (17, 130, 4096), (32, 48, 1024), (33, 65, 512), (70, 40, 256)])
def test_w4_parity(kind, group, T, N, K):
    _check_w4(T, N, K, group, kind, seed=T + N)


@pytest.mark.parametrize("group,K", [(32, 32), (32, 96), (32, 160), (64, 64), (64, 192), (64, 2112), (128, 128),
                                     (128, 3200), (32, 8224), (128, 16384)])
@pytest.mark.parametrize("kind", [BF16, E4M3])
def test_w4_inner_sizes(group, K, kind):
    # one group; groups that end inside the steps that the kernel takes
    _check_w4(3, 70, K, group, kind, seed=K, out_dtype=F32)
    _check_w4(12, 19, K, group, kind, seed=K)


@pytest.mark.parametrize("T", [1, 7, 20])
def test_w4_layer_shapes(T):
    _check_w4(T, 5120, 2048, 128, E4M3, seed=T)
    _check_w4(T, 2048, 4096, 64, BF16, seed=T, out_dtype=F32)


def test_w4_rows_of_wider_ones():
    _check_w4(6, 50, 256, 64, BF16, pad=64)
    _check_w4(6, 50, 256, 64, E4M3, pad=48)
    _check_w4(20, 9, 128, 32, BF16, pad=8)


def _check_w4_large(T, N, K, group, kind, seed=0, out_dtype=F32, spread=None):
    """As _check_w4 for matrices of which 64-bit copies are made on the GPU, a
    block of columns at a time."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    ws = (torch.rand(N, K // group, generator=g, device=DEV) * 0.02 - 0.005).to(BF16)
    x = torch.randn(T, K, generator=g, device=DEV)
    if spread is not None:
        x = x * spread(x)
    xs = None
    if kind == E4M3:
        a = x.abs().amax(1, keepdim=True)
        xs = (a[:, 0] / 448).float()
        x = x * 448 / a
    x = x.to(kind)
    out = torch.full((T, N), 5.0, dtype=out_dtype, device=DEV)
    dm.decomoe_w4_linear(x, w, ws, out, x_scale=xs)
    again = torch.empty_like(out)
    dm.decomoe_w4_linear(x, w, ws, again, x_scale=xs)
    assert torch.equal(out, again)
    x64 = x.double() * (1.0 if xs is None else xs.double()[:, None])
    u = 2.0 ** -8 if out_dtype == BF16 else 2.0 ** -23
    for n in range(0, N, 4096):
        b = w[n:n + 4096].int()
        q = torch.stack([b % 16, b // 16], -1).flatten(1).double() - 8
        s = ws[n:n + 4096].double().repeat_interleave(group, 1)
        ref, mag = x64 @ (q * s).t(), x64.abs() @ s.abs().t() * 16
        err = (out[:, n:n + 4096].double() - ref).abs()
        assert (err <= u * ref.abs() + 2.0 ** -18 * mag).all(), (n, float((err / mag).max()))


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("T,N,K,group", [
    (1, 20000, 2048, 128), (3, 40001, 1024, 64), (8, 4111, 8224, 32), (9, 9000, 4096, 128), (16, 20001, 2112, 64),
    (17, 4500, 8192, 64), (32, 4500, 8192, 128), (33, 5000, 8000, 32), (32, 2100, 16384, 32), (5, 1100, 32768, 128),
    (2, 130000, 512, 128), (20, 80000, 512, 64), (12, 300, 131072, 64)])
def test_w4_large_matrices(kind, T, N, K, group):
    # the kernel that large matrices take: one pass and several over the columns, rows
    # cut inside a unit of k, x staged whole and in parts, on one block and on two
    _check_w4_large(T, N, K, group, kind, seed=T + N)


@pytest.mark.parametrize("N,K", [(500, 1024), (20000, 2048)])
def test_w4_values_of_every_size(N, K):
    # groups of values around 2^-40, 1, 2^40 and 2^100 side by side in a row, rows of one size
    def spread(x):
        e = torch.tensor([0, 40, -40, 100, 31, 35], device=DEV)
        f = 2.0 ** e[(torch.arange(K, device=DEV) // 64) % 6].float()
        f = f.expand_as(x).clone()
        f[1], f[2], f[3] = 2.0 ** 100, 2.0 ** -60, 1.0
        return f

    _check_w4_large(6, N, K, 64, BF16, spread=spread)
    _check_w4_large(6, N, K, 64, BF16, spread=spread, out_dtype=BF16)


def test_w4_large_matrix_keeps_non_finite_values_in_their_row():
    N, K = 20000, 2048
    w = torch.randint(0, 256, (N, K // 2), device=DEV, dtype=torch.uint8)
    ws = torch.full((N, K // 64), 0.01, dtype=BF16, device=DEV)
    x = torch.randn(9, K, device=DEV).to(BF16)
    out = [torch.empty(9, N, dtype=F32, device=DEV) for _ in range(2)]
    dm.decomoe_w4_linear(x, w, ws, out[0])
    x[4, 100], x[7, 5] = float("nan"), float("inf")
    dm.decomoe_w4_linear(x, w, ws, out[1])
    keep = [0, 1, 2, 3, 5, 6, 8]
    assert torch.isnan(out[1][4]).all() and not torch.isfinite(out[1][7]).any()
    assert torch.equal(out[0][keep], out[1][keep])


def test_w4_values_that_are_not_finite_stay_in_their_row():
    x, w, ws, _ = _w4(9, 40, 512, 64, BF16)
    out = [torch.empty(9, 40, dtype=F32, device=DEV) for _ in range(2)]
    for i in (0, 1):
        dm.decomoe_w4_linear(x.to(DEV), w.to(DEV), ws.to(DEV), out[i])
        x[4, 100] = float("nan")
    torch.cuda.synchronize()
    keep = [t for t in range(9) if t != 4]
    assert torch.isnan(out[1][4]).all() and torch.equal(out[0][keep], out[1][keep])


def test_w4_every_code():
    # the sixteen codes at every place of a word, one column each
    K, group = 128, 32
    x = torch.eye(K, dtype=F32).to(BF16)
    w = torch.arange(16, dtype=torch.uint8)[:, None].repeat(1, K // 2)
    w = w | (15 - w) << 4
    ws = torch.full((16, K // group), 0.5).to(BF16)
    out = torch.empty(K, 16, dtype=F32, device=DEV)
    dm.decomoe_w4_linear(x.to(DEV), w.to(DEV), ws.to(DEV), out)
    ref = O.w4_dequant(w.numpy(), _np(ws))
    assert np.array_equal(_np(out), ref.T)


def test_w4_refusals():
    x, w, ws, _ = _w4(2, 8, 128, 32, BF16)
    x, w, ws = x.to(DEV), w.to(DEV), ws.to(DEV)
    out = torch.empty(2, 8, dtype=BF16, device=DEV)
    x8, xs = x.to(E4M3), torch.ones(2, device=DEV)
    dm.decomoe_w4_linear(x, w, ws, out)
    dm.decomoe_w4_linear(x[:0], w, ws, out[:0])  # no rows: nothing to do
    for args, kw in (((x, w.view(torch.int8), ws, out), {}), ((x, w[:, :32], ws, out), {}), ((x, w, ws.float(), out), {}),
                     ((x, w, ws[:4], out), {}), ((x, w, ws, out[:1]), {}), ((x8, w, ws, out), {}),
                     ((x8, w, ws, out), {"x_scale": xs[:1]}), ((x, w.t(), ws, out), {}), ((x[:, ::2], w, ws, out), {}),
                     ((x.cpu(), w, ws, out), {})):
        with pytest.raises(ValueError):
            dm.decomoe_w4_linear(*args, **kw)
    for args, kw in (((x, w, ws, out), {"x_scale": xs}), ((x, w, ws[:, :2].contiguous()[:, :1].repeat(1, 8), out), {}),
                     ((x.float(), w, ws, out), {})):
        with pytest.raises(dm.DecomoeError) as e:
            dm.decomoe_w4_linear(*args, **kw)
        assert e.value.code == dm.DECOMOE_ERR_INVALID_ARG
    torch.cuda.synchronize()
