"""The norm with the residual's addition and int8 codes against its definition: every output has one right value (the sum of
squares in 64 bits, every other step one rounding to 32), so all are compared for equality."""
import pytest
import torch

import paper_2502_11880_amd as B
from tests import hip_runner as H

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rows(M, K, dtype, g, scale=1.0):
    gain = torch.exp(torch.randn(K, generator=g))
    return (torch.randn(M, K, generator=g) * gain * scale).to(T[dtype])


def _want(x, gamma, eps, res=None):
    r = x.float()
    if res is not None:
        r = (r + res.float()).to(res.dtype).float()
    K = x.shape[1]
    inv = (1.0 / torch.sqrt((r.double() ** 2).sum(1, keepdim=True) / K + torch.tensor(eps, dtype=torch.float32).double())).float()
    n = r * inv
    if gamma is not None:
        n = n * gamma
    s = torch.tensor(127.0) / n.abs().amax(1).clamp(min=1e-5)
    xq = torch.round(n * s[:, None]).clamp(-128, 127).to(torch.int8)
    return dict(r=r, y=n, x_scale=s, xq=xq, x_rowsum=xq.sum(1, dtype=torch.int32))


def _equal(got, want, what):
    assert got.dtype == want.dtype and torch.equal(got.cpu(), want), what


def _run(x, gamma, eps, res=None, y="f32", codes=True, rowsum=True, stored=True):
    M, K = x.shape
    d = dict(device=H.DEV)
    out = dict(xq=torch.full((M, K), 99, dtype=torch.int8, **d) if codes else None, x_scale=torch.full((M,), -1.0, **d) if codes else None,
               x_rowsum=torch.full((M,), 7, dtype=torch.int32, **d) if codes and rowsum else None,
               y=torch.full((M, K), float("nan"), dtype=T[y], **d) if y else None)
    if res is not None:
        out["residual_out"] = torch.full((M, K), float("nan"), dtype=res.dtype, **d) if stored else None
    B.bitnet_norm_quantize(x.to(H.DEV), None if gamma is None else gamma.to(H.DEV), eps,
                           residual=None if res is None else res.to(H.DEV), **out)
    return out


# every form of the kernel: one wave to 16 a row, one to 16 quads a thread, single values where rows are no quads, long rows
WIDTHS = [1, 2, 3, 4, 5, 63, 64, 67, 255, 256, 1023, 1024, 1028, 1030, 2048, 2052, 3200, 4096, 4097, 4100, 8190, 8192, 8640, 10240, 10244, 14336, 16384,
          16387, 16388, 33024, 65536, 65537, 65540, 70001]


@pytest.mark.parametrize("K", WIDTHS)
@pytest.mark.parametrize("M", [1, 3, 65])
def test_widths(M, K):
    print("case: norm", M, K, flush=True)
    g = torch.Generator().manual_seed(1000 * M + K)
    x, res, gamma = _rows(M, K, "f32", g), _rows(M, K, "f32", g, 3.0), 1 + 0.3 * torch.randn(K, generator=g)
    want, got = _want(x, gamma, 1e-5, res), _run(x, gamma, 1e-5, res)
    _equal(got["residual_out"], want["r"], "residual_out")
    for k in ("y", "x_scale", "xq", "x_rowsum"):
        _equal(got[k], want[k], k)


@pytest.mark.parametrize("K", [333, 640, 4096, 8640, 70001])
@pytest.mark.parametrize("x_t,r_t,y_t", [("f32", "bf16", "bf16"), ("f32", "f16", "f16"), ("bf16", "bf16", "f32"), ("f16", "f16", None),
                                         ("bf16", None, "f16"), ("f16", None, "bf16"), ("f32", None, "f32")])
def test_types(K, x_t, r_t, y_t):
    print("case: norm types", K, x_t, r_t, y_t, flush=True)
    g = torch.Generator().manual_seed(K)
    x, gamma = _rows(7, K, x_t, g), 1 + 0.3 * torch.randn(K, generator=g)
    res = _rows(7, K, r_t, g) if r_t else None
    want, got = _want(x, gamma, 1e-6, res), _run(x, gamma, 1e-6, res, y=y_t)
    if r_t:
        _equal(got["residual_out"], want["r"].to(T[r_t]), "residual_out")
    if y_t:
        _equal(got["y"], want["y"].to(T[y_t]), "y")
    for k in ("x_scale", "xq", "x_rowsum"):
        _equal(got[k], want[k], k)


@pytest.mark.parametrize("K", [100, 101, 70001])
def test_what_may_be_left_out(K):
    g = torch.Generator().manual_seed(K)
    x, res, gamma = _rows(5, K, "f32", g), _rows(5, K, "bf16", g), torch.randn(K, generator=g)
    for kw in (dict(y=None), dict(codes=False), dict(rowsum=False), dict(stored=False), dict(y=None, rowsum=False, stored=False)):
        print("case: norm without", kw, K, flush=True)
        want, got = _want(x, gamma, 1e-5, res), _run(x, gamma, 1e-5, res, **kw)
        for k in ("y", "x_scale", "xq", "x_rowsum"):
            if got[k] is not None:
                _equal(got[k], want[k], k)
    want, got = _want(x, None, 1e-5), _run(x, None, 1e-5)          # no gamma, no residual
    for k in ("y", "x_scale", "xq", "x_rowsum"):
        _equal(got[k], want[k], k)


@pytest.mark.parametrize("K", [4096, 4097, 70001])
@pytest.mark.parametrize("place", ["residual_out is residual", "residual_out is x", "y is x", "y is residual, sum not stored",
                                   "residual_out is residual, y is x", "residual_out is x, y is residual"])
def test_in_place(K, place):
    print("case: norm in place", K, place, flush=True)
    g = torch.Generator().manual_seed(K)
    x, res, gamma = _rows(70, K, "f32", g), _rows(70, K, "f32", g), torch.randn(K, generator=g)
    want = _want(x, gamma, 1e-5, res)
    dx, dr = x.to(H.DEV), res.to(H.DEV)
    out = dr if "residual_out is residual" in place else dx if "residual_out is x" in place else None
    y = dx if "y is x" in place else dr if "y is residual" in place else None
    xq, s = torch.empty(70, K, dtype=torch.int8, device=H.DEV), torch.empty(70, device=H.DEV)
    B.bitnet_norm_quantize(dx, gamma.to(H.DEV), 1e-5, xq, s, None, dr, out, y)
    _equal(xq, want["xq"], "xq")
    _equal(s, want["x_scale"], "x_scale")
    if out is not None:
        _equal(out, want["r"], "residual_out")
    if y is not None:
        _equal(y, want["y"], "y")


@pytest.mark.parametrize("K", [64, 67, 4096, 70001])
def test_extreme_values(K):
    """Squares that 32 bits cannot hold, rows of zeros, of denormals and of one value."""
    g = torch.Generator().manual_seed(K)
    x = torch.randn(8, K, generator=g)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] = 0.0
    x[3] = 3.0e38
    x[4] *= 1e-42
    x[5] = 0.0
    x[5, K - 1] = -1e-20
    x[6] = 1.0
    x[7] *= 1e-4
    want, got = _want(x, None, 1e-12), _run(x, None, 1e-12)
    for k in ("y", "x_scale", "xq", "x_rowsum"):
        _equal(got[k], want[k], k)


@pytest.mark.parametrize("K", [64, 67, 4096, 70001])
def test_values_that_are_not_finite_spoil_their_own_row(K):
    g = torch.Generator().manual_seed(K)
    x = torch.randn(70, K, generator=g)
    spoilt = x.clone()
    spoilt[1, 3], spoilt[4, K - 1], spoilt[68, 0] = float("nan"), float("inf"), -float("inf")
    want, got = _want(x, None, 1e-5), _run(spoilt, None, 1e-5)
    keep = [i for i in range(70) if i not in (1, 4, 68)]
    for k in ("y", "x_scale", "xq", "x_rowsum"):
        _equal(got[k][keep], want[k][keep], k)


@pytest.mark.parametrize("M,K", [(2, 4096), (70, 3200), (3, 335)])
def test_codes_are_those_of_the_quantiser(M, K):
    """bitnet_quantize_act on the normed rows gives the same codes, scales and sums."""
    g = torch.Generator().manual_seed(K)
    got = _run(_rows(M, K, "bf16", g), torch.randn(K, generator=g), 1e-5, _rows(M, K, "bf16", g))
    xq, s, rs = torch.empty_like(got["xq"]), torch.empty_like(got["x_scale"]), torch.empty_like(got["x_rowsum"])
    B.bitnet_quantize_act(got["y"], xq, s, rs)
    for a, b in ((xq, got["xq"]), (s, got["x_scale"]), (rs, got["x_rowsum"])):
        assert torch.equal(a, b)


def test_rows_past_two_to_the_31st_value():
    M, K = 131200, 16384
    print("case: norm of 2^31 values and more", flush=True)
    x = torch.zeros(M, K, dtype=torch.bfloat16, device=H.DEV)
    g = torch.Generator().manual_seed(5)
    last = _rows(3, K, "bf16", g)
    x[-3:] = last.to(H.DEV)
    xq, s, rs = torch.empty(M, K, dtype=torch.int8, device=H.DEV), torch.empty(M, device=H.DEV), torch.empty(M, dtype=torch.int32, device=H.DEV)
    B.bitnet_norm_quantize(x, None, 1e-5, xq, s, rs)
    want = _want(last, None, 1e-5)
    _equal(xq[-3:], want["xq"], "xq")
    _equal(s[-3:], want["x_scale"], "x_scale")
    _equal(rs[-3:], want["x_rowsum"], "x_rowsum")
    assert not bool(xq[:1000].any()) and not bool(rs[:-3].any())


def test_no_rows_and_refusals_of_the_binding():
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=H.DEV)  # noqa: E731
    B.bitnet_norm_quantize(e(0, 64), e(64), 1e-5, e(0, 64, t=torch.int8), e(0))
    x, xq, s = e(2, 64), e(2, 64, t=torch.int8), e(2)
    for kw, err in ((dict(gamma=e(63)), ValueError), (dict(xq=e(2, 65, t=torch.int8)), ValueError), (dict(x_scale=e(3)), ValueError),
                    (dict(residual=e(2, 64), residual_out=e(2, 64, t=torch.float16)), TypeError), (dict(gamma=e(64, t=torch.float16)), TypeError),
                    (dict(x=e(64, 2).t()), ValueError), (dict(x=torch.empty(2, 64)), TypeError), (dict(residual_out=e(2, 64)), B.BitnetError),
                    (dict(y=x.view(torch.int32)), TypeError), (dict(eps=0.0), B.BitnetError), (dict(x=e(2, 64, t=torch.float64)), TypeError)):
        a = dict(x=x, gamma=e(64), eps=1e-5, xq=xq, x_scale=s)
        a.update(kw)
        with pytest.raises(err):
            B.bitnet_norm_quantize(**a)
