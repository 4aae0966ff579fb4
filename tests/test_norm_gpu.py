"""The residual stream's norm on the GPU against the 64-bit reference.

With u = 2^-24 and half a step of the result's type for its last rounding: the sum of squares
passes at most 64 additions in a lane and 10 over lanes and waves, the rest of y 6 roundings, and
a fused or matrix sum may truncate, so an entry of y is within 80 * 2 u of itself.  dx adds a
second sum of the kind: 160 * 2 u of |dsum| + r (|u| + |n| mean |u n|).  dweight adds rows one
after the other in a lane (at most rows / (blocks rows of a block)), then 32 rows of a block and
the blocks' parts with compensation: (that + 32 + 80 + 8) 2 u of the sum's absolute terms.
In eight bits half a step is 2^-4 of a value, or 2^-10 of its scale below 2^-6 scales.
"""
import pytest
import torch

from oracle import gbla_block as ref
from paper_2606_07317_amd import gbla
from tests.test_decoder_gpu import BF16, F32, U, _check, _dev, _gen, _randn

pytestmark = pytest.mark.gpu

EPS = 1e-5
SIZES = [(1, 8), (3, 40), (5, 64), (17, 72), (9, 128), (33, 256), (6, 264), (2, 512), (7, 1000), (4, 1024), (5, 2048),
         (3, 2056), (2, 4096), (3, 5120), (2, 8200), (1, 16384), (300, 128), (2500, 512)]


def _case(rows, width, dtype, residual=True, seed=0):
    gen = _gen(seed)
    t = dict(x=_randn(gen, rows, width, dtype=dtype), res=_randn(gen, rows, width, dtype=dtype, scale=4.0),
             w=1 + 0.3 * _randn(gen, width), dy=_randn(gen, rows, width, dtype=dtype),
             ds=_randn(gen, rows, width, dtype=dtype))
    if rows > 2:
        t["x"][1], t["res"][1] = 0, 0
    if not residual:
        t["res"] = None
    return t


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm(rows, width, dtype):
    for residual in (True, False):
        t = _case(rows, width, dtype, residual)
        x, res, w = _dev(t["x"], t["res"], t["w"])
        y, s = gbla.add_rms_norm(x, w, res, EPS)
        want, total = ref.add_norm(t["x"], t["res"], t["w"], EPS)
        assert (s is x) == (not residual) and torch.equal(s.cpu().double(), total)
        _check(y, want, want.abs(), 80 * 2 * U, "y")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm_in_eight_bits(rows, width, dtype):
    t = _case(rows, width, dtype)
    x, res, w = _dev(t["x"], t["res"], t["w"])
    want, total = ref.add_norm(t["x"], t["res"], t["w"], EPS)
    for group in (0, 128) if width % 128 == 0 else (0,):
        y, scales, s = gbla.add_rms_norm_e4m3(x, w, res, EPS, group=group)
        assert torch.equal(s.cpu().double(), total)
        assert y.dtype == torch.float8_e4m3fn and scales.shape == (rows, width // (group or width))
        g = want.view(rows, scales.shape[1], -1)
        most = (g.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
        _check(scales, most, most, 84 * 2 * U, "scales")
        sc = scales.cpu().double()[..., None]
        got = y.cpu().float().double().view(g.shape)
        assert (got.abs() <= 448).all()
        off = (got * sc - g).abs()
        assert (off <= (2.0 ** -4 * g.abs()).clamp(min=2.0 ** -10 * sc.expand_as(g)) + 90 * 2 * U * g.abs()).all()
        # the same number wherever y / scale is further from a border than its error
        near = ref.to_e4m3(g / sc * (1 - 90 * 2 * U)) != ref.to_e4m3(g / sc * (1 + 90 * 2 * U))
        assert torch.equal(got[~near], ref.to_e4m3(g / sc)[~near])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,width", SIZES)
def test_norm_backward(rows, width, dtype):
    t = _case(rows, width, dtype)
    s = t["res"]
    for ds in (t["ds"], None):
        g = gbla.add_rms_norm_backward(*_dev(s, t["w"], t["dy"], ds), eps=EPS)
        dx, dw = ref.add_norm_backward(s, t["w"], t["dy"], ds, EPS)
        r = 1 / torch.sqrt(s.double().square().mean(-1, keepdim=True) + EPS)
        n, u = (s.double() * r).abs(), (t["dy"].double() * t["w"].double()).abs()
        size = r * (u + n * (u * n).mean(-1, keepdim=True)) + (0 if ds is None else ds.double().abs())
        _check(g["dx"], dx, size, 160 * 2 * U, "dx")
        adds = rows / 512 + 1
        _check(g["dweight"], dw, (t["dy"].double().abs() * n).sum(0), (adds + 120) * 2 * U, "dweight")


def test_norm_backward_over_more_rows_than_one_pass():
    """Each workgroup takes several rows; the same bits again."""
    t = _case(70001, 32, BF16)
    args = _dev(t["res"], t["w"], t["dy"], t["ds"])
    a, b = (gbla.add_rms_norm_backward(*args, eps=EPS) for _ in range(2))
    assert torch.equal(a["dx"], b["dx"]) and torch.equal(a["dweight"], b["dweight"])
    dx, dw = ref.add_norm_backward(t["res"], t["w"], t["dy"], t["ds"], EPS)
    s = t["res"].double()
    n = (s / torch.sqrt((s * s).mean(-1, keepdim=True) + EPS)).abs()
    _check(a["dweight"], dw, (t["dy"].double().abs() * n).sum(0), (70001 / 32 / 1024 + 1 + 120) * 2 * U, "dweight")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [40, 1024, 4096])
def test_norm_in_place(width, dtype):
    t = _case(5, width, dtype)
    x, res, w = _dev(t["x"], t["res"], t["w"])
    y, s = gbla.add_rms_norm(x, w, res, EPS)
    a, b = x.clone(), res.clone()
    y2, s2 = gbla.add_rms_norm(a, w, b, EPS, sum_out=b, out=a)
    assert y2 is a and s2 is b and torch.equal(a, y) and torch.equal(b, s)
    a, b = x.clone(), res.clone()
    y8, sc, s = gbla.add_rms_norm_e4m3(x, w, res, EPS)
    z8, zc, s3 = gbla.add_rms_norm_e4m3(a, w, b, EPS, sum_out=a)
    assert torch.equal(a, s) and torch.equal(y8.view(torch.uint8), z8.view(torch.uint8)) and torch.equal(sc, zc)
    dy, ds = _dev(t["dy"], t["ds"])
    want = gbla.add_rms_norm_backward(s, w, dy, ds, EPS)
    for into in (0, 1):
        dyc, dsc = dy.clone(), ds.clone()
        got = gbla.add_rms_norm_backward(s, w, dyc, dsc, EPS, grads=dict(dx=(dyc, dsc)[into]))
        assert got["dx"] is (dyc, dsc)[into] and torch.equal(got["dx"], want["dx"])
        assert torch.equal(got["dweight"], want["dweight"])


def test_norm_values_that_are_not_finite_stay_in_their_row():
    t = _case(6, 256, BF16)
    x, res, w = _dev(t["x"], t["res"], t["w"])
    y, s = gbla.add_rms_norm(x, w, res, EPS)
    y8, sc, _ = gbla.add_rms_norm_e4m3(x, w, res, EPS, group=128)
    bad = x.clone()
    bad[2, 7], bad[4, 200] = float("nan"), float("inf")
    z, _ = gbla.add_rms_norm(bad, w, res, EPS)
    z8, zc, _ = gbla.add_rms_norm_e4m3(bad, w, res, EPS, group=128)
    ok = [0, 1, 3, 5]
    assert torch.equal(z[ok], y[ok]) and torch.equal(z8.view(torch.uint8)[ok], y8.view(torch.uint8)[ok])
    assert torch.equal(zc[ok], sc[ok])
    assert torch.isnan(z[2]).all() and torch.isnan(z[4, 200]) and (z[4, :200] == 0).all()
    worth = z8.float() * zc.repeat_interleave(128, dim=1)
    assert torch.isnan(worth[2]).all() and torch.isnan(worth[4, 128:]).all() and (worth[4, :128] == 0).all()


def test_norm_of_no_rows():
    w = torch.ones(64, device="cuda")
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    y, s = gbla.add_rms_norm(x, w, x.clone())
    assert y.shape == s.shape == (0, 64)
    g = gbla.add_rms_norm_backward(x, w, x)
    assert g["dx"].shape == (0, 64) and torch.equal(g["dweight"], torch.zeros_like(w))


def test_norm_replayed_from_a_graph_and_on_another_stream():
    t = _case(64, 1024, BF16)
    x, res, w, dy, ds = _dev(*(t[n] for n in ("x", "res", "w", "dy", "ds")))
    ws = torch.empty(gbla.add_rms_norm_backward_workspace_bytes(gbla.norm_shape(x)), dtype=torch.uint8, device="cuda")
    y, s = gbla.add_rms_norm(x, w, res)
    g = gbla.add_rms_norm_backward(s, w, dy, ds, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gbla.add_rms_norm(x, w, res, sum_out=s, out=y)
        gbla.add_rms_norm_backward(s, w, dy, ds, workspace=ws, grads=g)
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=_gen(i)).to(BF16))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        a, b = gbla.add_rms_norm(x, w, res)
        want = gbla.add_rms_norm_backward(b, w, dy, ds)
        assert torch.equal(y, a) and torch.equal(s, b)
        assert torch.equal(g["dx"], want["dx"]) and torch.equal(g["dweight"], want["dweight"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z, _ = gbla.add_rms_norm(x, w, res, stream=side)
    side.synchronize()
    assert torch.equal(z, y)


def test_norm_refuses_tensors():
    x, w = torch.zeros(4, 96, dtype=BF16, device="cuda"), torch.ones(96, device="cuda")
    for call in (lambda: gbla.add_rms_norm(x, w[:64]), lambda: gbla.add_rms_norm(x, w.bfloat16()),
                 lambda: gbla.add_rms_norm(x, w, x[:2]), lambda: gbla.add_rms_norm(x.half(), w),
                 lambda: gbla.add_rms_norm(x.t(), w), lambda: gbla.add_rms_norm(x[:, :60].contiguous(), w[:60]),
                 lambda: gbla.add_rms_norm(x, w, eps=-1.0), lambda: gbla.add_rms_norm_e4m3(x, w, group=128),
                 lambda: gbla.add_rms_norm_e4m3(x, w, out=torch.empty_like(x)),
                 lambda: gbla.add_rms_norm_e4m3(x, w, scales=torch.ones(4, device="cuda")),
                 lambda: gbla.add_rms_norm_backward(x, w, x.float()),
                 lambda: gbla.add_rms_norm_backward(x, w, x, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, gbla.GblaError)):
            call()
