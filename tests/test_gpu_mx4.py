"""Microscaled 4-bit quantizer, GEMM and layer against their definitions in 64 bits."""
import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou

pytestmark = pytest.mark.gpu
F16, BF16, F32 = ou.F16, ou.BF16, ou.F32


def _x(M, K, dtype, seed=0, spread=True):
    g = torch.Generator().manual_seed(seed * 1000003 + M * 131 + K)
    x = torch.randn(M, K, generator=g)
    if spread:
        x = x * torch.exp(torch.randn(K, generator=g) * 1.5)
    return x.to(dtype)


def _mask(K, seed=0):
    g = torch.Generator().manual_seed(seed + K)
    return torch.exp(torch.randn(K, generator=g))


def _quantized(x, cm=None):
    code, e = ou.quantize_mx4(x, cm)
    return (*(t.cuda() for t in ou.pack_mx4(code, e)), ou.values_mx4(code, e))


@pytest.mark.parametrize("M,K", [(1, 32), (1, 1152), (3, 96), (5, 4608), (77, 1184), (130, 160), (1024, 64)])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("balanced", [False, True])
def test_codes_are_the_definitions(M, K, dtype, balanced):
    x, cm = _x(M, K, dtype), _mask(K) if balanced else None
    want_q, want_s = ou.pack_mx4(*ou.quantize_mx4(x, cm))
    q, s = vq.vq_mx4_quantize(x.cuda(), None if cm is None else cm.cuda())
    assert torch.equal(s.cpu(), want_s) and torch.equal(q.cpu(), want_q)
    for t in (F16, BF16, F32):
        back = vq.vq_mx4_dequantize(q, s, dtype=t)
        assert back.dtype == t and torch.equal(back.cpu().double(), ou.values_mx4(*ou.unpack_mx4(q, s)).to(t).double())


def test_codes_at_borders():
    # every tie and its neighbours in fp32, at several scales; the block's largest value fixes the scale
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.999999])
    near = torch.cat([ties, torch.nextafter(ties, torch.tensor(0.0)), torch.nextafter(ties, torch.tensor(9.0))])
    row = torch.cat([near, torch.tensor([4.0, 0.0])])   # 32 values, top in [4, 8)
    rows = torch.stack([row * 2.0 ** e * s for e in (-126, -100, -3, 0, 5, 100) for s in (1, -1)])
    q, s = vq.vq_mx4_quantize(rows.cuda())
    want_q, want_s = ou.pack_mx4(*ou.quantize_mx4(rows))
    assert torch.equal(s.cpu(), want_s) and torch.equal(q.cpu(), want_q)


def test_codes_of_zeros_subnormals_and_largest():
    x = torch.zeros(6, 64)
    x[1, 3] = 2.0 ** -149
    x[2, 40] = 2.0 ** -126
    x[3, 0], x[3, 1] = 3.0e38, -1.0e38
    x[4, 5], x[4, 6] = -2.0 ** -128, 2.0 ** -127
    x[5] = torch.linspace(-1, 1, 64) * 2.0 ** -125
    q, s = vq.vq_mx4_quantize(x.cuda())
    want_q, want_s = ou.pack_mx4(*ou.quantize_mx4(x))
    assert torch.equal(s.cpu(), want_s) and torch.equal(q.cpu(), want_q)
    assert torch.equal(vq.vq_mx4_dequantize(q, s, dtype=F32).cpu().double(), ou.values_mx4(*ou.unpack_mx4(q, s)))


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_blocks_that_are_not_finite(bad):
    x = _x(4, 128, F16)
    x[1, 70] = bad
    q, s = vq.vq_mx4_quantize(x.cuda())
    assert s[1, 2].item() == 255 and (s != 255).sum().item() == 15
    assert (q[1, 32:48] == 0).all()
    back = vq.vq_mx4_dequantize(q, s, dtype=F32).cpu()
    assert back[1, 64:96].isnan().all() and back.isnan().sum().item() == 32
    wq, ws, _ = _quantized(_x(40, 128, F32, 1))
    y = vq.vq_gemm_mx4(q, s, wq, ws).cpu()
    assert y[1].isnan().all() and not y[[0, 2, 3]].isnan().any()


def test_scales_behind_the_last_block_are_not_looked_at():
    x, w = _x(20, 160, F16), _x(36, 160, F32, 1) * 0.05
    xq, xs, xv = _quantized(x)
    wq, ws, wv = _quantized(w)
    want, off = ou.product(xv, wv, None, F16)
    for fill in (0, 255, 254):
        xs[:, 5:] = fill
        ws[:, 5:] = fill
        ou.check(vq.vq_gemm_mx4(xq, xs, wq, ws), want, off, fill)


SIZES = [(1, 1, 32), (1, 16, 64), (1, 3456, 1152), (2, 130, 4096), (15, 17, 96), (16, 32, 128), (17, 100, 160), (33, 65, 224),
         (64, 64, 512), (65, 255, 1184), (127, 513, 352), (240, 2304, 4096), (300, 1152, 1152), (257, 511, 1152), (1001, 2821, 1184),
         (100, 4090, 640), (2048, 1152, 256), (1030, 4600, 320)]


# the large tiles, several a workgroup: whole and half stages of K, one stage, rows and channels that end inside a tile
LARGE = [(8200, 4616, 1152), (16384, 2304, 320), (33000, 1160, 128), (4100, 8192, 512), (9000, 1153, 640), (20000, 1152, 96)]


@pytest.mark.parametrize("M,N,K", LARGE)
def test_large_product(M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M)
    xq = torch.randint(0, 256, (M, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    wq = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    xs, ws = (torch.randint(118, 128, (n, vq.MX4_SCALE_STRIDE(K)), generator=g, device="cuda", dtype=torch.uint8) for n in (M, N))
    bias = torch.randn(N, generator=g, device="cuda").to(F16)
    y = torch.full((M + 1, N), 7.0, dtype=F16, device="cuda")
    got = vq.vq_gemm_mx4(xq, xs, wq, ws, bias, y=y[:M])
    assert (y[M] == 7).all() and torch.equal(got, vq.vq_gemm_mx4(xq, xs, wq, ws, bias))
    grid = torch.tensor(ou.E2M1 + tuple(-v for v in ou.E2M1), dtype=torch.float64, device="cuda")

    def values(q, s):
        v = grid[torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], -1).long()].reshape(q.shape[0], -1, 32)
        return (v * torch.pow(2.0, s[:, :K // 32].double() - 127).unsqueeze(-1)).reshape(q.shape[0], K)

    x, w = values(xq, xs), values(wq, ws)
    for r in range(0, M, 8192):
        part = x[r:r + 8192]
        want, size = part @ w.t().contiguous() + bias.double(), part.abs() @ w.abs().t().contiguous() + bias.double().abs()
        off = ou.HALF[F16] * want.abs() + ou.TINY[F16] + (32 + K // 32 + 2) * 2.0 ** -24 * size
        assert ((got[r:r + 8192].double() - want).abs() <= off).all()


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_product(M, N, K, dtype):
    xq, xs, xv = _quantized(_x(M, K, F16))
    wq, ws, wv = _quantized(_x(N, K, F32, 1) * 0.02)
    bias = _x(1, N, dtype, 2, False)[0] if (M + N) % 3 else None
    want, off = ou.product(xv, wv, bias, dtype)
    y = torch.full((M + 1, N), 7.0, dtype=dtype, device="cuda")
    got = vq.vq_gemm_mx4(xq, xs, wq, ws, None if bias is None else bias.cuda(), y=y[:M])
    ou.check(got, want, off, (M, N, K))
    assert (y[M] == 7).all()           # nothing behind the last row
    again = vq.vq_gemm_mx4(xq, xs, wq, ws, None if bias is None else bias.cuda(), dtype=dtype)
    assert torch.equal(got, again)     # the order of the sums is fixed


@pytest.mark.parametrize("M,N,K", [(1, 3456, 1152), (3, 50, 96), (16, 1152, 4608), (17, 64, 160), (33, 257, 1184), (240, 2304, 4096), (700, 640, 1152)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("balanced", [False, True])
def test_layer_is_quantizer_and_product(M, N, K, dtype, balanced):
    x, cm = _x(M, K, dtype), _mask(K) if balanced else None
    wq, ws, wv = _quantized(_x(N, K, F32, 1) * 0.02)
    bias = _x(1, N, dtype, 2, False)[0]
    _, _, xv = _quantized(x, cm)
    want, off = ou.product(xv, wv, bias, dtype)
    c = None if cm is None else cm.cuda()
    got = vq.vq_linear_mx4(x.cuda(), c, wq, ws, bias.cuda())
    assert got.dtype == dtype
    ou.check(got, want, off, (M, N, K))
    ws_bytes = vq.vq_linear_mx4_workspace_bytes(M, N, K)
    kept = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    assert torch.equal(got, vq.vq_linear_mx4(x.cuda(), c, wq, ws, bias.cuda(), workspace=kept))


def test_layer_with_blocks_that_are_not_finite():
    for M in (2, 200):
        x = _x(M, 256, F16)
        x[1, 100] = float("inf")
        wq, ws, _ = _quantized(_x(48, 256, F32, 1))
        y = vq.vq_linear_mx4(x.cuda(), None, wq, ws)
        assert y[1].isnan().all() and not y[0].isnan().any()


@pytest.mark.parametrize("K", [32, 96, 128, 160, 288, 352, 1120, 2080])
def test_nan_blocks_reach_their_row_only(K):
    # in every kernel: the scale of one block of one token, and of one channel, NaN
    for M, N in ((5, 40), (60, 100), (300, 2000), (4000, 1160), (9000, 1152)):
        xq, ws = torch.full((M, K // 2), 0x22, dtype=torch.uint8, device="cuda"), torch.full((N, vq.MX4_SCALE_STRIDE(K)), 127, dtype=torch.uint8, device="cuda")
        wq, xs = torch.full((N, K // 2), 0x22, dtype=torch.uint8, device="cuda"), torch.full((M, vq.MX4_SCALE_STRIDE(K)), 127, dtype=torch.uint8, device="cuda")
        xs[M // 2, K // 32 - 1] = 255
        ws[N - 1, 0] = 255
        y = vq.vq_gemm_mx4(xq, xs, wq, ws)
        assert y[M // 2].isnan().all() and y[:, N - 1].isnan().all()
        assert y.isnan().sum().item() == M + N - 1
        assert (y[:M // 2, :N - 1] == K).all() and (y[M // 2 + 1:, :N - 1] == K).all()


def test_layer_into_its_own_activations():
    # y where x was: the one launch would read what it has written
    K = N = 256
    x = _x(4, K, F16).cuda()
    wq, ws, _ = _quantized(_x(N, K, F32, 1) * 0.1)
    want = vq.vq_linear_mx4(x, None, wq, ws)
    assert torch.equal(vq.vq_linear_mx4(x, None, wq, ws, y=x), want)


def test_empty_sizes():
    x = torch.empty(0, 64, dtype=F16, device="cuda")
    q, s = vq.vq_mx4_quantize(x)
    assert q.shape == (0, 32) and s.shape == (0, 4)
    assert vq.vq_mx4_dequantize(q, s).shape == (0, 64)
    wq, ws, _ = _quantized(_x(8, 64, F32))
    assert vq.vq_gemm_mx4(q, s, wq, ws).shape == (0, 8)
    assert vq.vq_linear_mx4(x, None, wq, ws).shape == (0, 8)
    assert vq.vq_linear_mx4(_x(3, 64, F16).cuda(), None, wq[:0], ws[:0]).shape == (3, 0)


@pytest.mark.parametrize("M", [2, 300])
def test_captured_and_replayed(M):
    K, N = 1152, 640
    x, x2 = _x(M, K, F16).cuda(), _x(M, K, F16, 5).cuda()
    wq, ws, _ = _quantized(_x(N, K, F32, 1))
    cm = _mask(K).cuda()
    work = torch.empty(vq.vq_linear_mx4_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    want = [vq.vq_linear_mx4(t, cm, wq, ws) for t in (x, x2)]
    inp, out = x.clone(), torch.empty(M, N, dtype=F16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vq.vq_linear_mx4(inp, cm, wq, ws, y=out, workspace=work)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vq.vq_linear_mx4(inp, cm, wq, ws, y=out, workspace=work)
    for i in (1, 0, 1):
        inp.copy_((x, x2)[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        vq.vq_linear_mx4(x, cm, wq, ws)


def test_on_another_stream():
    x = _x(300, 1152, F16).cuda()
    wq, ws, _ = _quantized(_x(256, 1152, F32, 1))
    want = vq.vq_linear_mx4(x, None, wq, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = vq.vq_linear_mx4(x, None, wq, ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
