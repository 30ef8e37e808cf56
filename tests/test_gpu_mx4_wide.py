"""Microscaled products whose rows of y are too long for 32-bit offsets within a tile: every sum is exact, so that y is too."""
import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou

# rows, channels, K: whole 16-byte pieces from 2^21 channels on, and an odd number whose rows of a tile span more than 2^31 bytes
WIDE = [(64, (1 << 21) + 8, 32), (130, (1 << 21) + 16, 96), (64, 17_200_001, 32)]


def _codes(rows, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(0, 256, (rows, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.zeros(rows, vq.MX4_SCALE_STRIDE(K), device="cuda", dtype=torch.uint8)
    s[:, :K // 32] = torch.randint(125, 129, (rows, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    return q, s


def _values(q, s):
    grid = torch.tensor(ou.E2M1 + tuple(-v for v in ou.E2M1), device="cuda")
    code = torch.stack((q & 15, q >> 4), -1).reshape(q.shape[0], -1).long()
    scale = torch.exp2(s[:, :code.shape[1] // 32].float() - 127)
    return (grid[code].reshape(q.shape[0], -1, 32) * scale.unsqueeze(-1)).reshape(q.shape[0], -1)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", WIDE)
def test_rows_of_many_channels(M, N, K):
    xq, xs = _codes(M, K, 1)
    wq, ws = _codes(N, K, 2)
    # (sums are multiples of 2^-6 below 2^14, and so are they with such a bias: fp32 holds them)
    bias = (torch.randint(-64, 65, (N,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") / 8).to(ou.F16)
    room = torch.full((M + 2, N), 7.0, dtype=ou.F16, device="cuda")        # the rows in front and behind stay
    lead = -(room.data_ptr() // 2 + N) % 8                                 # y on 16 bytes
    y = room.view(-1)[N + lead:N + lead + M * N].view(M, N)
    vq.vq_gemm_mx4(xq, xs, wq, ws, bias, y)
    x = _values(xq, xs).double()
    for n0 in range(0, N, 1 << 20):
        w = _values(wq[n0:n0 + (1 << 20)], ws[n0:n0 + (1 << 20)]).double()
        want = (x @ w.t().contiguous() + bias[n0:n0 + (1 << 20)].double()).to(ou.F16)
        assert torch.equal(y[:, n0:n0 + (1 << 20)], want), n0
    flat = room.view(-1)
    assert (flat[:N + lead] == 7).all() and (flat[N + lead + M * N:] == 7).all()
