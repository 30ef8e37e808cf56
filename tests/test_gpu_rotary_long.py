"""Rotary positions of so many tokens that pairs are numbered in 64 bits."""
import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
def test_more_pairs_than_32_bits_count(interleaved):
    # one head, 63 pairs one by one: 4.297e9 of them, 2^32 is 4.295e9
    T, D, R = 68_200_000, 128, 126
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB of device memory")
    g = torch.Generator(device="cuda").manual_seed(3)
    row = torch.randn(1, 1, D, generator=g, device="cuda").to(ou.F16)
    q = row.expand(T, 1, D).contiguous()
    p = torch.zeros(T, dtype=torch.int32, device="cuda")
    part = 3000
    spots = [0, T // 2, (1 << 32) // 63 - part // 2, T - part]        # (and around the first pair behind 2^32)
    for at in spots:
        p[at:at + part] = torch.randint(-(1 << 20), 1 << 20, (part,), generator=g, device="cuda", dtype=torch.int32)
    f, _ = vq.vq_rotary_frequencies(R)
    f = f.cuda()
    vq.vq_rotary(q, None, p, f, interleaved=interleaved, q_out=q)
    still = torch.ones(T, dtype=torch.bool, device="cuda")
    for at in spots:
        want, off = ou.rotary(row.expand(part, 1, D), p[at:at + part], f, interleaved, 1.0)
        got = q[at:at + part]
        ou.check(got[..., :R], want[..., :R], off[..., :R] + ou.HALF[ou.F16] * want[..., :R].abs() + ou.TINY[ou.F16], at)
        assert torch.equal(got[..., R:], row.expand(part, 1, D)[..., R:])
        still[at:at + part] = False
    # a position of zero turns nothing
    for at in range(0, T, 1 << 22):
        same = (q[at:at + (1 << 22)] == row).all(-1).all(-1)
        assert (same | ~still[at:at + (1 << 22)]).all(), at
