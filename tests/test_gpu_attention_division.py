"""Attention whose keys are divided by the rules for ragged sequences, and rows that are dealt in blocks behind shared keys, against the formula in 64 bits."""
import pytest
import torch

import paper_2406_02540_amd as vq
import operator_util as ou
import test_gpu_attention_prefix as prefix
import test_gpu_attention_window as window
from test_gpu_attention import _data
from test_gpu_attention_kernels import _lengths

pytestmark = pytest.mark.gpu
F16, BF16 = ou.F16, ou.BF16

# queries, keys, shared keys, heads, heads of k and v: prompts among single tokens, rows at the edges of blocks of 64, sequences without any
PROMPTS = {
    "one first": ([500] + [1] * 60, [500] + _lengths(1, 60, 0, 300), 4001, 8, 2),
    "one last": ([1] * 60 + [333], _lengths(2, 60, 0, 300) + [40], 4001, 8, 2),
    "edges": ([63, 64, 65, 0, 1, 127, 128, 129, 0, 2], [70, 64, 200, 9, 0, 127, 300, 1, 0, 50], 9000, 3, 3),
    "edges, grouped": ([15, 16, 17, 0, 1, 31, 33, 2], [15, 300, 17, 9, 0, 31, 1, 50], 9000, 8, 2),
    "six heads a head": ([11, 10, 22, 0, 21, 1], [900, 700, 22, 30, 1800, 0], 6000, 12, 2),
    "divided": ([40, 1, 1, 25, 1, 1], [1500, 700, 900, 1200, 40, 1100], 9000, 4, 2),
    "one sequence of many blocks and empty ones": ([0] * 5 + [700] + [0] * 5, [9] * 5 + [650] + [0] * 5, 5000, 2, 2),
}


@pytest.mark.parametrize("D", [64, 72, 96, 128])
@pytest.mark.parametrize("name", PROMPTS)
def test_prompts_behind_shared_keys(name, D):
    lq, lk, P, H, G = PROMPTS[name]
    prefix._run(lq, lk, P, H, G, D, F16, True, before=2, behind=3)
    prefix._run(lq, lk, P, H, G, D, BF16, False)


def test_offsets_outside_the_tensors_in_blocks():
    Tq, Tk, H, G, D = 100, 4000, 8, 2, 64
    for cu_q, cu_k in (([-20, 40, 100000, 300, 120], [-7, 30, 200000, 95, 1 << 30]), ([0, 40, 20, -5, -7], [0, 30, 10, -4, -9]),
                       ([90, 80, 70, 60, 50], [0, 1, 2, 3, 4]), ([2**31 - 1] * 5, [0] * 5)):
        room = torch.full((Tq + 64, H, D), 5.0, dtype=F16, device="cuda")
        q, k, v = _data(Tq, Tk, H, G, D, F16)
        cu = [torch.tensor(c, dtype=torch.int32).cuda() for c in (cu_q, cu_k)]
        vq.vq_attention_prefix(q, *prefix._prefix(9000, G, D, F16), k, v, *cu, causal=True, out=room[32:32 + Tq])
        torch.cuda.synchronize()
        assert (room[:32] == 5).all() and (room[32 + Tq:] == 5).all()


@pytest.mark.parametrize("causal", [False, True])
def test_ragged_tokens_without_a_window(causal):
    lk = [9000, 40, 0, 700, 2500, 1, 300, 5000]
    window._run([1] * 8, lk, 8, 2, 64, F16, None, 0 if causal else None, 0, causal)
    window._run([1, 2, 0, 3, 1, 1, 1, 2], lk, 4, 4, 72, BF16, 20000, 20000, 3, causal)
    prefix._run([1] * 8, lk, 16, 8, 2, 64, F16, causal)
    prefix._run([1, 2, 0, 3, 1, 1, 1, 2], lk, 0, 4, 4, 72, BF16, causal)
    prefix._run([1] * 8, lk, 5000, 8, 8, 128, BF16, causal)


@pytest.mark.parametrize("name", ["one last", "divided"])
def test_captured_prompts(name):
    lq, lk, P, H, G = PROMPTS[name]
    D = 128
    q, k, v = _data(sum(lq), sum(lk), H, G, D, F16)
    pk, pv = prefix._prefix(P, G, D, F16)
    cu_q, cu_k = ou.offsets(lq).cuda(), ou.offsets(lk).cuda()
    work = torch.empty(vq.vq_attention_prefix_workspace_bytes(len(lq), sum(lq), P, sum(lk), H, G, D), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True, out=out, workspace=work)
    for turn in (list(reversed(lq)), lq, lq[1:] + lq[:1]):      # the lengths change between replays, not the sums
        cu_q.copy_(ou.offsets(turn))
        q.mul_(0.9)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, vq.vq_attention_prefix(q, pk, pv, k, v, cu_q, cu_k, causal=True))
