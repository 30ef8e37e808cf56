"""Microscaled layers, rotary positions and attention where no GPU is needed: refusals of the C entry points and of the
binding, workspace sizes, frequency tables, and the 64-bit definitions that the GPU tests use."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import operator_util as ou  # noqa: E402
from test_binding_host import child  # noqa: E402

A = 0x10000  # a made-up, 16-byte aligned address; never dereferenced by validation
P, F = ctypes.c_void_p, ctypes.c_float
OK, NULL, SHAPE, ALIGN, WORKSPACE, ARCH, TYPE = 0, 1, 2, 3, 4, 6, 8


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2406_02540_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_02540_amd import build
        build.build(verbose=False)
    return binding.lib()


def test_quantizer_refusals(lib):
    def q(x=A, t=0, cm=None, xq=A, s=A, M=4, K=64):
        return lib.vq_mx4_quantize(P(x), t, P(cm), P(xq), P(s), M, K, None)

    def d(xq=A, s=A, x=A, t=0, M=4, K=64):
        return lib.vq_mx4_dequantize(P(xq), P(s), P(x), t, M, K, None)

    assert [q(t=3), q(t=-1), d(t=3)] == [TYPE] * 3
    assert [q(M=-1), q(K=0), q(K=-32), q(K=48), q(K=131072 + 32), d(M=-1), d(K=16)] == [SHAPE] * 7
    assert [q(x=None), q(xq=None), q(s=None), d(xq=None), d(s=None), d(x=None)] == [NULL] * 6
    assert [q(x=A + 2), q(cm=A + 4), q(xq=A + 8), q(s=A + 1), d(xq=A + 4), d(s=A + 4), d(x=A + 8)] == [ALIGN] * 7
    assert [q(x=None, M=0), d(xq=None, M=0)] == [OK] * 2
    assert [q(), q(t=1, cm=A), q(t=2), d(), d(t=2), q(K=131072)] == [ARCH] * 6


def test_product_refusals(lib):
    def g(xq=A, xs=A, wq=A, ws=A, b=None, y=A, t=0, M=4, N=8, K=64):
        return lib.vq_gemm_mx4(P(xq), P(xs), P(wq), P(ws), P(b), P(y), t, M, N, K, None)

    assert [g(t=2), g(t=9)] == [TYPE] * 2
    assert [g(M=-1), g(N=-1), g(K=0), g(K=33), g(K=1 << 20)] == [SHAPE] * 5
    assert [g(xq=None), g(xs=None), g(wq=None), g(ws=None), g(y=None)] == [NULL] * 5
    assert [g(xq=A + 1), g(xs=A + 4), g(wq=A + 8), g(ws=A + 4), g(b=A + 2), g(y=A + 2)] == [ALIGN] * 6
    assert [g(M=0, xq=None), g(N=0, wq=None)] == [OK] * 2
    assert [g(), g(t=1, b=A)] == [ARCH] * 2


def test_layer_refusals(lib):
    need = lib.vq_linear_mx4_workspace_bytes(4, 8, 64)
    assert need == 4 * 32 + 16
    assert lib.vq_linear_mx4_workspace_bytes(3, 8, 160) == 240 + 32
    assert [lib.vq_linear_mx4_workspace_bytes(*s) for s in ((-1, 8, 64), (4, -1, 64), (4, 8, 0), (4, 8, 40), (0, 8, 64))] == [0] * 5
    big = lib.vq_linear_mx4_workspace_bytes(2**31 - 1, 1, 131072)
    assert big == -(-(2**31 - 1) * 65536 // 16) * 16 + -(-(2**31 - 1) * 4096 // 16) * 16

    def g(x=A, cm=None, wq=A, ws=A, b=None, y=A, t=0, w=A, n=None, M=4, N=8, K=64):
        return lib.vq_linear_mx4(P(x), P(cm), P(wq), P(ws), P(b), P(y), t, P(w), need if n is None else n, M, N, K, None)

    assert [g(t=2), g(M=-1), g(K=96 + 16), g(n=need - 1), g(w=None), g(w=A + 8), g(x=None), g(x=A + 2), g(cm=A + 4)] == \
        [TYPE, SHAPE, SHAPE, WORKSPACE, NULL, ALIGN, NULL, ALIGN, ALIGN]
    assert [g(wq=None), g(ws=A + 4), g(y=A + 2), g(M=0, x=None), g(N=0, y=None), g()] == [NULL, ALIGN, ALIGN, OK, OK, ARCH]


def _strides(*s):
    return (ctypes.c_int64 * 8)(*s)


def test_rotary_refusals(lib):
    dense = (1024, 128) * 4

    def r(q=A, qo=2 * A, k=3 * A, ko=4 * A, t=0, p=A, f=A, amp=1.0, inter=0, T=4, hq=8, hk=8, D=128, R=128, s=dense):
        return lib.vq_rotary(P(q), P(qo), P(k), P(ko), t, P(p), P(f), F(amp), inter, T, hq, hk, D, R, _strides(*s) if s else None, None)

    assert [r(t=2), r(t=-1)] == [TYPE] * 2
    assert [r(T=-1), r(hq=0), r(hk=-1), r(D=0), r(D=12), r(D=136), r(R=0), r(R=21), r(R=136), r(inter=2), r(amp=math.inf),
            r(amp=math.nan), r(hq=1 << 17)] == [SHAPE] * 13
    assert [r(q=None), r(qo=None), r(k=None), r(ko=None), r(p=None), r(f=None), r(s=None)] == [NULL] * 7
    assert [r(q=A + 8), r(qo=A + 2), r(k=A + 4), r(ko=A + 8), r(p=A + 2), r(f=A + 4)] == [ALIGN] * 6
    # strides: whole 16 bytes, not negative; rows that are written lie apart
    assert [r(s=(1020,) + dense[1:]), r(s=(-8,) + dense[1:]), r(s=dense[:2] + (1024, 64) + dense[4:]), r(s=dense[:2] + (0, 128) + dense[4:]),
            r(qo=A, s=(1024, 128, 2048, 128) + dense[4:]), r(ko=3 * A, s=dense[:6] + (1024, 256))] == [SHAPE] * 6
    assert [r(T=0, q=None), r(), r(s=(0, 0) + dense[2:]), r(R=20), r(R=18), r(hk=0, k=None, ko=None), r(qo=A, ko=3 * A), r(p=A + 4), r(T=1, s=dense[:2] + (0, 128) + dense[4:])] == \
        [OK] + [ARCH] * 8


def test_attention_refusals(lib):
    dense = (1024, 128, 256, 128, 256, 128, 1024, 128)

    def a(q=A, k=A, v=A, o=2 * A, t=0, cq=A, ck=A, B=2, Tq=600, Tk=700, H=8, G=2, D=128, s=dense, scale=0.1, causal=0, w=None, n=0):
        return lib.vq_attention(P(q), P(k), P(v), P(o), t, P(cq), P(ck), B, Tq, Tk, H, G, D, _strides(*s) if s else None, F(scale), causal,
                                P(w), n, None)

    assert [a(t=2), a(t=7)] == [TYPE] * 2
    assert [a(B=-1), a(Tq=-1), a(Tk=-1), a(H=0), a(G=0), a(G=3), a(D=0), a(D=100), a(D=136), a(causal=2), a(scale=0.0), a(scale=-1.0),
            a(scale=math.inf), a(scale=math.nan), a(H=1 << 17, G=1), a(scale=1e-31), a(scale=1e31), a(Tq=1 << 28), a(Tk=2**31 - 1)] == [SHAPE] * 19
    assert [a(q=None), a(k=None), a(v=None), a(o=None), a(cq=None), a(ck=None), a(s=None)] == [NULL] * 7
    assert [a(q=A + 2), a(k=A + 8), a(v=A + 8), a(o=A + 4), a(cq=A + 2), a(ck=A + 1)] == [ALIGN] * 6
    assert [a(s=(1020,) + dense[1:]), a(s=dense[:2] + (-8,) + dense[3:]), a(s=dense[:6] + (0, 128)), a(s=dense[:6] + (1024, 64)),
            a(s=dense[:2] + ((1 << 23) + 8,) + dense[3:]), a(s=dense[:4] + (1 << 24,) + dense[5:])] == [SHAPE] * 6
    assert [a(B=0, q=None), a(Tq=0, q=None), a(), a(Tk=0, k=None, v=None), a(causal=1, t=1), a(s=(0, 0, 0, 0, 0, 0, 1024, 128))] == \
        [OK, OK] + [ARCH] * 4
    # few queries over many keys: the keys are divided, which takes a workspace
    few = dict(B=2, Tq=2, Tk=40000)
    need = lib.vq_attention_workspace_bytes(2, 2, 40000, 8, 2, 128)
    assert need > 0 and need % 4 == 0
    assert [a(**few), a(**few, w=A, n=need - 1), a(**few, w=A + 8, n=need), a(**few, w=A, n=need)] == [NULL, WORKSPACE, ALIGN, ARCH]
    bad = [(0, 2, 9, 8, 2, 128), (2, 0, 9, 8, 2, 128), (2, 2, -1, 8, 2, 128), (2, 2, 9, 8, 3, 128), (2, 2, 9, 8, 2, 100), (2, 2, 9, 8, 0, 128)]
    assert [lib.vq_attention_workspace_bytes(*s) for s in bad] == [0] * len(bad)


def test_frequency_tables():
    import paper_2406_02540_amd as vq
    R, base = 64, 10000.0
    plain = [base ** (-2 * i / R) for i in range(R // 2)]

    def near(table, want):
        assert table.dtype == torch.float32 and table.device.type == "cpu" and table.shape == (R // 2,)
        assert all(abs(a - b) <= 2.0 ** -24 * abs(b) * 1.001 for a, b in zip(table.tolist(), want))

    f, amp = vq.vq_rotary_frequencies(R, base)
    near(f, plain)
    assert amp == 1.0
    f, amp = vq.vq_rotary_frequencies(R, base, "linear", 4.0)
    near(f, [v / 4 for v in plain])
    f, amp = vq.vq_rotary_frequencies(R, base, "base", 4.0)
    near(f, [(base * 4.0 ** (R / (R - 2))) ** (-2 * i / R) for i in range(R // 2)])
    assert f[0] == 1.0 and abs(f[-1].item() * 4 / plain[-1] - 1) < 1e-6      # the slowest pair is slowed by the factor
    f, amp = vq.vq_rotary_frequencies(R, base, "parts", 8.0, 4096)
    turns = [4096 * v / (2 * math.pi) for v in plain]
    assert amp == pytest.approx(0.1 * math.log(8.0) + 1.0, abs=1e-6)
    for i, (v, n) in enumerate(zip(f.tolist(), turns)):
        if n >= 32:
            assert v == pytest.approx(plain[i], rel=1e-6)
        elif n <= 1 and turns[i - 1] <= 1:                                    # (the blend ends at a whole pair)
            assert v == pytest.approx(plain[i] / 8, rel=1e-6)
        else:
            assert plain[i] / 8 * 0.999 <= v <= plain[i] * 1.001
    assert all(a > b for a, b in zip(f.tolist(), f.tolist()[1:]))
    same, _ = vq.vq_rotary_frequencies(R, base, "parts", 1.0, 4096)
    near(same, plain)


def test_frequency_refusals(lib):
    import paper_2406_02540_amd as vq
    with pytest.raises(ValueError):
        vq.vq_rotary_frequencies(64, scaling="ntk")
    for kw in ({"rot_dim": 0}, {"rot_dim": 7}, {"base": 1.0}, {"base": math.nan}, {"factor": 0.5}, {"factor": math.inf},
               {"scaling": "parts", "factor": 2.0}, {"scaling": "parts", "original_length": -4}, {"scaling": "base", "rot_dim": 2}):
        with pytest.raises(vq.VqError, match="VQ_ERR_SHAPE"):
            vq.vq_rotary_frequencies(**{"rot_dim": 64, **kw})
    amp = F()
    assert lib.vq_rotary_frequencies(None, ctypes.byref(amp), 64, 1e4, 0, 1.0, 0) == NULL
    assert lib.vq_rotary_frequencies((F * 32)(), None, 64, 1e4, 0, 1.0, 0) == NULL
    assert lib.vq_rotary_frequencies((F * 32)(), ctypes.byref(amp), 64, 1e4, 4, 1.0, 0) == SHAPE


def test_binding_refusals():
    got = child("""
        bf16 = torch.bfloat16
        with FakeTensorMode():
            st = Stream()
            x, cm = fake(M, K), fake(K, dtype=f32)
            q, s, w, ws = fake(M, K // 2, dtype=u8), fake(M, 4, dtype=u8), fake(N, K // 2, dtype=u8), fake(N, 4, dtype=u8)
            y, wk = fake(M, N), fake(4096, dtype=u8)
            h, kv, p, f, cu = fake(6, 4, 64), fake(9, 2, 64), fake(6, dtype=torch.int32), fake(16, dtype=f32), fake(3, dtype=torch.int32)
            ho, kr, ko = fake(6, 4, 64), fake(6, 2, 64), fake(6, 2, 64)
            qz = lambda x=x, cm=cm, q=q, s=s: vq.vq_mx4_quantize(x, cm, q, s, stream=st)
            dq = lambda q=q, s=s, t=torch.float16, x=x: vq.vq_mx4_dequantize(q, s, t, x, stream=st)
            gm = lambda q=q, s=s, w=w, ws=ws, b=None, y=y, t=torch.float16: vq.vq_gemm_mx4(q, s, w, ws, b, y, t, stream=st)
            ln = lambda x=x, cm=cm, w=w, ws=ws, b=None, y=y, k=wk: vq.vq_linear_mx4(x, cm, w, ws, b, y, k, stream=st)
            ro = lambda q=h, k=kr, p=p, f=f, qo=ho, ko=ko, amp=1.0: vq.vq_rotary(q, k, p, f, False, amp, qo, ko, stream=st)
            at = lambda q=h, k=kv, v=kv, cq=cu, ck=cu, sc=None, o=ho, k_=wk: vq.vq_attention(q, k, v, cq, ck, sc, False, o, k_, stream=st)
            for name, call in {
                "quantize fits": lambda: qz(), "quantize type": lambda: qz(x=fake(M, K, dtype=i8)), "quantize host": lambda: qz(x=torch.empty(M, K, device="cpu")),
                "quantize view": lambda: qz(x=fake(M, 2 * K)[:, :K]), "quantize mask": lambda: qz(cm=fake(K + 1, dtype=f32)), "quantize mask type": lambda: qz(cm=fake(K)),
                "quantize K": lambda: vq.vq_mx4_quantize(fake(M, 40), stream=st), "quantize out": lambda: qz(q=fake(M, K, dtype=u8)), "quantize scale": lambda: qz(s=fake(M, 5, dtype=u8)),
                "quantize none": lambda: qz(x=None), "quantize rows": lambda: qz(x=fake(K)),
                "read fits": lambda: dq(), "read scale": lambda: dq(s=fake(M, 3, dtype=u8)), "read type": lambda: dq(t=torch.float64, x=None), "read dtype": lambda: dq(t="f16", x=None),
                "read out": lambda: dq(x=fake(M, K + 32)),
                "product fits": lambda: gm(), "product K": lambda: gm(w=fake(N, K, dtype=u8), ws=fake(N, 8, dtype=u8)), "product bias": lambda: gm(b=fake(N, dtype=bf16)),
                "product bias shape": lambda: gm(b=fake(N + 1)), "product type": lambda: gm(y=None, t=f32), "product y": lambda: gm(y=fake(M, N + 1)), "product scale": lambda: gm(ws=fake(N, 3, dtype=u8)),
                "layer fits": lambda: ln(), "layer type": lambda: ln(x=fake(M, K, dtype=f32)), "layer bias": lambda: ln(b=fake(N, dtype=bf16)), "layer y": lambda: ln(y=fake(M, N, dtype=bf16)),
                "layer K": lambda: ln(x=fake(M, K + 32), cm=None), "layer mask": lambda: ln(cm=fake(K + 32, dtype=f32)), "layer workspace": lambda: ln(k=fake(4096)),
                "rotary fits": lambda: ro(), "rotary positions": lambda: ro(p=fake(7, dtype=torch.int32)), "rotary positions type": lambda: ro(p=fake(6, dtype=torch.int64)),
                "rotary freq": lambda: ro(f=fake(2, 8, dtype=f32)), "rotary R": lambda: ro(f=fake(33, dtype=f32)), "rotary k type": lambda: ro(k=fake(6, 2, 64, dtype=bf16)), "rotary k tokens": lambda: ro(k=fake(7, 2, 64)),
                "rotary dims": lambda: ro(q=fake(6, 64)), "rotary channels": lambda: ro(q=fake(6, 4, 128)[..., ::2]), "rotary out": lambda: ro(qo=fake(6, 4, 72)), "rotary k_out": lambda: ro(k=None),
                "rotary amplitude": lambda: ro(amp="wide"), "rotary type": lambda: ro(q=fake(6, 4, 64, dtype=f32)),
                "attention fits": lambda: at(), "attention v": lambda: at(v=fake(9, 4, 64)), "attention k type": lambda: at(k=fake(9, 2, 64, dtype=bf16)), "attention D": lambda: at(k=fake(9, 2, 72), v=fake(9, 2, 72)),
                "attention cu": lambda: at(cq=fake(4, dtype=torch.int32)), "attention cu type": lambda: at(cq=fake(3, dtype=torch.int64)), "attention empty cu": lambda: at(cq=fake(0, dtype=torch.int32), ck=fake(0, dtype=torch.int32)),
                "attention heads": lambda: at(q=fake(6, 5, 64), o=fake(6, 5, 64)), "attention scale": lambda: at(sc=-1), "attention out": lambda: at(o=fake(6, 4, 64, dtype=bf16)),
                "attention workspace": lambda: at(k_=fake(10)), "attention host": lambda: at(k=torch.empty(9, 2, 64, device="cpu")),
            }.items():
                print(name, outcome(call), sep="=", flush=True)
    """)
    for k in [k for k in got if k.endswith(" fits")]:
        assert "VQ_ERR_NULL" in got.pop(k)      # (a fake tensor's address is null: everything before was accepted)
    library = {"quantize K", "rotary R", "attention heads", "attention scale"}
    for k, v in got.items():
        want = "VqError: " if k in library else ("TypeError: ", "ValueError: ", "AttributeError: ")
        assert v.startswith(want), (k, v)


def test_tensors_without_an_address_raise():
    got = child("""
        with FakeTensorMode():
            st = Stream()
            q, s, w, ws, y, wk = fake(M, K // 2, dtype=u8), fake(M, 4, dtype=u8), fake(N, K // 2, dtype=u8), fake(N, 4, dtype=u8), fake(M, N), fake(4096, dtype=u8)
            p, f, cu, h = fake(M, dtype=torch.int32), fake(16, dtype=f32), fake(2, dtype=torch.int32), fake(M, 2, 64)
            for name, a, call in (("quantize", fake(3, M, K), lambda a: vq.vq_mx4_quantize(a, None, q, s, stream=st)),
                                  ("read", fake(3, M, K // 2, dtype=u8), lambda a: vq.vq_mx4_dequantize(a, s, torch.float16, y, stream=st)),
                                  ("product", fake(3, M, K // 2, dtype=u8), lambda a: vq.vq_gemm_mx4(a, s, w, ws, None, y, stream=st)),
                                  ("layer", fake(3, M, K), lambda a: vq.vq_linear_mx4(a, None, w, ws, None, y, wk, stream=st)),
                                  ("rotary", fake(3, M, 2, 64), lambda a: vq.vq_rotary(a, None, p, f, q_out=h, stream=st)),
                                  ("attention", fake(3, M, 2, 64), lambda a: vq.vq_attention(a, h, h, cu, cu, out=h, workspace=wk, stream=st))):
                print(name, outcome(lambda: torch.func.vmap(call)(a)), sep="=", flush=True)
    """)
    assert len(got) == 6 and all(v.split(": ")[0] in ("RuntimeError", "ValueError") for v in got.values()), got


def test_the_definition_of_the_codes():
    grid = torch.tensor([[6.0, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -0.25, -5.0, 7.9, 0.0] + [0.0] * 20])
    code, e = ou.quantize_mx4(grid)
    assert e.tolist() == [[0]]
    assert code[0, :12].tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 8, 14, 7, 0]      # ties to the even code, beyond 6: 6
    q, s = ou.pack_mx4(code, e)
    assert s.tolist() == [[127, 0, 0, 0]] and q[0, 0] == 7 + 16 * 6
    back, eb = ou.unpack_mx4(q, s)
    assert torch.equal(back, code) and torch.equal(eb, e)
    assert ou.values_mx4(code, e)[0, :4].tolist() == [6.0, 4.0, 4.0, 2.0]
    for top, want in ((4.0, 0), (3.99, -1), (8.0, 1), (2.0 ** -130, -127), (0.0, -127)):
        x = torch.zeros(1, 32, dtype=torch.float32)
        x[0, 7] = top
        assert ou.quantize_mx4(x)[1].item() == want


def test_the_definition_of_attention():
    q, k, v = torch.randn(5, 4, 8), torch.randn(7, 2, 8), torch.randn(7, 2, 8)
    out, off = ou.attention(q, k, v, [2, 3], [1, 6], 0.3, True)
    assert (out[0] == 0).all()                                  # two queries, one key: the first sees none
    assert torch.allclose(out[1], v[0].double().repeat_interleave(2, 0))
    s = torch.einsum("hd,khd->hk", q[3].double(), k[1:6].double().repeat_interleave(2, 1)) * 0.3
    want = torch.einsum("hk,khd->hd", s.softmax(1), v[1:6].double().repeat_interleave(2, 1))
    assert torch.allclose(out[3], want) and (off >= 0).all()


def test_written_rows_that_share_memory_are_refused(lib):
    def rotary(T, H, D, token, head, k_out=False):
        own, dense = (H * D, D), (token, head)
        s = own + own + own + dense if k_out else own + dense + own + own
        return lib.vq_rotary(P(A), P(1 << 40), P(A), P(1 << 50), 0, P(A), P(A), F(1.0), 0, T, H, H, D, D, _strides(*s), None)

    def attention(T, H, D, token, head):
        s = (H * D, D) * 3 + (token, head)
        return lib.vq_attention(P(A), P(A), P(A), P(1 << 40), 0, P(A), P(A), 1, T, 1, H, H, D, _strides(*s), F(0.1), 0, None, 0, None)

    def both(*sizes):
        got = {attention(*sizes), rotary(*sizes), rotary(*sizes, k_out=True)}
        assert len(got) == 1
        return got.pop()

    # token t + 1, head h is token t, head h + 1; rows of neighbours overlap in part; far ones meet
    shared = [(4, 8, 128, 128, 128), (600, 8, 64, 128, 64), (600, 8, 64, 64, 128), (3, 2, 64, 64, 96), (3, 4, 8, 24, 16), (4, 3, 8, 16, 24),
              (1 << 20, 2, 8, 8, 8 * ((1 << 20) - 1)), (65536, 16, 8, 16, 8), (4, 65, 8, 512, 8), (1002, 1002, 8, 8008, 8000)]
    assert [both(*s) for s in shared] == [SHAPE] * len(shared)
    # token-major, head-major, with gaps, one token, one head, and rows that lie between each other's
    apart = [(600, 8, 64, 512, 64), (600, 8, 64, 64, 600 * 64), (600, 8, 64, 1024, 72), (1, 8, 64, 8, 64), (600, 1, 64, 64, 0), (3, 3, 8, 24, 16),
             (1 << 20, 2, 8, 8, 8 << 20), (65536, 2, 8, 16, 8), (4, 64, 8, 512, 8), (1000, 1000, 8, 8008, 8000), (1000, 1000, 8, 8008, 8), (2, 1000, 8, 8, 16), (2, 2, 8, 1 << 40, 1 << 39)]
    assert [both(*s) for s in apart] == [ARCH] * len(apart)


def test_microscaled_products_that_no_launch_takes_are_refused_up_front(lib):
    # (on an error nothing was enqueued: the layer may not find out behind its quantizer)
    def g(M, N, K=32):
        return lib.vq_gemm_mx4(P(A), P(A), P(A), P(A), None, P(A), 0, M, N, K, None)

    def l(M, N, K=32):
        return lib.vq_linear_mx4(P(A), None, P(A), P(A), None, P(A), 0, P(A), 1 << 62, M, N, K, None)

    most = 2**31 - 256
    for f in (g, l):
        assert [f(most + 1, 8), f(2**31 - 1, 1), f(8, most + 1), f(1, 2**31 - 1), f(most, most), f(1 << 25, 1 << 20)] == [SHAPE] * 6
        assert [f(0, 2**31 - 1), f(2**31 - 1, 0)] == [OK] * 2
        # (134 million tiles and more)
        assert [f(most, 8), f(8, most), f(1 << 20, 1 << 21), f(1 << 24, 1 << 19)] == [ARCH] * 4


def test_attention_that_no_launch_takes_is_refused_up_front(lib):
    def a(B, Tq, Tk, H, G):
        s = (8, 8) * 3 + (64 * H, 64)
        need = lib.vq_attention_workspace_bytes(B, Tq, Tk, H, G, 64)
        return lib.vq_attention(P(A), P(A), P(A), P(1 << 50), 0, P(A), P(A), B, Tq, Tk, H, G, 64, _strides(*s), F(0.1), 0, P(A), need, None)

    most = 2**31 - 256
    # workgroups of 2^32 threads and more: rows by the tile, rows by the sequence, by a wavefront a sequence
    beyond = [(1, most // 64, 2000, 64, 64), (3000, most, most, 1, 1), (1 << 21, 1 << 21, most, 8, 8), (1 << 25, 1 << 25, 1 << 25, 2, 2)]
    assert [a(*s) for s in beyond] == [SHAPE] * len(beyond)
    assert [lib.vq_attention_workspace_bytes(*s, 64) for s in beyond] == [0] * len(beyond)
    within = [(1, 1 << 24, 2000, 64, 64), (1, most - 4096, 2000, 1, 1), (1000, 1 << 30, most, 1, 1), ((1 << 21) - 8, 1 << 21, most, 8, 8),
              ((1 << 25) - 8, 1 << 25, 1 << 25, 2, 2), (1, 1, most, 1 << 16, 1)]
    assert [a(*s) for s in within] == [ARCH] * len(within)


@pytest.mark.parametrize("R,base,factor", [(64, 10000.0, 8.0), (128, 5e5, 32.0), (2, 10000.0, 4.0), (72, 100.0, 1.5)])
@pytest.mark.parametrize("length", [1, 4, 6, 7, 40, 201, 202, 4096, 1 << 30])
def test_frequencies_by_parts_follow_the_turns(R, base, factor, length):
    import paper_2406_02540_amd as vq
    f, _ = vq.vq_rotary_frequencies(R, base, "parts", factor, length)
    plain = [base ** (-2 * i / R) for i in range(R // 2)]
    turns = [length * v / (2 * math.pi) for v in plain]
    for i, (v, p, n) in enumerate(zip(f.tolist(), plain, turns)):
        if n > 32:
            assert v == pytest.approx(p, rel=1e-6), (i, n)
        elif n < 1 and (i == 0 or turns[i - 1] < 1):       # (the blend ends at a whole pair)
            assert v == pytest.approx(p / factor, rel=1e-6), (i, n)
        else:
            assert p / factor * 0.999999 <= v <= p * 1.000001, (i, n)
