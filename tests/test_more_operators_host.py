"""Rotary positions of several axes, norms of heads, attention in a window and behind a prefix where no GPU is needed: refusals of the C entry
points and of the binding, workspace sizes, and the 64-bit definitions that the GPU tests use."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import more_operator_util as mu  # noqa: E402
import operator_util as ou  # noqa: E402
from test_binding_host import child  # noqa: E402

A = 0x10000  # a made-up, 16-byte aligned address; never dereferenced by validation
P, F = ctypes.c_void_p, ctypes.c_float
OK, NULL, SHAPE, ALIGN, WORKSPACE, ARCH, TYPE = 0, 1, 2, 3, 4, 6, 8
MOST = 2**31 - 256


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2406_02540_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2406_02540_amd import build
        build.build(verbose=False)
    return binding.lib()


def _strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


def _ints(s):
    return (ctypes.c_int32 * len(s))(*s)


DENSE = (1024, 128) * 4


@pytest.mark.parametrize("norm", [None, 0, 1])
def test_rotary_refusals(lib, norm):
    def r(q=A, qo=2 * A, k=3 * A, ko=4 * A, t=0, p=A, f=A, amp=1.0, pair=0, axes=None, sec=(8, 24, 32), T=4, hq=8, hk=8, D=128, s=DENSE, w=(None,) * 4,
          eps=1e-6, n=norm):
        strides, sections = _strides(*s) if s else None, _ints(sec) if sec else None
        turn = (P(p), P(f), F(amp), pair, len(sec) if axes is None else axes, sections, T, hq, hk, D, strides, None)
        if n is None:
            return lib.vq_rotary_axes(P(q), P(qo), P(k), P(ko), t, *turn)
        return lib.vq_norm_rotary(P(q), P(qo), P(k), P(ko), t, n, F(eps), *(P(x) for x in w), *turn)

    assert [r(t=2), r(t=-1)] == [TYPE] * 2
    assert [r(T=-1), r(hq=0), r(hk=-1), r(D=0), r(D=12), r(D=136), r(amp=math.inf), r(amp=math.nan), r(hq=1 << 17), r(hk=1 << 17)] == [SHAPE] * 10
    assert [r(pair=3), r(pair=-1), r(axes=-1), r(sec=(8, 0)), r(sec=(8, -2, 4)), r(sec=(65,)), r(sec=(2**31 - 1, 2**31 - 1)), r(sec=(1,) * 5),
            r(sec=(20, 20, 25))] == [SHAPE] * 9
    assert [r(q=None), r(qo=None), r(k=None), r(ko=None), r(p=None), r(f=None), r(s=None), r(sec=None, axes=2)] == [NULL] * 8
    assert [r(q=A + 8), r(qo=A + 2), r(k=A + 4), r(ko=A + 8), r(p=A + 2), r(f=A + 4)] == [ALIGN] * 6
    assert [r(s=(1020,) + DENSE[1:]), r(s=(-8,) + DENSE[1:]), r(s=DENSE[:2] + (1024, 64) + DENSE[4:]), r(s=DENSE[:2] + (0, 128) + DENSE[4:]),
            r(qo=A, s=(1024, 128, 2048, 128) + DENSE[4:]), r(ko=3 * A, s=DENSE[:6] + (1024, 256))] == [SHAPE] * 6
    assert [r(T=0, q=None), r(), r(t=1, pair=1), r(pair=2, sec=(64,)), r(sec=(1, 1, 1, 1)), r(s=(0, 0) + DENSE[2:]), r(hk=0, k=None, ko=None), r(qo=A, ko=3 * A),
            r(p=A + 4), r(T=2**31 - 1, s=(1 << 40, 128) * 4)] == [OK] + [ARCH] * 9
    if norm is None:
        assert r(axes=0) == SHAPE
    else:
        assert [r(n=2), r(n=-1), r(eps=0.0), r(eps=-1.0), r(eps=math.nan), r(eps=math.inf), r(eps=1e-31)] == [SHAPE] * 7
        assert [r(w=tuple(A + 4 if i == j else A for j in range(4))) for i in range(4)] == [ALIGN] * 4
        assert [r(axes=0, sec=None, p=None, f=None, amp=math.nan, pair=9), r(w=(A,) * 4), r(hk=0, k=None, ko=None, w=(A, A, A + 4, None))] == [ARCH] * 3


def test_window_refusals(lib):
    dense = (1024, 128, 256, 128, 256, 128, 1024, 128)

    def a(q=A, k=A, v=A, o=2 * A, t=0, cq=A, ck=A, B=2, Tq=600, Tk=700, H=8, G=2, D=128, s=dense, scale=0.1, causal=0, left=100, right=0, sinks=4, w=None, n=0):
        return lib.vq_attention_window(P(q), P(k), P(v), P(o), t, P(cq), P(ck), B, Tq, Tk, H, G, D, _strides(*s) if s else None, F(scale), causal, left, right,
                                       sinks, P(w), n, None)

    assert [a(t=2), a(t=7)] == [TYPE] * 2
    assert [a(B=-1), a(Tq=-1), a(Tk=-1), a(H=0), a(G=0), a(G=3), a(D=0), a(D=100), a(D=136), a(causal=2), a(scale=0.0), a(scale=-1.0), a(scale=math.inf),
            a(scale=math.nan), a(H=1 << 17, G=1), a(scale=1e-31), a(Tq=1 << 28), a(Tk=2**31 - 1), a(left=-2), a(right=-2), a(sinks=-1), a(right=-2, causal=1)] == [SHAPE] * 22
    assert [a(q=None), a(k=None), a(v=None), a(o=None), a(cq=None), a(ck=None), a(s=None)] == [NULL] * 7
    assert [a(q=A + 2), a(k=A + 8), a(v=A + 8), a(o=A + 4), a(cq=A + 2), a(ck=A + 1)] == [ALIGN] * 6
    assert [a(s=(1020,) + dense[1:]), a(s=dense[:2] + (-8,) + dense[3:]), a(s=dense[:6] + (0, 128)), a(s=dense[:6] + (1024, 64)),
            a(s=dense[:2] + ((1 << 23) + 8,) + dense[3:]), a(s=dense[:4] + (1 << 24,) + dense[5:])] == [SHAPE] * 6
    assert [a(B=0, q=None), a(Tq=0, q=None), a(), a(Tk=0, k=None, v=None), a(causal=1, t=1), a(left=-1, right=-1, sinks=0),
            a(left=2**31 - 1, right=2**31 - 1, sinks=2**31 - 1)] == [OK, OK] + [ARCH] * 5
    few = dict(B=2, Tq=2, Tk=80000, left=30000)
    need = lib.vq_attention_window_workspace_bytes(2, 2, 80000, 8, 2, 128, 0, 30000, 0, 4)
    if need:
        assert [a(**few), a(**few, w=A, n=need - 1), a(**few, w=A + 8, n=need), a(**few, w=A, n=need)] == [NULL, WORKSPACE, ALIGN, ARCH]
    bad = [(0, 2, 9, 8, 2, 128, 0, 5, 5, 1), (2, 0, 9, 8, 2, 128, 0, 5, 5, 1), (2, 2, -1, 8, 2, 128, 0, 5, 5, 1), (2, 2, 9, 8, 3, 128, 0, 5, 5, 1),
           (2, 2, 9, 8, 2, 100, 0, 5, 5, 1), (2, 2, 9, 8, 0, 128, 0, 5, 5, 1), (2, 2, 9, 8, 2, 128, 2, 5, 5, 1), (2, 2, 9, 8, 2, 128, 0, -2, 5, 1),
           (2, 2, 9, 8, 2, 128, 0, 5, -2, 1), (2, 2, 9, 8, 2, 128, 0, 5, 5, -1)]
    assert [lib.vq_attention_window_workspace_bytes(*s) for s in bad] == [0] * len(bad)


def test_prefix_refusals(lib):
    dense = (1024, 128, 300 * 8, 128, 300 * 8, 128, 256, 128, 256, 128, 1024, 128)

    def a(q=A, pk=A, pv=A, k=A, v=A, o=2 * A, t=0, cq=A, ck=A, B=2, Tq=600, Pn=500, Tk=700, H=8, G=2, D=128, s=dense, scale=0.1, causal=0, w=1 << 30, n=1 << 62):
        return lib.vq_attention_prefix(P(q), P(pk), P(pv), P(k), P(v), P(o), t, P(cq), P(ck), B, Tq, Pn, Tk, H, G, D, _strides(*s) if s else None, F(scale), causal,
                                       P(w), n, None)

    assert [a(t=2), a(t=7)] == [TYPE] * 2
    assert [a(B=-1), a(Tq=-1), a(Tk=-1), a(Pn=-1), a(H=0), a(G=0), a(G=3), a(D=0), a(D=100), a(D=136), a(causal=2), a(scale=0.0), a(scale=math.inf),
            a(scale=math.nan), a(H=1 << 17, G=1), a(scale=1e-31), a(Tq=1 << 28), a(Tk=2**31 - 1), a(Pn=2**31 - 1), a(Pn=MOST, Tk=1), a(Tk=MOST, Pn=1),
            a(Tk=-100, Pn=200)] == [SHAPE] * 22
    assert [a(q=None), a(pk=None), a(pv=None), a(k=None), a(v=None), a(o=None), a(cq=None), a(ck=None), a(s=None)] == [NULL] * 9
    assert [a(q=A + 2), a(pk=A + 8), a(pv=A + 2), a(k=A + 8), a(v=A + 8), a(o=A + 4), a(cq=A + 2), a(ck=A + 1)] == [ALIGN] * 8
    wrong = [a(s=dense[:i] + (1020,) + dense[i + 1:]) for i in range(12)] + [a(s=dense[:i] + (-8,) + dense[i + 1:]) for i in range(12)]
    wrong += [a(s=dense[:i] + ((1 << 23) + 8,) + dense[i + 1:]) for i in (2, 4, 6, 8)] + [a(s=dense[:10] + (0, 128)), a(s=dense[:10] + (1024, 64))]
    assert wrong == [SHAPE] * 30
    assert [a(B=0, q=None), a(Tq=0, q=None), a(), a(Tk=0, k=None, v=None), a(Pn=0, pk=None, pv=None), a(causal=1, t=1), a(Tk=0, Pn=0, k=None, v=None, pk=None, pv=None)] == \
        [OK, OK] + [ARCH] * 5
    few = dict(B=40, Tq=40, Pn=20000, Tk=4000)
    need = lib.vq_attention_prefix_workspace_bytes(40, 40, 20000, 4000, 8, 2, 128)
    if need:
        assert [a(**few, w=None), a(**few, w=A, n=need - 1), a(**few, w=A + 8, n=need), a(**few, w=A, n=need)] == [NULL, WORKSPACE, ALIGN, ARCH]
    bad = [(0, 2, 9, 9, 8, 2, 128), (2, 0, 9, 9, 8, 2, 128), (2, 2, -1, 9, 8, 2, 128), (2, 2, 9, -1, 8, 2, 128), (2, 2, 9, 9, 8, 3, 128), (2, 2, 9, 9, 8, 2, 100),
           (2, 2, MOST, 1, 8, 2, 128), (2, 2, -5, 9, 8, 2, 128)]
    assert [lib.vq_attention_prefix_workspace_bytes(*s) for s in bad] == [0] * len(bad)


def test_written_rows_that_share_memory_are_refused(lib):
    def window(T, H, D, token, head):
        s = (H * D, D) * 3 + (token, head)
        return lib.vq_attention_window(P(A), P(A), P(A), P(1 << 40), 0, P(A), P(A), 1, T, 1, H, H, D, _strides(*s), F(0.1), 0, 1, 1, 0, None, 0, None)

    def prefix(T, H, D, token, head):
        s = (H * D, D) * 5 + (token, head)
        return lib.vq_attention_prefix(P(A), P(A), P(A), P(A), P(A), P(1 << 40), 0, P(A), P(A), 1, T, 1, 1, H, H, D, _strides(*s), F(0.1), 0, P(A), 1 << 62, None)

    def turn(T, H, D, token, head):
        s = (H * D, D, token, head) * 2
        return lib.vq_rotary_axes(P(A), P(1 << 40), P(A), P(1 << 50), 0, P(A), P(A), F(1.0), 0, 1, _ints((4,)), T, H, H, D, _strides(*s), None)

    def all_of(*sizes):
        got = {window(*sizes), prefix(*sizes), turn(*sizes)}
        assert len(got) == 1
        return got.pop()

    assert [all_of(*s) for s in ((4, 8, 128, 128, 128), (600, 8, 64, 128, 64), (3, 2, 64, 64, 96), (65536, 16, 8, 16, 8))] == [SHAPE] * 4
    assert [all_of(*s) for s in ((600, 8, 64, 512, 64), (600, 8, 64, 64, 600 * 64), (1, 8, 64, 8, 64), (3, 3, 8, 24, 16))] == [ARCH] * 4


def test_binding_refusals():
    got = child("""
        bf16, i32 = torch.bfloat16, torch.int32
        with FakeTensorMode():
            st = Stream()
            h, kv, p, f, cu = fake(6, 4, 64), fake(9, 2, 64), fake(2, 6, dtype=i32), fake(16, dtype=f32), fake(3, dtype=i32)
            ho, kr, ko, pf, w, wk = fake(6, 4, 64), fake(6, 2, 64), fake(6, 2, 64), fake(5, 2, 64), fake(64, dtype=f32), fake(1 << 20, dtype=u8)
            ax = lambda q=h, k=kr, p=p, f=f, s=(8, 8), pair="halves", amp=1.0, qo=ho, ko=ko: vq.vq_rotary_axes(q, k, p, f, s, pair, amp, qo, ko, stream=st)
            nr = lambda q=h, k=kr, qw=w, kw=w, qb=None, kb=None, n="rms", e=1e-6, p=p, f=f, s=(8, 8), pair="halves", qo=ho, ko=ko: vq.vq_norm_rotary(
                q, k, qw, kw, qb, kb, n, e, p, f, s, pair, 1.0, qo, ko, stream=st)
            wi = lambda q=h, k=kv, v=kv, cq=cu, ck=cu, l=3, r=None, s=1, sc=None, o=ho, k_=wk: vq.vq_attention_window(q, k, v, cq, ck, l, r, s, sc, False, o, k_, stream=st)
            pr = lambda q=h, pk=pf, pv=pf, k=kv, v=kv, cq=cu, ck=cu, sc=None, o=ho, k_=wk: vq.vq_attention_prefix(q, pk, pv, k, v, cq, ck, sc, False, o, k_, stream=st)
            for name, call in {
                "axes fits": lambda: ax(), "axes list fits": lambda: ax(s=[8, 8]), "axes none fits": lambda: ax(k=None, ko=None),
                "axes pairing": lambda: ax(pair="thirds"), "axes sections": lambda: ax(s=(8, 9)), "axes sections type": lambda: ax(s=(8, 8.0)), "axes no sections": lambda: ax(s=None),
                "axes positions": lambda: ax(p=fake(1, 6, dtype=i32)), "axes positions T": lambda: ax(p=fake(2, 7, dtype=i32)), "axes positions type": lambda: ax(p=fake(2, 6, dtype=torch.int64)),
                "axes positions none": lambda: ax(p=None), "axes freq": lambda: ax(f=fake(16)), "axes k type": lambda: ax(k=fake(6, 2, 64, dtype=bf16)), "axes k_out": lambda: ax(k=None),
                "axes q": lambda: ax(q=fake(6, 4, 64, dtype=f32)), "axes dims": lambda: ax(q=fake(6, 64)), "axes out": lambda: ax(qo=fake(6, 4, 72)), "axes amplitude": lambda: ax(amp="wide"),
                "LIB axes many": lambda: ax(s=(1,) * 5, p=fake(5, 6, dtype=i32), f=fake(5, dtype=f32)), "LIB axes empty": lambda: ax(s=()), "LIB axes zero": lambda: ax(s=(0, 16)),
                "LIB axes wide": lambda: ax(s=(2**40, 16)), "LIB axes heads": lambda: ax(s=(20, 20), f=fake(40, dtype=f32)),
                "norm fits": lambda: nr(), "norm alone fits": lambda: nr(p=None, f=None, s=None), "norm biases fits": lambda: nr(qb=w, kb=w, n="layer"),
                "norm kind": lambda: nr(n="max"), "norm weight": lambda: nr(qw=fake(32, dtype=f32)), "norm weight type": lambda: nr(kw=fake(64)), "norm bias": lambda: nr(kb=fake(65, dtype=f32)),
                "norm k weight": lambda: nr(k=None, ko=None), "norm positions alone": lambda: nr(s=None), "norm no positions": lambda: nr(p=None), "norm eps text": lambda: nr(e="small"),
                "LIB norm eps": lambda: nr(e=0.0), "norm pairing": lambda: nr(pair="x"),
                "window fits": lambda: wi(), "window none fits": lambda: wi(l=None), "window v": lambda: wi(v=fake(9, 4, 64)), "window k type": lambda: wi(k=fake(9, 2, 64, dtype=bf16)),
                "window D": lambda: wi(k=fake(9, 2, 72), v=fake(9, 2, 72)), "window cu": lambda: wi(cq=fake(4, dtype=i32)), "window cu type": lambda: wi(cq=fake(3, dtype=torch.int64)),
                "window left text": lambda: wi(l="far"), "window left real": lambda: wi(l=2.5), "LIB window left": lambda: wi(l=-2), "LIB window right": lambda: wi(r=-7), "LIB window sinks": lambda: wi(s=-1),
                "LIB window wide": lambda: wi(l=2**31), "LIB window heads": lambda: wi(q=fake(6, 5, 64), o=fake(6, 5, 64)), "LIB window scale": lambda: wi(sc=-1), "window out": lambda: wi(o=fake(6, 4, 64, dtype=bf16)),
                "window workspace": lambda: wi(k_=fake(10)), "window host": lambda: wi(k=torch.empty(9, 2, 64, device="cpu")),
                "prefix fits": lambda: pr(), "prefix tokens": lambda: pr(pv=fake(6, 2, 64)), "prefix heads": lambda: pr(pk=fake(5, 4, 64), pv=fake(5, 4, 64)), "prefix v heads": lambda: pr(pv=fake(5, 4, 64)),
                "prefix D": lambda: pr(pk=fake(5, 2, 72), pv=fake(5, 2, 72)), "prefix type": lambda: pr(pk=fake(5, 2, 64, dtype=bf16)), "prefix v": lambda: pr(v=fake(9, 4, 64)), "prefix none": lambda: pr(pk=None),
                "prefix cu": lambda: pr(ck=fake(4, dtype=i32)), "LIB prefix scale": lambda: pr(sc=0), "prefix out": lambda: pr(o=fake(7, 4, 64)), "prefix workspace": lambda: pr(k_=fake(10)),
            }.items():
                print(name, outcome(call), sep="=", flush=True)
    """)
    for k in [k for k in got if k.endswith(" fits")]:
        assert "VQ_ERR_NULL" in got.pop(k), k      # (a fake tensor's address is null: everything before was accepted)
    for k, v in got.items():
        want = "VqError: " if k.startswith("LIB ") else ("TypeError: ", "ValueError: ", "AttributeError: ")
        assert v.startswith(want), (k, v)


def test_tensors_without_an_address_raise():
    got = child("""
        with FakeTensorMode():
            st = Stream()
            p, f, cu, h, wk = fake(1, M, dtype=torch.int32), fake(16, dtype=f32), fake(2, dtype=torch.int32), fake(M, 2, 64), fake(1 << 20, dtype=u8)
            for name, call in (("axes", lambda a: vq.vq_rotary_axes(a, None, p, f, (16,), q_out=h, stream=st)),
                               ("norm", lambda a: vq.vq_norm_rotary(a, None, q_out=h, stream=st)),
                               ("window", lambda a: vq.vq_attention_window(a, h, h, cu, cu, 5, out=h, workspace=wk, stream=st)),
                               ("prefix", lambda a: vq.vq_attention_prefix(h, a, h, h, h, cu, cu, out=h, workspace=wk, stream=st))):
                print(name, outcome(lambda: torch.func.vmap(call)(fake(3, M, 2, 64))), sep="=", flush=True)
    """)
    assert len(got) == 4 and all(v.split(": ")[0] in ("RuntimeError", "ValueError") for v in got.values()), got


def test_the_definition_of_the_pairs():
    assert [c[2:] for c in mu.channels_of((2, 1), "halves")] == [(0, 3), (1, 4), (2, 5)]
    assert [c[2:] for c in mu.channels_of((2, 1), "neighbours")] == [(0, 1), (2, 3), (4, 5)]
    assert [c[2:] for c in mu.channels_of((2, 1), "axis_halves")] == [(0, 2), (1, 3), (4, 5)]
    assert [c[0] for c in mu.channels_of((2, 1), "halves")] == [0, 0, 1]
    x = torch.randn(5, 2, 8, dtype=torch.float64)
    p, f = torch.arange(10).view(2, 5), torch.tensor([1.0, 0.5, 0.25])
    y, _ = mu.turn(x, torch.zeros_like(x), p, f, (2, 1), "neighbours", 1.0)
    assert torch.equal(y[..., 6:], x[..., 6:])
    for t in range(5):
        for i, (a, n) in enumerate(((0, 0), (0, 1), (1, 2))):
            angle = float(p[a, t]) * float(f[n])
            z = torch.complex(x[t, :, 2 * i], x[t, :, 2 * i + 1]) * complex(math.cos(angle), math.sin(angle))
            assert torch.allclose(y[t, :, 2 * i], z.real) and torch.allclose(y[t, :, 2 * i + 1], z.imag)
    # one axis is what operator_util has
    for pairing, interleaved in (("halves", False), ("neighbours", True), ("axis_halves", False)):
        y, _ = mu.turn(x, torch.zeros_like(x), p[:1], f, (3,), pairing, 1.5)
        assert torch.allclose(y, ou.rotary(x, p[0], f, interleaved, 1.5)[0])


def test_the_definition_of_the_norms():
    x, w, b = torch.randn(3, 2, 8), torch.randn(8), torch.randn(8)
    y, off = mu.norm(x, w, b, "layer", 1e-5)
    assert torch.allclose(y, torch.nn.functional.layer_norm(x.double(), (8,), w.double(), b.double(), 1e-5)) and (off > 0).all()
    y, _ = mu.norm(x, w, None, "rms", 1e-5)
    assert torch.allclose(y, torch.nn.functional.rms_norm(x.double(), (8,), w.double(), 1e-5))


def test_the_definition_of_the_window():
    s = mu.window(1, 2, 1, False)(3, 6)          # queries at 3, 4, 5
    assert [r.nonzero().flatten().tolist() for r in s] == [[0, 2, 3, 4, 5], [0, 3, 4, 5], [0, 4, 5]]
    s = mu.window(1, 2, 2, True)(4, 2)           # at -2, -1, 0, 1
    assert [r.nonzero().flatten().tolist() for r in s] == [[], [], [0], [0, 1]]
    s = mu.window(0, 1, 0, False)(4, 2)
    assert [r.nonzero().flatten().tolist() for r in s] == [[], [0], [0, 1], [1]]
    assert mu.window(None, None, 0, False)(3, 5).all()
    assert torch.equal(mu.window(-1, -1, 0, True)(3, 5), mu.behind(True)(3, 5))
    q, k, v = torch.randn(5, 4, 8), torch.randn(7, 2, 8), torch.randn(7, 2, 8)
    for causal in (False, True):
        for a, b in zip(mu.attention(q, k, v, [2, 3], [1, 6], 0.3, mu.behind(causal)), ou.attention(q, k, v, [2, 3], [1, 6], 0.3, causal)):
            assert torch.allclose(a, b)
    pk, pv = torch.randn(4, 2, 8), torch.randn(4, 2, 8)
    out, _ = mu.attention(q, k, v, [2, 3], [1, 6], 0.3, mu.behind(True), 0, 0, pk, pv)
    want, _ = ou.attention(q[2:], torch.cat((pk, k[1:])), torch.cat((pv, v[1:])), [3], [10], 0.3, True)
    assert torch.allclose(out[2:], want)
