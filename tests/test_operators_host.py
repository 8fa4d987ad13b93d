"""Operators next to the linear, without a GPU: what their calls refuse, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2412_14590_amd as mx
from paper_2412_14590_amd import binding

FAKE = 0x1000   # never dereferenced: validation fails first
EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -3


def epilogue(**kw):
    e = binding._Epilogue(None, None, 0, 0)
    for n, v in kw.items():
        setattr(e, n, v)
    return e


def call_epilogue(d, e, ptr=FAKE, scratch=FAKE, nbytes=1 << 30):
    L = mx.lib()
    e = None if e is None else C.byref(e)
    return (L.mixllm_mixed_linear_epilogue(C.byref(d), ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, e, ptr, None, 0, None),
            L.mixllm_mixed_linear_fp16_epilogue(C.byref(d), ptr, ptr, ptr, ptr, ptr, ptr, ptr, e, ptr, scratch, nbytes, None))


@pytest.mark.parametrize("dims,e", [
    ((4, 256, 64, 8), None),
    ((4, 256, 64, 8), epilogue(activation=5)), ((4, 256, 64, 8), epilogue(activation=-1)), ((4, 256, 64, 8), epilogue(gated=2)),
    ((4, 256, 63, 8), epilogue(gated=1)), ((4, 256, 64, 7), epilogue(gated=1)), ((0, 256, 63, 8), epilogue(gated=1)),
    ((4, 256, 64, 8), epilogue(bias=FAKE + 1)), ((4, 256, 64, 8), epilogue(residual=FAKE + 8)),
])
def test_bad_epilogues_are_refused(dims, e):
    assert call_epilogue(binding._desc(*dims), e) == (EINVAL, EINVAL)


def test_epilogue_calls_refuse_what_the_linear_refuses():
    d, e = binding._desc(4, 256, 64, 8), epilogue(activation=2)
    assert call_epilogue(d, e, ptr=None) == (EINVAL, EINVAL)
    assert call_epilogue(d, e, ptr=FAKE + 4) == (EINVAL, EINVAL)
    assert call_epilogue(binding._desc(4, 200, 64, 8), e) == (EUNSUPPORTED, EUNSUPPORTED)
    big = binding._desc(40, 4096, 64, 8)
    assert call_epilogue(big, e, scratch=FAKE, nbytes=100)[1] == EWORKSPACE
    assert call_epilogue(big, e, scratch=None)[1] == EINVAL
    assert call_epilogue(binding._desc(1 << 22, 4096, 64, 8), e, nbytes=1 << 40) == (EUNSUPPORTED, EUNSUPPORTED)   # 2^34 activations
    assert call_epilogue(binding._desc(0, 256, 64, 8), e, ptr=None) == (0, 0)


def route(ptr=FAKE, ws=FAKE, nbytes=1 << 30, logits=FAKE, bias=None, **kw):
    r = binding._RouteDesc(T=100, E=16, top_k=2, logits_fp16=0, logits_stride=16, score=0, groups=1, top_groups=1, group_score=0,
                           renormalize=1, scale=1.0)
    for n, v in kw.items():
        setattr(r, n, v)
    return mx.lib().mixllm_route_experts(C.byref(r), logits, bias, None, ptr, ptr, ptr, ptr, ptr, ws, nbytes, None)


@pytest.mark.parametrize("kw", [
    dict(T=-1), dict(E=0), dict(top_k=0), dict(top_k=17), dict(groups=0), dict(groups=3), dict(top_groups=0), dict(top_groups=2),
    dict(logits_stride=15), dict(score=2), dict(score=-1), dict(group_score=2), dict(logits_fp16=2), dict(renormalize=3),
    dict(ptr=None), dict(ptr=FAKE + 2), dict(logits=None), dict(logits=FAKE + 2), dict(logits=FAKE + 1, logits_fp16=1), dict(bias=FAKE + 1),
    dict(ws=None), dict(ws=FAKE + 8),
])
def test_bad_routes_are_refused(kw):
    assert route(**kw) == EINVAL


def test_routes_beyond_the_limits_are_refused():
    assert route(E=1025, logits_stride=1025) == EUNSUPPORTED
    assert route(E=64, logits_stride=64, top_k=33) == EUNSUPPORTED
    assert route(E=130, logits_stride=130, groups=65, top_groups=1) == EUNSUPPORTED
    assert route(T=(1 << 24) + 1) == EUNSUPPORTED
    assert route(nbytes=25 * 16 * 2 - 1) == EWORKSPACE   # 100 tokens: 25 blocks of four
    L = mx.lib()
    assert L.mixllm_route_experts(None, *[FAKE] * 9, 0, None) == EINVAL


def test_route_workspace():
    need = lambda T, E: mx.lib().mixllm_route_workspace(C.byref(binding._RouteDesc(T, E, 1, 0, E, 0, 1, 1, 0, 0, 1.0)))
    assert need(0, 16) == need(16, 16) == 0
    assert need(17, 16) == 5 * 16 * 2 and need(1025, 16) == 129 * 16 * 2 and need(16384, 16) == 256 * 16 * 2
    assert need(16385, 10) == 129 * 16 * 2               # 128 tokens a block from there on
    assert need((1 << 24) - (1 << 14), 1023) == 256 * 1024 * 2 and need(1 << 24, 1023) == 257 * 1024 * 2
    # a block's tokens, all with one expert, fit its 16-bit count
    for T in (17, 100, 16384, 16385, 1 << 20, (1 << 24) - 16384, 1 << 24):
        assert T <= need(T, 8) // 16 * 0xffff, T
    assert need(10, 1025) == 0                            # (refused)


def experts_call(d, E=4, table=FAKE, ptr=FAKE, offsets=FAKE, rows=FAKE, gather=2, e=None, ws=FAKE, nbytes=1 << 34):
    L, e = mx.lib(), C.byref(epilogue() if e is None else e)
    return (L.mixllm_experts_linear(C.byref(d), E, table, ptr, ptr, offsets, rows, gather, e, ptr, None),
            L.mixllm_experts_linear_fp16(C.byref(d), E, table, ptr, offsets, rows, gather, e, ptr, ws, nbytes, None))


def test_bad_calls_of_the_experts_are_refused():
    d = binding._desc(8, 256, 64, 0)
    for kw in (dict(E=0), dict(table=None), dict(table=FAKE + 8), dict(ptr=None), dict(ptr=FAKE + 2), dict(offsets=None), dict(offsets=FAKE + 1),
               dict(rows=None), dict(gather=-1), dict(gather=33), dict(e=epilogue(residual=FAKE)), dict(e=epilogue(activation=9)),
               dict(e=epilogue(bias=FAKE + 1))):
        assert experts_call(d, **kw) == (EINVAL, EINVAL), kw
    assert experts_call(binding._desc(8, 256, 63, 0), e=epilogue(gated=1)) == (EINVAL, EINVAL)
    assert experts_call(d, E=1025) == (EUNSUPPORTED, EUNSUPPORTED)
    assert experts_call(binding._desc(8, 200, 64, 0)) == (EUNSUPPORTED, EUNSUPPORTED)
    assert experts_call(binding._desc(1 << 20, 4096, 64, 0)) == (EUNSUPPORTED, EUNSUPPORTED)
    assert experts_call(binding._desc(8, 131072, 1 << 15, 0)) == (EUNSUPPORTED, EUNSUPPORTED)
    assert experts_call(d, nbytes=8 * 256 + 255)[1] == EWORKSPACE
    assert experts_call(d, ws=None)[1] == EINVAL
    assert experts_call(binding._desc(0, 256, 64, 0), ptr=None, table=None, offsets=None, rows=None) == (0, 0)
    need = mx.lib().mixllm_experts_workspace
    assert need(C.byref(d)) == 8 * 256 + 256 and need(C.byref(binding._desc(3, 384, 64, 9, 128))) == 1280 + 256


def test_bad_tables_of_experts_are_refused():
    L = mx.lib()
    good = binding._Expert(*[FAKE] * 6, 8, 0)
    def table(entries, d=binding._desc(0, 256, 64, 0), out=FAKE, E=None):
        arr = (binding._Expert * len(entries))(*entries)
        return L.mixllm_experts_table(C.byref(d), len(entries) if E is None else E, arr, out, None)
    assert table([good, good], out=None) == EINVAL and table([good], out=FAKE + 8) == EINVAL
    assert table([good], E=0) == EINVAL
    for n, v in (("n8", 65), ("n8", -1), ("packed_w4", None), ("packed_w8", FAKE + 4), ("scales4", None), ("scales8", None), ("zeros4", None),
                 ("feature_perm", None)):
        bad = binding._Expert(*[FAKE] * 6, 8, 0)
        setattr(bad, n, v)
        assert table([good, bad]) == EINVAL, n
    assert table([good], d=binding._desc(0, 200, 64, 0)) == EUNSUPPORTED
    assert L.mixllm_experts_table_bytes(0) == 0 and L.mixllm_experts_table_bytes(3) == 3 * 64


def test_bad_sums_are_refused():
    f = mx.lib().mixllm_experts_combine
    assert f(-1, 2, 64, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EINVAL
    assert f(4, 0, 64, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EINVAL
    assert f(4, 2, 0, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EINVAL
    assert f(4, 33, 64, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EUNSUPPORTED
    assert f(4, 2, 65535 * 256 + 1, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EUNSUPPORTED
    assert f((1 << 24) + 1, 2, 64, 8, FAKE, FAKE, FAKE, None, FAKE, None) == EUNSUPPORTED
    for bad in range(5):
        args = [FAKE, FAKE, FAKE, FAKE, FAKE]
        args[bad] = FAKE + 2
        assert f(4, 2, 64, 8, *args, None) == EINVAL, bad
    for bad in (0, 1, 2, 4):
        args = [FAKE, FAKE, FAKE, None, FAKE]
        args[bad] = None
        assert f(4, 2, 64, 8, *args, None) == EINVAL, bad
    assert f(0, 2, 64, 8, None, None, None, None, None, None) == 0


def refused(f, *words):
    with pytest.raises((AssertionError, ValueError, mx.MixllmError)) as e:
        f()
    assert any(w in str(e.value) for w in words), e.value


def test_python_calls_refuse_wrong_operands(monkeypatch):
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)
    L = binding.PackedLayer(256, 64, 8, 256, u8(16 * 256), u8(64 * 128), u8(32), u8(64 * 16), u8(64 * 4), torch.zeros(64, dtype=torch.int32))
    x = torch.zeros((4, 256), dtype=torch.float16)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)
    for f in (lambda **kw: mx.linear_fp16_epilogue(x, L, **kw),
              lambda **kw: mx.mixed_linear_epilogue(x.to(torch.int8), half(4, 1), L, **kw)):
        refused(lambda: f(activation="tanh"), "activation")
        refused(lambda: f(bias=half(63)), "bias")
        refused(lambda: f(bias=torch.zeros(64)), "bias")
        refused(lambda: f(residual=half(4, 32)), "residual")
        refused(lambda: f(residual=half(3, 64)), "residual")
        refused(lambda: f(residual=half(4, 64), gated=True), "residual")
        refused(lambda: f(), "device")                    # a tensor of the host is last
    refused(lambda: mx.linear_fp16_epilogue(x.float(), L), "fp16 matrix")
    refused(lambda: mx.mixed_linear_epilogue(x.to(torch.int8), half(4, 3), L), "xs")
    refused(lambda: mx.mixed_linear_epilogue(x, half(4, 1), L), "xq")
    logits = torch.zeros((4, 16))
    refused(lambda: mx.route_experts(logits.double(), 2), "logits")
    refused(lambda: mx.route_experts(logits, 2, score="max"), "score")
    refused(lambda: mx.route_experts(logits, 2, group_score="sum"), "group_score")
    refused(lambda: mx.route_experts(logits, 2), "device")
    route = mx.Route(torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2)), torch.zeros(4, dtype=torch.int32), torch.zeros(8, dtype=torch.int32),
                     torch.zeros((4, 2), dtype=torch.int32))
    E = mx.PackedExperts(256, 64, 256, [L] * 3, u8(3 * 64), 8)
    refused(lambda: mx.experts_linear_fp16(x[:3], E, route), "a row per token")
    refused(lambda: mx.experts_linear_fp16(x, E, route, gather=False), "a row per token")
    refused(lambda: mx.experts_linear_fp16(x[:, :128], E, route), "columns")
    refused(lambda: mx.experts_linear_fp16(x, E, route, bias=half(64)), "bias")
    refused(lambda: mx.experts_linear_fp16(x, mx.PackedExperts(256, 64, 256, [L] * 2, u8(128), 8), route), "experts")
    refused(lambda: mx.experts_linear(x.to(torch.int8), half(4, 2, 1), E, route), "xs")
    refused(lambda: mx.experts_linear_fp16(x, E, route), "device")
    refused(lambda: mx.experts_combine(half(8, 64), route, residual=half(4, 63)), "residual")
    refused(lambda: mx.experts_combine(half(8, 64), route, out=half(3, 64)), "out")
    refused(lambda: mx.experts_combine(half(8, 64), route), "device")
    odd = mx.PackedExperts(256, 64, 256, [L] * 3, u8(3 * 64), 8, pairs=False)
    refused(lambda: mx.experts_linear_fp16(x, odd, route, gated=True), "even number")
    refused(lambda: mx.experts_linear(x.to(torch.int8), half(4, 1), odd, route, gated=True), "even number")
    refused(lambda: mx.pack_experts([]), "experts of one size")
    other = binding.PackedLayer(128, 64, 8, 128, L.w8, L.w4, L.s8, L.s4, L.z4, L.perm)
    refused(lambda: mx.pack_experts([L, other]), "experts of one size")


LOAD = "\t;;#ASMSTART\n\tglobal_load_dwordx4 v[0:3], v4, s[6:7] offset:0\n\t;;#ASMEND\n"


@pytest.mark.parametrize("between,ok", [
    ("", False), ("\tv_add_u32_e32 v9, v8, v7\n" * 4, False), ("\tv_add_u32_e32 v9, v8, v7\n" * 5, True), ("\ts_nop 4\n", True), ("\ts_nop 3\n", False),
    ("\ts_add_u32 s6, s6, 16\n\ts_addc_u32 s7, s7, 0\n", True),       # rewritten by the scalar unit
    ("\ts_add_u32 s6, s6, 16\n", False),                              # ... half of it
    (".LBB0_1:\n\ts_branch .LBB0_2\n", False),
])
def test_the_build_checks_the_distance_of_a_scalar_base(between, ok):
    from paper_2412_14590_amd import build
    text = "\tv_readlane_b32 s6, v40, s3\n\tv_readfirstlane_b32 s7, v41\n" + between + LOAD
    if ok:
        build.check_scalar_bases(text, "x")
    else:
        with pytest.raises(RuntimeError):
            build.check_scalar_bases(text, "x")
    build.check_scalar_bases(text.replace("s6, v40", "s8, v40").replace("s7, v41", "s9, v41"), "x")
