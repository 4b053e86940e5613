"""CPU-only checks of include/gptq_w4a16_serving.h: exports, refusals before any GPU work, scratch sizes."""
import ctypes
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gptq_w4a16_serving.h")


@pytest.fixture(scope="module")
def S():
    from paper_2511_19438_amd import binding, build, serving

    if not os.path.exists(binding.LIB_PATH):
        build.build()
    serving._load()
    return serving


P, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008)  # never dereferenced: every call below fails validation first


def test_the_binding_and_the_library_have_every_declared_function(S):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = re.findall(r"GPTQ_API\s+[\w\s\*]+?\b(gptq_w4a16_\w+)\s*\(", text)
    assert sorted(names) == sorted(S.EXPORTS) and len(names) == len(set(names)) == 7
    for name in names:
        assert hasattr(S._load(), name) and callable(getattr(S, name))


def test_route_refuses(S):
    f = S._load().gptq_w4a16_moe_route
    good = dict(logits=P, kind=0, ids=P, weights=P, M=1, experts=8, top_k=2)

    def call(**kw):
        a = dict(good, **kw)
        return f(a["logits"], a["kind"], a["ids"], a["weights"], a["M"], a["experts"], a["top_k"], 1, None)

    for kw in (dict(logits=None), dict(ids=None), dict(weights=None), dict(kind=2), dict(kind=-1), dict(M=0), dict(experts=0),
               dict(top_k=0), dict(M=-1)):
        assert call(**kw) == -1, kw
    for kw in (dict(experts=1025), dict(top_k=9), dict(experts=64, top_k=33)):
        assert call(**kw) == -2, kw
    for kw in (dict(logits=ODD), dict(ids=ODD), dict(weights=ODD)):
        assert call(**kw) == -3, kw


def layer(S, **kw):
    e = S.Experts(*[0x1000] * 6, 8, 256, 128, 64)
    for k, v in kw.items():
        setattr(e, k, v)
    return e


def test_experts_refuse(S):
    lib = S._load()

    def calls(e, x=P, second=P, third=P, out=P, M=4, top_k=2):
        ref = ctypes.byref(e) if e is not None else None
        return {lib.gptq_w4a16_moe_experts(x, second, third, ref, out, M, top_k, None),
                lib.gptq_w4a16_moe(x, second, 0, ref, out, M, top_k, 1, None)}

    good = layer(S)
    for kw in (dict(x=None), dict(second=None), dict(out=None), dict(M=0), dict(top_k=0), dict(M=-3)):
        assert calls(good, **kw) == {-1}, kw
    assert calls(None) == {-1}
    for field in ("gate_up_qweight", "gate_up_qzeros", "gate_up_scales", "down_qweight", "down_qzeros", "down_scales"):
        assert calls(layer(S, **{field: None})) == {-1}, field
        assert calls(layer(S, **{field: 0x1004})) == {-3}, field
    for kw in (dict(experts=0), dict(hidden=0), dict(inter=-64), dict(group_size=0)):
        assert calls(layer(S, **kw)) == {-1}, kw
    for kw in (dict(group_size=16), dict(group_size=48), dict(hidden=224), dict(inter=96), dict(experts=1025),
               dict(hidden=1 << 21), dict(inter=1 << 21), dict(hidden=1 << 17, inter=1 << 16)):
        assert calls(layer(S, **kw)) == {-2}, kw
    assert calls(good, M=2049) == {-2} and calls(good, top_k=33) == {-2}
    for kw in (dict(x=ODD), dict(second=ODD), dict(out=ODD)):
        assert calls(good, **kw) == {-3}, kw
    assert lib.gptq_w4a16_moe(P, P, 2, ctypes.byref(good), P, 4, 2, 1, None) == -1
    assert lib.gptq_w4a16_moe(P, P, 0, ctypes.byref(layer(S, experts=1)), P, 4, 2, 1, None) == -2  # more places than experts
    assert lib.gptq_w4a16_moe_experts(P, P, None, ctypes.byref(good), P, 4, 2, None) == -1
    assert lib.gptq_w4a16_moe_experts(P, P, ODD, ctypes.byref(good), P, 4, 2, None) == -3


def test_adapters_refuse(S):
    lib = S._load()
    good = dict(x=P, a=P, b=P, scaling=P, adapter=P, base=P, out=ctypes.c_void_p(0x2000), M=4, K=64, N=32, rank=16, adapters=3,
                ldx=64, ld_base=32, ld_out=32)

    def call(**kw):
        a = dict(good, **kw)
        return lib.gptq_w4a16_lora_add(*[a[k] for k in good], None)

    for name in ("x", "a", "b", "scaling", "adapter", "base", "out"):
        assert call(**{name: None}) == -1, name
        assert call(**{name: ODD}) == -3, name
    for kw in (dict(M=0), dict(K=0), dict(N=-8), dict(rank=0), dict(adapters=0), dict(ldx=56), dict(ld_base=24), dict(ld_out=24),
               dict(out=P, ld_out=40)):
        assert call(**kw) == -1, kw
    for kw in (dict(K=60), dict(N=28), dict(rank=12), dict(rank=264), dict(ldx=68), dict(ld_base=36), dict(ld_out=36),
               dict(K=1 << 23, ldx=1 << 23), dict(adapters=1 << 30, rank=256)):
        assert call(**kw) == -2, kw

    def product(M=4, K=128, N=32, group=128, rank=16, count=3, x=P, a=P):
        return lib.gptq_w4a16_gemm_lora(x, P, P, P, a, P, P, P, ctypes.c_void_p(0x2000), M, K, N, group, rank, count, None)

    assert [product(x=None), product(a=None), product(M=0), product(group=0), product(rank=0), product(count=0)] == [-1] * 6
    assert [product(group=96), product(N=12), product(rank=20), product(rank=512)] == [-2] * 4
    assert [product(x=ODD), product(a=ODD)] == [-3] * 2


def test_workspace_bytes(S):
    f = S.gptq_w4a16_moe_workspace_bytes
    # the arrival counters, the activations of every pair in fp16 and its output in fp32
    assert f(64, 4096, 11008, 8, 2, 128) >= 262144 + 128 * (2 * 11008 + 4 * 4096)
    assert f(64, 4096, 11008, 8, 2, 128) < 1.1 * (262144 + 128 * (2 * 11008 + 4 * 4096))
    assert f(0, 4096, 11008, 8, 2, 128) == f(1, 4096, 11008, 8, 2, 100) == f(4097, 4096, 11008, 8, 1, 128) == 0
    g = S.gptq_w4a16_lora_workspace_bytes
    from paper_2511_19438_amd import binding

    assert g(16, 4096, 4096, 16) >= 262144 + 16 * 16 * 4
    assert g(16, 4096, 4096, 16, 128) >= max(binding.gptq_w4a16_workspace_bytes(16, 4096, 4096, 128), 262144) + 16 * 16 * 4
    assert g(16, 4096, 4096, 12) == g(0, 4096, 4096, 16) == g(16, 4100, 4096, 16) == g(16, 4096, 4096, 16, 100) == 0


def test_the_binding_names_what_is_wrong(S):
    """Tensors of the wrong shape, type or place are refused with a message before the library is called."""
    half = lambda *s: torch.empty(*s, dtype=torch.float16)  # noqa: E731
    with pytest.raises(ValueError, match="device memory"):
        S.gptq_w4a16_moe_route(half(2, 8), torch.empty(2, 2, dtype=torch.int32), torch.empty(2, 2))
    with pytest.raises(TypeError, match="logits"):
        S.gptq_w4a16_moe_route(torch.empty(2, 8, dtype=torch.float64), torch.empty(2, 2, dtype=torch.int32), torch.empty(2, 2))
    with pytest.raises(ValueError, match="weights"):
        S.gptq_w4a16_moe_route(half(2, 8), torch.empty(2, 2, dtype=torch.int32), torch.empty(2, 3))
    with pytest.raises(ValueError, match=r"b must be \[3, 32, 16\]"):
        S.gptq_w4a16_lora_add(half(4, 64), half(3, 16, 64), half(3, 16, 32), torch.empty(3), torch.empty(4, dtype=torch.int32),
                              half(4, 32), half(4, 32))
    words = lambda *s: torch.empty(*s, dtype=torch.int32)  # noqa: E731
    gate_up, down = (words(2, 8, 64), words(2, 2, 8), half(2, 2, 64)), (words(2, 4, 64), words(2, 1, 8), half(2, 1, 64))
    with pytest.raises(ValueError, match="out must be"):
        S.gptq_w4a16_moe(half(3, 64), half(3, 2), gate_up, down, half(3, 32), 1, 32)
    with pytest.raises(ValueError, match="gate_up qzeros"):
        S.gptq_w4a16_moe(half(3, 64), half(3, 2), (gate_up[0], words(2, 2, 4), gate_up[2]), down, half(3, 64), 1, 32)
    with pytest.raises(ValueError, match="gate_up qweight must live"):
        S.gptq_w4a16_moe(half(3, 64), half(3, 2), gate_up, down, half(3, 64), 1, 32)
