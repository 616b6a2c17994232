"""What the calls for microscaled experts refuse, and their sizes, without a GPU: every refusal comes before any CUDA call."""
import ctypes

import pytest

from paper_2512_12990_b200 import binding as B

p = ctypes.c_void_p


def _route(**kw):
    a = dict(logits=p(4096), dtype=B.F32, T=1, E=64, ld=64, score=0, bias=None, n_group=1, topk_group=1, best=1, k=6, renorm=0, scale=1.0,
             tau=2.0, rank_high=0, ids=p(4096), w=p(4096), prec=None, stream=None)
    a.update(kw)
    return B.lib().slicemoe_route_scored(*a.values())


@pytest.mark.parametrize("kw", [dict(logits=None), dict(ids=None), dict(w=None), dict(T=0), dict(T=-1), dict(E=0), dict(ld=63), dict(k=0), dict(k=17),
                                dict(E=4, ld=4), dict(n_group=5, topk_group=5), dict(n_group=4, topk_group=5), dict(n_group=4, topk_group=0),
                                dict(n_group=64, topk_group=64, best=2) | dict(E=64, n_group=32, topk_group=2, k=5),
                                dict(E=8, ld=8, n_group=8, topk_group=8, best=2), dict(logits=p(4098)), dict(logits=p(4097), dtype=B.BF16)])
def test_route_refuses(kw):
    assert _route(**kw) == B.E_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(E=513, ld=513), dict(E=66, ld=66, n_group=33, topk_group=33), dict(best=3), dict(best=0), dict(dtype=3), dict(score=2)])
def test_route_does_not_support(kw):
    assert _route(**kw) == B.E_UNSUPPORTED


def _quant(call, **kw):
    a = dict(x=p(4096), dtype=B.BF16, rows=1, K=64, ld=64, codes=p(4096), scale=p(4096), stream=None)
    a.update(kw)
    if call == "slicemoe_mx4_quantize":
        return B.lib().slicemoe_mx4_quantize(*a.values())
    return B.lib().slicemoe_mx4_dequantize(a["codes"], a["scale"], a["rows"], a["K"], a["x"], a["dtype"], a["ld"], None)


@pytest.mark.parametrize("call", ["slicemoe_mx4_quantize", "slicemoe_mx4_dequantize"])
@pytest.mark.parametrize("kw,rc", [(dict(x=None), -1), (dict(codes=None), -1), (dict(scale=None), -1), (dict(rows=0), -1), (dict(K=0), -1), (dict(K=48), -1),
                                   (dict(ld=63), -1), (dict(x=p(4097)), -1), (dict(codes=p(4104)), -1), (dict(scale=p(4098)), -1), (dict(dtype=7), -2)])
def test_quantize_refuses(call, kw, rc):
    assert _quant(call, **kw) == rc


def test_sizes():
    L = B.lib()
    assert [L.slicemoe_mx4_scale_pitch(K) for K in (0, 32, 128, 160, 1408)] == [0, 4, 4, 8, 44]
    assert L.slicemoe_mx4_codes_bytes(128, 64, 0) == 4096 and L.slicemoe_mx4_codes_bytes(129, 96, 0) == 4 * 4096
    assert L.slicemoe_mx4_codes_bytes(64, 64, 1) == 4096 and L.slicemoe_mx4_codes_bytes(65, 64, 1) == 2 * 4096
    assert L.slicemoe_mx4_scale_bytes(128, 64, 0) == 512 and L.slicemoe_mx4_scale_bytes(1408, 2048, 1) == 22 * 16 * 512
    assert L.slicemoe_mx4_codes_bytes(0, 64, 0) == 0 and L.slicemoe_mx4_codes_bytes(16, 48, 0) == 0
    ws = L.slicemoe_mx4_workspace_bytes
    assert ws(0, 1, 1, 64) == 0 and ws(1, 17, 1, 64) == 0 and ws(1, 1, 1025, 64) == 0 and ws(1 << 21, 16, 8, 64) == 0 and ws(1, 1, 1, 48) == 0
    assert ws(1, 6, 64, 2048) >= 256
    for T in (1, 5, 16, 100, 223, 224, 225, 1000, 5000):          # one of a larger call serves smaller ones
        for k in (1, 3, 16):
            for E in (1, 8, 1000):
                assert all(ws(T, k, E, 160) <= ws(*more) for more in ((T + 1, k, E, 160), (T, min(k + 1, 16), E, 160), (T, k, E + 1, 160), (T, k, E, 192)))


@pytest.mark.parametrize("kw,rc", [(dict(W=None), -1), (dict(N=0), -1), (dict(K=33), -1), (dict(ld=10), -1), (dict(W=p(4098)), -1), (dict(up=p(4098)), -1),
                                   (dict(codes=p(4104)), -1), (dict(scale=p(4100)), -1), (dict(dtype=9), -2), (dict(N=(1 << 24) + 1), -2)])
def test_pack_refuses(kw, rc):
    a = dict(W=p(4096), up=None, dtype=B.F32, N=16, K=64, ld=64, codes=p(4096), scale=p(4096), stream=None)
    a.update(kw)
    assert B.lib().slicemoe_mx4_pack(*a.values()) == rc


def test_unpack_refuses():
    L = B.lib()
    assert L.slicemoe_mx4_unpack(p(4096), p(4096), 16, 64, 0, 1, p(4096), p(4096), None) == B.E_INVALID_ARG
    assert L.slicemoe_mx4_unpack(p(4096), p(4096), 16, 64, 1, 2, p(4096), p(4096), None) == B.E_INVALID_ARG
    assert L.slicemoe_mx4_unpack(None, p(4096), 16, 64, 0, 0, p(4096), p(4096), None) == B.E_INVALID_ARG


@pytest.mark.parametrize("kw,rc", [
    (dict(mats=None), -1), (dict(codes=None), -1), (dict(scale=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(E=0), -1), (dict(N=0), -1),
    (dict(K=40), -1), (dict(T=0), -1), (dict(k=0), -1), (dict(ids=None), -1), (dict(codes=p(4104)), -1), (dict(scale=p(4097)), -1), (dict(out=p(4104)), -1),
    (dict(ids=p(4097)), -1), (dict(ws=p(4096 + 16)), -1), (dict(ws_bytes=16), -1), (dict(mats=p(4100)), -1),
    (dict(E=1025), -2), (dict(k=17), -2), (dict(dtype=3), -2), (dict(T=1 << 23, k=4), -2), (dict(K=1 << 21), -2), (dict(N=(1 << 24) + 1), -2)])
def test_product_refuses(kw, rc):
    a = dict(mats=p(4096), E=8, N=64, K=64, gated=0, codes=p(4096), scale=p(4096), T=4, k=2, per_pair=0, ids=p(4096), out=p(4096), dtype=B.BF16,
             ws=p(4096), ws_bytes=1 << 30, stream=None)
    a.update(kw)
    assert B.lib().slicemoe_mx4_product(*a.values()) == rc


def test_workspace_init_refuses():
    L = B.lib()
    assert L.slicemoe_mx4_workspace_init(None, 1 << 20, None) == B.E_INVALID_ARG
    assert L.slicemoe_mx4_workspace_init(p(4096), 8, None) == B.E_INVALID_ARG
    assert L.slicemoe_mx4_workspace_init(p(4096 + 128), 1 << 20, None) == B.E_INVALID_ARG


@pytest.mark.parametrize("kw,rc", [(dict(rows=None), -1), (dict(w=None), -1), (dict(out=None), -1), (dict(T=0), -1), (dict(k=0), -1), (dict(N=0), -1),
                                   (dict(ids=p(4096)), -1), (dict(rows=p(4097)), -1), (dict(out=p(4097)), -1), (dict(base=p(4097)), -1),
                                   (dict(k=17), -2), (dict(rd=3), -2), (dict(od=-1), -2)])
def test_combine_refuses(kw, rc):
    a = dict(rows=p(4096), rd=B.BF16, T=1, k=2, N=8, w=p(4096), ids=None, E=0, base=None, out=p(4096), od=B.BF16, stream=None)
    a.update(kw)
    assert B.lib().slicemoe_combine(*a.values()) == rc


def test_the_binding_wants_device_tensors():
    import torch
    x = torch.zeros((2, 64))
    with pytest.raises(ValueError):
        B.slicemoe_mx4_quantize(x)
    with pytest.raises(ValueError):
        B.slicemoe_route_scored(x, 2)
    with pytest.raises(KeyError):
        B.slicemoe_route_scored(x, 2, score="tanh")
    with pytest.raises(ValueError):
        B.slicemoe_combine(torch.zeros((1, 2, 8)), torch.zeros((1, 2)), dtype=torch.float32)
    with pytest.raises(ValueError):
        B.slicemoe_mx4_pack(x)
    with pytest.raises(ValueError):
        B.slicemoe_mx4_dequantize(torch.zeros((1, 32), dtype=torch.uint8), torch.zeros((1, 4), dtype=torch.uint8), torch.float32)
    with pytest.raises(TypeError):
        B.slicemoe_mx4_quantize([1.0])


# Sizes that a kernel's counters would step past an int with, and arrays off their type's alignment.
@pytest.mark.parametrize("kw,rc", [(dict(T=(1 << 30) + 1), -2), (dict(bias=p(4097)), -1), (dict(ids=p(4098)), -1), (dict(w=p(4097)), -1)])
def test_route_refuses_long_lists_and_misaligned_arrays(kw, rc):
    assert _route(**kw) == rc


@pytest.mark.parametrize("call", ["slicemoe_mx4_quantize", "slicemoe_mx4_dequantize"])
@pytest.mark.parametrize("K", [(1 << 30) + 32, (1 << 31) - 32])
def test_quantize_refuses_longer_rows(call, K):
    assert _quant(call, K=K, ld=K) == B.E_UNSUPPORTED
    assert B.lib().slicemoe_mx4_scale_pitch(K) == 0


@pytest.mark.parametrize("kw,rc", [(dict(N=(1 << 30) + 1), -2), (dict(N=(1 << 31) - 1), -2), (dict(w=p(4097)), -1), (dict(ids=p(4098), E=4), -1)])
def test_combine_refuses_longer_rows_and_misaligned_arrays(kw, rc):
    a = dict(rows=p(4096), rd=B.BF16, T=1, k=2, N=8, w=p(4096), ids=None, E=0, base=None, out=p(4096), od=B.BF16, stream=None)
    a.update(kw)
    assert B.lib().slicemoe_combine(*a.values()) == rc


def test_a_table_wants_matrices_of_its_device():
    import torch
    at = {d: B.Mx4Mat(128, 64, False, torch.zeros(4096, dtype=torch.uint8, device=d), torch.zeros(512, dtype=torch.uint8, device=d)) for d in ("cpu", "meta")}
    assert B.mx4_table([at["cpu"]]).n_experts == 1
    for mats, device in (([at["cpu"], at["cpu"]], "meta"), ([at["cpu"], B.Mx4Mat(128, 64, False, at["cpu"].codes, at["meta"].scale)], "cpu")):
        with pytest.raises(ValueError):
            B.mx4_table(mats, device)
