"""Refusals of the calls over 4-bit weights and of the log probabilities.  Everything here is refused (or fails for want of a GPU) before
anything is launched; the pointers are numbers that nobody follows."""
import ctypes as C

import pytest

import __graft_entry__ as entry

INVALID, UNSUPPORTED = 1, 2
P = 1 << 20                                                    # an aligned address


@pytest.fixture(scope="module")
def pb():
    entry.build()
    from paper_2607_27591_b200 import binding
    return binding


def w4(pb, codes=P, scales=P, zeros=None):
    return C.byref(pb.ProxW4(codes, scales, zeros))


def linear(pb, w=None, N=16, K=64, group=32, x=P, xs=64, xt=0, B=1, y=P, ys=16, yt=0):
    return pb.raw("prox_w4_linear")(w4(pb) if w is None else w, N, K, group, x, xs, xt, B, y, ys, yt, None)


@pytest.mark.parametrize("change,status", [
    (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(B=0), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(xt=1), INVALID), (dict(xt=3), INVALID),
    (dict(yt=3), INVALID), (dict(yt=-1), INVALID), (dict(x=P + 1), INVALID), (dict(y=P + 2, yt=1), INVALID), (dict(B=2, xs=63), INVALID), (dict(B=2, ys=15), INVALID),
    (dict(K=40), UNSUPPORTED), (dict(K=65568), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=-1), UNSUPPORTED), (dict(group=256), UNSUPPORTED),
    (dict(N=2 ** 31 - 1), UNSUPPORTED)])
def test_linear_refuses(pb, change, status):
    assert linear(pb, **change) == status


def test_linear_refuses_matrices(pb):
    assert pb.raw("prox_w4_linear")(None, 16, 64, 32, P, 64, 0, 1, P, 16, 0, None) == INVALID


def ffn(pb, gate=None, up=None, down=None, D=256, F=512, group=128, x=P, B=1, sel=P, stride=10, count=None, k2=10, y=P, yt=0, ws=P, bytes=1 << 40):
    one = w4(pb)
    return pb.raw("prox_w4_stage2_ffn")(gate or one, up or one, down or one, D, F, group, x, B, sel, stride, count, k2, y, yt, ws, bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(sel=None), INVALID), (dict(y=None), INVALID), (dict(ws=None), INVALID), (dict(B=0), INVALID), (dict(B=9), INVALID), (dict(k2=-1), INVALID),
    (dict(k2=513), INVALID), (dict(B=2, stride=9), INVALID), (dict(yt=2), INVALID), (dict(x=P + 2), INVALID), (dict(ws=P + 8), INVALID), (dict(sel=P + 2), INVALID),
    (dict(count=P + 1), INVALID), (dict(y=P + 2, yt=1), INVALID), (dict(bytes=100), INVALID), (dict(D=0), INVALID), (dict(F=0), INVALID),
    (dict(D=192), UNSUPPORTED), (dict(D=16512), UNSUPPORTED), (dict(F=65537), UNSUPPORTED), (dict(group=64), UNSUPPORTED)])
def test_ffn_refuses(pb, change, status):
    assert ffn(pb, **change) == status


def test_ffn_refuses_zero_points_on_some_matrices(pb):
    assert ffn(pb, gate=w4(pb, zeros=P)) == INVALID
    assert ffn(pb, down=w4(pb, zeros=P)) == INVALID


def test_workspace(pb):
    sizes = [pb.prox_w4_stage2_workspace(4096, 12288, b) for b in range(1, 9)]
    assert sizes == sorted(sizes) and sizes[0] >= 4 * 12288
    f = pb.raw("prox_w4_stage2_workspace")
    n = C.c_int64()
    assert f(4096, 12288, 0, C.byref(n)) == INVALID and f(4096, 12288, 9, C.byref(n)) == INVALID and f(4096, 12288, 1, None) == INVALID
    assert f(100, 12288, 1, C.byref(n)) == UNSUPPORTED
    assert ffn(pb, D=4096, F=12288, bytes=sizes[0] - 1) == INVALID


@pytest.mark.parametrize("change,status", [
    (dict(w=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(rows=0), INVALID), (dict(cols=0), INVALID), (dict(w=P + 2), INVALID),
    (dict(cols=48), UNSUPPORTED), (dict(group=48), UNSUPPORTED)])
def test_quantize_refuses(pb, change, status):
    a = dict(w=P, rows=4, cols=64, group=32, codes=P, scales=P) | change
    assert pb.raw("prox_w4_quantize")(a["w"], a["rows"], a["cols"], a["group"], a["codes"], a["scales"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(dt=3), INVALID), (dict(dt=-1), INVALID), (dict(T=0), INVALID), (dict(V=0), INVALID), (dict(stride=99), INVALID), (dict(temperature=0.0), INVALID),
    (dict(temperature=-1.0), INVALID), (dict(temperature=float("nan")), INVALID), (dict(temperature=float("inf")), INVALID), (dict(given=None), INVALID),
    (dict(logprob=None), INVALID), (dict(n_given=-1), INVALID), (dict(top=-1), INVALID), (dict(top=101), INVALID), (dict(top_logprob=None), INVALID), (dict(top_index=None), INVALID),
    (dict(x=P + 1), INVALID), (dict(x=P + 2, dt=1), INVALID), (dict(logprob=P + 2), INVALID), (dict(n_given=0, top=0, entropy=None), INVALID), (dict(top=33), UNSUPPORTED)])
def test_logprobs_refuses(pb, change, status):
    a = dict(x=P, dt=0, T=2, V=100, stride=100, temperature=1.0, given=P, n_given=1, logprob=P, entropy=P, top=5, top_logprob=P, top_index=P) | change
    assert pb.raw("prox_token_logprobs")(a["x"], a["dt"], a["T"], a["V"], a["stride"], a["temperature"], a["given"], a["n_given"], a["logprob"], a["entropy"], a["top"],
                                         a["top_logprob"], a["top_index"], None) == status


def test_without_a_gpu_the_calls_say_so(pb):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert linear(pb) == 4 and ffn(pb) == 4


def test_binding_raises(pb):
    with pytest.raises(pb.ProxError):
        pb.prox_token_logprobs(None, 0, 1, 1, 1, 1.0, None, 0, None, None, 0, None, None)
    with pytest.raises(pb.ProxError):
        pb.prox_w4_linear((P, P, None), 0, 64, 32, P, 64, 0, 1, P, 1, 0)


def test_loading_kernels_without_a_gpu_says_so(pb):
    import torch
    if torch.cuda.is_available():
        pytest.skip("there is a GPU")
    assert pb.raw("prox_load_kernels")() == 4
    with pytest.raises(pb.ProxError):
        pb.prox_load_kernels()
