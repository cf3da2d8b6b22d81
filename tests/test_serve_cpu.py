"""Checks of the serving operators that need no GPU: the C entry points refuse bad
arguments before any CUDA call, and the tensor-level wrappers refuse bad tensors."""

import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def kd():
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    return kashin


A, NULL = 4096, None  # an aligned address that is never read


def _norm(kd, **k):
    a = dict(x=A, dtype=kd.KD_F16, n=64, rows=2, ldx=64, weight=A, weight_dtype=kd.KD_F16, eps=1e-5, residual=NULL,
             ld_residual=0, new_residual=NULL, ld_new_residual=0, q=A, ldq=64, scale=A, y=NULL, y_dtype=0, ldy=0)
    a.update(k)
    return kd.kd_rmsnorm(*a.values(), None)


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=2 ** 31), dict(dtype=3), dict(dtype=9), dict(weight_dtype=2), dict(eps=-1.0),
    dict(eps=float("nan")), dict(ldx=63), dict(ldq=63), dict(x=NULL), dict(weight=NULL), dict(q=NULL), dict(scale=NULL),
    dict(q=NULL, scale=NULL), dict(residual=A, ld_residual=63), dict(new_residual=A, ld_new_residual=64),
    dict(residual=A, ld_residual=64, new_residual=A, ld_new_residual=63), dict(y=A, ldy=63), dict(y=A, ldy=64, y_dtype=3),
    dict(x=A + 1), dict(weight=A + 1), dict(scale=A + 2), dict(y=A + 2, ldy=64), dict(residual=A + 1, ld_residual=64)])
def test_rmsnorm_refusals(kd, bad):
    assert _norm(kd, **bad) == kd.KD_ERR_INVALID_ARG


def test_rmsnorm_lengths_and_nothing_to_do(kd):
    assert _norm(kd, n=0) == kd.KD_ERR_UNSUPPORTED_N
    assert _norm(kd, n=16385, ldx=16385, ldq=16385) == kd.KD_ERR_UNSUPPORTED_N
    assert _norm(kd, rows=0, x=NULL, weight=NULL, q=NULL, scale=NULL) == kd.KD_OK


def _w4(kd, **k):
    a = dict(codes=A, scales=A, zeros=NULL, n=64, m=4, group=32, scale_dtype=kd.KD_F16)
    a.update(k)
    return kd.KdWeight4(*a.values())


BAD_W4 = [dict(n=0), dict(n=2 ** 31), dict(m=-1), dict(m=2 ** 31), dict(group=16), dict(group=0), dict(scale_dtype=0),
          dict(scale_dtype=3), dict(codes=NULL), dict(scales=NULL), dict(codes=A + 8), dict(scales=A + 1)]


@pytest.mark.parametrize("bad", BAD_W4)
def test_weight4_refusals(kd, bad):
    w = _w4(kd, **bad)
    big = 2 ** 32
    assert kd.kd_quantise_4bit(A, 0, big, ctypes.addressof(w), None) == kd.KD_ERR_INVALID_ARG
    assert kd.kd_dequantise_4bit(ctypes.addressof(w), 0, A, big, None) == kd.KD_ERR_INVALID_ARG
    assert kd.kd_matmul_4bit(ctypes.addressof(w), A, 1, None, 1, big, A, 0, big, None) == kd.KD_ERR_INVALID_ARG


def test_weight4_call_refusals(kd):
    w = _w4(kd)
    ref, bad = ctypes.addressof(w), kd.KD_ERR_INVALID_ARG
    assert kd.kd_quantise_4bit(A, 3, 64, ref, None) == bad          # e4m3 is no input type
    assert kd.kd_quantise_4bit(A, 0, 63, ref, None) == bad          # ld < n
    assert kd.kd_quantise_4bit(NULL, 0, 64, ref, None) == bad
    assert kd.kd_quantise_4bit(A + 2, 0, 64, ref, None) == bad
    assert kd.kd_quantise_4bit(A, 0, 64, None, None) == bad
    assert kd.kd_dequantise_4bit(ref, 3, A, 64, None) == bad
    assert kd.kd_dequantise_4bit(ref, 0, A, 63, None) == bad
    assert kd.kd_dequantise_4bit(ref, 0, NULL, 64, None) == bad
    assert kd.kd_dequantise_4bit(None, 0, A, 64, None) == bad
    ok = dict(x=A, x_dtype=kd.KD_F16, x_scale=NULL, rows=2, ldx=64, y=A, y_dtype=kd.KD_F32, ldy=4)
    for b in (dict(x_dtype=0), dict(x_dtype=4), dict(rows=-1), dict(ldx=63), dict(ldy=3), dict(y_dtype=3), dict(x=NULL),
              dict(y=NULL), dict(x=A + 1), dict(y=A + 2), dict(x_scale=A + 2)):
        assert kd.kd_matmul_4bit(ref, *dict(ok, **b).values(), None) == bad, b
    assert kd.kd_matmul_4bit(None, *ok.values(), None) == bad
    # nothing to do: no pointer is wanted and no device
    assert kd.kd_matmul_4bit(ref, *dict(ok, rows=0, x=NULL, y=NULL).values(), None) == kd.KD_OK
    none = _w4(kd, m=0, codes=NULL, scales=NULL)
    assert kd.kd_matmul_4bit(ctypes.addressof(none), *dict(ok, x=NULL, y=NULL).values(), None) == kd.KD_OK
    assert kd.kd_quantise_4bit(NULL, 0, 64, ctypes.addressof(none), None) == kd.KD_OK
    assert kd.kd_dequantise_4bit(ctypes.addressof(none), 0, NULL, 64, None) == kd.KD_OK


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(rows=2 ** 31), dict(vocab=0), dict(vocab=2 ** 30 + 1, ld=2 ** 31), dict(ld=99), dict(tokens=-1),
    dict(top=-1), dict(top=33), dict(vocab=5, top=6), dict(dtype=3), dict(logits=NULL), dict(ids=NULL),
    dict(logprobs=NULL), dict(top_ids=NULL), dict(top_logprobs=NULL), dict(logits=A + 1), dict(ids=A + 4),
    dict(logprobs=A + 2), dict(lse=A + 2), dict(entropy=A + 2), dict(top_ids=A + 4), dict(top_logprobs=A + 2)])
def test_token_logprobs_refusals(kd, bad):
    a = dict(logits=A, dtype=kd.KD_F16, rows=2, vocab=100, ld=100, ids=A, tokens=1, top=2, logprobs=A, lse=A, entropy=A,
             top_ids=A, top_logprobs=A)
    a.update(bad)
    assert kd.kd_token_logprobs(*a.values(), None) == kd.KD_ERR_INVALID_ARG


def test_token_logprobs_nothing_to_do(kd):
    assert kd.kd_token_logprobs(NULL, 0, 0, 100, 100, NULL, 1, 2, NULL, NULL, NULL, NULL, NULL, None) == kd.KD_OK


def test_wrappers_refuse_host_tensors_and_shapes(kd):
    x, w = torch.zeros(2, 64), torch.ones(64)
    with pytest.raises(ValueError, match="CUDA"):
        kd.rmsnorm(x, w)
    with pytest.raises(ValueError, match="2-D"):
        kd.rmsnorm(x[0], w)
    with pytest.raises(ValueError, match="dtype"):
        kd.rmsnorm(x.double(), w)
    with pytest.raises(ValueError, match="CUDA"):
        kd.quantise_4bit(x)
    with pytest.raises(ValueError, match="group"):
        kd.Weight4(torch.zeros((2, 8), dtype=torch.int32), torch.zeros((2, 2)).half(), n=64, group=16)
    with pytest.raises(ValueError, match="codes"):
        kd.Weight4(torch.zeros((2, 7), dtype=torch.int32), torch.zeros((2, 1)).half(), n=64)
    with pytest.raises(ValueError, match="scales"):
        kd.Weight4(torch.zeros((2, 8), dtype=torch.int32), torch.zeros((2, 2)).half(), n=64)
    with pytest.raises(ValueError, match="zeros"):
        kd.Weight4(torch.zeros((2, 8), dtype=torch.int32), torch.zeros((2, 1)).half(), torch.zeros((2, 1)), n=64)
    with pytest.raises(ValueError, match="CUDA"):
        kd.Weight4(torch.zeros((2, 8), dtype=torch.int32), torch.zeros((2, 1)).half(), n=64)
    with pytest.raises(ValueError, match="CUDA"):
        kd.token_logprobs(x, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="2-D"):
        kd.token_logprobs(x[0], torch.zeros(2, dtype=torch.int64))
