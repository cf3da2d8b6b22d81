"""Decomposition, reconstruction, P and the 2-bit products with ``stream=``: outputs and scratch
come from that stream's pool.  On stand-ins for torch and the library: no GPU."""

import contextlib
import types

import pytest


class Tensor:
    is_cuda = True

    def __init__(self, shape, dtype, pool=None):
        self.shape = (shape,) if isinstance(shape, int) else tuple(shape)
        self.dtype, self.device, self.pool = dtype, "cuda:0", pool

    def stride(self, i):
        return self.shape[1] if i == 0 else 1

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def record_stream(self, stream):
        pass


class Torch:
    """torch.empty and the stream functions that it answers to."""

    float32, float16, bfloat16, int32, int8, uint8 = "float32", "float16", "bfloat16", "int32", "int8", "uint8"

    def __init__(self):
        self.stack = [types.SimpleNamespace(cuda_stream=0, device="cuda:0")]
        self.cuda = self
        self.taken = []

    def empty(self, shape, dtype=None, device=None):
        self.taken.append(Tensor(shape, dtype, self.stack[-1]))
        return self.taken[-1]

    def empty_like(self, t):
        return self.empty(t.shape, t.dtype)

    @contextlib.contextmanager
    def stream(self, stream):
        self.stack.append(stream)
        yield
        self.stack.pop()

    def current_stream(self, device=None):
        return self.stack[-1]


class Library:
    def __getattr__(self, name):
        return lambda *a: 256 if "size" in name else 0


@pytest.fixture
def kd(monkeypatch):
    from paper_2609_11687_gb300 import build
    build.build()
    from paper_2609_11687_gb300 import kashin
    fake = Torch()
    monkeypatch.setattr(kashin, "_torch", lambda: fake)
    monkeypatch.setattr(kashin, "lib", Library())
    return kashin, fake


def _calls(kd):
    w, x = Tensor((5, 64), "float16"), Tensor((3, 64), "float32")
    h = Tensor((3, 64), "float16")
    d = kd.Decomposed(*[Tensor((5, 4), "int32")] * 2, *[Tensor((5, 4), "float32")] * 2, None, None, None, None, None)
    ws = types.SimpleNamespace(ptr=4096, nbytes=256)
    return {
        "decompose": lambda s: kd.decompose(w, 4, 1, factors=True, trace=True, stream=s),
        "decompose_batch": lambda s: kd.decompose_batch([w, w], 4, [1, 2], coeffs=True, stream=s),
        "matmul_2bit": lambda s: kd.matmul_2bit(d, x, x, stream=s),
        "matmul_2bit_batch": lambda s: kd.matmul_2bit_batch([d], [x], [x], stream=s),
        "matmul_2bit_f16": lambda s: kd.matmul_2bit_f16(d, h, h, stream=s),
        "apply_p": lambda s: kd.apply_p(x, 1, stream=s),
        "apply_p_batch": lambda s: kd.apply_p_batch([x, x], [1, 2], stream=s),
        "prepare_p": lambda s: kd.prepare_p(64, [1], stream=s),
        "apply_p_prepared": lambda s: kd.apply_p_prepared([x], ws, stream=s),
        "dequantise": lambda s: kd.dequantise(d.codes_u, d.centres_u, 64, stream=s),
        "dequantise_batch": lambda s: kd.dequantise_batch([(d.codes_u, d.centres_u)], 64, stream=s),
        "rht": lambda s: kd.rht(x, 1, stream=s),
        "reconstruct": lambda s: kd.reconstruct(d, 64, 1, stream=s),
        "reconstruct_batch": lambda s: kd.reconstruct_batch([d, d], 64, [1, 2], stream=s),
    }


NAMES = ["decompose", "decompose_batch", "matmul_2bit", "matmul_2bit_batch", "matmul_2bit_f16", "apply_p", "apply_p_batch", "prepare_p",
         "apply_p_prepared", "dequantise", "dequantise_batch", "rht", "reconstruct", "reconstruct_batch"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_comes_from_the_pool_of_the_stream_that_writes_it(kd, name):
    kd, fake = kd
    side = types.SimpleNamespace(cuda_stream=7, device="cuda:0")
    _calls(kd)[name](side)
    assert fake.taken and all(t.pool is side for t in fake.taken)
    fake.taken.clear()
    _calls(kd)[name](None)
    assert fake.taken and all(t.pool is fake.stack[0] for t in fake.taken)
