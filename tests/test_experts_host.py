"""Checks of the calls around the experts that need no GPU: what the C entries and the binding refuse before anything is launched."""
import ctypes
import os

import pytest
import torch

import paper_2508_12801_amd as ms
from paper_2508_12801_amd import binding

one, null = ctypes.c_void_p(256), None       # never dereferenced: every call below is refused


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ms.lib_path()):
        from paper_2508_12801_amd.build import build
        build()
    return ms.load_library()


CALLS = {
    "maxscore_expert_matmul": dict(x=one, W=one, dtype=0, transposed=0, offsets=one, E=4, C=8, K=16, N=16, y=one, stream=null),
    "maxscore_expert_matmul_wgrad": dict(x=one, dy=one, dtype=0, offsets=one, E=4, C=8, K=16, N=16, out_dtype=1, dW=one, stream=null),
    "maxscore_expert_swiglu": dict(x=one, W=one, dtype=0, transposed=0, offsets=one, E=4, C=8, K=16, N=16, h=one, gate_up=one, stream=null),
    "maxscore_expert_swiglu_backward": dict(gate_up=one, dh=one, dtype=0, offsets=one, E=4, C=8, N=16, dgate_up=one, h=one, stream=null),
    "maxscore_combine_backward": dict(dy=one, expert_out=one, dtype=0, assign=one, pos=one, gates=one, offsets=one, T=8, d=16, E=4, k=2, C=8,
                                      dexpert_out=one, dgates=one, stream=null),
    "maxscore_mxfp4_quantise": dict(x=one, dtype=0, rows=4, d=32, q=one, scales=one, stream=null),
    "maxscore_mxfp4_dequantise": dict(q=one, scales=one, rows=4, d=32, dtype=0, x=one, stream=null),
    "maxscore_expert_matmul_mxfp4": dict(xq=one, xs=one, Wq=one, Ws=one, offsets=one, E=4, C=8, K=32, N=16, y=one, stream=null),
    "maxscore_expert_swiglu_mxfp4": dict(xq=one, xs=one, Wq=one, Ws=one, offsets=one, E=4, C=8, K=32, N=16, h=one, stream=null),
}
OPTIONAL = {("maxscore_expert_swiglu", "gate_up"), ("maxscore_expert_swiglu_backward", "h")}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_c_entries_refuse_on_the_host(lib, name):
    args = CALLS[name]
    call = lambda **kw: getattr(lib, name)(*dict(args, **kw).values())      # noqa: E731
    for a, v in args.items():
        if v is one and (name, a) not in OPTIONAL:
            assert call(**{a: null}) == -1, a
        if a in ("E", "C", "K", "N", "d", "T", "k", "rows"):
            assert call(**{a: 0}) == -2 and call(**{a: -1}) == -2, a
        if a in ("K", "N", "d"):
            assert call(**{a: (1 << 20) + 32}) == -2, a
        if a in ("dtype", "out_dtype"):
            assert call(**{a: 2}) == -4 and call(**{a: -1}) == -4, a
    if "E" in args:
        assert call(E=1025) == -2 and call(C=(1 << 21) + 1) == -2
    if name == "maxscore_expert_matmul_wgrad":
        assert call(dtype=1, out_dtype=0) == -4            # fp32 rows have fp32 gradients
    if name == "maxscore_combine_backward":
        assert call(k=5) == -2 and call(k=65, E=100) == -2 and call(T=(1 << 21) + 1) == -2
    if "mxfp4" in name:
        assert call(**{"d" if "d" in args else "K": 48}) == -2


class FakeCuda:
    """Lets the binding's own checks run on CPU tensors: these count as the current device's."""

    def __init__(self, current=0):
        self.cuda = self
        self.current = current

    def current_device(self):
        return self.current

    def __getattr__(self, name):
        return getattr(torch, name)


class Tensor:
    """A CPU tensor that says it is on GPU `index`."""

    def __init__(self, t, index=0):
        self.t, self.index, self.is_cuda = t, index, True

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture
def bound(monkeypatch):
    monkeypatch.setattr(binding, "_torch", lambda: FakeCuda())
    monkeypatch.setattr(binding, "_TORCH", torch)
    monkeypatch.setattr(binding, "_stream", lambda: None)
    launched = []

    class Library:
        def maxscore_status_string(self, code):
            return b"refused"

        def __getattr__(self, name):
            return lambda *a: launched.append(name) or 0

    monkeypatch.setattr(binding, "load_library", lambda: Library())
    return launched


def t(*shape, dtype=torch.bfloat16, index=0):
    return Tensor(torch.zeros(shape, dtype=dtype), index)


def off(E=4, index=0):
    return t(E + 1, dtype=torch.int32, index=index)


def refused(fn, *args, **kw):
    with pytest.raises((ms.MaxScoreError, TypeError)):
        fn(*args, **kw)


def test_binding_refuses_what_the_kernels_would_misread(bound):
    x, w = t(4, 8, 32), t(4, 32, 16)
    refused(ms.expert_matmul, t(4, 8, 32, dtype=torch.float16), t(4, 32, 16, dtype=torch.float16), off())
    refused(ms.expert_matmul, t(4, 8, 32, dtype=torch.float64), w, off())
    refused(ms.expert_matmul, x, t(4, 32, 16, dtype=torch.float32), off())          # types differ
    refused(ms.expert_matmul, x, t(4, 16, 32), off())                               # layout not the one named
    refused(ms.expert_matmul, x, t(3, 32, 16), off())
    refused(ms.expert_matmul, x, w, off(), transposed=True)
    refused(ms.expert_matmul, x, w, off(3))
    refused(ms.expert_matmul, x, w, t(5, dtype=torch.int64))
    refused(ms.expert_matmul, t(8, 32), w, off())
    refused(ms.expert_matmul, t(4, 8, 32, index=1), w, off())                       # another device than the current one
    refused(ms.expert_matmul, x, t(4, 32, 16, index=1), off())
    refused(ms.expert_matmul, x, w, off(index=1))
    refused(ms.expert_matmul, torch.zeros(4, 8, 32, dtype=torch.bfloat16), w, off())    # host memory
    refused(ms.expert_matmul, Tensor(x.t.transpose(0, 1).contiguous().transpose(0, 1)), w, off())
    refused(ms.expert_matmul, x, w, off(), out=t(4, 8, 17))
    refused(ms.expert_matmul, x, w, off(), out=t(4, 8, 16, dtype=torch.float32))
    refused(ms.expert_matmul_wgrad, x, t(4, 9, 16), off())
    refused(ms.expert_matmul_wgrad, x, t(4, 8, 16, dtype=torch.float32), off())
    refused(ms.expert_matmul_wgrad, x, t(4, 8, 16), off(), dtype=torch.float16)
    refused(ms.expert_swiglu, x, t(4, 32, 15), off())                               # no pairs of gate and up
    refused(ms.expert_swiglu_backward, t(4, 8, 16), t(4, 8, 16), off())
    refused(ms.expert_swiglu_backward, t(4, 8, 32, dtype=torch.float32), t(4, 8, 16), off())
    f32, i32 = torch.float32, torch.int32
    good = dict(dy=t(6, 32, dtype=f32), expert_out=x, assign=t(6, 2, dtype=i32), token_pos=t(6, 2, dtype=i32), gate=t(6, 2, dtype=f32), expert_offsets=off())
    for name, bad in (("dy", t(6, 32)), ("dy", t(5, 32, dtype=f32)), ("dy", t(6, 31, dtype=f32)), ("assign", t(6, 2, dtype=torch.int64)),
                      ("token_pos", t(6, 3, dtype=i32)), ("gate", t(6, 2)), ("gate", t(2, 6, dtype=f32)), ("expert_offsets", off(5))):
        refused(ms.combine_backward, **dict(good, **{name: bad}))
    u8 = torch.uint8
    refused(ms.mxfp4_quantise, t(4, 48))
    refused(ms.mxfp4_quantise, t(0, 32))
    refused(ms.mxfp4_quantise, t(4, 32, dtype=torch.float16))
    refused(ms.mxfp4_dequantise, t(4, 16, dtype=u8), t(4, 2, dtype=u8))
    refused(ms.mxfp4_dequantise, t(4, 24, dtype=u8), t(4, 1, dtype=u8))
    refused(ms.mxfp4_dequantise, t(4, 16, dtype=torch.int8), t(4, 1, dtype=u8))
    mx = (t(4, 8, 32, dtype=u8), t(4, 8, 2, dtype=u8), t(4, 16, 32, dtype=u8), t(4, 16, 2, dtype=u8), off())
    for i, bad in ((0, t(4, 8, 32, dtype=torch.int8)), (1, t(4, 8, 4, dtype=u8)), (2, t(4, 16, 16, dtype=u8)), (3, t(4, 8, 2, dtype=u8)), (4, off(3))):
        refused(ms.expert_matmul_mxfp4, *(bad if n == i else a for n, a in enumerate(mx)))
    refused(ms.expert_swiglu_mxfp4, mx[0], mx[1], t(4, 15, 32, dtype=u8), t(4, 15, 2, dtype=u8), off())
    assert bound == []


def test_without_a_gpu_the_calls_fail_loudly():
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    x = torch.zeros(4, 8, 32)
    with pytest.raises(ms.MaxScoreError):
        ms.expert_matmul(x, torch.zeros(4, 32, 16), torch.zeros(5, dtype=torch.int32))
    with pytest.raises(ms.MaxScoreError):
        ms.mxfp4_quantise(x)
