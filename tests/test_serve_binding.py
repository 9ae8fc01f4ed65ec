"""The binding of the serving operators without a GPU: host tensors that say they are on one, and a library that notes its calls."""
import pytest
import torch

from paper_2603_12617_amd import binding as B


class _On:
    """A host tensor that says it is on GPU 0."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


class _Library:
    def __init__(self):
        self.calls = {}

    def __getattr__(self, name):
        def call(*args):
            self.calls[name] = args
            return 0
        return call


def _i32(*shape):
    return _On(torch.zeros(shape, dtype=torch.int32))


def _bf16(*shape):
    return _On(torch.zeros(shape, dtype=torch.bfloat16))


def _f32(*shape):
    return _On(torch.zeros(shape))


def _bytes(n):
    return _On(torch.zeros(n, dtype=torch.uint8))


def _calls(**kw):
    """One call of each operator: name -> function."""
    return {
        "sd_pages": lambda: B.sd_pages(_i32(2), _i32(2), _i32(2), _i32(2, 4), _i32(8), _i32(1), 16, _i32(2), _i32(2), _i32(2), _i32(1), _i32(3), _i32(5), _i32(5), **kw),
        "sd_cache_store": lambda: B.sd_cache_store(_bf16(5, 2, 64), _bf16(5, 2, 64), _i32(5), _bf16(8, 16, 2, 64), _bf16(8, 16, 2, 64), **kw),
        "sd_attend": lambda: B.sd_attend(_bf16(5, 4, 64), _bf16(8, 16, 2, 64), _bf16(8, 16, 2, 64), _i32(3), _i32(2), _i32(2, 4), _bf16(5, 4, 64), 0.125, ws=_bytes(16), **kw),
        "sd_verify_logits": lambda: B.sd_verify_logits(_f32(5, 9), _f32(3, 9), _i32(3), _f32(3), _f32(2, 9), _f32(2), _i32(3), _i32(2), _i32(2), _bytes(64), **kw)}


class _Stream:
    cuda_stream = 0x5678


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(B, "lib", lambda: lib)
    monkeypatch.setattr(B, "_SD_DTYPE", {})
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0x1234)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: type("S", (), {"cuda_stream": 0x1234}))
    return lib


@pytest.mark.parametrize("name", sorted(_calls()))
def test_calls_go_to_the_current_stream(library, name):
    """The stream that torch's own operations go to, unless one is given."""
    _calls()[name]()
    assert library.calls[name][-1] == 0x1234
    _calls(stream=_Stream)[name]()
    assert library.calls[name][-1] == 0x5678


@pytest.mark.parametrize("ws", [None, torch.zeros(64, dtype=torch.uint8), _On(torch.zeros((8, 16), dtype=torch.uint8)[:, :8])])
def test_workspaces_that_are_refused(library, ws):
    """A workspace on the host, or one that is not whole: a refusal, not an assertion, which optimised Python leaves out."""
    with pytest.raises(ValueError):
        B.sd_attend(_bf16(5, 4, 64), _bf16(8, 16, 2, 64), _bf16(8, 16, 2, 64), _i32(3), _i32(2), _i32(2, 4), _bf16(5, 4, 64), 0.125, ws=ws)
    with pytest.raises(ValueError):
        B.sd_verify_logits(_f32(5, 9), _f32(3, 9), _i32(3), _f32(3), _f32(2, 9), _f32(2), _i32(3), _i32(2), _i32(2), ws)
    assert not library.calls
