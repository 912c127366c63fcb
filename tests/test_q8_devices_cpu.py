"""Where the tensors of a call lie: the 8-bit operators refuse a tensor that is not on the call's GPU
before anything is launched, and launch on that GPU's stream.  No GPU is used: stand-ins claim to be
on one, and the library is a recorder."""
from __future__ import annotations

import contextlib

import pytest
import torch

from paper_2112_13896_amd import ops


class OnGpu(torch.Tensor):
    """Host memory that says it is on GPU `gpu`."""
    gpu = 0
    is_cuda = property(lambda self: self.gpu >= 0)
    device = property(lambda self: torch.device("cuda", self.gpu) if self.gpu >= 0
                      else torch.device("cpu"))

    def get_device(self):
        return self.gpu


def at(gpu, *shape, dtype=torch.float32):
    t = torch.Tensor._make_subclass(OnGpu, torch.zeros(shape, dtype=dtype))
    t.gpu = gpu
    return t


class Recorder:
    """Stands for the library: entry points that note their arguments and succeed."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def f(*args):
            if name.endswith("_bytes"):
                return 64
            self.calls.append((name, args))
            return 0
        return f


@pytest.fixture
def rec(monkeypatch):
    r = Recorder()
    r.entered = []

    @contextlib.contextmanager
    def device(gpu):
        r.entered.append(gpu)
        yield
    monkeypatch.setattr(ops, "lib", lambda: r)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(ops, "_current_gpu", lambda: 0, raising=False)
    monkeypatch.setattr(ops, "_current_stream", lambda gpu: 1000 + gpu, raising=False)
    return r


def cache(*gpus, pages=4):
    k, v, ks, vs = gpus if len(gpus) > 1 else gpus * 4
    return ops.PagedCache(at(k, pages, 2, 16, 32, dtype=torch.int8),
                          at(v, pages, 2, 16, 32, dtype=torch.int8), at(ks, pages, 2, 16),
                          at(vs, pages, 2, 16))


def calls(gpu):
    """name -> (function of its tensors, the tensors) of a good call on a GPU."""
    i8, i32, i64 = torch.int8, torch.int32, torch.int64
    return {
        "quantise_rows": (lambda x, q, scale: ops.quantise_rows(x, q=q, scale=scale),
                          dict(x=at(gpu, 4, 32), q=at(gpu, 4, 32, dtype=i8), scale=at(gpu, 4))),
        "linear_q8": (lambda x, w, sw, sx, bias, ws, out: ops.linear_q8(
            x, w, sw, sx=sx, bias=bias, ws=ws, out=out),
            dict(x=at(gpu, 4, 32, dtype=i8), w=at(gpu, 8, 32, dtype=i8), sw=at(gpu, 8), sx=at(gpu, 4),
                 bias=at(gpu, 8), ws=at(gpu, 64, dtype=torch.uint8), out=at(gpu, 4, 8))),
        "cache_write": (lambda cache, k, v, slots: ops.cache_write(cache, k, v, slots),
                        dict(cache=cache(gpu), k=at(gpu, 3, 2, 32), v=at(gpu, 3, 2, 32),
                             slots=at(gpu, 3, dtype=i64))),
        "cache_read": (lambda cache, slots, a, b: ops.cache_read(cache, slots, torch.float32,
                                                                 out=(a, b)),
                       dict(cache=cache(gpu), slots=at(gpu, 3, dtype=i64), a=at(gpu, 3, 2, 32),
                            b=at(gpu, 3, 2, 32))),
        "paged_attention": (lambda q, cache, table, lens, starts, ws, out: ops.paged_attention(
            q, cache, table, lens, starts, ws=ws, out=out),
            dict(q=at(gpu, 3, 4, 32), cache=cache(gpu), table=at(gpu, 2, 3, dtype=i32),
                 lens=at(gpu, 2, dtype=i32), starts=at(gpu, 3, dtype=i32),
                 ws=at(gpu, 64, dtype=torch.uint8), out=at(gpu, 3, 4, 32))),
    }


NAMES = list(calls(0))


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("gpu", [0, 1])
def test_the_tensors_gpu_is_used(rec, name, gpu):
    """On the current GPU nothing is switched; on another one it is, for the launch."""
    f, tensors = calls(gpu)[name]
    f(**tensors)
    assert [c[0] for c in rec.calls] == ["cs_" + name]
    assert rec.calls[0][1][-1] == 1000 + gpu                  # the stream is the last argument
    assert rec.entered == ([gpu] if gpu else [])


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("other", [-1, 1])
def test_a_tensor_elsewhere_is_refused(rec, name, other):
    f, tensors = calls(0)[name]
    for arg, t in tensors.items():
        if arg == "cache":
            moved = cache(other)
        else:
            moved = at(other, *t.shape, dtype=t.dtype)
        with pytest.raises(ValueError):
            f(**{**tensors, arg: moved})
    assert not rec.calls


@pytest.mark.parametrize("which", [1, 2, 3])
@pytest.mark.parametrize("other", [-1, 1])
def test_a_cache_lies_on_one_device(which, other):
    gpus = [0, 0, 0, 0]
    gpus[which] = other
    with pytest.raises(ValueError):
        cache(*gpus)
