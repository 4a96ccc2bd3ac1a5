"""A call that is given a stream allocates in that stream's pool: a block of the current stream's may still be in use there by work
that was enqueued before, and `stream` does not wait for it.  Allocations, streams and the library's calls are replaced; no GPU needed."""
import contextlib

import pytest
import torch

from tests import test_cache_host as H


@pytest.fixture(scope="module")
def B():
    from paper_2507_08143_amd import compactor
    return compactor


class _Stream:
    def __init__(self, name):
        self.name, self.cuda_stream, self.device = name, 0, torch.device("cpu")


class _Tensor(torch.Tensor):
    is_cuda = True

    def record_stream(self, stream):
        self.__dict__.setdefault("waits", []).append(stream)


class _Lib:
    """The library, whose calls that would reach a GPU succeed."""

    def __init__(self, lib):
        self.lib, self.called = lib, []

    def __getattr__(self, name):
        if name in ("compactor_layout", "compactor_workspace_size", "compactor_attention_workspace_size",
                    "compactor_cache_attention_workspace_size", "compactor_cache_evict_workspace_size"):
            return getattr(self.lib, name)
        return lambda *a: self.called.append(name) or 0


@pytest.fixture
def world(B, monkeypatch):
    """main is current; -> (main, side, list of (tensor, stream that was current when it was made))"""
    main, side = _Stream("main"), _Stream("side")
    current, made = [main], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        try:
            yield
        finally:
            current.pop()

    def noted(make):
        def f(*a, **kw):
            t = make(*a, **kw).as_subclass(_Tensor)
            made.append((t, current[-1]))
            return t
        return f

    lib = _Lib(B._lib)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[-1])
    monkeypatch.setattr(B, "_raw_stream", lambda *a: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", lambda *a: contextlib.nullcontext())
    monkeypatch.setattr(torch, "empty", noted(torch.empty))
    monkeypatch.setattr(torch, "empty_like", noted(torch.empty_like))
    monkeypatch.setattr(_Tensor, "new_empty", noted(torch.Tensor.new_empty))
    monkeypatch.setattr(B, "_lib", lib)
    return main, side, made, lib


def _g(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(_Tensor)


def _calls(B):
    params = B.Params(2, 4)
    k = _g(2, 4, 100, 128, dtype=torch.bfloat16)
    reqs = [B.Request(k_score=k, v_cache=k, ratio=0.5)]
    idx, cnt, scores = _g(2 * 4 * 50, dtype=torch.int32), _g(8, dtype=torch.int32), _g(800)
    attn = B.AttnRequest(q=_g(2, 8, 100, 128, dtype=torch.bfloat16), k=k)
    cache = H._handle(B, N=5000)
    q = _g(3, 2, 1, 8, 128, dtype=torch.bfloat16)
    return {
        "score": lambda s: B.compactor_score(params, reqs, stream=s),
        "select": lambda s: B.compactor_select(params, reqs, scores, stream=s),
        "compact": lambda s: B.compactor_compact(params, reqs, idx, cnt, stream=s),
        "compress": lambda s: tuple(B.compactor_compress(params, reqs, want_scores=True, stream=s).values()),
        "attention_scores": lambda s: (B.compactor_attention_scores(B.AttnParams(2, 4, 8), [attn], stream=s),),
        "srht_phi": lambda s: (B.compactor_srht_phi(2, [0] * 128, [0, 1], "cpu", stream=s),),
        "cache_attention": lambda s: B.compactor_cache_attention(cache, q, accumulate=True, want_lse=True, stream=s),
        "cache_evict": lambda s: B.compactor_cache_evict(cache, budget=3, scope=1, stream=s) or (),
    }


@pytest.mark.parametrize("name", ["score", "select", "compact", "compress", "attention_scores", "srht_phi", "cache_attention", "cache_evict"])
def test_allocations_belong_to_the_stream_that_uses_them(B, world, name):
    main, side, made, lib = world
    call = _calls(B)[name]
    del made[:]
    got = call(side)
    assert lib.called == ["compactor_" + name] and made
    for t, s in made:
        assert s is side, "a block of %s elements comes from the pool of another stream" % t.numel()
    for t in got:            # the caller goes on with these on its own stream
        assert t.waits == [main]
    del made[:]
    for t in call(None):
        assert not hasattr(t, "waits")
    assert made and all(s is main for _, s in made)
