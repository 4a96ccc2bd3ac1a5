"""A call on another stream allocates from that stream's pool, and what it hands out waits for the caller's: the calls of caches in 4 bits,
of rotation and of pages."""
import pytest
import torch

from tests import test_mx_host as M
from tests import test_rotate_host as R
from tests.test_binding_streams import B, _g, _Lib, world      # noqa: F401


class _More(_Lib):
    def __getattr__(self, name):
        if name.endswith("_workspace_size"):
            return getattr(self.lib, name)
        return super().__getattr__(name)


def _calls(B):
    i32, bf = torch.int32, torch.bfloat16
    cache, rotation, refs = M._handle(B, N=5000), R._made(B), _g(20, dtype=i32)
    q, k, pos = _g(3, 2, 5, 8, 128, dtype=bf), _g(3, 2, 5, 4, 128, dtype=bf), _g(3, 5, dtype=i32)
    return {
        "mx_attention": lambda s: B.compactor_mx_attention(cache, q, accumulate=True, want_lse=True, stream=s),
        "mx_evict": lambda s: B.compactor_mx_evict(cache, budget=3, scope=1, stream=s) or (),
        "mx_read": lambda s: B.compactor_mx_read(cache, 5, stream=s),
        "rotate": lambda s: B.compactor_rotate(rotation, q, k, pos, want_plain=True, stream=s),
        "mx_append_rotated": lambda s: (B.compactor_mx_append_rotated(cache, rotation, k, k, q, stream=s),),
        "pages_reserve": lambda s: B.compactor_pages_reserve(cache, refs, 1, stream=s),
        "pages_compact": lambda s: B.compactor_pages_compact(cache, refs, stream=s),
    }


@pytest.mark.parametrize("name", ["mx_attention", "mx_evict", "mx_read", "rotate", "mx_append_rotated", "pages_reserve", "pages_compact"])
def test_allocations_belong_to_the_stream_that_uses_them(B, world, monkeypatch, name):      # noqa: F811
    main, side, made, lib = world
    more = _More(lib.lib)
    monkeypatch.setattr(B, "_lib", more)
    monkeypatch.setattr(M, "_g", _g)          # tensors whose allocations are noted
    monkeypatch.setattr(R, "_g", _g)
    call = _calls(B)[name]
    del made[:]
    got = call(side)
    assert more.called == ["compactor_" + name] and made
    for t, s in made:
        assert s is side, "a block of %s elements comes from the pool of another stream" % t.numel()
    for t in got:            # the caller goes on with these on its own stream
        assert t.waits == [main]
    del made[:]
    for t in call(None):
        assert not hasattr(t, "waits")
    assert made and all(s is main for _, s in made)
