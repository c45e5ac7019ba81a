"""What the classes of the paged cache and of the rotary positions refuse or take besides test_pages_cpu.py's cases (CPU; the library's
calls are replaced by recorders)."""
import pytest
import torch

from paper_2412_14838_amd import dkv
from paper_2412_14838_amd.pages import PagedCache
from test_pages_cpu import _desc

CALLS = ("clear", "resize", "fork", "store", "store_layers", "append", "attention", "attention_layers")


def _bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.fixture
def seen(monkeypatch):
    """The calls that reach the library, as (name, arguments)."""
    calls = []
    for name in CALLS:
        monkeypatch.setattr(dkv, "dkv_pages_" + name, lambda *a, _name=name, **kw: calls.append((_name, a)))
    monkeypatch.setattr(PagedCache, "_on", lambda self, call, *args: call(*args))
    return calls


def test_layers_of_one_call_are_laid_out_alike(seen):
    """The kernel takes one pair of strides for all layers: a layer of another order would be permuted, a shorter one read past its end."""
    d = _desc()
    cache = PagedCache(d, n_pages=10, device="cpu")
    rest = (_i32(4), _i32(4, 3, 2, d.layer_max), _i32(3, 4))
    like, other = _bf(2, 60, 128), _bf(60, 2, 128).transpose(0, 1)
    for bad in (other, _bf(2, 5, 128), _bf(2, 61, 128), _bf(2, 60, 256)[..., :128], _bf(2, 80, 128)[:, 20:], _bf(3, 60, 128), _bf(60, 256),
                _bf(2, 60, 128).flatten()):
        for layer in (0, 1, 2):
            for turn in (False, True):
                xs = [like] * 3
                xs[layer] = bad
                ks, vs = (xs, [like] * 3) if turn else ([like] * 3, xs)
                with pytest.raises(ValueError):
                    cache.store_layers(0, ks, vs, *rest)
                with pytest.raises(ValueError):
                    cache.store_layers(0, ks, vs, *rest, stride_token=128)
    assert [name for name, _ in seen] == ["clear"]
    # all of another order, and strides along dimensions of one element, which are no part of the layout
    cache.store_layers(0, [other] * 3, [_bf(60, 2, 128).transpose(0, 1) for _ in range(3)], *rest)
    assert seen[-1][1][5:7] == (256, 128)
    one = PagedCache(_desc(n_q_heads=2, n_kv_heads=1), n_pages=10, device="cpu")
    one.store_layers(0, [_bf(1, 60, 128), _bf(60, 1, 128).transpose(0, 1)], [_bf(1, 60, 128)] * 2, _i32(4), _i32(4, 3, 1, d.layer_max), _i32(3, 4))
    assert seen[-1][0] == "store_layers" and seen[-1][1][5:7] == (128, 60 * 128)
    # given strides say how all of them lie, whatever their shapes
    cache.store_layers(0, [_bf(60 * 2 * 128)] * 2, [_bf(60, 2, 128)] * 2, *rest, stride_token=256, stride_head=128)
    assert seen[-1][1][5:7] == (256, 128)


def test_room_for_new_tokens_by_default(seen):
    """A layer that holds all that a prompt can leave still takes new rows; attention goes on expecting what a prompt leaves."""
    d = _desc()                                           # 16 + 64 rows of a prompt
    cache = PagedCache(d, n_pages=10, page_rows=16, device="cpu")
    assert cache.max_rows >= 80 + 1024 and cache.table.shape == (3, 4, cache.max_rows // 16)
    q, out = _bf(2, 3, 4, 128), torch.zeros(2, 3, 4, 128)

    def hints(cache):
        seen.clear()
        for rows in (0, 33):
            cache.attention(0, q[0], out[0], expected_rows=rows)
            cache.attention_layers(0, 2, q, out, expected_rows=rows)
        return [a[4 if name == "attention_layers" else 3] for name, a in seen]

    assert hints(cache) == [80, 80, 33, 33]
    assert hints(PagedCache(d, n_pages=10, page_rows=64, device="cpu")) == [128, 128, 33, 33]        # what two pages hold
    named = PagedCache(d, n_pages=10, page_rows=16, max_rows=80, device="cpu")
    assert named.max_rows == 80 and hints(named) == [0, 0, 33, 33]
    # tables of the caller's own say themselves how long they are
    tensors = {name: getattr(named, name) for name in ("k", "v", "k_scale", "v_scale", "table", "rows", "refs", "missing")}
    for length in (5, 7):
        tensors["table"] = _i32(3, 4, length)
        own = PagedCache(d, n_pages=10, page_rows=16, device="cpu", **tensors)
        assert own.max_rows == 16 * length and own.pages.table_len == length and hints(own) == [0, 0, 33, 33]
    for bad in (_i32(3, 4, 0), _i32(3, 4), _i32(4, 3, 5)):
        with pytest.raises(ValueError):
            PagedCache(d, n_pages=10, page_rows=16, device="cpu", **dict(tensors, table=bad))
