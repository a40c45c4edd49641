"""The Python binding of the calls of a cache in 8 or 4 bits: what it refuses before
the library is called (no GPU)."""
import pytest
import torch

import paper_2608_11368_amd as pair


def on_cpu(dtype=torch.float8_e4m3fn):
    return pair.mx_cache(2, 16, 2, 64, dtype, device="cpu")


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.float4_e2m1fn_x2])
def test_cache(dtype):
    k, v, ks, vs = on_cpu(dtype)
    width = 64 if dtype == torch.float8_e4m3fn else 32
    assert k.shape == v.shape == (2, 16, 2, width) and ks.shape == vs.shape == (2, 16, 2, 2)
    assert k.dtype == v.dtype == dtype and ks.dtype == torch.float8_e8m0fnu
    # the slots of a head side by side
    assert k.stride() == (32 * width, width, 16 * width, 1) and ks.stride() == (64, 2, 32, 1)
    assert not k.view(torch.uint8).any() and not ks.view(torch.uint8).any()
    for bad in (dict(dtype=torch.bfloat16), dict(dim=0), dict(dim=80), dict(dim=320)):
        with pytest.raises((TypeError, ValueError)):
            pair.mx_cache(**{**dict(pages=2, page=16, kv_heads=2, dim=64, device="cpu"), **bad})


def test_native_calls_take_no_other_tensors(monkeypatch):
    """None for what is not a GPU tensor; the library is not called."""
    native, never = pair._native(), 1 << 40            # an address that must not be called
    cache = on_cpu()
    k, slots = torch.zeros(3, 2, 64).bfloat16(), torch.zeros(3, dtype=torch.int64)
    for call in (native.store_mx, native.load_mx):
        assert call(never, k, k, slots, *cache, None, 0, 0) is None
        assert call(never, None, k, slots, *cache, None, 0, 0) is None
        assert call(never, k, k, slots, 1, "x", None, k, None, 0, 0) is None
        for bad in ((never, k), (never, k, k, slots, *cache, None, "device", 0),
                    ("address", k, k, slots, *cache, None, 0, 0)):
            with pytest.raises(TypeError):
                call(*bad)
    args = [never, k, *cache, slots, slots, slots, 1, 1, 0.5, k, None, slots, None, 0, 0]
    assert native.attention_mx(*args) is None
    for i, bad in ((9, "one"), (10, None), (11, "scale"), (16, "device"), (0, "address")):
        with pytest.raises(TypeError):
            native.attention_mx(*args[:i], bad, *args[i + 1:])
    with pytest.raises(TypeError):
        native.attention_mx(*args[:-1])


def test_tensors_on_the_host_are_refused(monkeypatch):
    monkeypatch.setattr(pair, "_device_index", lambda: 0)
    monkeypatch.setattr(pair, "_stream", lambda stream: 0)
    cache = on_cpu()
    k, slots = torch.zeros(3, 2, 64).bfloat16(), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="k_cache must be a 4-D CUDA tensor"):
        pair.pair_cache_store_mx(k, k, slots, *cache)
    with pytest.raises(ValueError, match="k_cache must be a 4-D CUDA tensor"):
        pair.pair_cache_load_mx(slots, *cache, k, k)
    with pytest.raises(ValueError, match="k_cache must be a 4-D CUDA tensor"):
        pair.pair_paged_attention_mx(k, *cache, slots, slots, slots, 1, 1, 0.5, k, None, slots)
