"""The native reader of tensor arguments: refusals without a GPU; on one, its
addresses, sizes and types against torch's own."""
import array

import pytest
import torch

import paper_2608_11368_amd as pair

DEV = "cuda:0"


def test_address_refusals():
    address = pair._native().address
    assert address(None, "x", torch.int32, 3, True) is None
    for bad in (None, 3, "t", torch.ones(4)):
        with pytest.raises(ValueError, match="^x "):
            address(bad, "x", torch.float32, 1)
    for call in ((), (None,), (None, "x", torch.int32, 1, True, 0), (torch.ones(1), "x", "int32")):
        with pytest.raises(TypeError):
            address(*call)


def test_table_refusals():
    table = pair._native().grad_table
    for bad in ([torch.ones(3)], [3], [None], ["t", torch.ones(2)]):
        with pytest.raises(ValueError, match="^grads must be"):
            table(bad, "grads")
    for call in (((torch.ones(2),), "grads"), ([],), (None, "grads")):
        with pytest.raises(TypeError):
            table(*call)
    assert table([], "grads") == (b"", b"", b"")


@pytest.mark.gpu
def test_against_torch():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    address, table = pair._native().address, pair._native().grad_table
    flat = torch.zeros(1000, device=DEV)
    views = [flat[1:8], flat[:0], flat[8:400].view(4, 98), torch.nn.Parameter(flat[500:]),
             torch.zeros(7, device=DEV).bfloat16(), torch.zeros(3, device=DEV).half()[1:]]
    ptrs, sizes, codes = table(views, "grads")
    assert array.array("Q", ptrs).tolist() == [v.data_ptr() for v in views]
    assert array.array("q", sizes).tolist() == [v.numel() for v in views]
    assert array.array("i", codes).tolist() == [0, 0, 0, 0, 1, 2]
    with pytest.raises(TypeError, match="got torch.float64"):
        table([flat, flat.double()], "grads")
    for bad in (flat[::2], torch.zeros(4, 4, device=DEV).t()):
        with pytest.raises(ValueError, match="contiguous"):
            table([flat, bad], "grads")
        with pytest.raises(ValueError, match="contiguous"):
            address(bad, "x", torch.float32)
    with pytest.raises(ValueError, match="one device"):
        table([flat, torch.ones(2)], "grads")
    assert address(flat[3:], "x", torch.float32, 997) == flat.data_ptr() + 12
    with pytest.raises(ValueError, match="holds 997 elements, needs 998"):
        address(flat[3:], "x", torch.float32, 998)
    with pytest.raises(TypeError, match="must be torch.int32, got torch.float32"):
        address(flat, "x", torch.int32)


def test_parts_refusals():
    parts = pair._native().parts
    for call in ((), (0,), (0, torch.int32), (0, torch.int32, 3, 4), ("0", torch.int32, 3),
                 (0, "int32", 3), (0, torch.int32, (1, 2, 3, 4, 5)), (0, torch.int32, None),
                 (0,) + (torch.int32, 1) * 17):
        with pytest.raises(TypeError):
            parts(*call)
    for call in ((-1, torch.int32, 3), (0, torch.int32, -1), (0, torch.int32, (1 << 40, 1 << 40))):
        with pytest.raises(ValueError):
            parts(*call)


def test_layouts_of_others_are_none():
    native = pair._native()
    x = torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16)      # not on a GPU
    assert native.cache(x, x) is None and native.cache(None, x) is None
    assert native.rows(x[0], 1, 2, 64) is None and native.rows("x", 1, 2, 64) is None
    for call in ((), (x,), (x, x, x)):
        with pytest.raises(TypeError):
            native.cache(*call)
    with pytest.raises(TypeError):
        native.rows(x[0], 1, 2)


@pytest.mark.gpu
def test_layouts_against_torch():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    native = pair._native()
    both = torch.zeros(3, 5, 16, 2, 2, 64, dtype=torch.float16, device=DEV)
    k, v = both[1:, :, 2:, 0, :1].transpose(1, 2)[:, :, 0], both[1:, :, 2:, 1, :1].transpose(1, 2)[:, :, 0]
    assert k.dim() == 4
    assert native.cache(k, v) == (k.data_ptr(), v.data_ptr(), 2, *k.stride()[:3], *k.shape)
    assert native.cache(k, v[:1]) is None and native.cache(k, v.bfloat16()) is None
    assert native.cache(k, v.contiguous()) is None and native.cache(k.float(), v.float()) is None
    assert native.cache(k[..., ::2], v[..., ::2]) is None and native.cache(k[0], v[0]) is None
    q = torch.zeros(7, 9, 128, dtype=torch.bfloat16, device=DEV)[1:, ::2, :64]
    assert native.rows(q, 1, 0, 64) == (q.data_ptr(), 9 * 128, 256, 6, 5)
    assert native.rows(q, 1, 5, 64) == native.rows(q, 1, 0, 64)
    for other in ((q, 2, 5, 64), (q, 1, 4, 64), (q, 1, 5, 32), (q[0], 1, 5, 64),
                  (q[..., ::2], 1, 5, 32)):
        assert native.rows(*other) is None


@pytest.mark.gpu
def test_parts():
    """Parts of one allocation are tensors like others: shapes, types, places
    apart, written without touching each other, alive on their own."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    want = [(torch.uint8, 7), (torch.int32, (3, 5)), (torch.float32, 0), (torch.int64, 33),
            (torch.bfloat16, (2, 3, 4)), (torch.float32, (1, 1))]
    got = pair._native().parts(0, *[x for pair_ in want for x in pair_])
    spans = []
    for k, (t, (dtype, shape)) in enumerate(zip(got, want)):
        assert t.dtype is dtype and t.device == torch.device(DEV) and t.is_contiguous()
        assert tuple(t.shape) == (shape if isinstance(shape, tuple) else (shape,))
        assert t.data_ptr() % 256 == 0 and not t.requires_grad and t._base is None
        if t.numel():                 # an empty tensor's address reads as 0
            spans.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
        t.fill_(k + 1)
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    for k, t in enumerate(got):
        assert bool((t == k + 1).all())
    last, first = got[3], got[0]
    del got, t
    torch.zeros(1 << 20, device=DEV)
    assert bool((last == 4).all()) and bool((first == 1).all())
    leaf = pair._native().parts(0, torch.float32, 4)[0].fill_(2.0).requires_grad_()
    (leaf * leaf).sum().backward()
    assert leaf.grad.tolist() == [4.0] * 4
    with torch.inference_mode():
        assert pair._native().parts(0, torch.float32, 4)[0].fill_(1.0).sum().item() == 4.0
    with pytest.raises(torch.OutOfMemoryError):
        pair._native().parts(0, torch.uint8, 1 << 44)
