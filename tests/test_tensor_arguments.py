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
