"""4-bit float operators on the device, at the corners that their other tests leave out, against the definitions in 64 bits (fp4_ref)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def code_of(lib, call, *args, **kw):
    with pytest.raises(lib.B2CError) as e:
        call(*args, **kw)
    return e.value.code


def test_empty_matrices_are_refused(lib):
    """A stack of matrices without rows, a layer without an inner or a hidden size, all on the device."""
    q, s = lib.fp4_empty(3, 64, lib.NVFP4)
    b, bs = lib.fp4_empty((4, 0), 64, lib.NVFP4)
    offsets = torch.zeros(5, dtype=torch.int32, device="cuda")
    assert code_of(lib, lib.fp4_matmul, q, s, b, bs, torch.zeros(3, 0, device="cuda"), offsets=offsets) == lib.E_INVALID_ARG
    ids, weights, ws = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, 1, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    for hidden, inter in ((64, 0), (0, 64)):
        (w1, s1), (w2, s2) = lib.fp4_empty((2, 2, inter), hidden, lib.NVFP4), lib.fp4_empty((2, hidden), inter, lib.NVFP4)
        x, y = (torch.zeros(3, hidden, device="cuda") for _ in range(2))
        assert code_of(lib, lib.fp4_experts, x, ids, weights, w1, s1, w2, s2, y, ws) == lib.E_INVALID_ARG
