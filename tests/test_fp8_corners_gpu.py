"""8-bit float operators where their results hang on the numbers in between: slots that cancel, scores far below one, biases of both signs."""
import math

import pytest
import torch

import fp8_ref as ref

pytestmark = pytest.mark.gpu

E4 = torch.float8_e4m3fn
WIDE = [torch.float32, torch.float16, torch.bfloat16]


@pytest.mark.parametrize("xt", WIDE, ids=str)
@pytest.mark.parametrize("tokens", [1, 20, 30, 100, 700])
def test_experts_slots_that_cancel(lib, tokens, xt):
    """Two slots of 784 * 257 and 784 * -256: in fewer than 14 bits their sum is another number, in 16-bit floats they are infinite.
    Everything is a whole number of few bits, so the result is exact up to the rounding of y."""
    H = I = 128
    x = torch.zeros(tokens, H, device="cuda")
    x[:, 0] = 448.0                                          # scale 1
    w1 = torch.zeros(2, 2, I, H, device="cuda")
    w1[:, :, :, 0] = 1.0
    s1 = torch.tensor([1.0, 2.0 ** -8], device="cuda").repeat(2).reshape(2, 2, 1, 1)  # gate 448, up 1.75: h = 784 = 448 * 1.75
    w2 = torch.zeros(2, H, I, device="cuda")
    n = torch.arange(H, device="cuda")
    w2[0, :, 0], w2[0, :, 1] = 256.0, 1.0
    w2[1, :, 0], w2[1, :, 1] = -256.0, (n % 8).float()
    s2 = torch.ones(2, 1, 1, device="cuda")
    ids = torch.tensor([0, 1], dtype=torch.int32, device="cuda").repeat(tokens, 1)
    ids[1::2] = ids[1::2].flip(1)
    w = torch.ones(tokens, 2, device="cuda") * 2.0 ** -(torch.arange(tokens, device="cuda") % 3)[:, None]
    y = torch.full((tokens, H), math.nan, device="cuda", dtype=xt)
    kind = {torch.float32: lib.F32, torch.float16: lib.F16, torch.bfloat16: lib.BF16}[xt]
    ws = torch.empty(lib.experts_workspace_bytes(H, I, 2, 2, tokens, dtype=kind), dtype=torch.uint8, device="cuda")
    lib.fp8_experts(x.to(xt), ids, w, w1.to(E4), s1, w2.to(E4), s2, y, ws)
    assert lib.fp8_status() == lib.OK
    want = 784.0 * (1.0 + (n % 8).float()) * w[:, :1]
    assert torch.equal(y, want.to(xt))
