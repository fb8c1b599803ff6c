"""The layer norm of no tokens through the C entry points, which ask nothing of the addresses of matrices without rows."""
import ctypes as C

import pytest
import torch

from paper_2504_18454_b200 import block as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [5, 256, 3001, 16384])
@pytest.mark.parametrize("address", [None, 4, 0x7FFC])
@pytest.mark.parametrize("past", [False, True])
def test_weight_gradients_of_no_tokens_are_zero_and_no_row_is_read(dtype, D, address, past):
    K, es = 2, torch.finfo(dtype).bits // 8
    stream = torch.cuda.current_stream().cuda_stream
    w = torch.ones(K, D, device="cuda", dtype=dtype)
    out = torch.full((2, K, D + 3), 7.0, device="cuda", dtype=dtype)
    none, mat = B.Mat(address, D, D), lambda t: B.Mat(t.data_ptr(), t.stride(0), 0)
    r = C.byref
    s = B.NormShape(K, 1 if es == 2 else 0, 0, D, 1e-5)
    size = C.c_size_t(0)
    call = lambda ws: B.lib().palsgd_layer_norm_backward(r(s), r(none), r(none), r(mat(w)), r(none), r(none), r(none) if past else None, r(none),
                                                         r(mat(out[0])), r(mat(out[1])), ws, r(size), stream)
    assert call(None) == 0 and size.value
    ws = torch.empty(size.value, device="cuda", dtype=torch.uint8)
    assert call(ws.data_ptr()) == 0
    torch.cuda.synchronize()
    assert not bool(out[:, :, :D].any()) and bool((out[:, :, D:] == 7).all())
    assert B.lib().palsgd_layer_norm_forward(r(s), r(none), None, r(mat(w)), r(mat(w)), r(none), None, None, None, stream) == 0
