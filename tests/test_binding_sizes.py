"""Counts that do not fit the library's 32 bits are refused by the bindings, not cut
off (CPU; tensors of such shapes without memory)."""
import pytest

from paper_2504_03651_amd import echo, fp8, moe


def _meta(*shape, dtype=None):
    import torch
    return torch.empty(shape, dtype=dtype or torch.float32, device="meta")


@pytest.mark.parametrize("rows, cols", [(2 ** 32, 16), (2 ** 31, 16), (3, 2 ** 32 + 16)])
def test_quantize(rows, cols):
    import torch
    for lead in ((), (2,)):
        with pytest.raises(echo.EchoError, match="2\\^31"):
            fp8.quantize(_meta(*lead, rows, cols, dtype=torch.bfloat16), _meta(*lead, rows, cols, dtype=torch.uint8),
                         _meta(*lead, rows, fp8.blocks(cols)))
    with pytest.raises(echo.EchoError, match="2\\^31"):
        fp8.quantize(_meta(rows, 1, 16, dtype=torch.bfloat16) if rows > 3 else _meta(2 ** 32, 1, 16), None, None)


@pytest.mark.parametrize("T, N, K", [(2 ** 32 + 137, 16, 16), (2, 2 ** 31, 16), (2, 16, 2 ** 32)])
def test_gemm(T, N, K):
    import torch
    u8 = torch.uint8
    with pytest.raises(echo.EchoError, match="2\\^31"):
        fp8.gemm(_meta(T, K, dtype=u8), _meta(T, fp8.blocks(K)), _meta(N, K, dtype=u8),
                 _meta(fp8.blocks(N), fp8.blocks(K)), _meta(T, N))
    with pytest.raises(echo.EchoError, match="2\\^31"):
        fp8.gemm_workspace_bytes(T, N, K)


def test_route():
    import torch
    with pytest.raises(echo.EchoError, match="2\\^31"):
        moe.route(moe.Router(8, 2), _meta(2 ** 32, 8), _meta(2 ** 32, 2, dtype=torch.int32), _meta(2 ** 32, 2))
    with pytest.raises(echo.EchoError, match="2\\^31"):
        moe.Router(2 ** 32 + 8, 2)
    with pytest.raises(echo.EchoError, match="2\\^31"):
        moe.Router(8, 2, top_groups=2 ** 32 + 1)
    for logits, ids in [(_meta(), _meta()), (_meta(8), _meta(2)), (_meta(3, 8), _meta())]:
        with pytest.raises(echo.EchoError):
            moe.route(moe.Router(8, 2), logits, ids, ids)


class _Handle(moe.Experts):
    """Experts without device memory."""

    def __init__(self, device):
        self.device, self.num_experts, self.hidden, self.intermediate = device, 2, 16, 16
        self.c = moe.CExperts(2, 16, 16)
        import ctypes
        self.ref = ctypes.byref(self.c)


def test_experts():
    import torch
    ex = _Handle(fp8.types().device())
    T, i32, u8 = 2 ** 32 + 1, torch.int32, torch.uint8
    for shape in ((T, 2), (2, T)):
        with pytest.raises(echo.EchoError, match="2\\^31"):
            moe.experts(ex, _meta(shape[0], 16, dtype=u8), _meta(shape[0], 1), _meta(*shape, dtype=i32), _meta(*shape),
                        _meta(shape[0], 16, dtype=torch.bfloat16), None)
        with pytest.raises(echo.EchoError, match="2\\^31"):
            ex.workspace_bytes(*shape)
    with pytest.raises(echo.EchoError, match="2\\^31"):
        moe.Experts(_meta(2 ** 31, 32, 16, dtype=u8), _meta(2 ** 31, 2, 1, 1), _meta(2 ** 31, 16, 16, dtype=u8),
                    _meta(2 ** 31, 1, 1))
    with pytest.raises(echo.EchoError):
        moe.experts(ex, _meta(dtype=u8), _meta(), _meta(dtype=i32), _meta(), _meta(), None)
