"""binding.py's 4-bit calls refuse operands of other types than the kernels read, before anything is launched."""
import pytest
import torch

from paper_2606_07618_gb300 import binding as B


def z(*s, dt=torch.uint8):
    return torch.zeros(*s, dtype=dt)


def op(rows, cols, codes=torch.uint8, sf=torch.uint8, S=None):
    return z(rows, cols // 2, dt=codes), z(B.swizzled_bytes(rows, cols), dt=sf), S


BAD = [op(4, 64, S=z(1, dt=torch.float64)), op(4, 64, S=z(1, dt=torch.bfloat16)), op(4, 64, S=z(1, dt=torch.int32)),
       op(4, 64, S=z(0, dt=torch.float32)), op(4, 64, S=z(2, dt=torch.float32)), op(4, 64, codes=torch.int32),
       op(4, 64, codes=torch.float16), op(4, 64, sf=torch.float32)]


@pytest.mark.parametrize("bad", range(len(BAD)))
def test_operands(bad):
    bad, good, f = BAD[bad], op(4, 64), lambda *s: z(*s, dt=torch.bfloat16)
    for a, b in ((bad, good), (good, bad)):
        with pytest.raises(TypeError):
            B.fp4_matmul(0, a, b, f(4, 4))
        with pytest.raises(TypeError):
            B.fp4_matmul_backward(0, a, b, f(4, 4), f(4, 64), f(4, 64), z(1 << 16))
    for ops in ((bad, good, good), (good, bad, good), (good, good, bad)):
        with pytest.raises(TypeError):
            B.fp4_gated_ff(0, 0, *ops, f(4, 4))
        with pytest.raises(TypeError):
            B.fp4_gated_ff_backward(0, 0, *ops, f(4, 4), f(4, 64), f(4, 64), f(4, 64), None, z(1 << 16))


def test_bytes_of_other_names_are_operands():
    """Codes and scales held as int8, E4M3 or E8M0 reach the call, which refuses the CPU's memory."""
    for codes, sf in ((torch.int8, torch.float8_e4m3fn), (torch.uint8, torch.int8)):
        with pytest.raises(B.Nvfp4Error):
            B.fp4_matmul(0, op(4, 64, codes, sf, z(1, dt=torch.float32)), op(4, 64), z(4, 4, dt=torch.float32),
                         stream=0)


def test_codes_of_a_gated_result():
    x, w = op(4, 64), op(32, 64)
    with pytest.raises(TypeError):
        B.fp4_gated_ff(0, 0, x, w, w, None, z(4, 16, dt=torch.float16), z(512))


def test_status_words():
    """A status word shorter than an int would be written past its end."""
    f = lambda *s: z(*s, dt=torch.bfloat16)  # noqa: E731
    for st in (z(1), z(2), z(1, dt=torch.int16), z(0, dt=torch.int32), z(1, dt=torch.int64), f(1)):
        for call in (lambda: B.mxfp4_quantize(f(4, 64), z(4, 32), z(4, 2), None, st),
                     lambda: B.fp4_matmul(0, op(4, 64), op(4, 64), f(4, 4), st),
                     lambda: B.fp4_selftest_wait_timeout(0, op(4, 64), op(4, 64), f(4, 4), st),
                     lambda: B.fp4_matmul_backward(0, op(4, 64), op(4, 64), f(4, 4), f(4, 64), None, z(1 << 16), st),
                     lambda: B.fp4_gated_ff(0, 0, op(4, 64), op(4, 64), op(4, 64), f(4, 4), status=st),
                     lambda: B.fp4_gated_ff_backward(0, 0, op(4, 64), op(4, 64), op(4, 64), f(4, 4), f(4, 64), status=st,
                                                     workspace=z(1 << 16))):
            with pytest.raises(TypeError):
                call()
