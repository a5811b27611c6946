"""step.py without a GPU: tensors that the grouped call would misread are refused when the step is made."""
import pytest
import torch

from paper_2606_07618_gb300 import binding as B
from paper_2606_07618_gb300.step import QuantizeStep


def z(*s, dt=torch.bfloat16):
    return torch.zeros(*s, dtype=dt)


def test_one_type_for_all_tensors():
    """The call takes one type for all of them: an fp32 first tensor would have bf16 ones read to twice their size."""
    QuantizeStep([z(4, 32), z(8, 16)])
    QuantizeStep([z(4, 32, dt=torch.float32)], activation=True)
    for xs in ([z(4, 32, dt=torch.float32), z(4, 32)], [z(4, 32), z(4, 32, dt=torch.float32)], [z(4, 32, dt=torch.float16)],
               [z(4, 32), z(4, 32, dt=torch.float16)], [z(4, 32, dt=torch.float64)]):
        with pytest.raises(TypeError):
            QuantizeStep(xs)


def test_tensors_are_rows_of_consecutive_elements():
    for x in (z(64, 32).t(), z(4, 64)[:, :32], z(4, 64)[:, ::2], z(1, 32).expand(4, 32), z(2, 4, 32)):
        with pytest.raises(ValueError):
            QuantizeStep([z(4, 32), x])


def test_importance_weights():
    """fp32, with an element for each column (or, with a row stride, for each element)."""
    xs, f32 = [z(4, 32), z(8, 64)], torch.float32
    step = lambda *ws, **kw: QuantizeStep(xs, list(ws), objective=B.NVFP4_OBJ_WMSE, **kw)  # noqa: E731
    step(z(32, dt=f32), z(64, dt=f32))
    step(z(4, 32, dt=f32), z(8, 80, dt=f32)[:, :64], w_row_strides=[32, 80])
    for w in (z(32), z(32, dt=torch.float64)):
        with pytest.raises(TypeError):
            step(w, z(64, dt=f32))
    for w in (z(63, dt=f32), z(32, dt=f32), z(128, dt=f32)[::2], z(1, dt=f32).expand(64)):
        with pytest.raises(ValueError):
            step(z(32, dt=f32), w)
    with pytest.raises(ValueError):
        step(z(4, 32, dt=f32), z(8, 64, dt=f32), w_row_strides=[32, 65])
