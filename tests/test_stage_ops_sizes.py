"""Sizes at the ends of what the stage operators take, without a GPU: the C ABI checks them before it looks at a device."""
import pytest

from test_stage_ops_refusals import EINVAL, EMBEDDING_GRAD, ENODEV, RECURRENCE, RECURRENCE_GRAD, called, lib, strides  # noqa: F401


@pytest.mark.parametrize("empty", [dict(batch=0), dict(steps=0), dict(width=0)])
def test_packed_tensors_without_elements_have_strides_of_zero(lib, empty):  # noqa: F811
    """The strides of a packed [batch][steps][width] are steps * width and width, whichever of them is 0."""
    sizes = dict(dict(batch=4, steps=5000, width=66), **empty)
    packed = [sizes["steps"] * sizes["width"], sizes["width"]]
    assert called(lib.fpsched_op_recurrence, RECURRENCE, strides=strides(*packed * 3), **empty) == ENODEV
    assert called(lib.fpsched_op_recurrence_grad, RECURRENCE_GRAD, strides=strides(*packed * 5), **empty) == ENODEV
    assert called(lib.fpsched_op_recurrence, RECURRENCE, strides=strides(*[0, 0] * 3)) == EINVAL


def test_rows_of_the_largest_table(lib):  # noqa: F811
    most = (1 << 31) - 1
    assert called(lib.fpsched_op_embedding_grad, EMBEDDING_GRAD, rows=most) == ENODEV
    assert called(lib.fpsched_op_embedding_grad, EMBEDDING_GRAD, rows=most + 1) == EINVAL
    assert lib.fpsched_op_embedding_grad_workspace_bytes(most, 64, 5) > 0 == lib.fpsched_op_embedding_grad_workspace_bytes(most + 1, 64, 5)
