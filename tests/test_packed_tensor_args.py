"""Packed tensors that the binding refuses before it looks at their memory (no GPU: shapes, strides and addresses alone)."""
import pytest
import torch


class Device:
    """What the binding looks at of a device tensor."""

    dtype, is_cuda = torch.bfloat16, True

    def __init__(self, *shape, last=1):
        self.shape, at = shape, [last]
        for n in reversed(shape[1:]):
            at.insert(0, at[0] * n)
        self.at = tuple(at)

    def stride(self):
        return self.at

    def data_ptr(self):
        return 4096


def test_only_rows_of_128_elements():
    from paper_2502_08910_amd import binding as b
    t = b._packed_tensor(Device(10, 4, 128), "k", 10, 4)
    assert (t.ptr, t.stride_b, t.stride_h, t.stride_t) == (4096, 0, 128, 512)
    for wrong in (Device(10, 4, 64), Device(10, 4, 256), Device(10, 4, 0), Device(10, 128), Device(1, 10, 4, 128), Device(10, 4, 128, last=2)):
        with pytest.raises(b.IhipError, match="128"):
            b._packed_tensor(wrong, "k", 10, 4)
