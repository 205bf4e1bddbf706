"""Which tensors the token operators take as rows: exactly those whose elements
lie where rows, length and distance say, found on the CPU by reading them there."""
import itertools

import numpy as np
import pytest

from paper_2108_02416_amd import aspis


def _where(x):
    """The index in memory of every element, as rows [rows, d]."""
    at = np.zeros(x.shape, dtype=np.int64)
    for i, (n, stride) in enumerate(zip(x.shape, x.stride())):
        at += stride * np.arange(n).reshape([-1 if j == i else 1 for j in range(x.dim())])
    return at.reshape(-1, x.shape[-1])


def _rows_of(x):
    """(rows, d, ld) with row i's element j at i * ld + j and ld >= d, or None."""
    at = _where(x)
    rows, d = at.shape
    ld = int(at[1, 0] - at[0, 0]) if rows > 1 else d
    same = (at == ld * np.arange(rows)[:, None] + np.arange(d)).all()
    return (rows, d, ld) if same and ld >= d else None


def test_layouts_of_every_small_shape_and_stride():
    import torch
    memory, taken = torch.arange(400.0), 0
    for dims in (1, 2, 3, 4):
        sizes = (1, 2, 3) if dims < 4 else (1, 2)
        strides = (0, 1, 2, 3, 4, 6, 12) if dims < 4 else (0, 1, 2, 4)
        for shape in itertools.product(sizes, repeat=dims):
            for stride in itertools.product(strides, repeat=dims):
                x = memory.as_strided(shape, stride)
                want, got = _rows_of(x), aspis._tensors().layout(x)
                assert got == want, (shape, stride)
                taken += want is not None
    assert taken > 1000


@pytest.mark.parametrize("shape,to", [((4, 1, 8), (4, 100, 8)), ((1, 8), (5, 8)), ((1, 1, 8), (3, 4, 8)),
                                      ((4, 1, 1), (4, 3, 1)), ((2, 1, 3, 8), (2, 5, 3, 8)),
                                      ((4, 1), (4, 8)), ((1, 3, 8), (4, 3, 8))])
def test_expanded_tensors_hold_no_rows(shape, to):
    import torch
    assert aspis._tensors().layout(torch.randn(shape).expand(to)) is None


def test_the_binding_by_attributes_takes_the_same():
    """_rows, which asks a tensor's attributes where the native call gives none."""
    import torch

    class OnGpu(torch.Tensor):
        is_cuda = True

    memory = torch.arange(400.0)
    for shape in itertools.product((1, 2, 3), repeat=3):
        for stride in itertools.product((0, 1, 2, 3, 6), repeat=3):
            x = memory.as_strided(shape, stride)
            try:
                got = aspis._rows("x", x.as_subclass(OnGpu))[:3]
            except aspis.AspisError:
                got = None
            assert got == aspis._tensors().layout(x), (shape, stride)


def test_tensors_without_elements_and_dimensions_are_left_to_the_binding():
    import torch
    for x in (torch.tensor(1.0), torch.zeros(0), torch.zeros(3, 0), torch.zeros(0, 3)):
        assert aspis._tensors().layout(x) is None
    assert aspis._tensors().layout([1.0]) is None
