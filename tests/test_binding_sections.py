"""The sections of xattn_rope_kvcache in the binding: whole numbers, whatever calls came before (host code only)."""
import numpy as np
import pytest
import torch

import paper_2510_14686_amd as xa
from paper_2510_14686_amd import binding

A = 4096                                # an address that is never looked at


def call(sections):
    """A call that the library refuses for its last argument, once it has the sections."""
    xa.xattn_rope_kvcache(A, A, A, 1024, 256, 256, A, A, sections, 0, A, A, A, A, 2, 9, 8, 2, 128, A + 8)


@pytest.mark.parametrize("sections", [(16, 24, 24), [16, 24, 24], np.array([16, 24, 24]), torch.tensor([16, 24, 24], dtype=torch.int32)], ids=lambda s: type(s).__name__)
def test_whole_numbers(sections):
    with pytest.raises(xa.XattnError) as e:
        call(sections)
    assert e.value.status == binding.XATTN_EINVAL and "q_out" in str(e.value)
    assert list(binding._sections_array(sections)) == [16, 24, 24]


def test_equal_numbers_of_other_types_are_refused_also_after_whole_ones():
    for other in ((40.0,), (np.float32(40),), ("40",)):
        with pytest.raises(TypeError):
            call(other)
    with pytest.raises(xa.XattnError):
        call((40,))
    for other in ((40.0,), (np.float32(40),), ("40",)):
        with pytest.raises(TypeError):
            call(other)


def test_arrays_are_kept_by_value():
    """A tensor that changes between calls names the new sections, and asking for the same ones keeps one array."""
    t = torch.tensor([8, 8], dtype=torch.int32)
    assert list(binding._sections_array(t)) == [8, 8]
    t[1] = 16
    assert list(binding._sections_array(t)) == [8, 16]
    before = len(binding._sections_arrays)
    for _ in range(10):
        binding._sections_array(t)
    assert len(binding._sections_arrays) == before
