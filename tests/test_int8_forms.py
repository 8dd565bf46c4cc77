"""The form that an 8-bit product takes (no GPU needed): each is the choice somewhere, and the sizes that the rule was measured at keep theirs."""
import pytest

from tests.int8_util import INT8_FORMS, int8_form

CHOICES = [((1, 61440, 5), "few rows"), ((1, 61441, 5), "32, shared k"), ((2, 30720, 5), "few rows"), ((2, 30721, 5), "32, shared k"), ((2, 3072, 12288), "few rows"),
           ((3, 3072, 12288), "32, shared k"), ((128, 12288, 3072), "32, shared k"), ((256, 12288, 3072), "64, shared k"), ((512, 4096, 4096), "64"),
           ((300, 2000, 4000), "64"), ((333, 3072, 9216), "128"), ((1280, 12288, 3072), "128"), ((1280, 3072, 9216), "256 x 192"), ((20480, 3072, 12288), "256 x 256")]


@pytest.mark.parametrize("size,want", CHOICES)
def test_forms_by_size(size, want):
    assert int8_form(*size) == want


def test_every_form_is_the_choice_somewhere():
    assert {w for _, w in CHOICES} == set(INT8_FORMS)
