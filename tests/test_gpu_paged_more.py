"""The cases of paged_more on the GPU, checked as test_gpu_paged checks its own."""
import pytest

import paged_more as more
import test_gpu_paged as t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("c", more.ROWS, ids=range(len(more.ROWS)))
def test_rows_are_transformed_and_find_their_pages(c):
    t.test_rows_are_transformed_and_find_their_pages(c)


@pytest.mark.parametrize("c", more.MANY, ids=range(len(more.MANY)))
def test_attention_over_pages(c):
    t.test_attention_over_pages(c)


@pytest.mark.parametrize("kind", ["bad_pages", "beyond", "masked_infinity", "masked_nan", "one_component"])
@pytest.mark.parametrize("c", [more.MANY[0], more.MANY[1], more.MANY[5], more.MANY[7]], ids=range(4))
def test_what_is_not_seen_has_no_influence(c, kind):
    t.test_what_is_not_seen_has_no_influence(c, kind)
