"""Numbers that the C entry points' arguments cannot hold are refused by the extension, not cut to ones that they can."""
import pytest
import torch

from test_paged_calls import Library, attention, i32, reserve


@pytest.fixture()
def library():
    return Library()


@pytest.mark.parametrize("page", [2 ** 32 + 16, 2 ** 31, -2 ** 32 + 16])
def test_tokens_of_a_page(library, page):
    with pytest.raises(ValueError):
        library.calls.kv_pages_reserve(*reserve(page=page).values())
    with pytest.raises(ValueError):
        library.calls.kv_pages_free(i32(3, 5), i32(9), i32(3), page, None, -1, 0)
    for other in (2 ** 70, "sixteen", None, 16.5):
        with pytest.raises(TypeError):
            library.calls.kv_pages_free(i32(3, 5), i32(9), i32(3), other, None, -1, 0)
    assert not library.made


@pytest.mark.parametrize("shape", [(1, 2 ** 32 + 5), (2 ** 32 + 3, 5)])
def test_a_table_beyond_32_bits(library, shape):
    """(No memory behind it.)"""
    table = torch.empty(shape, dtype=torch.int32, device="meta")
    with pytest.raises(ValueError):
        library.calls.kv_pages_fork(table, i32(9), i32(3), i32(3), -1, 0)
    assert not library.made


def test_a_scale_that_float32_rounds_to_nothing(library):
    for scale in (1e-46, -1e-50):
        with pytest.raises(ValueError):
            library.calls.verify_attention_paged(*attention(scale=scale).values())
    assert not library.made
    assert library.calls.verify_attention_paged(*attention(scale=1e-44).values()) == 0 and library.made[0][0].scale > 0
