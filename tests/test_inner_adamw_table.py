"""AdamW's tensor table: what does not describe every element is refused, before any device call."""
import pytest


@pytest.fixture(scope="module")
def inner():
    import __graft_entry__ as g
    g.build()
    from paper_2508_15706_b200 import inner
    return inner


@pytest.mark.parametrize("shapes", [[(2, 3, 4)], [(8, 8), (2, 3, 4)], [()], [(4,), (1, 1, 4)]])
def test_shapes_that_are_no_matrix_are_refused(inner, shapes):
    """Only the first two of three dimensions would be updated otherwise."""
    from paper_2508_15706_b200.binding import SL_ERR_INVALID_ARG, SlError
    with pytest.raises(SlError) as e:
        inner.AdamW(shapes)
    assert e.value.status == SL_ERR_INVALID_ARG and "[rows, cols] or a vector" in str(e.value)


@pytest.mark.parametrize("offsets", [[], [0], [0, 16, 32]])
def test_offsets_of_another_number_are_refused(inner, offsets):
    from paper_2508_15706_b200.binding import SL_ERR_INVALID_ARG, SlError
    with pytest.raises(SlError) as e:
        inner.AdamW([(4, 4), (4,)], offsets)
    assert e.value.status == SL_ERR_INVALID_ARG and "offsets for 2 tensors" in str(e.value)
