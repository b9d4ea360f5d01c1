"""What the gradient of the windowed attention refuses, and what it takes, without a GPU."""
import pytest

from paper_2512_23049_amd import binding as b
from pc_inputs import Call
from tests.test_window_refusals import OK, cache  # noqa: F401


@pytest.mark.parametrize("calls,window,n_sink,code", [
    ([OK], 0, 0, b.PC_ERR_INVALID_ARG), ([OK], 5, -1, b.PC_ERR_INVALID_ARG), ([], 0, 0, b.PC_ERR_INVALID_ARG),
    ([Call([(3, 0)], 1, 40, 7, None)], 5, 0, b.PC_ERR_BAD_MSG_ID), ([Call([(0, 0)], 1, 40, 8, None)], 5, 0, b.PC_ERR_SHAPE)])
def test_refused(cache, calls, window, n_sink, code):  # noqa: F811
    with pytest.raises(b.PcError) as e:
        cache.attend_window_backward(calls, window, n_sink, 0, 0, 0, 0, 0, 0, 0)
    assert e.value.code == code


def test_taken(cache):  # noqa: F811
    cache.attend_window_backward([OK, OK], 2147483647, 2147483647, 0, 0, 0, 0, 0, 0, 0)
    cache.attend_window_backward([], 1, 0, 0, 0, 0, 0, 0, 0, 0)
