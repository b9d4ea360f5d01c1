"""What the windowed attention refuses, and what it takes, without a GPU."""
import pytest

from paper_2512_23049_amd import binding as b
from pc_inputs import Call


@pytest.fixture
def cache():
    c = b.Cache(8, 2, 128, b.PC_BF16, 10000.0, 1024, 8, max_position=5000, flags=b.PC_FLAG_HOST_ONLY)
    c.append_message(0, 0, 40)
    c.append_message(0, 0, 7)
    yield c
    c.close()


OK = Call([(0, 0)], 1, 40, 7, None)


@pytest.mark.parametrize("name", ["attend_window", "attend_window_static"])
@pytest.mark.parametrize("calls,window,n_sink,code", [
    ([OK], 0, 0, b.PC_ERR_INVALID_ARG), ([OK], -5, 0, b.PC_ERR_INVALID_ARG), ([OK], 5, -1, b.PC_ERR_INVALID_ARG), ([], 0, 0, b.PC_ERR_INVALID_ARG),
    ([Call([(3, 0)], 1, 40, 7, None)], 5, 0, b.PC_ERR_BAD_MSG_ID), ([Call([(0, 0)], 1, 40, 8, None)], 5, 0, b.PC_ERR_SHAPE),
    ([Call([(0, 4970)], 1, 40, 7, None)], 5, 0, b.PC_ERR_INVALID_ARG), ([OK, Call([(0, 0)], 9, 40, 7, None)], 5, 0, b.PC_ERR_BAD_MSG_ID)])
def test_refused(cache, name, calls, window, n_sink, code):
    with pytest.raises(b.PcError) as e:
        getattr(cache, name)(calls, window, n_sink, 0, 0)
    assert e.value.code == code and name in str(e.value) or "call" in str(e.value)


@pytest.mark.parametrize("name", ["attend_window", "attend_window_static"])
def test_taken(cache, name):
    getattr(cache, name)([OK], 1, 0, 0, 0)
    getattr(cache, name)([OK, OK], 2147483647, 2147483647, 0, 0)
    getattr(cache, name)([], 1, 0, 0, 0)
