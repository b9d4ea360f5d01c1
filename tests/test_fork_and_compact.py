"""Forks and the cache closing up: bookkeeping and refusals, without a GPU."""
import numpy as np
import pytest

from paper_2512_23049_amd import binding as b

AUTO = None


def make(capacity=4096, messages=400, flags=0, max_position=10000):
    return b.Cache(8, 2, 128, b.PC_BF16, 10000.0, capacity, messages, max_position=max_position, flags=b.PC_FLAG_HOST_ONLY | flags)


def room(n):
    return (n + 31) // 32 * 32


def test_fork_takes_ids_lengths_slots_and_base():
    c = make()
    a = c.append_message(0, 0, 100, 120)
    c.reposition(a, 50)
    ids = c.message_fork([(a, 0, 100, 0, AUTO), (a, 33, 5, 64, AUTO), (a, 99, 1, 0, -700)])
    assert ids == [1, 2, 3]
    assert c.message_info(1) == (100, 128, 100) and c.message_info(2) == (5, 256, 64) and c.message_info(3) == (1, 320, 1)
    assert [c.message_base(m) for m in ids] == [50, 83, -700] and c.message_base(a) == 50
    c.append_tokens(2, 0, 0, 59)
    assert c.message_info(2)[0] == 64
    assert c.message_fork([]) == []
    c.close()


@pytest.mark.parametrize("fork,code", [
    ((5, 0, 1, 0, AUTO), b.PC_ERR_BAD_MSG_ID), ((-1, 0, 1, 0, AUTO), b.PC_ERR_BAD_MSG_ID), ((1, 0, 1, 0, AUTO), b.PC_ERR_BAD_MSG_ID), ((0, -1, 1, 0, AUTO), b.PC_ERR_INVALID_ARG),
    ((0, 0, 0, 0, AUTO), b.PC_ERR_INVALID_ARG), ((0, 0, 101, 0, AUTO), b.PC_ERR_INVALID_ARG), ((0, 100, 1, 0, AUTO), b.PC_ERR_INVALID_ARG),
    ((0, 2147483647, 2147483647, 0, AUTO), b.PC_ERR_INVALID_ARG), ((0, 0, 1, 0, 10001), b.PC_ERR_INVALID_ARG), ((0, 0, 1, 0, -10001), b.PC_ERR_INVALID_ARG),
    ((0, 0, 10, 5000, AUTO), b.PC_ERR_NO_SPACE), ((2, 5, 1, 0, AUTO), b.PC_ERR_INVALID_ARG)])
def test_a_refused_fork_changes_nothing(fork, code):
    c = make()
    c.append_message(0, 0, 100)
    c.append_message(0, 0, 10)
    c.append_message(0, 0, 20)
    c.message_free(1)
    c.reposition(2, 9996)                                # (token 5 is stored at 10001)
    before = c.cache_info()
    with pytest.raises(b.PcError) as e:
        c.message_fork([(0, 0, 10, 0, AUTO), fork])
    assert e.value.code == code and "fork 1" in str(e.value)
    assert c.cache_info() == before
    assert c.message_fork([(0, 0, 10, 0, AUTO)]) == [3] and c.message_info(3)[1] == 128        # the span that was freed
    c.close()


def test_a_full_table_refuses():
    c = make(messages=3)
    c.append_message(0, 0, 10)
    with pytest.raises(b.PcError) as e:
        c.message_fork([(0, 0, 1, 0, AUTO)] * 3)
    assert e.value.code == b.PC_ERR_NO_SPACE
    assert c.message_fork([(0, 0, 1, 0, AUTO)] * 2) == [1, 2]
    c.close()


def test_close_up():
    c = make()
    for n in (40, 10, 70, 33, 5):
        c.append_message(0, 0, n)
    assert c.compact() == 0
    c.message_free(0)
    c.message_free(3)
    assert c.compact() == 32 + 96 + 32
    assert [c.message_info(m)[1] for m in (1, 2, 4)] == [0, 32, 128]
    assert c.cache_info()[1] == 160
    assert c.compact() == 0
    c.message_free(4)
    assert c.cache_info()[1] == 128
    assert c.append_message(0, 0, 7) == 5 and c.message_info(5)[1] == 128
    c.close()


def test_close_up_a_little_at_a_time():
    c = make()
    for n in (32, 64, 96, 32, 160, 32):
        c.append_message(0, 0, n)
    c.message_free(0)
    c.message_free(3)
    assert c.compact(100) == 64                          # the next one, of 96, would be too much
    assert [c.message_info(m)[1] for m in (1, 2, 4, 5)] == [0, 96, 224, 384]
    assert c.append_message(0, 0, 30) == 6 and c.message_info(6)[1] == 64          # the gap has moved up
    assert c.compact(1) == 160                           # the first extent moves whatever its size
    assert c.compact(1) == 32
    assert [c.message_info(m)[1] for m in (1, 6, 2, 4, 5)] == [0, 64, 96, 192, 352]
    assert c.compact(1) == 0 and c.cache_info()[1] == 384
    with pytest.raises(b.PcError) as e:
        c.compact(-1)
    assert e.value.code == b.PC_ERR_INVALID_ARG
    c.close()


def test_what_does_not_fit_fits_behind():
    c = make(capacity=512)
    ids = [c.append_message(0, 0, 32) for _ in range(16)]
    for m in ids[::2]:
        c.message_free(m)
    with pytest.raises(b.PcError):
        c.append_message(0, 0, 200)
    c.compact()
    assert c.message_info(c.append_message(0, 0, 256))[1] == 256
    c.close()


@pytest.mark.parametrize("seed", range(4))
def test_random_programs(seed):
    """Appends, growth into extents, forks, frees and closing up, against a plain model: every live message's extents in slot
    order, none overlapping, all of them inside what is used."""
    r = np.random.default_rng(seed)
    c = make(capacity=8192, messages=4000, flags=b.PC_FLAG_GROW_EXTENTS)
    live = {}                                            # id -> (length, reserves by extent)
    for _ in range(400):
        what = r.integers(0, 6)
        try:
            if what <= 1:
                n, res = int(r.integers(1, 120)), int(r.integers(0, 200))
                m = c.append_message(0, 0, n, res)
                live[m] = n
            elif what == 2 and live:
                m = int(r.choice(list(live)))
                n = int(r.integers(1, 90))
                c.append_tokens(m, 0, 0, n)
                live[m] += n
            elif what == 3 and live:
                m = int(r.choice(list(live)))
                first = int(r.integers(0, live[m]))
                n = int(r.integers(1, live[m] - first + 1))
                f, = c.message_fork([(m, first, n, int(r.integers(0, 100)), AUTO)])
                live[f] = n
            elif what == 4 and live:
                m = int(r.choice(list(live)))
                c.message_free(m)
                del live[m]
            elif what == 5:
                before = sorted((c.message_extents(m)[0][0], m) for m in live)
                c.compact(int(r.choice([0, 0, 100, 1000])))
                assert [m for _, m in before] == [m for _, m in sorted((c.message_extents(m)[0][0], m) for m in live)]
        except b.PcError as e:
            assert e.code == b.PC_ERR_NO_SPACE
        spans, used = [], c.cache_info()[1]
        for m, n in live.items():
            ext = c.message_extents(m)
            assert c.message_info(m)[0] == n == sum(length for _, length in ext)
            spans += [(s, s + max(room(length), 32)) for s, length in ext]
        spans.sort()
        assert all(a[1] <= z[0] for a, z in zip(spans, spans[1:])) and (not spans or spans[-1][1] <= used)
    while c.compact(500) > 0:
        pass
    spans = sorted(s for m in live for s, _ in c.message_extents(m))
    assert not spans or spans[0] == 0
    c.close()
