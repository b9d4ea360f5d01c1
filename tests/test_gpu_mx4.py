"""Attention over PC_MX4 caches against fp64 on the values held: head layouts, rows, windows, masks that leave a row empty, lists of every kind,
splits, recorded and replayed calls, long caches, tokens of no number, messages that grow, fork, move and swap."""
import numpy as np
import pytest

from oracle import project_oracle as po
from tests.project_cases import THETA, Layer4, Rows, cache_of, same
from tests.window_cases import say

pytestmark = pytest.mark.gpu

HEADS = [(4, 4), (8, 2), (32, 2), (6, 2), (5, 1), (64, 8)]
LENS = [31, 1, 64, 33, 100, 90]
SEL = [(0, 0), (4, 40), (1, 7), (2, 300), (0, 500), (3, 140)]


@pytest.mark.parametrize("h_q,h_kv", HEADS)
@pytest.mark.parametrize("n_q", [1, 2, 33, 90])
def test_heads_rows_and_windows(h_q, h_kv, n_q):
    layer = Layer4(LENS, h_q, h_kv)
    for window, n_sink in [(0, 0), (1, 0), (2, 1), (31, 0), (33, 32), (64, 33), (400, 0), (2147483647, 3), (5, 1 << 30)]:
        layer.run([(SEL, 5, 600, n_q)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("h_q,h_kv", HEADS)
def test_rows_over_a_copy(h_q, h_kv):
    """Every prefill call over a copy of what it lists (the caller's word), with single tokens, short and empty calls among them; and none of them."""
    layer = Layer4(LENS, h_q, h_kv)
    calls = [(SEL, 5, 600, 90), ([], 5, 0, 90), (SEL, 5, 600, 1), (SEL[2:], 3, 300, 33), ([], -1, 5, 70), (SEL[:1], -1, 40, 65, [-7 * i for i in range(65)]), (SEL, 4, -10 ** 6, 17)]
    for mode in (2, 1, 0):
        layer.cache.set_key_gather(mode)
        layer.run(calls, what=f"mode {mode}")
        for n_q in (2, 5, 18, 32, 64, 90):
            layer.run([(SEL, 5, 600, n_q)], what=f"mode {mode} rows {n_q}")
    layer.cache.close()


def test_tuned_and_timed():
    """The same calls in splits of the caller's length, with kernels timed: rows over the cache and over a copy, tokens."""
    layer = Layer4(LENS, 8, 2)
    calls = [(SEL, 5, 600, 90), (SEL, 5, 600, 1), (SEL[::-1], 4, 500, 100)]
    for tiles, gather in ((0, 2), (1, 2), (3, 2), (1, 1)):
        layer.cache.set_tuning(tiles, tiles)
        layer.cache.set_key_gather(gather)
        layer.cache.profile_enable(True)
        layer.run(calls, what=f"splits of {tiles} gather {gather}")
        of = list(layer.cache.profile_read().values())   # (by class: 2 rows, 3 tokens, 8 copies)
        layer.cache.profile_enable(False)
        assert of[2][1] >= 1 and of[3][1] >= 1 and of[8][1] == (2 if gather == 2 else 0)
        assert sum(ms for ms, _ in of) > 0
    layer.cache.close()


@pytest.mark.parametrize("h_q,h_kv", [(8, 2), (4, 4)])
@pytest.mark.parametrize("static", [False, True])
def test_batches(h_q, h_kv, static):
    """One row and many side by side; calls that see nothing, without a new message, with their own tokens alone; a message twice; positions
    stated, negative, repeated; a window behind every key."""
    lens = [int(x) for x in np.random.default_rng(3).integers(20, 300, size=12)] + [20, 70, 1]
    layer = Layer4(lens, h_q, h_kv)
    long = [(m, 300 * m) for m in range(12)]
    calls = [(long, 14, 3700, 1), (long[::-1], 13, 100, 70), ([(0, 5)], -1, 0, 3, [900, 5, 700]), ([], 12, 0, 20), ([(0, -5000)], -1, 9000, 1),
             ([(3, 50), (3, 50)], 13, 80, 40), (long[:3], -1, 0, 5, [-40, 3, 3, 10 ** 6, 90]), ([], -1, 7, 2), ([], 14, 0, 1), (long, -1, 2000, 1), ([], -1, 3, 1)]
    for window, n_sink in [(0, 0), (50, 0), (333, 7), (4000, 500)]:
        layer.run(calls, window, n_sink, static)
    layer.cache.close()


@pytest.mark.parametrize("calls_n", [1, 3, 17, 40])
def test_parallel_single_tokens(calls_n):
    """Calls that list the same messages and some of their own, in each its order; the same calls give the same bits."""
    rng = np.random.default_rng(calls_n)
    lens = [700] + [int(x) for x in rng.integers(1, 400, size=20)] + [int(x) for x in rng.integers(1, 70, size=calls_n)]
    layer = Layer4(lens, 16, 2)
    calls = []
    for i in range(calls_n):
        sel, at = [(0, 0)], 700
        for m in rng.permutation(20)[:8] + 1:
            sel.append((int(m), at + int(rng.integers(-5, 20))))
            at += lens[m]
        calls.append((sel, 21 + i, at, 1))
    q = layer.normal(calls_n, 16, 128)
    for window, n_sink in [(0, 0), (900, 4)]:
        a = layer.run(calls, window, n_sink, q=q)
        b = layer.attend(calls, q, window, n_sink)
        assert layer.torch.equal(a[0], b[0]) and layer.torch.equal(a[1], b[1])
    layer.cache.close()


@pytest.mark.parametrize("mode", [1, 2])
def test_sharing_as_the_caller_says(mode):
    layer = Layer4([200, 64, 100, 40, 40, 40], 8, 2)
    layer.cache.set_decode_sharing(mode)
    calls = [([(0, 0), (1, 200 + 7 * i)], 3 + i, 400, 1) for i in range(3)] + [([(2, 10), (0, 130)], -1, 500, 1), ([(0, 0), (0, 300)], -1, 900, 1)]
    for window, n_sink in [(0, 0), (120, 3)]:
        layer.run(calls, window, n_sink)
        layer.run(calls[:3], window, n_sink)
    layer.cache.close()


def test_large_scores_and_powers():
    """Keys and values over forty orders of magnitude: scores of some thousands, values whose powers differ by 2^100 from token to token; rows that
    see the large ones alone, and the small ones alone."""
    def spoil(i, k, v):
        if i == 1:
            v *= np.float32(2.0) ** 50
        if i == 2:
            v *= np.float32(2.0) ** -50
        if i == 3:
            k *= 300
    layer = Layer4([64, 64, 64, 64], 8, 2, spoil=spoil)
    for n_q in (1, 40):
        q = layer.normal(n_q, 8, 128)
        for m in (1, 2):
            out, lse = layer.attend([([(m, 0)], -1, 64, n_q)], q)
            want, want_lse = layer.want([([(m, 0)], -1, 64, n_q)], q)
            unit = 2.0 ** 50 if m == 1 else 2.0 ** -50
            same(out.double() / unit, lse, want / unit, want_lse, f"values by {unit}")
        # scores of some thousands: a turned query's values are off by 2^-8 of themselves at most, a score then by 2^-8 sum |q_i k_i| / sqrt(128), at most
        # 2^-8 |q| |k| / sqrt(128) (a turn keeps the norms), and a log-sum-exp by no more than its scores; 1e-6 of the same for sums in 32 bits
        call = [([(3, 0)], -1, 64, n_q)]
        out, lse = layer.attend(call, q)
        want, want_lse = layer.want(call, q)
        size = np.linalg.norm(q, axis=-1) * np.repeat(np.linalg.norm(layer.ks[3], axis=-1).max(axis=0), 4) / np.sqrt(128)
        assert (np.abs(lse.double().cpu().numpy() - want_lse) <= (2.0 ** -8 + 1e-6) * size).all()
        assert np.abs(want_lse).max() > 500
    layer.cache.close()


@pytest.mark.parametrize("spoilt", ["", "keys", "query", "no number"])
def test_many_rows_over_long_lists(spoilt):
    """Calls of 1.3e8 scores among short ones, with a message twice, one of a single token, parts of messages grown and placed at odd positions; and keys
    and queries outside what 16 bits hold, or none at all, which any call may have."""

    def spoil(i, k, v):
        if spoilt == "keys" and i == 1:
            k[5] *= 1e6
        if spoilt == "no number" and i == 1:
            v[5, 0, 3] = np.nan
    from paper_2512_23049_amd import binding as b
    lens = [1900, 33, 2500, 1, 1030, 70, 1100, 1099, 40]
    layer = Layer4(lens, 16, 2, spoil=spoil)
    long = [(0, 0), (4, 2000), (2, 3007), (3, 9000), (5, 5600), (0, 5700)]
    calls = [([(0, 3)], 8, 1950, 40), (long, 6, 8000, 1100), (long[:3], -1, 7000, 1), (long + [(1, -70)], 7, 8100, 1000), (long, 7, 8000, 1001), ([], 8, 0, 1)]
    q = layer.normal(sum(c[3] for c in calls), 16, 128)
    if spoilt == "query":
        q[40 + 1100 + 1 + 7] *= 3e4
    if spoilt in ("keys", "query"):
        out, lse = layer.attend(calls, q)
        want, want_lse = layer.want(calls, q)
        # rows that see a large key, or are large: one key takes all, or two near each other do; a score is off by 2^-8 |q| |k| / sqrt(128)
        far = np.abs(want_lse) > 60
        assert far.any() and (far.sum(axis=1) == 0).sum() > 2000
        rows = ~far.any(axis=1)
        same(out[rows], lse[rows], want[rows], want_lse[rows], spoilt)
        assert out.isfinite().all()
        top = 1e6 * 20 if spoilt == "keys" else 20.0
        norm = np.linalg.norm(q, axis=-1)
        assert (np.abs(lse.double().cpu().numpy() - want_lse)[far] <= (2.0 ** -8 + 1e-6) * (norm * top / np.sqrt(128))[far] + 1e-3).all()
        # where the large key's score is below all others it is not seen; it comes within its own error of them, 2^-8 x 11 deviations, in 4 rows of 100
        off = np.abs(out.double().cpu().numpy() - want).max(axis=-1)[~far] > 4e-2
        assert off.mean() < 0.05
        return
    if spoilt:
        out, lse = layer.attend(calls, q)
        rows = np.zeros(len(q), bool)
        rows[1141:2141] = True                           # (the call that lists it)
        assert out[rows][:, :8].isnan().all() and out[rows][:, 8:].isfinite().all()
        layer.ks[1][np.isnan(layer.ks[1])] = 0
        layer.vs[1][np.isnan(layer.vs[1])] = 0
        want, want_lse = layer.want(calls, q)
        same(out[~rows], lse[~rows], want[~rows], want_lse[~rows], "the others")
        same(out[rows][:, 8:], lse[rows][:, 8:], want[rows][:, 8:], want_lse[rows][:, 8:], "the other head")
        return
    out, _ = layer.run(calls, q=q)
    tq = layer.dev(q)
    again = layer.torch.full_like(tq, 7.0)
    layer.cache.attend(layer.calls(calls), tq.data_ptr(), again.data_ptr())              # (no sums asked for; the same bits)
    layer.torch.cuda.synchronize()
    assert layer.torch.equal(again, out)
    for q_ptr, out_ptr in ((0, again.data_ptr()), (tq.data_ptr(), 0), (tq.data_ptr() + 2, again.data_ptr())):
        with pytest.raises(b.PcError):
            layer.cache.attend(layer.calls(calls), q_ptr, out_ptr)
    layer.cache.close()


def test_queries_that_are_no_numbers():
    """A row's head whose query holds a NaN or an infinity is NaN, and no other is touched: tokens on their own and shared, rows, rows over a copy."""
    layer = Layer4([300, 90, 40, 40, 40, 40], 16, 2)
    sel = [(0, 0), (1, 310)]
    tokens, rows = [(sel, 2 + i, 400, 1) for i in range(4)], [(sel, 2, 400, 40), (sel[::-1], 3, 420, 33)]
    for calls, sharing, gather in ((tokens, 1, 0), (tokens, 2, 0), (rows, 0, 1), (rows, 0, 2)):
        layer.cache.set_decode_sharing(sharing)
        layer.cache.set_key_gather(gather)
        n = sum(c[3] for c in calls)
        q = layer.normal(n, 16, 128)
        spoilt = q.copy()
        bad = np.zeros((n, 16), bool)
        for r, h, d, x in ((0, 3, 5, np.nan), (1, 9, 127, np.inf), (n - 1, 15, 64, -np.inf), (n - 2, 0, 0, np.nan)):
            spoilt[r, h, d], bad[r, h] = x, True
        out, lse = layer.attend(calls, spoilt)
        want, want_lse = layer.want(calls, q)
        assert out[layer.torch.from_numpy(bad)].isnan().all()
        same(out[layer.torch.from_numpy(~bad)], lse[layer.torch.from_numpy(~bad)], want[~bad], want_lse[~bad], f"sharing {sharing} gather {gather}")
    layer.cache.close()


def test_windows_that_leave_all():
    """Rows whose window reaches just to the first token that they list, and one short of it; positions that a call states, sinks, messages in front."""
    layer = Layer4([100, 90, 200, 70], 16, 2)
    layer.cache.set_key_gather(2)
    sel = [(0, 0), (1, 130)]
    for window in (299, 300, 301, 369, 370, 371, 1 << 20, 2147483647):
        # rows at 300 to 369: the last sees all from a window of 370 on
        layer.run([(sel, 3, 300, 70)], window, 0)
        layer.run([(sel, 3, 300, 70), (sel, -1, 300, 1), (sel, 2, -50, 200), (sel[:1], -1, 0, 40, [100 + 5 * i for i in range(40)])], window, 3)
    layer.cache.close()


@pytest.mark.parametrize("powers", [(13, -11), (14, 0), (0, -16), (40, -40)])
def test_values_inside_and_outside_fp16(powers):
    """Values by powers of two that fp16 holds, and that it does not, for single tokens that share their messages and for rows, short and long: each sees
    those of one power alone, with scores from near zero to some tens, and long lists of keys of small probabilities beside one of a large one."""
    up, down = powers

    def spoil(i, k, v):
        v *= np.float32(2.0) ** {1: up - 2, 2: down}.get(i, 0)       # (normal values: blocks of 32 have exponents of 0 or 1 below theirs)
        if i == 3:
            k[::40] *= 6
    layer = Layer4([300, 300, 300, 1500, 20, 20, 20, 20], 16, 2, spoil=spoil)
    layer.cache.set_decode_sharing(2)
    for m, power in ((0, 0), (1, up - 2), (2, down), (3, 0)):
        unit = 2.0 ** power
        for calls in ([([(m, 5 * i)], -1, 300 + i, 1) for i in range(4)], [([(m, 0)], -1, 400, 50), ([(m, 7)], -1, 200, 3)]):
            q = layer.normal(sum(c[3] for c in calls), 16, 128)
            out, lse = layer.attend(calls, q)
            want, want_lse = layer.want(calls, q)
            same(out.double() / unit, lse, want / unit, want_lse, f"values by {unit}") if m != 3 else None
            if m == 3:                                   # (scores of some tens: errors by their size, 2^-8 |q| |k| / sqrt(128), as far as one key takes all)
                size = np.linalg.norm(q, axis=-1) * np.linalg.norm(layer.ks[3], axis=-1).max() / np.sqrt(128)
                assert (np.abs(lse.double().cpu().numpy() - want_lse) <= (2.0 ** -8 + 1e-6) * size).all()
                assert out.isfinite().all()
            layer.cache.set_key_gather(2)
            if calls[0][3] > 1 and m != 3:
                out, lse = layer.attend(calls, q)
                same(out.double() / unit, lse, want / unit, want_lse, f"values by {unit}, copied")
            layer.cache.set_key_gather(0)
    layer.run([([(0, 3 * i)], 4 + i, 320, 1) for i in range(4)], what="with tails")
    layer.cache.close()


@pytest.mark.parametrize("n_q", [1, 5, 40])
def test_tokens_that_are_no_numbers(n_q):
    """Rows that see one are NaN in that head's query heads; what others do not see does not touch them."""
    def spoil(i, k, v):
        if i == 1:
            k[3, 0, 5], v[40, 1, 100] = np.inf, np.nan
    layer = Layer4([64, 50, 64], 8, 2, spoil=spoil)
    q = layer.normal(n_q, 8, 128)
    out, _ = layer.attend([([(0, 0), (1, 64)], 2, 114, n_q)], q)
    assert out.isnan().all()
    # a window that leaves both out, and one that leaves the first out: head 1 sees the second
    calls = [([(1, 0), (0, 50)], 2, 114, n_q)]
    layer.ks[1][np.isnan(layer.ks[1])] = 0               # (not seen)
    for window in (60, 70):
        out, lse = layer.attend(calls, q, window)
        want, want_lse = layer.want(calls, q, window)
        same(out, lse, want, want_lse, f"window {window}")
    first = 114 + 64 - n_q                               # position of the first row
    window = first - 40 + 1                              # it sees positions from 40 on, the others from later on
    out, lse = layer.attend(calls, q, window)
    want, want_lse = layer.want(calls, q, window)
    assert out[0, 4:].isnan().all() and out[0, :4].isfinite().all()
    if n_q > 1:
        same(out[1:], lse[1:], want[1:], want_lse[1:], "the others")
    layer.cache.close()


def test_recorded_and_replayed():
    """A step of single tokens and a prefill recorded into one graph, replayed on other queries with eager work and waits between."""
    torch = __import__("torch")
    layer = Layer4([300, 64, 200, 40, 70], 8, 2)
    calls = [([(0, 0), (2, 300)], 3, 500, 1), ([(1, 0), (0, 90)], 4, 400, 70), ([(0, 5)], -1, 700, 1)]
    q = layer.normal(72, 8, 128)
    tq = layer.dev(q)
    out, lse = torch.zeros_like(tq), torch.zeros(72, 8, device="cuda:0")
    out2, lse2 = torch.zeros_like(tq), torch.zeros(72, 8, device="cuda:0")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    cs = layer.calls(calls)
    with torch.cuda.graph(graph, stream=s):
        st = torch.cuda.current_stream().cuda_stream
        layer.cache.attend_static(cs, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), st)
        layer.cache.attend_window_static(cs, 90, 4, tq.data_ptr(), out2.data_ptr(), lse2.data_ptr(), st)
        with pytest.raises(Exception, match="captured"):
            layer.cache.attend(cs, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), st)
    for step in range(4):
        q = layer.normal(72, 8, 128)
        tq.copy_(layer.dev(q))
        out.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        same(out, lse, *layer.want(calls, q), f"replay {step}")
        same(out2, lse2, *layer.want(calls, q, 90, 4), f"replay {step}, window")
        layer.run(calls[:2])                             # (eager work between the replays)
    layer.cache.close()


def test_what_is_not_recorded():
    """A decode step, and what brings long lists, is refused on a stream that is being captured, before the books change."""
    from paper_2512_23049_amd import binding as b
    torch = __import__("torch")
    layer = Layer4([40, 33, 64] + [1] * 200, 8, 2, reserves=[64, 64, 64] + [32] * 200)
    k = layer.dev(layer.normal(300, 2, 128))
    q = layer.dev(layer.normal(1, 8, 128))
    out = torch.zeros_like(q)
    call = layer.calls([([(0, 0)], 1, 40, 1)])
    layer.cache.attend(call, q.data_ptr(), out.data_ptr())
    before = [layer.cache.message_info(i) for i in layer.ids]
    s = torch.cuda.Stream()
    with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
        st = torch.cuda.current_stream().cuda_stream
        out.zero_()
        with pytest.raises(b.PcError):
            layer.cache.decode_step([layer.ids[1]], k.data_ptr(), k.data_ptr(), call, q.data_ptr(), out.data_ptr(), stream=st)
        with pytest.raises(b.PcError):
            layer.cache.append_tokens_batch(layer.ids[3:], k.data_ptr(), k.data_ptr(), stream=st)
        with pytest.raises(b.PcError):
            layer.cache.messages_read(layer.ids, k.data_ptr(), k.data_ptr(), stream=st)
    torch.cuda.synchronize()
    assert [layer.cache.message_info(i) for i in layer.ids] == before
    layer.run([([(0, 0), (2, 50)], 1, 140, 1)], what="behind it")
    layer.cache.close()


def test_recorded_long_lists():
    """Lists that neither arguments nor a slot hold are recorded with the call."""
    torch = __import__("torch")
    rng = np.random.default_rng(6)
    lens = [int(x) for x in rng.integers(1, 60, size=120)] + [40]
    layer = Layer4(lens, 8, 2)
    calls = [([(int(m), 70 * j) for j, m in enumerate(rng.permutation(120)[:90])], -1, 6500, 1) for _ in range(6)] + [([(m, 60 * m) for m in range(60)], 120, 4000, 40)]
    q = layer.normal(46, 8, 128)
    tq, cs = layer.dev(q), layer.calls(calls)
    out, lse = torch.zeros_like(tq), torch.zeros(46, 8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        layer.cache.attend_static(cs, tq.data_ptr(), out.data_ptr(), lse.data_ptr(), torch.cuda.current_stream().cuda_stream)
    want = layer.want(calls, q)
    for _ in range(3):
        out.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        same(out, lse, *want, "replay")
        layer.run(calls[:1])
    layer.run(calls)
    layer.cache.close()


def test_static_refuses_what_does_not_fit():
    from paper_2512_23049_amd import binding as b
    layer = Layer4([20000, 40], 64, 8)
    q = layer.normal(40, 64, 128)
    with pytest.raises(b.PcError) as e:
        layer.attend([([(0, 0)], 1, 20000, 40)], q, static=True)
    assert e.value.code == b.PC_ERR_NO_SPACE
    layer.run([([(0, 0)], 1, 20000, 40)], q=q)
    layer.run([([(0, 0)], 1, 20000, 1)], static=True)
    layer.cache.close()


def test_growth_forks_moves_and_swaps():
    """A generation over a 4-bit cache: tokens join, the line is forked in its middle, its oldest message leaves, the cache closes up, a message is away for
    a while; what is attended to is always what was appended."""
    from paper_2512_23049_amd import binding as b
    torch = __import__("torch")
    layer = Layer4([100, 70, 45, 33], 8, 2, reserves=[100, 70, 64, 40], flags=b.PC_FLAG_GROW_EXTENTS, room=600)
    for step in range(9):                                # (the last message outgrows its reserve)
        k, v, q = layer.normal(2, 2, 128), layer.normal(2, 2, 128), layer.normal(2, 8, 128)
        tk, tv, tq = layer.dev(k), layer.dev(v), layer.dev(q)
        out, lse = torch.zeros_like(tq), torch.zeros(2, 8, device="cuda:0")
        layer.grow(2, k[:1], v[:1])
        layer.grow(3, k[1:], v[1:])
        calls = [([(0, 0), (1, 90)], 2, 200, 1), ([(1, 0)], 3, 70, 1)]
        layer.cache.decode_step([layer.ids[2], layer.ids[3]], tk.data_ptr(), tv.data_ptr(), layer.calls(calls), tq.data_ptr(), out.data_ptr(), lse.data_ptr())
        torch.cuda.synchronize()
        same(out, lse, *layer.want(calls, q), f"step {step}")
    assert len(layer.cache.message_extents(layer.ids[3])) == 2
    forks = [(3, 5, 37), (3, 13, 20), (2, 0, 54), (0, 33, 1)]
    ids = layer.cache.message_fork([(layer.ids[m], first, n, n + 3, None) for m, first, n in forks])
    for (m, first, n), new in zip(forks, ids):           # (a fork's keys stay turned as they are: base first)
        layer.ids.append(new)
        layer.raw.append(tuple(x[first:first + n] for x in layer.raw[m]))
        layer.ks.append(layer.ks[m][first:first + n].copy())
        layer.vs.append(layer.vs[m][first:first + n].copy())
    calls = [([(0, 0), (4, 100), (5, 150)], 6, 300, 1), ([(7, 5), (2, 9)], 5, 200, 20)]
    layer.run(calls, what="forks")
    k, v = layer.normal(1, 2, 128), layer.normal(1, 2, 128)
    tk, tv = layer.dev(k), layer.dev(v)
    layer.cache.append_tokens(layer.ids[5], tk.data_ptr(), tv.data_ptr(), 1)
    torch.cuda.synchronize()
    at = 13 + 20                                         # (turned to base + index)
    from oracle.choreo_oracle import rope
    layer.ks[5] = np.concatenate([layer.ks[5], rope(po.to_mx4(rope(k.astype(np.float64), np.array([at]), THETA)), -np.array([at]), THETA)])
    layer.vs[5] = np.concatenate([layer.vs[5], po.to_mx4(v)])
    layer.run([([(0, 0)], 5, 300, 21)], what="a fork that grew")
    blob = torch.empty(layer.cache.message_swap_bytes(layer.ids[1]), dtype=torch.uint8).pin_memory()
    layer.cache.message_swap_out(layer.ids[1], blob.data_ptr())
    layer.cache.message_free(layer.ids[0])
    assert layer.cache.compact() > 0
    calls = [([(4, 100), (5, 150), (2, 20)], 6, 300, 1), ([(7, 5), (2, 9)], 3, 200, 2)]
    layer.run(calls, what="closed up")
    layer.cache.message_swap_in(layer.ids[1], blob.data_ptr())
    layer.run([([(1, 0), (4, 100)], 3, 300, 2), ([(1, 40)], 2, 120, 30)], 45, 2, what="back")
    layer.cache.close()


def test_many_rows_over_grown_and_forked_messages():
    """Rows of a long prefill over a message of several extents, one that grew in its last tile, forks from their middles on, and behind a compaction."""
    from paper_2512_23049_amd import binding as b
    layer = Layer4([1500, 70, 45, 512], 32, 2, reserves=[1500, 70, 64, 512], flags=b.PC_FLAG_GROW_EXTENTS, room=3000)
    for n in (9, 1, 40):
        for m in (1, 2):
            k, v = layer.normal(n, 2, 128), layer.normal(n, 2, 128)
            tk, tv = layer.dev(k), layer.dev(v)
            layer.cache.append_tokens(layer.ids[m], tk.data_ptr(), tv.data_ptr(), n)
            layer.torch.cuda.synchronize()
            layer.grow(m, k, v)
    assert len(layer.cache.message_extents(layer.ids[1])) > 1
    for m, first, n in [(0, 333, 777), (1, 65, 50)]:
        layer.ids += layer.cache.message_fork([(layer.ids[m], first, n, n, None)])
        layer.raw.append(tuple(x[first:first + n] for x in layer.raw[m]))
        layer.ks.append(layer.ks[m][first:first + n].copy())
        layer.vs.append(layer.vs[m][first:first + n].copy())
    sel = [(1, 5), (0, 100), (4, 1500), (5, 2300), (2, 2301)]
    layer.run([(sel, 3, 2500, 500), ([(0, 0)], -1, 1500, 2), (sel[::-1], 3, 2600, 512), (sel[1:], 3, 2000, 1)], what="grown")
    layer.cache.message_free(layer.ids[4])
    assert layer.cache.compact() > 0
    layer.run([(sel[:2] + sel[3:], 3, 2500, 512), (sel[:2] + [(0, 1700)], 3, 2500, 511)], what="closed up")
    layer.cache.close()


def test_many_moves():
    """Closing up over many messages, in steps and at once: chunks of tiles that do not end with a message."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(1, 260, size=60)]
    layer = Layer4(lens, 4, 4)
    for m in range(0, 60, 3):
        layer.cache.message_free(layer.ids[m])
    while layer.cache.compact(1000) > 0:
        pass
    keep = [m for m in range(60) if m % 3]
    layer.run([([(m, 50 * m) for m in keep], -1, 6000, 1), ([(m, 50 * m) for m in keep[::2]], -1, 5000, 9)], what="moved")
    layer.cache.close()


def test_offsets_past_32_bits():
    """A cache whose stores are 2.3 GB each: messages at its end."""
    from paper_2512_23049_amd import binding as b
    torch = __import__("torch")
    H, cap = 8, 4 << 20
    c = b.Cache(16, H, 128, b.PC_MX4, THETA, cap + 64, 16)
    rng = np.random.default_rng(2)

    def normal(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)
    front = normal(32, H, 128).to("cuda:0")
    c.append_message(front.data_ptr(), front.data_ptr(), 32, cap - 320)
    ks, vs, ids = [], [], []
    for n in (100, 90, 70):
        k, v = normal(n, H, 128), normal(n, H, 128)
        dk, dv = k.to("cuda:0"), v.to("cuda:0")
        ids.append(c.append_message(dk.data_ptr(), dv.data_ptr(), n))
        torch.cuda.synchronize()
        a, e = po.held(k.double().numpy(), v.double().numpy(), THETA)
        ks.append(a)
        vs.append(e)
    assert c.message_info(ids[0])[1] * H * 68 > 1 << 31 and (cap * 7 + c.message_info(ids[0])[1]) * 68 > 1 << 31
    from oracle import window_oracle as win
    from pc_inputs import Call
    for n_q in (1, 70):
        q = normal(n_q, 16, 128)
        tq = q.to("cuda:0")
        out, lse = torch.zeros_like(tq), torch.zeros(n_q, 16, device="cuda:0")
        c.attend([Call([(ids[0], 0), (ids[1], 100)], ids[2], 200, n_q, None)], tq.data_ptr(), out.data_ptr(), lse.data_ptr())
        torch.cuda.synchronize()
        same(out, lse, *win.attend_call_window(ks, vs, [(0, 0), (1, 100)], 2, 200, n_q, None, q.double().numpy(), THETA, 1 << 40, 0), f"{n_q} rows")
    k, v = (torch.zeros(260, H, 128, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    c.messages_read(ids, k.data_ptr(), v.data_ptr())
    assert np.array_equal(v.double().cpu().numpy(), np.concatenate(vs))
    c.close()


@pytest.mark.parametrize("rows_n", [1, 64])
def test_a_projected_layer_over_four_bits(rows_n):
    """As in serving: projected rows join a 4-bit cache, and attend over it with the queries that came out."""
    torch = __import__("torch")
    from oracle import window_oracle as win
    from pc_inputs import Call
    h_q, h_kv = 8, 2
    c = cache_of("mx4", h_q, h_kv, 128, 1024)
    old = Rows("mx4", 150, h_q, h_kv, 128, seed=1, queries=False)
    parents = c.append_projected(old.c, [100, 50], 0)
    rows = Rows("mx4", rows_n, h_q, h_kv, 128, seed=2)
    me, = c.append_projected(rows.c, [rows_n], rows.out_ptr, [rows_n + 8])
    out, lse = torch.empty_like(rows.q_out), torch.empty(rows_n, h_q, device="cuda:0")
    c.attend([Call([(parents[1], 0), (parents[0], 60)], me, 170, rows_n, None)], rows.q_out.data_ptr(), out.data_ptr(), lse.data_ptr())
    torch.cuda.synchronize()
    held = [po.held(r.k[a:b], r.v[a:b], THETA, r.kw, r.eps) for r, a, b in ((old, 0, 100), (old, 100, 150), (rows, 0, rows_n))]
    ks, vs = [x[0] for x in held], [x[1] for x in held]
    q = rows.q_out.double().cpu().numpy()
    same(out, lse, *win.attend_call_window(ks, vs, [(1, 0), (0, 60)], 2, 170, rows_n, None, q, THETA, 1 << 40, 0), "prefill")
    more = Rows("mx4", 1, h_q, h_kv, 128, seed=5)        # and the next token
    c.append_projected_tokens(more.c, [me], more.out_ptr)
    out, lse = torch.empty_like(more.q_out), torch.empty(1, h_q, device="cuda:0")
    c.attend([Call([(parents[1], 0), (parents[0], 60)], me, 170, 1, None)], more.q_out.data_ptr(), out.data_ptr(), lse.data_ptr())
    torch.cuda.synchronize()
    k, v = np.concatenate([rows.k, more.k]), np.concatenate([rows.v, more.v])
    ks[2], vs[2] = po.held(k, v, THETA, None, None)
    normed = np.concatenate([po.norm(rows.k, rows.kw, rows.eps), po.norm(more.k, more.kw, more.eps)])
    from oracle.choreo_oracle import rope
    at = np.arange(len(k))
    ks[2] = rope(po.to_mx4(rope(normed, at, THETA)), -at, THETA)
    q = more.q_out.double().cpu().numpy()
    same(out, lse, *win.attend_call_window(ks, vs, [(1, 0), (0, 60)], 2, 170, 1, None, q, THETA, 1 << 40, 0), "token")
    c.close()


def test_tables_and_two_caches_at_once():
    """pc_build_tables of a 4-bit cache; two caches on two streams."""
    torch = __import__("torch")
    a, b = Layer4([40, 33, 50], 8, 2, seed=1), Layer4([40, 33, 50], 8, 2, seed=2)
    calls = [([(0, 0), (1, 50)], 2, 100, 50), ([(1, 0)], 2, 60, 1)]
    call = a.calls(calls)[0]
    n = a.cache.build_tables(call, 0, 0, 0)
    assert n == 123
    slot, pos = torch.zeros(n, dtype=torch.int32, device="cuda:0"), torch.zeros(n, dtype=torch.int32, device="cuda:0")
    a.cache.build_tables(call, slot.data_ptr(), pos.data_ptr(), n)
    torch.cuda.synchronize()
    assert pos.tolist() == list(range(40)) + list(range(50, 83)) + list(range(100, 150))
    assert slot.tolist() == list(range(40)) + list(range(64, 97)) + list(range(128, 178))
    q = a.normal(51, 8, 128)
    tq = a.dev(q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for layer, s in zip((a, b), streams):
        s.wait_stream(torch.cuda.current_stream())
        out, lse = torch.zeros_like(tq), torch.zeros(51, 8, device="cuda:0")
        outs.append((out, lse))
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, s, (out, lse) in zip((a, b), streams, outs):
            layer.cache.attend(layer.calls(calls), tq.data_ptr(), out.data_ptr(), lse.data_ptr(), s.cuda_stream)
    torch.cuda.synchronize()
    for layer, (out, lse) in zip((a, b), outs):
        same(out, lse, *layer.want(calls, q), "two streams")
        layer.cache.close()
