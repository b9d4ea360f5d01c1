"""pc_attend_window against the fp64 oracle: window and sink edges inside tiles, ragged messages, rows that see nothing, head
layouts, both types, splits, one row and many; values that are not finite where a row does not see them."""
import numpy as np
import pytest

from tests.window_cases import Layer, compare, say

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 4, 4, 128), ("bf16", 8, 2, 128), ("bf16", 32, 2, 128), ("bf16", 6, 2, 128), ("bf16", 5, 1, 128), ("bf16", 16, 2, 128),
          ("f32", 4, 2, 64), ("f32", 3, 1, 128), ("f32", 32, 2, 64), ("f32", 40, 2, 128)]
LENS = [31, 1, 64, 33, 100, 90]
SEL = [(0, 0), (4, 40), (1, 7), (2, 300), (0, 500), (3, 140)]


def run(layer, calls, window, n_sink, what="", static=False):
    q = layer.normal(layer.rows(calls), layer.h_q, layer.D)
    out, lse = layer.attend(calls, window, n_sink, q, static)
    want, want_lse = layer.want(calls, window, n_sink, q)
    compare(layer.dtype, out, lse, want, want_lse, what or f"w {window} s {n_sink}")


@pytest.mark.parametrize("dtype,h_q,h_kv,D", SHAPES)
@pytest.mark.parametrize("n_q", [1, 2, 33, 90])
def test_windows_and_sinks(dtype, h_q, h_kv, D, n_q):
    layer = Layer(dtype, LENS, h_q, h_kv, D)
    for window, n_sink in [(1, 0), (2, 1), (31, 0), (32, 5), (33, 32), (64, 33), (100, 40), (400, 0), (1 << 30, 0), (2147483647, 3), (5, 1 << 30)]:
        run(layer, [(SEL, 5, 600, n_q)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_a_window_over_everything_is_pc_attend(dtype, h_q, h_kv, D):
    import torch
    layer = Layer(dtype, LENS, h_q, h_kv, D)
    for n_q in (1, 90):
        calls = [(SEL, 5, 600, n_q)]
        q = layer.normal(n_q, h_q, D)
        out, lse = layer.attend(calls, 1 << 20, 0, q)
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        tq = layer.dev(q)
        layer.cache.attend(layer.calls(calls), tq.data_ptr(), o2.data_ptr(), l2.data_ptr())
        torch.cuda.synchronize()
        compare(dtype, out, lse, o2.double().cpu().numpy(), l2.double().cpu().numpy())
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("bf16", 4, 4, 128), ("f32", 6, 2, 64), ("f32", 4, 1, 128)])
@pytest.mark.parametrize("static", [False, True])
def test_batches(dtype, h_q, h_kv, D, static):
    """Calls of one row and of many side by side; some see nothing, some have no new message, some only their own tokens; the
    same message twice; positions stated, negative, repeated, in front of every key; a window behind every key."""
    lens = [int(x) for x in np.random.default_rng(3).integers(20, 300, size=12)] + [20, 70, 1]
    layer = Layer(dtype, lens, h_q, h_kv, D)
    long = [(m, 300 * m) for m in range(12)]
    calls = [(long, 14, 3700, 1), (long[::-1], 13, 100, 70), ([(0, 5)], -1, 0, 3, [900, 5, 700]), ([], 12, 0, 20), ([(0, -5000)], -1, 9000, 1),
             ([(3, 50), (3, 50)], 13, 80, 40), (long[:3], -1, 0, 5, [-40, 3, 3, 10 ** 6, 90]), ([], -1, 7, 2), ([], 14, 0, 1), (long, -1, 2000, 1)]
    for window, n_sink in [(50, 0), (333, 7), (1500, 64), (4000, 500)]:
        run(layer, calls, window, n_sink, static=static)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 4, 1, 128), ("f32", 2, 1, 64)])
@pytest.mark.parametrize("n_q", [1, 3, 40])
def test_long_walks_are_split(dtype, h_q, h_kv, D, n_q):
    lens = [700] * 9 + [50]
    layer = Layer(dtype, lens, h_q, h_kv, D)
    sel = [(m, 650 * m) for m in range(9)]
    for window, n_sink in [(5000, 40), (6500, 0), (90, 900)]:
        run(layer, [(sel, 9, 5850, n_q)], window, n_sink)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_moved_messages_far_positions_and_extents(dtype, h_q, h_kv, D):
    from paper_2512_23049_amd.binding import PC_FLAG_GROW_EXTENTS
    layer = Layer(dtype, [40, 70, 33, 20], h_q, h_kv, D, flags=PC_FLAG_GROW_EXTENTS, max_position=2147483647, room=2000)
    layer.cache.reposition(0, 1000)
    layer.cache.reposition(1, -77)
    import torch
    for n in (50, 45):                                   # the last message grows into further extents
        k, v = layer.normal(n, h_kv, D), layer.normal(n, h_kv, D)
        tk, tv = layer.dev(k), layer.dev(v)
        layer.cache.append_tokens(3, tk.data_ptr(), tv.data_ptr(), n)
        torch.cuda.synchronize()
        layer.ks[3], layer.vs[3] = np.concatenate([layer.ks[3], k]), np.concatenate([layer.vs[3], v])
    assert len(layer.cache.message_extents(3)) > 1
    for far in (0, 2147483647 - 2000):
        for n_q in (1, 12):
            for window, n_sink in [(60, 3), (150, 45), (1 << 30, 1)]:
                run(layer, [([(0, far), (2, far + 40), (3, far + 100), (1, far + 77)], 3, far + 300, n_q)], window, n_sink)
    lowest = -2147483647
    run(layer, [([(0, lowest), (1, 2147483647 - 100)], -1, 0, 3, [lowest, lowest + 50, 2147483647])], 2147483647, 2)
    run(layer, [([(0, lowest), (1, 2147483647 - 100)], -1, 0, 1, [lowest + 20])], 2147483647, 0)
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("bf16", 4, 4, 128), ("f32", 6, 2, 64), ("f32", 2, 1, 128)])
@pytest.mark.parametrize("n_q", [1, 70])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, h_q, h_kv, D, n_q):
    """Keys and values out of the window, in its tiles and in front of them, and behind a row's own token."""
    bad = [np.inf, -np.inf, np.nan]

    def spoil(ks, vs):
        for i, t in enumerate((0, 3, 64, 70)):           # message 0, in front of the window: every row's or only the later ones'
            vs[0][t, :, i::7] = bad[i % 3]
            ks[0][t, 0, 5 + i] = bad[i % 3]
        vs[1][60, 0, 3], vs[1][61, 0, 3], vs[1][62, 0, 4] = np.inf, -np.inf, np.nan        # own tokens that the earlier rows do not see
        ks[1][66, 0, 9] = np.nan
    layer = Layer(dtype, [100, 70], h_q, h_kv, D, spoil=spoil)
    calls = [([(0, 0)], 1, 100, n_q)]
    q = layer.normal(n_q, h_q, D)
    for window, n_sink in [(30, 0), (60, 2), (101, 0)]:
        out, lse = layer.attend(calls, window, n_sink, q)
        want, want_lse = layer.want(calls, window, n_sink, q)
        got = out.float().cpu().numpy().astype(np.float64)
        # A row that sees a key that is not finite: a turn of (inf, y) is (+-inf, +-inf), whichever the angle, so what its score
        # is depends on how many turns the key and the query went through; nothing is said of those rows.  The others are the test.
        from oracle import window_oracle as win
        keys, vis = np.concatenate([layer.ks[0], layer.ks[1]]), win.visible(np.arange(170), 170 - n_q + np.arange(n_q), 170 - n_q + np.arange(n_q), window, n_sink)
        dead = np.repeat(np.stack([(vis & ~np.isfinite(keys[:, h]).all(axis=1)).any(axis=1) for h in range(h_kv)], axis=1), h_q // h_kv, axis=1)
        g, w = got[~dead], want[~dead]
        off = np.argwhere((np.isnan(g) != np.isnan(w)) | ((g == np.inf) != (w == np.inf)) | ((g == -np.inf) != (w == -np.inf)))
        if len(off):
            say(f"  w {window} s {n_sink}: differ at {off[:5].tolist()}: got {[g[tuple(i)] for i in off[:5]]}, want {[w[tuple(i)] for i in off[:5]]}")
        assert np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(g == np.inf, w == np.inf) and np.array_equal(g == -np.inf, w == -np.inf)
        fine = np.isfinite(w)
        say(f"  w {window}: {dead.sum()} rows left out, {(~fine).sum()} values not finite, {fine.sum()} finite")
        if n_q > 1 and window == 30:
            assert dead.any() and fine.any() and (h_kv == 1 or (~fine).any())
        assert np.abs(g[fine] - w[fine]).max(initial=0) <= {"f32": 3e-5, "bf16": 4e-2}[dtype]
    layer.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 6, 2, 64)])
def test_large_scores_move_the_reference(dtype, h_q, h_kv, D):
    """Scores of several hundred in the logarithm's units, the largest first, last and in the middle, of one sign and both: exact scores
    (one-token messages at the rows' own position, a scale of a power of two in the logarithm's base), so that bf16's roundings of keys and
    queries have no part in them."""
    from paper_2512_23049_amd import binding
    import torch
    from pc_inputs import Call
    for order in ([-400, 0, 400], [400, 0, -400], [0, 700, -100], [-900, -890, -880], [0, 90, 150, 300, 500]):
        cache = binding.Cache(h_q, h_kv, D, binding.PC_BF16 if dtype == "bf16" else binding.PC_F32, 10000.0, 4096, 64, softmax_scale=0.25 * float(np.log(2.0)))
        kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        vals = []
        for i, s in enumerate(order):
            k, v = torch.zeros(1, h_kv, D, device="cuda:0", dtype=kind), torch.full((1, h_kv, D), float(i + 1), device="cuda:0", dtype=kind)
            k[:, :, 0] = s / 2.0
            cache.append_message(k.data_ptr(), v.data_ptr(), 1)
            vals.append(s * 2.0 * np.log(2.0))           # 0.25 ln 2 x 16 x s / 2
            torch.cuda.synchronize()
        for n_q in (1, 40):
            q = torch.zeros(n_q, h_q, D, device="cuda:0", dtype=kind)
            q[:, :, 0] = 16.0
            out, lse = torch.empty_like(q), torch.empty(n_q, h_q, device="cuda:0")
            cache.attend_window([Call([(i, 0) for i in range(len(order))], -1, 0, n_q, [0] * n_q)], 1, 0, q.data_ptr(), out.data_ptr(), lse.data_ptr())
            torch.cuda.synchronize()
            x = np.array(vals)
            p = np.exp(x - x.max())
            want, want_lse = (p * np.arange(1, len(x) + 1)).sum() / p.sum(), x.max() + np.log(p.sum())
            assert np.abs(out.float().cpu().numpy() - want).max() <= 2 ** -7 * want
            assert np.abs(lse.cpu().numpy() - want_lse).max() <= 1e-6 * abs(want_lse) + 1e-5
        cache.close()
