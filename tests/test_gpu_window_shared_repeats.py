"""Single tokens of calls that list a message twice at the same place, or their new message as a parent where it is: such keys are
seen twice (a score more in the sum, its value twice), whatever way the batch goes.  Against the fp64 oracle; the bars of compare()."""
import numpy as np
import pytest

from tests.window_cases import Layer, compare

pytestmark = pytest.mark.gpu


def check(layer, calls, window, n_sink, q, some=None, what=""):
    some = list(range(len(calls))) if some is None else some
    out, lse = layer.attend(calls, window, n_sink, q)
    compare("bf16", out[some], lse[some], *layer.want([calls[i] for i in some], window, n_sink, q[some]), f"{what} w {window} s {n_sink}")


@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("h_q,h_kv,n_calls", [(16, 2, 24), (3, 1, 23), (16, 1, 6)])
def test_a_message_twice_at_the_same_place(h_q, h_kv, n_calls, mode):
    layer = Layer("bf16", [200, 31, 333, 1, 150] + [7] * 4, h_q, h_kv, 128)
    layer.cache.set_decode_sharing(mode)
    base = [(0, 0), (1, 200), (2, 231), (3, 564), (4, 565)]
    more = [[], [(0, 0)], [(2, 231)], [(2, 231), (2, 231)], [(3, 564)], [(0, 0), (4, 565)]]
    q = layer.normal(n_calls, h_q, 128)
    for every in (1, 5):                                 # of all calls, of some
        calls = [(base + (more[i // every % len(more)] if i % every == 0 else []), 5 + i % 4 if i % 3 else -1, 715, 1) for i in range(n_calls)]
        for window, n_sink in [(1 << 30, 0), (1 << 30, 40), (500, 0), (500, 64), (300, 800), (200, 3)]:
            check(layer, calls, window, n_sink, q, what=f"mode {mode}")
    layer.cache.close()


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_the_new_message_as_a_parent_where_it_is(mode):
    layer = Layer("bf16", [300, 260] + [40] * 3, 16, 2, 128)
    layer.cache.set_decode_sharing(mode)
    q = layer.normal(24, 16, 128)
    for window, n_sink in [(1 << 30, 0), (350, 0), (100, 33), (20, 700)]:
        calls = [([(0, 0), (1, 300)] + ([(2 + i % 3, 560)] if i % 2 else []), 2 + i % 3, 560, 1) for i in range(24)]
        check(layer, calls, window, n_sink, q, what=f"mode {mode}")
    layer.cache.close()


def test_a_batch_that_shares_by_its_cost():
    """64 calls over the same 5120 tokens, which go together by themselves; one call in three has a message twice."""
    layer = Layer("bf16", [640] * 8, 32, 4, 128)
    base = [(m, 640 * m) for m in range(8)]
    q = layer.normal(64, 32, 128)
    some = [0, 1, 33, 63]
    for what, calls in [("once", [(base, -1, 5119 + i, 1) for i in range(64)]), ("twice", [(base + ([(3, 1920)] if i % 3 == 0 else []), -1, 5119 + i, 1) for i in range(64)])]:
        for window, n_sink in [(1 << 30, 0), (4000, 100)]:
            check(layer, calls, window, n_sink, q, some, what)
            layer.cache.set_decode_sharing(1)
            out, lse = layer.attend(calls, window, n_sink, q)
            layer.cache.set_decode_sharing(0)
            shared, shared_lse = layer.attend(calls, window, n_sink, q)
            # (probabilities rounded relative to another maximum: each sum is off by 2^-8 of itself at most)
            assert (lse - shared_lse).abs().max().item() <= 2 * 2.0 ** -8 and (out.float() - shared.float()).abs().max().item() <= 4e-2
    layer.cache.close()


def test_the_prompts_of_such_calls():
    """The same lists with a few rows a call, and fp32."""
    for dtype in ("bf16", "f32"):
        layer = Layer(dtype, [100, 70, 40], 8, 2, 128)
        for n_q in (1, 3, 40):
            calls = [([(0, 0), (1, 100), (0, 0)], 2, 170, n_q), ([(1, 0), (1, 0), (2, 70)], 2, 70, n_q)]
            q = layer.normal(2 * n_q, 8, 128)
            for window, n_sink in [(1 << 30, 0), (120, 30)]:
                out, lse = layer.attend(calls, window, n_sink, q)
                compare(dtype, out, lse, *layer.want(calls, window, n_sink, q), f"n_q {n_q} w {window}")
        layer.cache.close()
