"""pc_append_projected* and pc_messages_read against fp64: types, head layouts, strides, ragged lengths, weights, rows of zeros, growing messages,
spans that are taken again."""
import numpy as np
import pytest

from oracle import project_oracle as po
from oracle.choreo_oracle import rope
from tests.project_cases import THETA, Layer4, Rows, cache_of, check, kinds, read

pytestmark = pytest.mark.gpu

SHAPES = [("bf16", 8, 2, 128), ("bf16", 5, 5, 128), ("bf16", 24, 12, 128), ("f32", 4, 2, 64), ("f32", 9, 3, 128), ("mx4", 8, 2, 128), ("mx4", 11, 11, 128)]


def want_held(rows, a, b, first, dtype):
    """(keys as stored, values) of rows [a, b), whose first token has index `first` in its message."""
    k = rope(rows.want_k(a, b), first + np.arange(b - a), THETA)
    return (po.to_mx4(k), po.to_mx4(rows.v[a:b])) if dtype == "mx4" else (k, rows.v[a:b])


def compare_held(got_k, got_v, want_k, want_v, dtype, what):
    assert np.array_equal(got_v, want_v), what
    if dtype == "mx4":
        assert np.array_equal(got_k, want_k), what
    else:
        check(got_k, want_k, dtype, what)


@pytest.mark.parametrize("dtype,h_q,h_kv,D", SHAPES)
@pytest.mark.parametrize("fused,extra,weights", [(True, 0, True), (True, 64, False), (False, 0, True)])
def test_messages(dtype, h_q, h_kv, D, fused, extra, weights):
    import torch
    lens, reserves = [1, 7, 8, 33, 64, 100, 2], [40, 0, 9, 0, 0, 128, 0]
    rows = Rows(dtype, sum(lens), h_q, h_kv, D, fused=fused, extra=extra, weights=weights, spoil=lambda x: x[3].zero_())
    c = cache_of(dtype, h_q, h_kv, D, 1024)
    ids = c.append_projected(rows.c, lens, rows.out_ptr, reserves)
    torch.cuda.synchronize()
    check(rows.q_out.double().cpu().numpy(), rows.want_q(), dtype, "q")
    k, v = read(c, ids, sum(lens), h_kv, D, rows.kind)
    at = 0
    for n in lens:
        compare_held(k[at:at + n], v[at:at + n], *want_held(rows, at, at + n, 0, dtype), dtype, f"message of {n}")
        at += n
    for m in ids[::2]:                                   # other messages where these were
        c.message_free(m)
    again = Rows(dtype, 70, h_q, h_kv, D, seed=5, queries=False)
    ids2 = c.append_projected(again.c, [40, 1, 29], 0)
    k, v = read(c, ids2 + [ids[1]], 77, h_kv, D, rows.kind)
    for a, b in ((0, 40), (40, 41), (41, 70)):
        compare_held(k[a:b], v[a:b], *want_held(again, a, b, 0, dtype), dtype, "again")
    compare_held(k[70:], v[70:], *want_held(rows, 1, 8, 0, dtype), dtype, "what stayed")
    c.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", SHAPES)
def test_tokens(dtype, h_q, h_kv, D):
    """Token after token, across groups of eight slots, tiles and extents; beside them plain tokens."""
    import torch
    from paper_2512_23049_amd import binding as b
    c = cache_of(dtype, h_q, h_kv, D, 2048, flags=b.PC_FLAG_GROW_EXTENTS)
    lens = [1, 30, 7]
    first = Rows(dtype, sum(lens), h_q, h_kv, D)
    ids = c.append_projected(first.c, lens, first.out_ptr)
    held = [want_held(first, a, a + n, 0, dtype) for a, n in zip((0, 1, 31), lens)]
    for step in range(11):
        order = [2, 0, 1][:1 + step % 3]
        rows = Rows(dtype, len(order), h_q, h_kv, D, seed=10 + step)
        c.append_projected_tokens(rows.c, [ids[m] for m in order], rows.out_ptr)
        torch.cuda.synchronize()
        check(rows.q_out.double().cpu().numpy(), rows.want_q(), dtype, "q")
        for j, m in enumerate(order):
            k, v = want_held(rows, j, j + 1, len(held[m][0]), dtype)
            held[m] = (np.concatenate([held[m][0], k]), np.concatenate([held[m][1], v]))
    k, v = read(c, ids, sum(len(x[0]) for x in held), h_kv, D, first.kind)
    at = 0
    for wk, wv in held:
        compare_held(k[at:at + len(wk)], v[at:at + len(wk)], wk, wv, dtype, f"{len(wk)} tokens")
        at += len(wk)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_norms_it_is_what_plain_appends_store(dtype):
    """Rows of norm one and weights of one: the same messages by pc_append_messages, compared slot by slot."""
    import torch
    h_q, h_kv, D = 4, 2, 128
    lens = [37, 5, 64]
    rows = Rows(dtype, sum(lens), h_q, h_kv, D, weights=False)
    c = cache_of(dtype, h_q, h_kv, D, 512)
    ids = c.append_projected(rows.c, lens, rows.out_ptr)
    normed = torch.from_numpy(po.norm(rows.k, None, rows.eps)).to("cuda:0", torch.float32)
    k, v = normed.to(rows.kind), rows.parts[2].reshape(sum(lens), h_kv, D).contiguous()
    starts = [0, 37, 42]
    ids2 = c.append_messages([k[a:].data_ptr() for a in starts], [v[a:].data_ptr() for a in starts], lens)
    a, b = read(c, ids, sum(lens), h_kv, D, rows.kind), read(c, ids2, sum(lens), h_kv, D, rows.kind)
    (k1, v1), (k2, v2) = tuple(a), tuple(b)
    assert np.array_equal(v1, v2)
    if dtype == "f32":
        check(k1, k2, dtype, "keys")
    else:
        # Of the plain append the normed key was rounded before its turn: a and b of a pair are off by 2^-8 of themselves at most, a c - b s then by
        # 2^-8 (|a c| + |b s|) <= 2^-8 sqrt(a^2 + b^2), the pair's norm, which a turn keeps.  Both results are rounded after it, by
        # 2^-8 of themselves each (of the exact ones, which the other's errors move by 2^-8 more: 2.1 for both).
        pair = np.sqrt(k2[..., :D // 2] ** 2 + k2[..., D // 2:] ** 2)
        bar = 2.0 ** -8 * (1.01 * np.concatenate([pair, pair], axis=-1) + 2.1 * np.abs(k2)) + 1e-6
        assert (np.abs(k1 - k2) <= bar).all()
    c.close()


def test_many_messages_and_long_lists():
    """Lists that the arguments do not hold."""
    import torch
    lens = [int(x) for x in np.random.default_rng(2).integers(1, 20, size=150)]
    for dtype, h_q, h_kv, D in (("bf16", 8, 2, 128), ("mx4", 8, 2, 128), ("f32", 4, 2, 64)):
        rows = Rows(dtype, sum(lens), h_q, h_kv, D)
        c = cache_of(dtype, h_q, h_kv, D, 32 * 400, messages=400)
        ids = c.append_projected(rows.c, lens, rows.out_ptr, [n + 1 for n in lens])
        more = Rows(dtype, 150, h_q, h_kv, D, seed=9)
        c.append_projected_tokens(more.c, ids, more.out_ptr)
        torch.cuda.synchronize()
        check(rows.q_out.double().cpu().numpy(), rows.want_q(), dtype, "q")
        k, v = read(c, ids, sum(lens) + 150, h_kv, D, rows.kind)
        at = src = 0
        for j, n in enumerate(lens):
            compare_held(k[at:at + n], v[at:at + n], *want_held(rows, src, src + n, 0, dtype), dtype, f"message {j}")
            compare_held(k[at + n:at + n + 1], v[at + n:at + n + 1], *want_held(more, j, j + 1, n, dtype), dtype, f"token {j}")
            at += n + 1
            src += n
        c.close()


@pytest.mark.parametrize("dtype", ["bf16", "mx4"])
def test_another_stream_and_large_values(dtype):
    import torch
    h_q, h_kv, D = 8, 2, 128

    def spoil(x):
        x[1] *= 1e12
        x[2] *= 1e-12
        x[4] *= 3e18                                     # (squares up to 1e38 x 128: their sum passes 32 bits)
    rows = Rows(dtype, 40, h_q, h_kv, D, spoil=spoil, eps=0.0)
    c = cache_of(dtype, h_q, h_kv, D, 512)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ids = c.append_projected(rows.c, [40], rows.out_ptr, stream=s.cuda_stream)
    s.synchronize()
    fine = [i for i in range(40) if i != 4]
    check(rows.q_out.double().cpu().numpy()[fine], rows.want_q()[fine], dtype, "q")
    k, v = read(c, ids, 40, h_kv, D, rows.kind)
    wk, wv = want_held(rows, 0, 40, 0, dtype)
    compare_held(k[fine], v[fine], wk[fine], wv[fine], dtype, "held")
    c.close()


def test_what_is_no_number_in_four_bits():
    """A token with an infinity or a NaN has keys of NaN in that head, and no other does."""
    def spoil(i, k, v):
        if i == 1:
            k[3, 0, 5], v[6, 1, 100], k[9, 1, 64], v[10, 0, 0] = np.inf, np.nan, np.nan, -np.inf
    layer = Layer4([20, 40, 33], 8, 2, spoil=spoil)
    k, _ = read(layer.cache, layer.ids, 93, 2, 128, layer.torch.bfloat16)
    none = np.isnan(k).any(axis=-1)
    assert sorted(map(tuple, np.argwhere(none))) == [(23, 0), (26, 1), (29, 1), (30, 0)]
    assert np.isnan(k[none]).all()
    layer.cache.close()


@pytest.mark.parametrize("h_kv", [1, 2, 9])
def test_four_bit_messages_hold_what_they_say(h_kv):
    """Plain appends, tokens one by one and many at once, values that are ties, zeros, larger and smaller than there are powers for."""
    from paper_2512_23049_amd import binding as b

    def spoil(i, k, v):
        if i == 2:
            k[:4] = np.round(k[:4] * 4) / 4
            v[:8] = np.round(v[:8] * 4) / 4
            v[8] = 0
            v[9] *= 2.0 ** 70
            v[10] *= 2.0 ** -80
            k[11] *= 2.0 ** 90
            v[12, :, 32:64] = 0
    lens = [1, 31, 64, 33]
    layer = Layer4(lens, h_kv, h_kv, spoil=spoil, reserves=[10, 40, 0, 0], flags=b.PC_FLAG_GROW_EXTENTS, room=512)
    for m, n in ((0, 3), (1, 1), (0, 20), (3, 50)):
        k, v = layer.normal(n, h_kv, 128), layer.normal(n, h_kv, 128)
        tk, tv = layer.dev(k), layer.dev(v)
        layer.cache.append_tokens(layer.ids[m], tk.data_ptr(), tv.data_ptr(), n)
        layer.torch.cuda.synchronize()
        layer.grow(m, k, v)
    for _ in range(3):
        k, v = layer.normal(2, h_kv, 128), layer.normal(2, h_kv, 128)
        tk, tv = layer.dev(k), layer.dev(v)
        layer.cache.append_tokens_batch([layer.ids[1], layer.ids[0]], tk.data_ptr(), tv.data_ptr())
        layer.torch.cuda.synchronize()
        layer.grow(1, k[:1], v[:1])
        layer.grow(0, k[1:], v[1:])
    total = sum(len(x) for x in layer.ks)
    k, v = read(layer.cache, layer.ids, total, h_kv, 128, layer.torch.bfloat16)
    want = [po.to_mx4(rope(np.asarray(a, np.float64), np.arange(len(a)), THETA)) for a, _ in layer.raw]
    assert np.array_equal(k, np.concatenate(want))
    assert np.array_equal(v, np.concatenate(layer.vs))
    layer.cache.close()
