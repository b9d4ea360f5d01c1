"""Forks and the cache closing up on the GPU: what the stores hold afterwards, bit for bit where nothing is turned, and that
attention goes on as before."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


class Store:
    """A cache in an arena of the test's own, whose stores can be read: k, v [kv_heads, slots, dim]."""

    def __init__(self, dtype, h_kv, D, slots, messages=2000, flags=0, h_q=None):
        import torch
        from paper_2512_23049_amd import binding
        self.torch, self.h_kv, self.D, self.slots = torch, h_kv, D, slots
        self.kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        es = 2 if dtype == "bf16" else 4
        self.arena = torch.empty(2 * slots * h_kv * D * es, dtype=torch.uint8, device="cuda:0")
        self.cache = binding.Cache(h_q or h_kv, h_kv, D, binding.PC_BF16 if dtype == "bf16" else binding.PC_F32, 10000.0, slots, messages,
                                   max_position=1 << 20, flags=flags, arena=self.arena.data_ptr(), arena_bytes=self.arena.numel())
        self.bits = torch.int16 if dtype == "bf16" else torch.int32
        self.grouped = dtype == "bf16"

    def put(self, n, seed, reserve=0):
        g = self.torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        k, v = (self.torch.randn(n, self.h_kv, self.D, generator=g, device="cuda:0").to(self.kind) for _ in range(2))
        m = self.cache.append_message(k.data_ptr(), v.data_ptr(), n, reserve)
        self.torch.cuda.synchronize()
        return m

    def read(self):
        self.torch.cuda.synchronize()
        half = self.arena.numel() // 2
        k = self.arena[:half].view(self.kind).view(self.h_kv, self.slots, self.D)
        v = self.arena[half:].view(self.kind)
        v = v.view(self.h_kv, self.slots // 8, self.D, 8).permute(0, 1, 3, 2).reshape(self.h_kv, self.slots, self.D) if self.grouped else v.view(self.h_kv, self.slots, self.D)
        return k.clone(), v.clone()

    def message(self, m, stores=None):
        k, v = stores or self.read()
        at = [np.arange(s, s + n) for s, n in self.cache.message_extents(m, 256)]
        at = self.torch.from_numpy(np.concatenate(at)).to("cuda:0")
        return k[:, at], v[:, at]

    def same(self, a, b):
        return all(self.torch.equal(x.view(self.bits), y.view(self.bits)) for x, y in zip(a, b))


TYPES = [("bf16", 3, 128), ("f32", 2, 64), ("f32", 3, 128)]


@pytest.mark.parametrize("dtype,h_kv,D", TYPES)
def test_forks_are_exact_copies(dtype, h_kv, D):
    s = Store(dtype, h_kv, D, 8192)
    for i, n in enumerate((1, 31, 32, 33, 257, 400)):
        s.put(n, i)
    s.put(60, 9)
    s.cache.message_free(6)                              # (the forks' spans hold leftovers)
    forks = [(m, first, n, reserve, None) for m, first, n, reserve in
             [(0, 0, 1, 0), (1, 0, 31, 0), (1, 7, 24, 40), (3, 32, 1, 0), (4, 1, 256, 0), (4, 5, 33, 100), (5, 9, 391, 0), (5, 399, 1, 70), (5, 16, 200, 0), (5, 11, 8, 0)]]
    ids = s.cache.message_fork(forks)
    stores = s.read()
    for (m, first, n, reserve, _), f in zip(forks, ids):
        k, v = s.message(m, stores)
        assert s.same(s.message(f, stores), (k[:, first:first + n].contiguous(), v[:, first:first + n].contiguous()))
        assert s.cache.message_base(f) == first
        start, end = s.cache.message_info(f)[1] + n, s.cache.message_info(f)[1] + (max(n, reserve) + 31) // 32 * 32
        assert (stores[0][:, start:end] == 0).all() and (stores[1][:, start:end] == 0).all()
    s.cache.close()


@pytest.mark.parametrize("dtype,h_kv,D", TYPES)
def test_forks_of_several_extents_and_of_what_is_not_finite(dtype, h_kv, D):
    from paper_2512_23049_amd.binding import PC_FLAG_GROW_EXTENTS
    import torch
    s = Store(dtype, h_kv, D, 4096, flags=PC_FLAG_GROW_EXTENTS)
    m = s.put(37, 1)
    for i, n in enumerate((45, 3, 70)):
        s.put(10, 20 + i)
        k = torch.randn(n, h_kv, D, device="cuda:0").to(s.kind)
        k[0, 0, 0], k[1, 0, 3], k[2, 0, 5] = float("nan"), float("inf"), -float("inf")
        s.cache.append_tokens(m, k.data_ptr(), k.data_ptr(), n)
        torch.cuda.synchronize()
    assert len(s.cache.message_extents(m)) > 2
    total = s.cache.message_info(m)[0]
    forks = [(m, first, n, 0, None) for first, n in [(0, total), (30, 20), (36, 2), (5, 100), (38, 90)]]
    ids = s.cache.message_fork(forks)
    stores = s.read()
    k, v = s.message(m, stores)
    for (_, first, n, _, _), f in zip(forks, ids):
        assert s.same(s.message(f, stores), (k[:, first:first + n].contiguous(), v[:, first:first + n].contiguous()))
        assert len(s.cache.message_extents(f)) == 1
    s.cache.close()


@pytest.mark.parametrize("dtype,h_kv,D", TYPES)
def test_turned_forks(dtype, h_kv, D):
    """Keys against the stored ones turned in 64 bits: one rounding to the cache's type of a product of numbers of which each
    was rounded to 24 bits.  bf16: half a step of the result, 2^-8 of a number no larger than the pair it is a part of; fp32: three
    roundings of 2^-24 of that."""
    from oracle import choreo_oracle as orc
    s = Store(dtype, h_kv, D, 8192)
    for i, n in enumerate((5, 64, 333)):
        s.put(n, i)
    s.cache.reposition(1, 500)
    forks = [(0, 0, 5, 0, -3), (1, 10, 50, 0, 12), (2, 3, 330, 0, 700000), (2, 40, 1, 0, 0), (1, 0, 64, 0, 500)]
    ids = s.cache.message_fork(forks)
    stores = s.read()
    bar = (2.0 ** -8 + 3 * 2.0 ** -24) if dtype == "bf16" else 3 * 2.0 ** -24
    for (m, first, n, _, base), f in zip(forks, ids):
        k, v = s.message(m, stores)
        fk, fv = s.message(f, stores)
        assert s.same((fv,), (v[:, first:first + n].contiguous(),))
        src = k[:, first:first + n].double().cpu().numpy().transpose(1, 0, 2)
        turn = base - ((500 if m == 1 else 0) + first)
        want = orc.rope(src, np.full(n, turn), 10000.0)
        size = np.sqrt(src[..., :D // 2] ** 2 + src[..., D // 2:] ** 2)
        got = fk.double().cpu().numpy().transpose(1, 0, 2)
        assert (np.abs(got - want) <= bar * np.concatenate([size, size], axis=-1) + 1e-30).all()
        if turn == 0:
            assert s.same((fk,), (k[:, first:first + n].contiguous(),))
    s.cache.close()


@pytest.mark.parametrize("dtype,h_kv,D", TYPES)
@pytest.mark.parametrize("seed,gap", [(0, 32), (1, 300), (2, 2000), (3, None)])
def test_closing_up_moves_bits(dtype, h_kv, D, seed, gap):
    """A small gap in front of everything, large ones, scattered ones; all at once and in parts; reserves with room."""
    r = np.random.default_rng(seed)
    s = Store(dtype, h_kv, D, 40960)
    ids = []
    if gap:
        ids.append(s.put(gap, 1000))
    for i in range(60):
        n = int(r.integers(1, 900))
        ids.append(s.put(n, i, n + int(r.choice([0, 0, 5, 200]))))
    gone = ids[:1] if gap else [m for m in ids if r.random() < 0.4]
    stores = s.read()
    kept = {m: s.message(m, stores) for m in ids if m not in gone}
    for m in gone:
        s.cache.message_free(m)
    moved, times = 0, 0
    while True:
        step = s.cache.compact(0 if seed % 2 else 7000)
        if step == 0:
            break
        moved, times = moved + step, times + 1
        stores = s.read()
        for m, was in kept.items():
            assert s.same(s.message(m, stores), was), (m, times)
    used = 0
    for m in kept:
        n, start, reserved = s.cache.message_info(m)
        end = start + (reserved + 31) // 32 * 32
        assert start == used and (stores[0][:, start + n:end] == 0).all() and (stores[1][:, start + n:end] == 0).all()
        used = end
    assert s.cache.cache_info()[1] == used
    say(f"  {dtype} {D}: {moved} slots moved in {times}")
    s.cache.close()


def test_closing_up_a_cache_of_millions_of_slots():
    """Tiles beyond 4 GiB of a store, a gap of one tile in front of them."""
    import torch
    s = Store("bf16", 4, 128, 6 << 20)                   # 6 GiB each of keys and values
    first = s.put(20, 1)
    big = [s.put(1 << 18, i) for i in range(22)]
    last = s.put(77, 99)
    before = {m: s.message(m) for m in (big[0], big[21], last)}
    torch.cuda.synchronize()
    s.cache.message_free(first)
    assert s.cache.compact() == 22 * (1 << 18) + 96
    for m, was in before.items():
        assert s.same(s.message(m), was)
    s.cache.close()


@pytest.mark.parametrize("dtype,h_q,h_kv,D", [("bf16", 8, 2, 128), ("f32", 4, 2, 64)])
def test_a_generation_that_branches_and_forgets(dtype, h_q, h_kv, D):
    """Branches of a common prompt generate in a windowed layer; the worse half is given up, its best branch is forked, the cache
    closes up, and the generation goes on: every step against the oracle, pc_attend beside it."""
    import torch
    from tests.window_cases import Layer, compare
    window, sinks = 90, 4
    layer = Layer(dtype, [70, 45], h_q, h_kv, D, room=4000)
    c = layer.cache
    lines = []                                           # (message, keys, values)

    def tail(n):
        return layer.normal(n, h_kv, D), layer.normal(n, h_kv, D)
    for _ in range(4):
        k, v = tail(20)
        tk, tv = layer.dev(k), layer.dev(v)
        lines.append([c.append_message(tk.data_ptr(), tv.data_ptr(), 20, 64), k, v])
        torch.cuda.synchronize()
    for step in range(30):
        k, v = tail(len(lines))
        tk, tv = layer.dev(k), layer.dev(v)
        c.append_tokens_batch([x[0] for x in lines], tk.data_ptr(), tv.data_ptr())
        for i, x in enumerate(lines):
            x[1], x[2] = np.concatenate([x[1], k[i:i + 1]]), np.concatenate([x[2], v[i:i + 1]])
        if step in (9, 19):
            given_up, lines = lines[::2], lines[1::2]
            best = lines[0]
            ids = c.message_fork([(best[0], 0, len(best[1]), 64, None), (best[0], 0, 15, 64, 40), (1, 3, 41, 0, None)])
            for x in given_up:
                c.message_free(x[0])
            assert c.compact() > 0
            lines += [[ids[0], best[1].copy(), best[2].copy()], [ids[1], best[1][:15].copy(), best[2][:15].copy()]]
            c.message_free(ids[2])
        calls = [([(0, 0), (1, 75)], x[0], 120, 1) for x in lines] + [([(1, 0)], lines[0][0], 50, 12)]
        ks, vs = list(layer.ks), list(layer.vs)
        for x in lines:
            while len(ks) <= x[0]:
                ks.append(np.zeros((0, h_kv, D)))
                vs.append(np.zeros((0, h_kv, D)))
            ks[x[0]], vs[x[0]] = x[1], x[2]
        q = layer.normal(layer.rows(calls), h_q, D)
        keep, layer.ks, layer.vs = (layer.ks, layer.vs), ks, vs
        out, lse = layer.attend(calls, window, sinks, q)
        compare(dtype, out, lse, *layer.want(calls, window, sinks, q), what=f"step {step}")
        if step in (9, 29):                              # the full attention reads the same cache
            tq, o2, l2 = layer.dev(q), torch.empty_like(out), torch.empty_like(lse)
            c.attend(layer.calls(calls), tq.data_ptr(), o2.data_ptr(), l2.data_ptr())
            torch.cuda.synchronize()
            compare(dtype, o2, l2, *layer.want(calls, 1 << 30, 0, q), what="all")
        layer.ks, layer.vs = keep
    c.close()


def test_captured_streams_are_refused():
    import torch
    from paper_2512_23049_amd.binding import PC_ERR_INVALID_ARG, PcError
    s = Store("bf16", 2, 128, 2048)
    a, z = s.put(40, 1), s.put(50, 2)
    s.cache.message_free(a)
    g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    x = torch.zeros(8, device="cuda:0")
    with torch.cuda.graph(g, stream=st):
        for f in (lambda: s.cache.message_fork([(z, 0, 1, 0, None)], st.cuda_stream), lambda: s.cache.compact(0, st.cuda_stream)):
            with pytest.raises(PcError) as e:
                f()
            assert e.value.code == PC_ERR_INVALID_ARG and "captured" in str(e.value)
        x.add_(1)
    g.replay()
    torch.cuda.synchronize()
    assert (x == 1).all() and s.cache.message_info(z)[1] == 64
    assert s.cache.compact() == 64
    s.cache.close()


@pytest.mark.parametrize("dtype,h_kv,D", TYPES)
def test_many_forks_at_once_and_calls_in_a_row(dtype, h_kv, D):
    """More forks than a kernel's arguments hold, from the same messages, some turned; and calls that follow each other without a wait."""
    s = Store(dtype, h_kv, D, 1 << 16)
    for i, n in enumerate((40, 100, 33)):
        s.put(n, i)
    rng = np.random.default_rng(3)
    whole = [s.message(m) for m in range(3)]
    lens = (40, 100, 33)

    def one():
        m = int(rng.integers(0, 3))
        first = int(rng.integers(0, lens[m]))
        return m, first, int(rng.integers(1, lens[m] - first + 1)), int(rng.integers(0, 60)), None
    batches = [[one() for _ in range(n)] for n in (150, 1, 75, 3, 74, 200, 2)]
    ids = [s.cache.message_fork(b) for b in batches]
    stores = s.read()
    for b, got in zip(batches, ids):
        for (m, first, n, _, _), f in zip(b, got):
            assert s.same(s.message(f, stores), tuple(x[:, first:first + n].contiguous() for x in whole[m]))
    s.cache.close()
