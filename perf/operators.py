"""Windowed attention over choreographed messages, and the cache's own copies, as cases that can be timed and compared.

A case is a plain dict: the shape of the attention layer, how the cache is laid out and what one pass asks for.

  decode   parallel generations in a layer with a sliding window: the attention of one query row for each call
  prefill  the attention of one or more new messages in such a layer
  train    a prefill that keeps the log-sum-exp, zeroed gradients, the gradient, the turn of the keys' gradient, and
           gradients in the type of what they are the gradients of
  fork     branches of cached messages: part of a message copied into a new one (which is given back at the end, as a
           branch that was not taken), its keys turned to another position or as they are
  beams    one step of a search: the survivors are forked, the others freed, and the cache closes up
  roll     a cache that is full: its oldest messages are freed, it closes up, and as many new ones are appended

A key is visible to a row if the row's call lists it (own tokens: up to the row's own one) and its position is above the
row's position less the window, or if it is one of the first `sinks` tokens of the call's list.  Layouts follow from the
case; K, V, Q and the output gradients, N(0,1) like in this repository's workloads, from the seed.
"""
import math

import numpy as np
import torch

own = False                            # False: the plain forms; True: the framework's calls

DEV = "cuda:0"
IDS = 1 << 22                          # a message id is never given out twice: room for the messages of many passes
ALIGN = 32                             # messages start on such slots


# ------------------------------------------------------------------------------------------------------- the cases
def _b8(**kw):                         # 8B-shaped attention
    return dict(heads=32, kv_heads=8, dim=128, dtype="bf16", theta=500000.0, **kw)


def _b70(**kw):                        # 70B-shaped attention
    return dict(heads=64, kv_heads=8, dim=128, dtype="bf16", theta=500000.0, **kw)


def listed():
    return [
        # a few agents generate after a short common prompt: launches and host work count
        _b8(name="decode_few", kind="decode", layout=11, window=512, sinks=4, shared=300, pool=16, len_lo=40, len_hi=300, n_sel=3, n_calls=4, tail=17),
        # the parallel decode workload in a windowed layer: a system message, 8 of 512 pool messages and a tail per call
        _b8(name="decode_parallel", kind="decode", layout=12, window=1024, sinks=4, shared=2048, pool=512, len_lo=128, len_hi=512, n_sel=8, n_calls=64, tail=64),
        # long-context generation: 32 calls over about 64k tokens each, a wide window
        _b70(name="decode_long", kind="decode", layout=13, window=16384, sinks=64, shared=0, pool=512, len_lo=64, len_hi=256, n_sel=410, n_calls=32, tail=1),
        # a short ragged message after a few others: the small everyday prefill
        _b8(name="prefill_short", kind="prefill", layout=21, window=256, sinks=1, pool=12, len_lo=30, len_hi=400, n_sel=5, n_new=1, new_lo=77, new_hi=77),
        # a long document read in one call
        _b8(name="prefill_long", kind="prefill", layout=22, window=4096, sinks=4, pool=16, len_lo=64, len_hi=1024, n_sel=8, n_new=1, new_lo=8192, new_hi=8192),
        # reference precision, sizes that fill no tile
        dict(name="prefill_fp32", kind="prefill", heads=8, kv_heads=2, dim=64, dtype="f32", theta=10000.0, layout=23, window=333, sinks=0, pool=24, len_lo=17,
             len_hi=300, n_sel=6, n_new=2, new_lo=100, new_hi=501),
        # fine-tuning on a workflow trace: four new messages over shared cached ones
        _b8(name="train_bf16", kind="train", layout=31, window=512, sinks=4, pool=16, len_lo=64, len_hi=512, n_sel=7, n_new=4, new_lo=150, new_hi=320),
        # the same at reference precision
        dict(name="train_fp32", kind="train", heads=8, kv_heads=2, dim=64, dtype="f32", theta=10000.0, layout=32, window=100, sinks=3, pool=10, len_lo=20,
             len_hi=200, n_sel=5, n_new=2, new_lo=50, new_hi=110),
        # one answer is taken up again from its middle
        _b8(name="fork_one", kind="fork", layout=41, pool=4, len_lo=200, len_hi=700, n_forks=1, turned=False),
        # branches of cached messages, each of which goes on at a position of its own
        _b8(name="fork_branches", kind="fork", layout=42, pool=8, len_lo=1500, len_hi=2500, n_forks=32, turned=True),
        # a search with 64 beams of which 16 survive
        _b8(name="beams", kind="beams", layout=51, beams=64, survivors=16, len_lo=300, len_hi=900),
        # a full cache: the two oldest of 512 messages leave
        _b8(name="roll", kind="roll", layout=52, pool=512, len_lo=64, len_hi=256, leaving=2),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))
    layout = rng.randrange(1000, 1 << 30)
    lo = log(16, 200)
    lens = dict(layout=layout, len_lo=lo, len_hi=lo + log(8, 800))
    mid = (lens["len_lo"] + lens["len_hi"]) // 2

    def history(most, pool_most=512):                    # how many messages a call lists for about that many tokens, of how many
        n_sel = max(1, min(pool_most // 2, log(min(50, most), most) // mid))
        return dict(n_sel=n_sel, pool=min(pool_most, n_sel + log(1, 3 * n_sel + 8)), **lens)
    shape = rng.choice((_b8, _b70))
    f32 = dict(dtype="f32", theta=10000.0, kv_heads=rng.choice((2, 4)), heads=rng.choice((4, 8, 16)), dim=rng.choice((64, 128)))
    kind = rng.choice(("decode", "decode", "prefill", "prefill", "train", "fork", "beams", "roll"))
    seen = dict(window=log(1, 8192), sinks=rng.choice((0, 1, 4, log(1, 100))))
    exact32 = rng.random() < 0.3
    if kind == "decode":
        calls = log(1, 64)
        kw = dict(kind=kind, shared=rng.choice((0, log(64, 2048))), n_calls=calls, tail=log(1, 200), **seen, **history(min(32768, 400000 // calls)))
        return dict(f32, **kw) if exact32 else shape(**kw)
    if kind == "prefill":
        n_new = rng.choice((1, 1, 2, log(2, 8)))
        new = log(2, max(4, (700 if exact32 else 4096) // n_new))
        kw = dict(kind=kind, n_new=n_new, new_lo=max(2, new // 2), new_hi=new, **seen, **history(2000 if exact32 else 6000, 64))
        return dict(f32, **kw) if exact32 else shape(**kw)
    if kind == "train":
        n_new = rng.randint(1, 4)
        new = log(8, 160 if exact32 else 700)
        kw = dict(kind=kind, n_new=n_new, new_lo=max(4, new // 2), new_hi=new, **seen, **history(600 if exact32 else 3000, 32))
        return dict(f32, **kw) if exact32 else _b8(**kw)
    if kind == "fork":
        n = log(1, 64)
        top = max(8, log(8, 60000 // n))
        kw = dict(kind=kind, layout=layout, pool=rng.randint(1, 16), len_lo=max(2, top // 3), len_hi=top, n_forks=n, turned=rng.random() < 0.6)
    elif kind == "beams":
        n = log(4, 96)
        top = log(8, 1200)
        kw = dict(kind=kind, layout=layout, beams=n, survivors=rng.randint(1, max(1, n // 3)), len_lo=max(2, top // 3), len_hi=top)
    else:
        n = log(4, 512)
        kw = dict(kind=kind, layout=layout, pool=n, leaving=rng.randint(1, max(1, n // 4)), len_lo=lo, len_hi=lo + log(8, 200))
    return dict(f32, **kw) if exact32 else shape(**kw)


# ------------------------------------------------------------------------------------------------------ the layouts
def _room(n):
    return (n + ALIGN - 1) // ALIGN * ALIGN


def _attention_layout(case):
    """(message lengths, cached ones first; calls: (list of (message, start), own message, its start, query rows))."""
    r = np.random.default_rng(case["layout"])
    lens = [int(x) for x in r.integers(case["len_lo"], case["len_hi"] + 1, size=case["pool"])]
    first = 1 if case.get("shared", 0) > 0 else 0
    if first:
        lens.insert(0, case["shared"])
    decode = case["kind"] == "decode"
    new = [case["tail"]] * case["n_calls"] if decode else [int(x) for x in r.integers(case["new_lo"], case["new_hi"] + 1, size=case["n_new"])]
    overlap, calls = case["n_sel"] > 64, []
    for c, n in enumerate(new):
        sel, at = ([(0, 0)], lens[0]) if first else ([], 0)
        for i in r.permutation(case["pool"])[:case["n_sel"]]:
            m = int(i) + first
            at += -int(r.integers(0, min(32, lens[m]) // 2 + 1)) if overlap else int(r.integers(0, 33))     # overlapping, or with gaps
            at = max(at, 0)
            sel.append((m, at))
            at += lens[m]
        calls.append((sel, len(lens) + c, at, 1 if decode else n))
    return lens + new, calls


def _fork_layout(case):
    """(message lengths, forks: (message, first token, tokens, base or None))."""
    r = np.random.default_rng(case["layout"])
    lens = [int(x) for x in r.integers(case["len_lo"], case["len_hi"] + 1, size=case["pool"])]
    forks = []
    for _ in range(case["n_forks"]):
        m = int(r.integers(0, len(lens)))
        first = int(r.integers(0, lens[m] // 4 + 1))
        n = int(r.integers(max(1, (lens[m] - first) * 3 // 4), lens[m] - first + 1))
        forks.append((m, first, n, int(r.integers(-4000, 4001)) if case["turned"] else None))
    return lens, forks


def _beams_layout(case):
    """(lengths of the lines, line of each beam, the beams that survive, line of each fork).  The step leaves what it found:
    survivor j is a beam of line j, and behind the survivors come the forks, in whose places the next step's survivors are."""
    r = np.random.default_rng(case["layout"])
    n, s = case["beams"], case["survivors"]
    lens = [int(x) for x in r.integers(case["len_lo"], case["len_hi"] + 1, size=s)]
    keep = [0] + sorted(int(x) for x in r.choice(np.arange(s, n), size=s - 1, replace=False)) if s > 1 else [0]
    forks = [int(x) for x in r.integers(0, s, size=n - s)]
    for j, at in enumerate(keep):
        if at >= s:
            forks[at - s] = j
    return lens, list(range(s)) + forks, keep, forks


def _roll_lens(case):
    r = np.random.default_rng(case["layout"])
    return [int(x) for x in r.integers(case["len_lo"], case["len_hi"] + 1, size=case["pool"])]


def _starts(lens):
    return np.concatenate([[0], np.cumsum([_room(n) for n in lens])]).astype(np.int64)


def _pairs(case, lens, calls):
    """Visible (row, key) pairs of the calls, and the tokens that some row sees (cached tokens of several calls once)."""
    total, seen = 0, [np.zeros(n, dtype=bool) for n in lens]
    for sel, me, start, n_q in calls:
        p = start + lens[me] - n_q + np.arange(n_q)
        at = 0
        for m, s in sel + [(me, start)]:
            t = np.arange(lens[m])
            up = p - start if m == me and s == start else np.full(n_q, lens[m] - 1)      # the last token a row may see
            low = np.clip(p - case["window"] + 1 - s, 0, lens[m])
            sinks = min(max(case["sinks"] - at, 0), lens[m])
            n_low = np.minimum(low, up + 1)
            total += int(np.sum(up + 1 - n_low + np.minimum(sinks, n_low)))
            seen[m] |= (t >= low.min()) & (t <= up.max()) | (t < sinks) & (t <= up.max())
            at += lens[m]
    return total, int(sum(x.sum() for x in seen))


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    kv = 2 * case["kv_heads"] * case["dim"] * es                                   # one token's K and V
    if case["kind"] in ("decode", "prefill", "train"):
        lens, calls = _attention_layout(case)
        pairs, seen = _pairs(case, lens, calls)
        rows = sum(c[3] for c in calls)
        row = case["heads"] * case["dim"] * es                                     # one query or output row
        by, fl = kv * seen + 2 * row * rows, 4 * case["dim"] * case["heads"] * pairs
        if case["kind"] == "train":                                                # S, dP, dQ, dK, dV besides the forward; dO, dQ, and a gradient for every slot
            fl += 10 * case["dim"] * case["heads"] * pairs
            by += 2 * row * rows + kv * sum(_room(n) for n in lens)
        return {"bytes": by, "flops": fl}
    if case["kind"] == "fork":
        lens, forks = _fork_layout(case)
        used = [np.zeros(n, dtype=bool) for n in lens]
        for m, first, n, _ in forks:
            used[m][first:first + n] = True
        out = sum(n for _, _, n, _ in forks)
        return {"bytes": kv * (int(sum(u.sum() for u in used)) + out), "flops": 3 * case["kv_heads"] * case["dim"] * out if case["turned"] else 0}
    if case["kind"] == "beams":
        lens, line, keep, forks = _beams_layout(case)
        read = sum(lens)                                                           # a fork's tokens are read from their line once, and written in their final place;
        moved = sum(lens[j] for j, at in enumerate(keep) if at != j)               # the survivors behind the first freed beam move there too
        return {"bytes": kv * (read + moved + sum(lens[j] for j in forks)), "flops": 0}
    lens = _roll_lens(case)
    gone = sum(lens[:case["leaving"]])
    return {"bytes": 2 * kv * sum(lens), "flops": 3 * case["kv_heads"] * case["dim"] * gone}


# ------------------------------------------------------------------------------------------------------- the inputs
class _State:
    pass


def _normal(g, dt, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dt)


def _inputs(case, seed):
    """The tensors of a case, from the seed alone; k, v: every message on slots of its own, [slots, kv_heads, dim]."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    s = _State()
    s.case, s.dt = case, torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    kind = case["kind"]
    if kind in ("decode", "prefill", "train"):
        s.lens, s.calls = _attention_layout(case)
    elif kind == "fork":
        s.lens, s.forks = _fork_layout(case)
    elif kind == "beams":
        s.lens = _beams_layout(case)[0]                  # (k, v: one message for each line)
    else:
        s.lens = _roll_lens(case)
    s.starts = _starts(s.lens)
    n, H, D = int(s.starts[-1]), case["kv_heads"], case["dim"]
    there = np.zeros(n, dtype=bool)
    for a, length in zip(s.starts, s.lens):
        there[a:a + length] = True
    there = torch.from_numpy(there).to(DEV)[:, None, None]
    s.k, s.v = _normal(g, s.dt, n, H, D) * there, _normal(g, s.dt, n, H, D) * there
    if kind in ("decode", "prefill", "train"):
        s.rows = sum(c[3] for c in s.calls)
        s.q = _normal(g, s.dt, s.rows, case["heads"], D)
        if kind == "train":
            s.d_out = _normal(g, s.dt, s.rows, case["heads"], D)
    return s


def _ptrs(t, starts, lens):
    return [t[a:a + n].data_ptr() for a, n in zip(starts, lens)]


def prepare(case, seed):
    s = _inputs(case, seed)
    attention = case["kind"] in ("decode", "prefill", "train")
    if own:
        _cache(s)
        if attention:
            _batch(s)
    elif attention:
        _padded(s)
    else:
        _plain_cache(s)
    torch.cuda.synchronize()
    return s


def run(s):
    kind = s.case["kind"]
    if kind in ("decode", "prefill"):
        return _own_attention(s) if own else _plain_attention(s)
    if kind == "train":
        return _own_train(s) if own else _plain_train(s)
    if kind == "fork":
        return _own_fork(s) if own else _plain_fork(s)
    if kind == "beams":
        return _own_beams(s) if own else _plain_beams(s)
    return _own_roll(s) if own else _plain_roll(s)


# -------------------------------------------------------------------------------------------- the framework's calls
def _cache(s):
    from paper_2512_23049_amd.binding import PC_BF16, PC_F32, Cache
    case, kind = s.case, s.case["kind"]
    H, D, es = case["kv_heads"], case["dim"], s.k.element_size()
    heads = case.get("heads", H)
    order = list(range(len(s.lens)))
    cap = int(s.starts[-1])
    if kind == "fork":
        cap += sum(_room(n) for _, _, n, _ in s.forks)
    elif kind == "beams":
        order = _beams_layout(case)[1]
        cap = 2 * sum(_room(s.lens[j]) for j in order)
    attention = kind in ("decode", "prefill", "train")
    s.arena = torch.empty(2 * cap * H * D * es, dtype=torch.uint8, device=DEV)
    s.cache = Cache(heads, H, D, PC_BF16 if s.dt == torch.bfloat16 else PC_F32, case["theta"], cap, len(s.lens) + 8 if attention else IDS,
                    arena=s.arena.data_ptr(), arena_bytes=s.arena.numel())
    s.ids = []
    for i in range(0, len(order), 64):
        part = order[i:i + 64]
        s.ids += s.cache.append_messages(_ptrs(s.k, s.starts[part], [s.lens[j] for j in part]), _ptrs(s.v, s.starts[part], [s.lens[j] for j in part]),
                                         [s.lens[j] for j in part])
        torch.cuda.synchronize()
    half = s.arena.numel() // 2
    s.k_store = s.arena[:half].view(s.dt).view(H, cap, D)
    if s.dt == torch.bfloat16:                           # values: groups of eight tokens, by dimension
        s.v_store = s.arena[half:].view(s.dt).view(H, cap // 8, D, 8).permute(0, 1, 3, 2)
    else:
        s.v_store = s.arena[half:].view(s.dt).view(H, cap // 8, 8, D)


class _Call:
    def __init__(self, sel, self_msg, self_start, n_q):
        self.sel, self.self_msg, self.self_start, self.n_q, self.q_pos = sel, self_msg, self_start, n_q, None


def _batch(s):
    from paper_2512_23049_amd.binding import marshal_calls
    s.batch = [_Call(*c) for c in s.calls]
    s.marshalled = marshal_calls(s.batch)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty(s.q.shape[:2], dtype=torch.float32, device=DEV)
    if s.case["kind"] == "train":
        s.d_q = torch.empty(s.q.shape, dtype=torch.float32, device=DEV)
        s.d_k = torch.empty(s.k.shape, dtype=torch.float32, device=DEV)
        s.d_v = torch.empty_like(s.d_k)


def _own_attention(s):
    exact32 = s.dt == torch.float32
    s.cache.attend_window(s.batch, s.case["window"], s.case["sinks"], s.q.data_ptr(), s.out.data_ptr(), s.lse.data_ptr() if exact32 else 0,
                          marshalled=s.marshalled)
    return [s.out, s.lse] if exact32 else [s.out]


def _own_train(s):
    c, w, n = s.cache, s.case["window"], s.case["sinks"]
    c.attend_window(s.batch, w, n, s.q.data_ptr(), s.out.data_ptr(), s.lse.data_ptr(), marshalled=s.marshalled)
    s.d_k.zero_()
    s.d_v.zero_()
    c.attend_window_backward(s.batch, w, n, s.q.data_ptr(), s.out.data_ptr(), s.lse.data_ptr(), s.d_out.data_ptr(), s.d_q.data_ptr(), s.d_k.data_ptr(),
                             s.d_v.data_ptr(), marshalled=s.marshalled)
    c.grad_keys_finalize(s.d_k.data_ptr())
    return [s.out, s.d_q.to(s.dt), s.d_k.to(s.dt), s.d_v.to(s.dt)]


def _own_fork(s):
    ids = s.cache.message_fork([(s.ids[m], first, n, 0, base) for m, first, n, base in s.forks])
    for m in ids:
        s.cache.message_free(m)
    a = int(s.starts[-1])
    return [s.k_store[:, a:], s.v_store[:, a // 8:]]


def _own_beams(s):
    _, line, keep, forks = _beams_layout(s.case)
    kept = [s.ids[at] for at in keep]
    ids = s.cache.message_fork([(kept[j], 0, s.lens[j], 0, None) for j in forks])
    for at in set(range(len(line))) - set(keep):
        s.cache.message_free(s.ids[at])
    s.cache.compact()
    s.ids = kept + ids
    n = sum(_room(s.lens[j]) for j in line)
    return [s.k_store[:, :n], s.v_store[:, :n // 8]]


def _own_roll(s):
    n = s.case["leaving"]
    for m in s.ids[:n]:
        s.cache.message_free(m)
    s.cache.compact()
    if not hasattr(s, "order"):
        s.order = list(range(len(s.lens)))
    back = s.order[:n]
    ids = s.cache.append_messages(_ptrs(s.k, s.starts[back], [s.lens[j] for j in back]), _ptrs(s.v, s.starts[back], [s.lens[j] for j in back]),
                                  [s.lens[j] for j in back])
    s.order, s.ids = s.order[n:] + back, s.ids[n:] + ids
    return [s.k_store, s.v_store]


# --------------------------------------------------------------------------------------------------- the plain forms
def _turn(x, pos, theta):
    """Pairs (i, i + D/2) of x [..., heads, D] turned by pos [...] theta^(-2i/D); angles in 64 bits."""
    D = x.shape[-1]
    freq = torch.arange(D // 2, device=x.device, dtype=torch.float64) * (-2.0 / D) * math.log(theta)
    angle = pos.double()[..., None, None] * freq.exp()
    cos, sin = angle.cos().float(), angle.sin().float()
    lo, hi = x[..., :D // 2].float(), x[..., D // 2:].float()
    return torch.cat([lo * cos - hi * sin, lo * sin + hi * cos], dim=-1)


def _padded(s):
    """Calls side by side, padded to the longest: slots and positions of the listed tokens, of the query rows, and what
    the mask needs.  (A token that is not there: slot 0, order beyond every row's limit.)"""
    case, lens, calls = s.case, s.lens, s.calls
    C, R = len(calls), max(c[3] for c in calls)
    N = max(sum(lens[m] for m, _ in c[0]) + lens[c[1]] for c in calls)
    slot, pos, order = np.zeros((C, N), np.int64), np.zeros((C, N), np.int64), np.full((C, N), 1 << 30, np.int64)
    q_row, q_pos, limit = np.zeros((C, R), np.int64), np.zeros((C, R), np.int64), np.full((C, R), -1, np.int64)
    packed, row0 = np.zeros(s.rows, np.int64), 0
    for c, (sel, me, start, n_q) in enumerate(calls):
        n = 0
        for m, at in sel + [(me, start)]:
            slot[c, n:n + lens[m]] = s.starts[m] + np.arange(lens[m])
            pos[c, n:n + lens[m]] = at + np.arange(lens[m])
            n += lens[m]
        order[c, :n] = np.arange(n)
        q_row[c, :n_q] = row0 + np.arange(n_q)
        q_pos[c, :n_q] = start + lens[me] - n_q + np.arange(n_q)
        limit[c, :n_q] = n - n_q + np.arange(n_q)        # the row's own token, in list order
        packed[row0:row0 + n_q] = c * R + np.arange(n_q)
        row0 += n_q
    for name, x in (("slot", slot), ("pos", pos), ("order", order), ("q_row", q_row), ("q_pos", q_pos), ("limit", limit), ("packed", packed)):
        setattr(s, name, torch.from_numpy(x).to(DEV))


def _scores(s):
    """(queries [C, Hkv, g R, D] and keys [C, Hkv, N, D] at their positions, values, probabilities, log-sum-exp)."""
    case = s.case
    Hq, H, D = case["heads"], case["kv_heads"], case["dim"]
    g, (C, R), N = Hq // H, s.q_row.shape, s.slot.shape[1]
    q = _turn(s.q[s.q_row], s.q_pos, case["theta"]).reshape(C, R, H, g, D).permute(0, 2, 3, 1, 4).reshape(C, H, g * R, D)
    k = _turn(s.k[s.slot], s.pos, case["theta"]).permute(0, 2, 1, 3).contiguous()
    v = s.v[s.slot].float().permute(0, 2, 1, 3).contiguous()
    sees = (s.order[:, None] <= s.limit[..., None]) & ((s.pos[:, None] > s.q_pos[..., None] - case["window"]) | (s.order[:, None] < case["sinks"]))
    x = torch.matmul(q, k.transpose(2, 3)).reshape(C, H, g, R, N) * D ** -0.5
    x = x.masked_fill(~sees[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x = (x - top).exp()
    total = x.sum(-1, keepdim=True)
    p = (x / total.clamp_min(1e-38)).reshape(C, H, g * R, N)
    return q, k, v, p, (top + total.log()).reshape(C, H, g, R)


def _by_row(s, x):
    """[C, Hkv, g R, D] as packed rows [rows, Hq, D]."""
    C, H, gR, D = x.shape
    R = s.q_row.shape[1]
    return x.reshape(C, H, gR // R, R, D).permute(0, 3, 1, 2, 4).reshape(C * R, H * (gR // R), D)[s.packed]


def _plain_attention(s):
    _, _, v, p, lse = _scores(s)
    out = _by_row(s, torch.matmul(p, v)).to(s.dt)
    if s.dt != torch.float32:
        return [out]
    return [out, lse.permute(0, 3, 1, 2).reshape(-1, s.case["heads"])[s.packed]]


def _plain_train(s):
    case = s.case
    H, D, R = case["kv_heads"], case["dim"], s.q_row.shape[1]
    q, k, v, p, _ = _scores(s)
    o = torch.matmul(p, v)
    d_o = s.d_out[s.q_row].float() * (s.limit >= 0)[..., None, None]
    d_o = d_o.reshape(*s.q_row.shape, H, -1, D).permute(0, 2, 3, 1, 4).reshape(o.shape)
    d_s = p * (torch.matmul(d_o, v.transpose(2, 3)) - (d_o * o).sum(-1, keepdim=True)) * D ** -0.5
    d_q = torch.matmul(d_s, k)
    d_k = torch.matmul(d_s.transpose(2, 3).contiguous(), q).permute(0, 2, 1, 3)
    d_v = torch.matmul(p.transpose(2, 3).contiguous(), d_o).permute(0, 2, 1, 3)
    d_q = _turn(_by_row(s, d_q), -s.q_pos.reshape(-1)[s.packed], case["theta"])
    d_k = _turn(d_k, -s.pos, case["theta"])
    there = (s.order < 1 << 30).reshape(-1)
    at = s.slot.reshape(-1)[there]
    sums = [torch.zeros(s.k.shape, dtype=torch.float32, device=DEV).index_add_(0, at, x.reshape(-1, H, D)[there]) for x in (d_k, d_v)]
    return [_by_row(s, o).to(s.dt), d_q.to(s.dt), sums[0].to(s.dt), sums[1].to(s.dt)]


def _plain_cache(s):
    """Keys, turned to their place in the message, and values, [kv_heads, slots, dim]; messages one after the other."""
    case, kind = s.case, s.case["kind"]
    s.place = torch.from_numpy(np.concatenate([np.arange(_room(n)) for n in s.lens])).to(DEV)
    stored = _turn(s.k, s.place, case["theta"]).to(s.dt).permute(1, 0, 2)
    values = s.v.permute(1, 0, 2)
    at = torch.arange(stored.shape[1], device=DEV)
    s.extra = 0
    if kind == "fork":
        s.extra = sum(_room(n) for _, _, n, _ in s.forks)
    elif kind == "beams":
        at = _slots(s, _beams_layout(case)[1])
    else:
        s.order = list(range(len(s.lens)))
    s.k_store = torch.cat([stored[:, at], stored.new_zeros(stored.shape[0], s.extra, stored.shape[2])], 1)
    s.v_store = torch.cat([values[:, at], values.new_zeros(values.shape[0], s.extra, values.shape[2])], 1)


def _slots(s, order):
    """Slots (of the inputs) of whole messages in that order."""
    return torch.from_numpy(np.concatenate([np.arange(s.starts[j], s.starts[j + 1]) for j in order])).to(DEV)


def _groups(v):
    return v.reshape(v.shape[0], -1, 8, v.shape[2])


def _plain_fork(s):
    src, there, by = [], [], []
    for m, first, n, base in s.forks:
        src.append(np.concatenate([s.starts[m] + first + np.arange(n), np.zeros(_room(n) - n, np.int64)]))
        there.append(np.arange(_room(n)) < n)
        by.append(np.full(_room(n), 0 if base is None else base - first))
    src, there, by = (torch.from_numpy(np.concatenate(x)).to(DEV) for x in (src, there, by))
    k, v = s.k_store[:, src] * there[:, None], s.v_store[:, src] * there[:, None]
    if s.case["turned"]:
        k = _turn(k.permute(1, 0, 2), by, s.case["theta"]).to(s.dt).permute(1, 0, 2)
    a = int(s.starts[-1])
    s.k_store[:, a:] = k
    s.v_store[:, a:] = v
    return [s.k_store[:, a:], _groups(s.v_store[:, a:])]


def _plain_beams(s):
    _, line, keep, forks = _beams_layout(s.case)
    first = np.concatenate([[0], np.cumsum([_room(s.lens[j]) for j in line])])
    src = [np.arange(first[at], first[at + 1]) for at in keep]
    src = torch.from_numpy(np.concatenate(src + [src[j] for j in forks])).to(DEV)
    n = src.numel()
    s.k_store[:, :n] = s.k_store[:, src]
    s.v_store[:, :n] = s.v_store[:, src]
    return [s.k_store[:, :n], _groups(s.v_store[:, :n])]


def _plain_roll(s):
    n = s.case["leaving"]
    gone = s.order[:n]
    off = sum(_room(s.lens[j]) for j in gone)
    s.k_store[:, :-off] = s.k_store[:, off:].clone()
    s.v_store[:, :-off] = s.v_store[:, off:].clone()
    at = _slots(s, gone)
    s.k_store[:, -off:] = _turn(s.k[at], s.place[at], s.case["theta"]).to(s.dt).permute(1, 0, 2)
    s.v_store[:, -off:] = s.v[at].permute(1, 0, 2)
    s.order = s.order[n:] + gone
    return [s.k_store, _groups(s.v_store)]


# ------------------------------------------------------------------------------------------------ in 64 bits, apart
def _spin(x, pos, theta):
    """The same turn as a product of complex numbers; x [tokens, heads, D], pos: one for each token."""
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half].double(), x[..., half:].double())
    rate = torch.tensor([theta ** (-i / half) for i in range(half)], dtype=torch.float64, device=x.device)
    angle = torch.as_tensor(pos, dtype=torch.float64, device=x.device).reshape(-1, 1, 1) * rate
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    s = _inputs(case, seed)
    kind, theta = case["kind"], case["theta"]
    if kind in ("decode", "prefill", "train"):
        return _exact_attention(s)
    if kind == "fork":
        k, v = [], []
        for m, first, n, base in s.forks:
            a = int(s.starts[m]) + first
            start = first if base is None else base
            pad = (0, 0, 0, 0, 0, _room(n) - n)
            k.append(torch.nn.functional.pad(_spin(s.k[a:a + n], np.arange(start, start + n), theta), pad))
            v.append(torch.nn.functional.pad(s.v[a:a + n].double(), pad))
    else:
        order = _beams_layout(case)[1] if kind == "beams" else list(range(case["leaving"], case["pool"])) + list(range(case["leaving"]))
        lines = [(_spin(s.k[a:b], np.arange(b - a), theta), s.v[a:b].double()) for a, b in ((int(s.starts[j]), int(s.starts[j + 1])) for j in range(len(s.lens)))]
        k, v = [lines[j][0] for j in order], [lines[j][1] for j in order]
    return [torch.cat(k).transpose(0, 1), torch.cat(v).transpose(0, 1).unflatten(1, (-1, 8))]


def _exact_attention(s):
    """Call by call and head by head."""
    case = s.case
    Hq, H, D, theta = case["heads"], case["kv_heads"], case["dim"], case["theta"]
    out = torch.zeros(s.rows, Hq, D, dtype=torch.float64, device=DEV)
    lse = torch.full((s.rows, Hq), -math.inf, dtype=torch.float64, device=DEV)
    d_q = torch.zeros_like(out)
    d_k, d_v = torch.zeros(s.k.shape, dtype=torch.float64, device=DEV), torch.zeros(s.k.shape, dtype=torch.float64, device=DEV)
    at = 0
    for sel, me, start, n_q in s.calls:
        parts = [(int(s.starts[m]), s.lens[m], p) for m, p in sel + [(me, start)]]
        pos = np.concatenate([p + np.arange(n) for _, n, p in parts])
        k = _spin(torch.cat([s.k[a:a + n] for a, n, _ in parts]), pos, theta)
        v = torch.cat([s.v[a:a + n] for a, n, _ in parts]).double()
        n_kv = len(pos)
        mine = np.arange(n_kv - n_q, n_kv)
        q = _spin(s.q[at:at + n_q], pos[mine], theta)
        row, col = torch.from_numpy(mine).to(DEV)[:, None], torch.arange(n_kv, device=DEV)[None]
        where = torch.from_numpy(pos).to(DEV)
        hidden = (col > row) | ((where[None] <= where[mine][:, None] - case["window"]) & (col >= case["sinks"]))
        d_rot = torch.zeros_like(k)
        for h in range(Hq):
            kh = h // (Hq // H)
            x = torch.where(hidden, -math.inf, q[:, h] @ k[:, kh].T / math.sqrt(D))
            lse[at:at + n_q, h] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            out[at:at + n_q, h] = p @ v[:, kh]
            if case["kind"] == "train":
                d_o = s.d_out[at:at + n_q, h].double()
                d_p = d_o @ v[:, kh].T
                d_x = p * (d_p - (p * d_p).sum(1, keepdim=True)) / math.sqrt(D)
                d_q[at:at + n_q, h] = d_x @ k[:, kh]
                d_rot[:, kh] += d_x.T @ q[:, h]
                first = 0
                d_val = p.T @ d_o
                for a, n, _ in parts:
                    d_v[a:a + n, kh] += d_val[first:first + n]
                    first += n
        if case["kind"] == "train":
            d_q[at:at + n_q] = _spin(d_q[at:at + n_q], -pos[mine], theta)
            d_rot, first = _spin(d_rot, -pos, theta), 0
            for a, n, _ in parts:
                d_k[a:a + n] += d_rot[first:first + n]
                first += n
        at += n_q
    if case["kind"] == "train":
        return [out, d_q, d_k, d_v]
    return [out] if s.dt != torch.float32 else [out, lse]
