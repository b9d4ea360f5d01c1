"""Long prefills over a PC_MX4 cache on a card that is full but for a few hundred MB: what has no room is refused before anything is written, or served
without the copy."""
import contextlib

import pytest

from pc_inputs import Call

pytestmark = pytest.mark.gpu
MB = 1 << 20


@contextlib.contextmanager
def all_but(left):
    """The card's memory taken, but for so many bytes."""
    import torch
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = []
    try:
        while torch.cuda.mem_get_info()[0] > left + 8 * MB:
            held.append(torch.empty(min(64 << 30, (torch.cuda.mem_get_info()[0] - left) // (4 * MB) * (4 * MB)), dtype=torch.uint8, device="cuda:0"))
        yield
    finally:
        torch.cuda.synchronize()
        held.clear()
        torch.cuda.empty_cache()


def layer(tokens, rows, h_q=64, h_kv=8):
    import torch
    from paper_2512_23049_amd import binding as b
    g = torch.Generator(device="cuda:0").manual_seed(tokens)
    k, v = (torch.randn(tokens, h_kv, 128, generator=g, device="cuda:0").to(torch.bfloat16) for _ in range(2))
    q = torch.randn(rows, h_q, 128, generator=g, device="cuda:0").to(torch.bfloat16)

    def cache():
        c = b.Cache(h_q, h_kv, 128, b.PC_MX4, 10000.0, tokens, 4)
        return c, [Call([(c.append_message(k.data_ptr(), v.data_ptr(), tokens), 0)], -1, tokens, rows, None)]
    return q, torch.full_like(q, 7.0), cache


def attend(c, calls, q, out):
    import torch
    c.attend(calls, q.data_ptr(), out.data_ptr())
    torch.cuda.synchronize()


def test_no_room_for_the_walk_behind_a_copy():
    """The walk over the cache, which follows a long prefill over its copy and does nothing unless it is marked, takes as much as the queries: where there is no
    room for it the call is refused, and its output left as it was."""
    from paper_2512_23049_amd import binding as b
    q, out, cache = layer(2048, 32768)                   # (512 MB of queries)
    first, calls = cache()
    attend(first, calls, q, out)                         # (what the kernels themselves take is there from here on)
    want = out.clone()
    first.close()
    c, calls = cache()
    out.fill_(7)
    with all_but(300 * MB), pytest.raises(b.PcError) as e:           # (torch's own kernels have no room to be loaded there)
        attend(c, calls, q, out)
    assert e.value.code == b.PC_ERR_HIP
    assert (out == 7).all()
    attend(c, calls, q, out)
    assert (out == want).all()
    c.close()


def test_no_room_for_a_copy():
    """A call whose copy has no room is served by the walk over the cache, then and at the next call."""
    q, out, cache = layer(65536, 128)                    # (268 MB of copy, half of it for the walk)
    first, calls = cache()
    attend(first, calls, q, out)
    first.set_key_gather(1)
    attend(first, calls, q, out)
    want = out.clone()
    out.fill_(7)
    first.close()
    c, calls = cache()
    for _ in range(2):
        outs = [out.clone(), out.clone()]
        with all_but(230 * MB):
            for x in outs:
                attend(c, calls, q, x)
        for x in outs:
            assert (x.float() - want.float()).norm() <= 5.8e-3 * want.float().norm()
    c.close()


def test_a_refused_call_behind_others():
    """A batch of short and long calls, of which a later one is refused: it is named by its place in the batch, and nothing has been written."""
    import torch
    from paper_2512_23049_amd import binding as b
    q, out, cache = layer(4096, 1600)
    c, calls = cache()
    msg = calls[0].sel[0][0]
    batch = [Call([(msg, 0)], -1, 4096, 3, None), Call([(msg, 0)], -1, 4096, 1024, None), Call([(msg, 5)], -1, 4200, 1, None), Call([(msg + 1, 0)], -1, 4096, 572, None)]
    with pytest.raises(b.PcError) as e:
        attend(c, batch, q, out)
    torch.cuda.synchronize()
    assert e.value.code == b.PC_ERR_BAD_MSG_ID and "call 3" in str(e.value)
    assert (out == 7).all()
    batch[3] = Call([(msg, 0)], -1, 4096, 572, None)
    attend(c, batch, q, out)
    want = out.clone()
    for first, n, call in ((0, 3, 0), (3, 1024, 1), (1027, 1, 2), (1028, 572, 3)):
        out.fill_(7)
        attend(c, [batch[call]], q[first:first + n], out[first:first + n])
        assert (out[first:first + n].float() - want[first:first + n].float()).norm() <= 5.8e-3 * want[first:first + n].float().norm()
    c.close()
