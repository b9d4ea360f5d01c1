"""Which way a batch of single tokens goes by itself: told by its bits (no sum depends on anything but the way and the calls)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


# calls over `pick` of `pool` messages; shared or not as measured on both sides (see plan_shared)
@pytest.mark.parametrize("h_q,h_kv,pool,pick,tokens,window,n_calls,together", [
    (64, 8, 512, 410, 160, 16384, 8, False), (64, 8, 512, 410, 160, 16384, 32, True), (32, 8, 512, 410, 160, 16384, 32, True),
    (16, 2, 512, 410, 160, 16384, 32, False), (16, 2, 512, 410, 160, 16384, 64, False), (4, 1, 512, 410, 160, 16384, 64, False),
    (16, 2, 48, 24, 160, 4096, 64, False), (64, 8, 48, 24, 160, 4096, 64, True)])
def test_the_way_a_batch_goes(h_q, h_kv, pool, pick, tokens, window, n_calls, together):
    import torch
    from paper_2512_23049_amd import binding
    from pc_inputs import Call
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    cache = binding.Cache(h_q, h_kv, 128, binding.PC_BF16, 1e4, pool * (tokens + 31) // 32 * 32 + 64, pool + 8, max_position=1 << 20)
    k, v = (torch.randn(pool * tokens, h_kv, 128, generator=g, device="cuda:0").bfloat16() for _ in range(2))
    for m in range(pool):
        cache.append_message(k[m * tokens:].data_ptr(), v[m * tokens:].data_ptr(), tokens)
    rng, calls = np.random.default_rng(3), []
    for _ in range(n_calls):
        order = rng.permutation(pool)[:pick]
        calls.append(Call([(int(m), tokens * i) for i, m in enumerate(order)], -1, tokens * pick, 1, None))
    q = torch.randn(n_calls, h_q, 128, generator=g, device="cuda:0").bfloat16()
    out = []
    for mode in (0, 1, 2):
        cache.set_decode_sharing(mode)
        o = torch.empty_like(q)
        cache.attend_window(calls, window, 4, q.data_ptr(), o.data_ptr())
        torch.cuda.synchronize()
        out.append(o)
    assert not torch.equal(out[1], out[2])               # (the ways differ in their last bits)
    assert torch.equal(out[0], out[2 if together else 1])
    cache.close()
