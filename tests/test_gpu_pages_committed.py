"""A handle's row goes to pages as far as it is committed, also where the host's count is ahead of the device's."""
import numpy as np
import pytest
import torch

import gpu_harness as H
import test_gpu_pages as T
from paper_2601_20357_b200 import binding as TB
from paper_2601_20357_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_positions_that_rounds_on_the_device_rejected_are_not_parked(dtype):
    """Rounds whose drafts are all rejected keep one position each, and the host counts gamma + 1 until it is told."""
    G, heads, d, L, n, cap = 3, 2, 128, 2, 30, 120
    wl = W.Workload(name="pages", config_id=97, drafter=W.DrafterCfg(L, d, heads, heads, 256, 1000, dtype), n_inputs=2, n_requests=1, gamma=G, window_h=4,
                    rounds=1, policy=W.POLICY_STATIC, kv_capacity=cap)
    g = H.make_gpu(wl, TB.weights_to_device(wl.drafter, W.make_weights(wl), T.DEV))
    r = np.random.default_rng(4)
    k, v = (torch.from_numpy(r.standard_normal((L, heads, n, 64)) * 0.5).to(T.DEV, T.TYPES[dtype]).contiguous() for _ in range(2))
    for row in range(2):
        g.load_prefix_kv(row, k, v)
    g.set_pending(T.ints([[5, 0]]), T.ints([1]))
    reject = np.full((1, G + 1, 1000), -30.0, np.float32)
    reject[:, :, 7] = 30.0
    toks, u, a = torch.empty((1, G), dtype=torch.int32, device=T.DEV), torch.full((1, G), 0.5, device=T.DEV), T.ints([0])
    for _ in range(5):
        g.draft_round(u, toks)
        g.verify(H.t(reject), u, u[:, 0].contiguous(), a, a.clone())
        g.update_weights()
    held = int(g.debug_view(TB.VIEW_KV_LEN)[0])
    assert n + 5 <= held < n + 5 * (G + 1)
    c = T.make([], L=L, Hkv=heads, ps=16, hd=64, spare=20, blocks=8, seqs=2)
    p = T.to_gpu(c)
    T.forked(c, p, [0], [0], [0], [cap])
    for start, length in [(0, held + 1), (held, 1), (held - 4, 8), (0, n + 5 * (G + 1))]:
        g.pages_store_row(p, 1, 0, start, length)
        assert p.last_error() == TB.ERR_INVALID_ARG, (start, length)
        T.same(T.from_gpu(p), c)
    g.pages_store_row(p, 1, 0, 0, held)                     # all that is committed
    assert p.last_error() == 0
    g.sync_lengths()                                        # the host knows it now, too
    with pytest.raises(TB.TabedError) as e:
        g.pages_store_row(p, 1, 0, 0, held + 1)
    assert e.value.code == TB.ERR_INVALID_ARG
    g.pages_store_row(p, 1, 0, held - 1, 1)
    assert p.last_error() == 0
    g.destroy()
