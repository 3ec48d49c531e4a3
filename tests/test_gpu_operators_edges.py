"""The serving operators at the edges of what their documentation allows, and what they refuse there."""
import numpy as np
import pytest
import torch

import cache_reference as ref
from test_gpu_operators import A, DEV, model

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------------------------------------------------------------- evict

@pytest.mark.parametrize("room", [12289, 30000, 70000])  # tokens: clusters of two, four and eight CTAs
def test_evict_refuses_one_by_one_across_a_cluster(room):
    """Bad blocks in the part of a table that only one CTA of the cluster looks at, and bad lengths: those sequences are
    left alone and the others are cut."""
    a = A()
    T, D, Hkv, budget, recent = 16, 8, 2, 48, 8
    width = -(-room // T)
    lens = [room, 300, room - 700, -1, 40, width * T + 1, room]
    S = len(lens)
    used = [-(-max(0, min(n, width * T)) // T) for n in lens]
    NB = sum(used) + 1
    g = torch.Generator().manual_seed(room)
    bt = torch.full((S, width), -1, dtype=torch.int32)
    ids, k = torch.randperm(NB, generator=g).to(torch.int32), 0
    for s, n in enumerate(used):
        bt[s, :n] = ids[k:k + n]
        k += n
    good = bt.clone()
    bt[0, used[0] - 1], bt[2, 0] = NB, -1  # the last block of a table, and the first
    layout = a.make_layout(model(2, Hkv, D), 1, NB, T)
    pool = torch.randn(1, NB, Hkv, 2, T, D, generator=g).to(torch.bfloat16)
    scores = torch.randn(1, NB, Hkv, T, generator=g)
    dpool, dscores, dbt = pool.to(DEV), scores.to(DEV), bt.to(DEV)
    dlens, new = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (lens, [99] * S))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.full((a.amoeba_evict_workspace_bytes(layout, 1, S, budget),), 0x7F, dtype=torch.uint8, device=DEV)
    a.amoeba_evict_kv(layout, 0, 1, [dpool], [dscores], dbt, dlens, dbt, budget, recent, new, status, ws)
    assert new.tolist() == [-1, budget, -1, -1, 40, -1, budget]
    assert int(status.item()) in (a.ERR_BAD_BLOCK_ID, a.ERR_INVALID_ARG)
    want, ws = pool.clone(), scores.clone()
    for s in (1, 6):
        n, b = lens[s], good[s].long()
        i = torch.arange(n)
        x = scores[0, b[i // T], :, i % T].numpy()
        for h in range(Hkv):
            f, j = torch.from_numpy(ref.kept(x[:, h].astype(np.float64), n, budget, recent)), torch.arange(budget)
            want[0, b[j // T], h, :, j % T] = pool[0, b[f // T], h, :, f % T]
            ws[0, b[j // T], h, j % T] = scores[0, b[f // T], h, f % T]
    assert torch.equal(dpool.cpu(), want) and torch.equal(dscores.cpu(), ws)
