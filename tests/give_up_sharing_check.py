"""Run against the checked build of the library: attention with shared prefixes and block copies with waits that run out after a few polls.
Every call returns, reports the timeout, and leaves the GPU as it was: the next call with ordinary waits is right."""
import numpy as np
import torch

from paper_2509_19729_b200 import binding as B
from test_gpu_sharing import A, Case, dev, model

set_polls = B._load().amoeba_checked_set_wait_polls
POLLS = (1, 2, 3, 5, 10, 20, 40, 80, 160, 320, 640)  # 1: at once, also where there is nothing to wait for


def attention(groups, shape, **kw):
    c = Case(groups, *shape, extra_rows=1, **kw).up()
    seen = set()
    for polls in POLLS:
        set_polls(polls)
        c.status.zero_()
        c.run()
        torch.cuda.synchronize()
        code = int(c.status.item())
        assert code in (0, A().ERR_TIMEOUT) and (polls > 1 or code == A().ERR_TIMEOUT), (polls, code)
        assert all((o[-1] == 7).all() for o in c.out)  # the row of no sequence
        seen.add(code)
        set_polls(0)
        c.status.zero_()
        c.run().check()
    return seen


def copies(order):
    layout = A().make_layout(model(8, 8, 128, 3), 2, 40, 16, kv_order=order)
    shape = (3, 40, 4, 2, 16, 128) if order == 0 else (3, 2, 40, 16, 4, 128)
    pools = [torch.randn(*shape, device="cuda").half() for _ in range(2)]
    want = [p.clone() for p in pools]
    for w in want:
        (w if order == 0 else w.transpose(1, 2))[:, 20:40] = (w if order == 0 else w.transpose(1, 2))[:, :20].clone()
    pairs, status = dev(np.stack([np.arange(20), np.arange(20, 40)], 1)), torch.zeros(1, dtype=torch.int32, device="cuda")
    for polls in POLLS:
        set_polls(polls)
        status.zero_()
        A().amoeba_copy_blocks(layout, pools, pairs, dev([20]), 0, 3, status)
        torch.cuda.synchronize()
        code = int(status.item())
        assert code in (0, A().ERR_TIMEOUT) and (polls > 1 or code == A().ERR_TIMEOUT), (polls, code)
        set_polls(0)
        status.zero_()
        A().amoeba_copy_blocks(layout, pools, pairs, dev([20]), 0, 3, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and all(torch.equal(p, w) for p, w in zip(pools, want))


if __name__ == "__main__":
    assert str(B.library_path()).endswith("libamoeba_checked.so")
    single, pieces = [(900, [(2, 1)] * 30), (300, [(5, 1)] * 9)], [(500, [(70, 70), (90, 66)]), (260, [(40, 40)] * 9)]
    for groups in (single, pieces):
        for shape, kw in (((8, 2, 128, 2), dict(seed=80)), ((8, 2, 64, 1), dict(seed=81, order=1)), ((8, 2, 128, 1, 5), dict(seed=82))):
            print(shape, attention(groups, shape, **kw))
    for order in (0, 1):
        copies(order)
    print("gave up and came back")
