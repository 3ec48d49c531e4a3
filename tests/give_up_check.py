"""Run against the checked build of the library: the kernels of many rows with waits that run out after a few polls.  Every call
returns, reports the timeout, and leaves the GPU as it was: the next call with ordinary waits is right."""
import torch

from paper_2509_19729_b200 import binding as B
from test_gpu_operators import A, Case, check_attend, check_scores

set_polls = B._load().amoeba_checked_set_wait_polls


def check(shape, **kw):
    c = Case(*shape, lens=[900, 300, 40], qlens=[150, 70, 1], extra_rows=1, **kw).up()
    scores = [torch.zeros(1, c.NB, c.m["Hkv"] // c.tp, c.T, device="cuda") for _ in range(c.tp)]

    def score():
        A().amoeba_accumulate_scores(c.layout, 1, 0, c.dpools, c.batch, c.dq, c.scale, 0, c.lse, None, scores, c.status)

    seen = set()
    for polls in (1, 2, 3, 5, 10, 20, 40, 80, 160, 320, 640):  # 1: at once, also where there is nothing to wait for
        for call in (c.attend, score):
            set_polls(polls)
            c.status.zero_()
            call()
            torch.cuda.synchronize()
            code = int(c.status.item())
            assert code in (0, A().ERR_TIMEOUT) and (polls > 1 or code == A().ERR_TIMEOUT), (polls, code)
            assert all((o[-1] == 7).all() for o in c.out)  # the row of no sequence
            seen.add(code)
        set_polls(0)
        c.status.zero_()
        c.attend()
        check_attend(c)
    check_scores(c)
    return seen


if __name__ == "__main__":
    assert str(B.library_path()).endswith("libamoeba_checked.so")
    for shape, kw in (((8, 2, 128, 2), dict(seed=80)), ((8, 2, 64, 1), dict(seed=81, order=1)), ((8, 2, 128, 1, 5), dict(seed=82))):
        print(shape, check(shape, **kw))
    print("gave up and came back")
