"""The serving operators at the edges of what their documentation allows, and what they refuse there."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import cache_reference as ref
from test_gpu_operators import A, DEV, Case, check_attend, check_evict, check_scores, draw_scores, model

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


# ------------------------------------------------------------------------------------------------------ lengths past 2^30

@pytest.mark.parametrize("length", [2 ** 30 + 1, 2 ** 31 - 100, 2 ** 31 - 1])
def test_lengths_past_2_to_the_30_are_refused(length):
    """A table that would hold them, of blocks of 65536 tokens: INVALID_ARG, nothing of that sequence is done, and the
    sequence beside it is."""
    a = A()
    T, width = 1 << 16, 1 << 15
    c = Case(1, 1, 64, T=T, lens=[100], seed=70, spare=1)
    c.bt = np.zeros((2, width), np.int32)
    c.bt[0, 0] = 1
    c.lens, c.qlens = np.array([100, 5], np.int32), np.array([1, 1])
    c.starts, c.rows = np.array([0, 1, 2], np.int32), 2
    c.q = torch.cat([c.q, c.q])
    c.up()
    c.dlens.copy_(torch.tensor([100, length], dtype=torch.int32))

    def refused():
        torch.cuda.synchronize()
        code, _ = int(c.status.item()), c.status.zero_()
        return code == a.ERR_INVALID_ARG

    for maxq in (1, 40):  # the kernels for few rows, and for many beside them
        c.batch = a.make_batch(c.dbt, c.dlens, c.dstarts, 2, maxq)
        c.ws = torch.full((a.amoeba_attend_workspace_bytes(c.layout, c.batch),), 0x7F, dtype=torch.uint8, device=DEV)
        c.out[0].fill_(7.0)
        c.attend()
        assert refused() and (c.out[0][1] == 7).all() and (c.out[0][0] != 7).any()
        scores = torch.full((1, c.NB, 1, T), 3.0, device=DEV)
        a.amoeba_accumulate_scores(c.layout, 1, 0, c.dpools, c.batch, c.dq, c.scale, 0, c.lse, None, [scores], c.status)
        assert refused() and (scores[0, 0] == 3).all() and (scores[0, 1, 0, :100] != 3).all() and (scores[0, 1, 0, 100:] == 3).all()
        pool, q_out = c.dpools[0].clone(), torch.full_like(c.dq[0], 7.0)
        a.amoeba_append_kv(c.layout, 1, 0, [pool], c.batch, c.dq, c.dq, c.dq, None, [q_out], c.status)
        assert refused() and torch.equal(pool[0, 0], c.dpools[0][0, 0]) and (q_out[1] == 7).all()
        assert torch.equal(pool[0, 1, 0, 0, 99], c.dq[0][0]) and torch.equal(q_out[0], c.dq[0][0])
    pool, scores, new = c.dpools[0].clone(), torch.rand(1, c.NB, 1, T, device=DEV), torch.full((2,), 99, dtype=torch.int32, device=DEV)
    before = scores.clone()
    ws = torch.empty(a.amoeba_evict_workspace_bytes(c.layout, 1, 2, 40), dtype=torch.uint8, device=DEV)
    a.amoeba_evict_kv(c.layout, 0, 1, [pool], [scores], c.dbt, c.dlens, c.dbt, 40, 8, new, c.status, ws)
    assert refused() and new.tolist() == [40, -1]
    assert torch.equal(pool[0, 0], c.dpools[0][0, 0]) and torch.equal(scores[0, 0], before[0, 0])


# ---------------------------------------------------------------------------------------------------------- waits that run out

def test_waits_that_run_out_end_the_call_with_a_status():
    """In the checked build, whose waits can be told to give up after a few polls (give_up_check.py)."""
    import paper_2509_19729_b200.build as b

    b.build(checked=True)
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, os.path.join(here, "give_up_check.py")], cwd=os.path.dirname(here), timeout=300,
                       env=dict(os.environ, AMOEBA_BINDING_BUILD="checked", PYTHONPATH=os.path.dirname(here)), capture_output=True, text=True)
    assert r.returncode == 0 and "gave up and came back" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


# -------------------------------------------------------------------------------------------------------------------- sessions

@pytest.mark.parametrize("as_handle", [False, True])
def test_a_workspace_is_taken_from_the_stream_that_uses_it(as_handle):
    """An eviction on another stream, which has to grow the workspace, beside a kernel on the current stream that still writes
    to memory freed there."""
    from paper_2509_19729_b200.session import CacheSession

    m, budget, recent = model(2, 2, 64), 100, 10
    s = CacheSession(m, 1, 60, 3, 20, device=DEV)
    g = torch.Generator().manual_seed(90)
    pool = torch.randn(1, 60, 2, 2, 16, 64, generator=g).to(torch.bfloat16)
    scores = torch.randn(1, 60, 2, 16, generator=g)
    s.pools[0].copy_(pool.flatten().view(torch.uint8))
    s.score_pools[0].copy_(scores)
    lens, bt = [320, 120, 50], torch.arange(60, dtype=torch.int32).view(3, 20)
    s.set_tables(lens, bt)
    s.workspace = torch.empty(0, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    freed = torch.empty(A().amoeba_evict_workspace_bytes(s.layout, 1, 3, budget), dtype=torch.uint8, device=DEV)
    at = freed.data_ptr()
    torch.cuda._sleep(200_000_000)
    freed.fill_(0x7F)
    del freed
    s.evict(budget, recent, stream=side.cuda_stream if as_handle else side)
    assert s.workspace.data_ptr() != at
    torch.cuda.synchronize()
    want, ws = pool.clone(), scores.clone()
    for q, n in enumerate(lens[:2]):
        i, j, b = torch.arange(n), torch.arange(budget), bt[q].long()
        for h in range(2):
            f = torch.from_numpy(ref.kept(scores[0, b[i // 16], h, i % 16].double().numpy(), n, budget, recent))
            want[0, b[j // 16], h, :, j % 16] = pool[0, b[f // 16], h, :, f % 16]
            ws[0, b[j // 16], h, j % 16] = scores[0, b[f // 16], h, f % 16]
    assert s.new_lens.tolist() == [100, 100, 50] and int(s.status.item()) == 0
    assert torch.equal(s.pools[0].cpu(), want.flatten().view(torch.uint8)) and torch.equal(s.score_pools[0].cpu(), ws)


# ---------------------------------------------------------------------------------------------------------------------- append

def append_beside_bad(lens, starts, rows, maxq, left, S=3, T=16):
    """Appends; sequences `left` must be left out, the others' tokens written; a row that two name is the first one's."""
    a = A()
    c = Case(2, 1, 64, T=T, lens=[40] * S, seed=91).up()
    c.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
    c.dstarts.copy_(torch.tensor(starts, dtype=torch.int32))
    c.batch = a.make_batch(c.dbt, c.dlens, c.dstarts, rows, maxq)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(rows, w, generator=g).to(torch.bfloat16).to(DEV) for w in (128, 64, 64))
    out, want = torch.full_like(q, 7.0), torch.full_like(q, 7.0)
    pool, host = c.dpools[0].clone(), c.dpools[0].clone()
    a.amoeba_append_kv(c.layout, 1, 0, [pool], c.batch, [q], [k], [v], None, [out], c.status)
    torch.cuda.synchronize()
    owners = [[s for s in range(S) if starts[s] <= r < starts[s + 1]] for r in range(rows)]
    for r, o in enumerate(owners):
        if o and o[0] not in left:
            s = o[0]
            i = lens[s] - (starts[s + 1] - starts[s]) + r - starts[s]
            b = int(c.bt[s, i // T])
            host[0, b, 0, 0, i % T], host[0, b, 0, 1, i % T], want[r] = k[r], v[r], q[r]
    assert torch.equal(pool, host) and torch.equal(out, want)
    return int(c.status.item())


@pytest.mark.parametrize("lens,starts,rows,maxq,left", [
    ([40, 40, 40], [0, 1, 0, 1], 1, 1, [1]),          # a decreasing row number: no row is the second's, row 0 two others'
    ([40, 40, 40], [0, 3, 1, 4], 4, 3, [1]),          # rows 1 and 2 are two sequences', 0 and 3 one's
    ([40, 40, 40], [0, 2, 2, 4], 4, 1, [0, 2]),       # more rows than announced
    ([40, -1, 40], [0, 1, 1, 3], 3, 2, [1]),          # bad lengths of sequences without rows
    ([40, 49, 40], [0, 1, 1, 3], 3, 2, [1]),
    ([40, 2 ** 31 - 1, 40], [0, 1, 1, 3], 3, 2, [1]),
    ([40, 40, 40], [0, 1, 2, 9], 2, 9, [2]),          # rows that leave the buffers
    ([40, 40, 40], [0, 1, 7, 9], 1, 9, [1, 2]),
    ([40, 40, 40], [-3, 1, 2, 3], 3, 9, [0]),
    ([40, 40, 1], [0, 1, 2, 4], 4, 2, [2]),           # more new tokens than cached ones
])
def test_append_reports_every_bad_sequence(lens, starts, rows, maxq, left):
    assert append_beside_bad(lens, starts, rows, maxq, left) == A().ERR_INVALID_ARG


def test_append_reports_the_last_of_many_sequences():
    lens, S = [40] * 1500, 1500
    starts = [min(s, 7) for s in range(S + 1)]
    assert append_beside_bad(lens, starts, 7, 1, [], S) == 0
    lens[-1] = -5
    assert append_beside_bad(lens, starts, 7, 1, [], S) == A().ERR_INVALID_ARG


# ---------------------------------------------------------------------------------------------------------------------- attend

@pytest.mark.parametrize("lens", [(20, 30, 40), (900, 30, 400)])
def test_rows_where_none_are_announced(lens):
    """max_q_len 0: sequences with rows are refused by every call, those without are fine."""
    a = A()
    for starts, lengths, status in (([0, 0, 0, 0], lens, 0), ([0, 0, 1, 1], lens, a.ERR_INVALID_ARG),
                                    ([0, 0, 0, 0], (lens[0], -1, lens[2]), a.ERR_INVALID_ARG)):
        c = Case(4, 2, 64, lens=lens, seed=92).up()
        c.dlens.copy_(torch.tensor(lengths, dtype=torch.int32))
        c.dstarts.copy_(torch.tensor(starts, dtype=torch.int32))
        c.batch = a.make_batch(c.dbt, c.dlens, c.dstarts, c.rows, 0)
        c.attend()
        torch.cuda.synchronize()
        assert int(c.status.item()) == status and (c.out[0] == 7).all() and (c.lse == 7).all()
        c.status.zero_()
        pool, k = c.dpools[0].clone(), torch.zeros(c.rows, 128, dtype=torch.bfloat16, device=DEV)
        a.amoeba_append_kv(c.layout, 1, 0, [pool], c.batch, c.dq, [k], [k], None, c.out, c.status)
        torch.cuda.synchronize()
        assert int(c.status.item()) == status and (c.out[0] == 7).all() and torch.equal(pool, c.dpools[0])
        c.status.zero_()
        a.amoeba_accumulate_scores(c.layout, 1, 0, c.dpools, c.batch, c.dq, c.scale, 0, c.lse, None,
                                   [torch.zeros(1, c.NB, 2, 16, device=DEV)], c.status)
        assert int(c.status.item()) == status


# ---------------------------------------------------------------------------------------------------------------------- scores

def scores_of(c, lse):
    got = [torch.zeros(1, c.NB, c.m["Hkv"] // c.tp, c.T, device=DEV) for _ in range(c.tp)]
    A().amoeba_accumulate_scores(c.layout, 1, 0, c.dpools, c.batch, c.dq, c.scale, 0, lse, None, got, c.status)
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0
    return got


@pytest.mark.parametrize("Hq,Hkv,D,q", [(4, 2, 64, 3), (8, 2, 128, 33), (8, 2, 64, 40), (6, 2, 128, 100), (2, 2, 64, 300)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 0.0])
def test_scores_rows_that_add_nothing_may_hold_anything(Hq, Hkv, D, q, bad):
    """Rows with lse -infinity, first and last of their sequences among them: the others' sums, to the bit."""
    c = Case(Hq, Hkv, D, lens=[700, q, 300], qlens=[q, q, 1], seed=100 + q).up()
    c.attend()
    lse = c.lse.clone()
    mute = torch.zeros(c.rows, dtype=torch.bool)
    mute[[0, q // 2, q - 1, q]] = True
    lse[mute.to(DEV)] = -np.inf
    want = scores_of(c, lse)
    for x in c.dq:
        x[mute.to(DEV)] = bad
    got = scores_of(c, lse)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(torch.isfinite(x).all() for x in got)


@pytest.mark.parametrize("Hq,Hkv,D,q", [(4, 2, 64, 3), (8, 2, 128, 33), (8, 2, 64, 40), (6, 2, 128, 100), (2, 2, 64, 300)])
def test_scores_of_a_key_that_no_row_wants(Hq, Hkv, D, q):
    """A key of -infinity that every row sees with a logit of -infinity: its score is 0, in passes that are not full too."""
    c = Case(Hq, Hkv, D, lens=[700, q], qlens=[q, q], seed=120 + q).up()
    at = 5
    for x in c.dq:
        x.view(c.rows, Hq, D)[..., at] = x.view(c.rows, Hq, D)[..., at].abs() + 0.5
    c.dpools[0][0, int(c.bt[0, 9]), :, 0, 7, at] = -np.inf  # token 151 of the first sequence
    c.attend()
    got = scores_of(c, c.lse)[0][0, int(c.bt[0, 9])]
    assert (got[:, 7] == 0).all() and torch.isfinite(got).all() and (got[:, 6] > 0).all()


@pytest.mark.parametrize("D,T,dtype", [(64, 16, "fp16"), (128, 8, "bf16"), (128, 5, "fp16")])
@pytest.mark.parametrize("q", [1, 8, 40])
def test_scores_of_large_logits(D, T, dtype, q):
    """Logits around a thousand, whose products and sums are exact: what is left is one rounding of the difference to lse and one
    of its product with log2(e), itself off by 2^-26 (3 half steps of 2^-24 of the exponent, with room for that), the exponential's
    2^-22 and the additions' 2^-24 each."""
    c = Case(8, 2, D, T=T, dtype=dtype, lens=[q + 200], qlens=[q], seed=140)
    n = q + 200
    g = np.random.default_rng(q)
    u, v = g.integers(120, 129, n).astype(float), g.integers(60, 65, (q, 8)).astype(float)  # whole numbers of 8 bits at most
    scale = np.float32(0.125 if D == 64 else 0.1)
    c.q.zero_()
    c.q[:, :, 3] = torch.from_numpy(v).to(c.q.dtype)
    for i in range(n):
        for h in range(2):
            k = c.cache.at(0, int(c.bt[0, i // T]), h, 0, i % T)
            k.zero_()
            k[3] = u[i]
    c.up()
    lse = (np.float64(scale) * v * 128 + 0.3 * v / 60).astype(np.float32)
    got = [torch.zeros(1, c.NB, 2, T, device=DEV)]
    A().amoeba_accumulate_scores(c.layout, int(dtype == "bf16"), 0, c.dpools, c.batch, c.dq, float(scale), 0,
                                 torch.from_numpy(lse).to(DEV), None, got, c.status)
    host = got[0].cpu().double().numpy()
    for i in range(n):
        x = np.float64(scale) * v * u[i] - lse.astype(np.float64)  # [q, 8]
        w = np.where((i <= n - q + np.arange(q))[:, None], np.exp(x), 0.0).reshape(q, 2, 4)
        tol = (w * (4 * 2.0 ** -24 * np.abs(x).reshape(q, 2, 4) + 2.0 ** -22 + 4 * q * 2.0 ** -24)).sum((0, 2))
        assert (np.abs(host[0, c.bt[0, i // T], :, i % T] - w.sum((0, 2))) <= tol).all()


@pytest.mark.parametrize("q", [1, 8, 12, 30])
def test_scores_of_logits_whose_sums_are_cut(q):
    """One product of 512 beside eight of 0.9 steps of it, one to each matrix instruction, which may cut what does not reach a
    step (2^-14).  Up to 8 rows there are four sums of two instructions: two steps cut and three half steps of rounding; up to 32
    two of four: four steps and a half.  One sum would lose seven steps.  Beside that the roundings of the exponent (as above)."""
    c = Case(2, 2, 128, lens=[q + 64], qlens=[q], seed=170)
    n = q + 64
    c.q.zero_()
    c.q[:, :, 0], c.q[:, :, 1::16] = 32.0, 2.0 ** -7
    for i in range(n):
        for h in range(2):
            k = c.cache.at(0, int(c.bt[0, i // 16]), h, 0, i % 16)
            k.zero_()
            k[0], k[1::16] = 16.0, 115 * 2.0 ** -14
    c.up()
    logit, lse = (512 + 8 * 115 * 2.0 ** -21) / 64, 8.5
    got = [torch.zeros(1, c.NB, 2, 16, device=DEV)]
    A().amoeba_accumulate_scores(c.layout, 1, 0, c.dpools, c.batch, c.dq, 1 / 64, 0, torch.full((q, 2), lse, device=DEV), None, got,
                                 c.status)
    host = got[0].cpu().double().numpy()
    off = (3.5 if q <= 8 else 4.5) * 2.0 ** -14 / 64 + 4 * 2.0 ** -24 * abs(logit - lse) + 2.0 ** -22 + q * 2.0 ** -24
    for i in range(n):
        rows = q if i <= n - q else n - i
        want = rows * np.exp(logit - lse)
        assert (np.abs(host[0, c.bt[0, i // 16], :, i % 16] - want) <= want * off).all(), (i, host[0, c.bt[0, i // 16], :, i % 16] / want - 1, off)


@pytest.mark.parametrize("tp,to,T,order", [(1, 2, 16, 0), (4, 1, 8, 1), (2, 4, 32, 0)])
def test_scores_go_along_with_a_transformation(tp, to, T, order):
    """Scores of one layout, moved by a second call for the same pairs: the eviction that follows keeps the same tokens."""
    from paper_2509_19729_b200.session import Session

    a = A()
    L, Hkv, D, lens, budget, recent = 2, 4, 64, [200, 90, 33], 64, 8
    m = model(4, Hkv, D, L=L)
    c = Case(4, Hkv, D, tp, T=T, order=order, lens=lens, L=L, seed=150)
    c.up()
    g = torch.Generator().manual_seed(2)
    scores = [torch.randn(L, c.NB, Hkv // tp, T, generator=g).to(DEV) for _ in range(tp)]
    t = Session(m, tp, to, c.NB, c.NB + 5, 3, c.bt.shape[1], c.bt.size, weights=False, block_tokens=T, device=DEV,
                src_kv_order=order, dst_kv_order=order)
    t.set_tables(lens, c.bt, free_list=np.random.default_rng(1).permutation(c.NB + 5))
    for x, y in zip(t.src_pools, c.dpools):
        x.copy_(y.flatten().view(torch.uint8))
    t.step()
    layout = lambda n, nb: a.make_layout(dict(m, D=8), n, nb, T // 8)  # noqa: E731
    plan = a.amoeba_plan_create(layout(tp, c.NB), layout(to, c.NB + 5))
    assert a.amoeba_layout_kv_pool_bytes(plan.src) == scores[0].nbytes
    moved = [torch.full((L, c.NB + 5, Hkv // to, T), -9.0, device=DEV) for _ in range(to)]
    a.amoeba_reshard_kv(plan, scores, moved, t.pairs, t.num_pairs, t.pairs_cap, 0, L, t.status)
    db = t.dst_bt.cpu().numpy()
    for s, n in enumerate(lens):
        i = np.arange(-(-n // T) * T)
        for h in range(Hkv):
            x = scores[h // (Hkv // tp)][:, c.bt[s, i // T], h % (Hkv // tp), i % T]
            y = moved[h // (Hkv // to)][:, db[s, i // T], h % (Hkv // to), i % T]
            assert torch.equal(x, y)
    kept = []
    for lay, pools, sc, bt in ((c.layout, c.dpools, scores, c.dbt), (t.dst_layout, t.dst_pools, moved, t.dst_bt)):
        new = torch.zeros(3, dtype=torch.int32, device=DEV)
        ws = torch.empty(a.amoeba_evict_workspace_bytes(lay, L, 3, budget), dtype=torch.uint8, device=DEV)
        a.amoeba_evict_kv(lay, 0, L, pools, sc, bt, c.dlens, bt, budget, recent, new, t.status, ws)
        hb = bt.cpu().numpy()
        n = len(pools)
        shape = (L, -1, Hkv // n, 2, T, D) if order == 0 else (L, 2, -1, T, Hkv // n, D)
        p = [x.view(torch.uint8).view(torch.bfloat16).view(*shape) for x in (y.flatten() for y in pools)]
        p = [x if order == 0 else x.permute(0, 2, 4, 1, 3, 5) for x in p]
        kept.append([torch.cat([x[:, hb[s, i // T], :, :, i % T] for x in p], 2) for s, i in ((s, np.arange(min(k, budget))) for s, k in enumerate(lens))])
    assert all(torch.equal(x, y) for x, y in zip(*kept)) and int(t.status.item()) == 0


# ------------------------------------------------------------------------------------------- tables much wider than the lengths

@pytest.mark.parametrize("extra", [0, 100, 5000])
@pytest.mark.parametrize("T", [8, 16])
def test_tables_wider_than_the_lengths(extra, T):
    """Launch shapes go by the table's width: short sequences in the tables of a session with room for long ones."""
    for qlens in ([1, 1, 1, 0, 1], [1, 20, 70, 0, 3]):
        c = Case(8, 2, 64, 2, T=T, lens=[5, 40, 130, 0, 300], qlens=qlens, seed=160, extra=extra).up()
        c.attend()
        check_attend(c)
        check_scores(c, scored=[4, 20, 60, 0, 297])


@pytest.mark.parametrize("extra", [100, 1000, 5000])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_in_tables_wider_than_the_lengths(extra, in_place):
    lens = [5, 64, 65, 130, 0, 301]
    c = Case(4, 2, 64, 2, T=16, lens=lens, L=2, seed=161, spare=60, extra=extra).up()
    free = np.setdiff1d(np.arange(c.NB), c.bt).astype(np.int32)
    dst, k = np.full((len(lens), 4), -1, np.int32), 0
    for s, n in enumerate(lens):
        m = -(-min(n, 64) // 16)
        dst[s, :m] = free[k:k + m]
        k += m
    check_evict(c, draw_scores(c, "ties"), 64, 10, in_place, dst_blocks=dst)


# ------------------------------------------------------------------------------------------------------------ captured calls

@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("wide", [0, 1000])  # one CTA, and a cluster, to each selection
def test_a_captured_step_with_an_eviction(in_place, wide):
    """Append, attend, accumulate and evict in one graph, replayed with other rows, lengths and tables: the same bits as the calls
    one by one, on another stream."""
    a = A()
    L, budget, recent, S, NB = 2, 40, 8, 3, 120
    layout = a.make_layout(model(8, 2, 64, L), 2, NB, 16)
    i32 = dict(dtype=torch.int32, device=DEV)
    bt, dst = torch.full((S, 12 + wide), -1, **i32), torch.full((S, 12 + wide), -1, **i32)
    lens, starts, new = torch.zeros(S, **i32), torch.zeros(S + 1, **i32), torch.zeros(S, **i32)
    status = torch.zeros(1, **i32)
    q, k, v = ([torch.zeros(60, w, dtype=torch.bfloat16, device=DEV) for _ in range(2)] for w in (256, 64, 64))
    q_out, out = ([torch.zeros_like(x) for x in q] for _ in range(2))
    lse = torch.zeros(60, 8, device=DEV)
    pools = [torch.zeros(L, NB, 1, 2, 16, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    scores = [torch.zeros(L, NB, 1, 16, device=DEV) for _ in range(2)]
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).to(DEV)
    rotation = a.make_rotation(inv_freq=freq, rot_dim=64)
    batch = a.make_batch(bt, lens, starts, 60, 50)
    ws = torch.zeros(a.amoeba_attend_workspace_bytes(layout, batch), dtype=torch.uint8, device=DEV)
    ews = torch.zeros(a.amoeba_evict_workspace_bytes(layout, L, S, budget), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        for l in range(L):
            a.amoeba_append_kv(layout, 1, l, pools, batch, q, k, v, rotation, q_out, status, stream)
            a.amoeba_attend(layout, 1, l, pools, batch, q_out, 0.125, 0, out, lse, status, ws, stream)
            a.amoeba_accumulate_scores(layout, 1, l, pools, batch, q_out, 0.125, 0, lse, None, scores, status, stream)
        a.amoeba_evict_kv(layout, 0, L, pools, scores, bt, lens, bt if in_place else dst, budget, recent, new, status, ews, stream)

    def fill(seed, n, rows):
        g = torch.Generator(device=DEV).manual_seed(seed)
        for t in q + k + v + pools + scores:
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        ids = torch.randperm(NB, generator=g, device=DEV).to(torch.int32).view(S, 40)
        bt[:, :12], dst[:, :12] = ids[:, :12], ids[:, 12:24]
        lens.copy_(torch.tensor(n))
        starts.copy_(torch.tensor([0, *np.cumsum(rows).tolist()]))

    def state():
        return [t.clone() for t in (*q_out, *out, lse, *pools, *scores, new)]

    fill(0, [5, 6, 7], [1, 1, 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed, n, rows in ((1, [150, 41, 30], [50, 1, 9]), (2, [30, 40, 192], [1, 1, 1]), (3, [100, 60, 50], [0, 33, 20])):
        fill(seed, n, rows)
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        want = state()
        fill(seed, n, rows)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(state(), want))
        assert int(status.item()) == 0 and new.tolist() == [min(x, budget) for x in n]
