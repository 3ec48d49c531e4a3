"""Tables from lengths, block copies and attention with shared prefixes against their definitions."""
import numpy as np
import pytest
import torch

import cache_reference as ref
import sharing_reference as share

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = ref.DT


def A():
    import paper_2509_19729_b200 as a

    return a


def model(Hq, Hkv, D, L=1):
    return dict(L=L, hidden=Hq * D, Hq=Hq, Hkv=Hkv, D=D, I=Hq * D)


def code(dtype):
    return A().DTYPE_FP16 if dtype == "fp16" else A().DTYPE_BF16


def dev(x, dt=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(DEV, dt)


# ---------------------------------------------------------------------------------------------------- tables

class Step:
    """One call with everything that it may be given, its outputs filled with what must not be there afterwards."""

    def __init__(self, T, table, refs, old, new, parents=None, shared=None, num_rows=None, first_pos=None, pairs_cap=0, in_place=False):
        self.args = (T, table, refs, old, new, parents, shared, num_rows, first_pos, pairs_cap)
        S, NB = len(old), len(refs)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.layout = A().make_layout(model(2, 2, 64), 1, NB, T)
        self.table, self.refs, self.old, self.new = dev(table), dev(refs), dev(old), dev(new)
        self.parents, self.shared = (None, None) if parents is None else (dev(parents), dev(shared))
        self.first = None if first_pos is None else dev(first_pos)
        self.lens = self.old if in_place else torch.full((S,), -7, **i32)
        rows = num_rows is not None
        self.rows = num_rows or 0
        self.starts = torch.full((S + 1,), -7, **i32) if rows else None
        self.positions = torch.full((self.rows,), -7, **i32) if rows else None
        self.slots = torch.full((self.rows,), -7, dtype=torch.int64, device=DEV) if rows else None
        self.pairs = torch.full((pairs_cap, 2), -7, **i32) if pairs_cap else None
        self.n_pairs = torch.full((1,), -7, **i32) if pairs_cap else None
        self.free, self.status = torch.full((1,), -7, **i32), torch.zeros(1, **i32)

    def run(self, stream=None):
        A().amoeba_advance_tables(self.layout, self.table, self.refs, self.old, self.new, self.parents, self.shared, self.lens, self.starts,
                                  self.rows, self.first, self.positions, self.slots, self.pairs, self.n_pairs, self.free, self.status, stream)
        return self

    def check(self):
        want = share.advance(*self.args)
        torch.cuda.synchronize()
        assert int(self.status.item()) == want["status"]
        for k, mine in (("lens", self.lens), ("refs", self.refs), ("table", self.table), ("starts", self.starts),
                        ("positions", self.positions), ("slots", self.slots)):
            if mine is not None:
                assert np.array_equal(mine.cpu().numpy(), want[k]), k
        assert int(self.free.item()) == want["free"]
        if self.pairs is not None:
            n = len(want["pairs"])
            assert int(self.n_pairs.item()) == n and np.array_equal(self.pairs[:n].cpu().numpy(), want["pairs"])
            assert (self.pairs[n:] == -7).all()
        else:
            assert len(want["pairs"]) == 0
        return want


def state(lens, T, NB, extra=2, seed=0):
    table = ref.tables(lens, T, NB, seed, extra)
    refs = np.zeros(NB, np.int32)
    np.add.at(refs, table[table >= 0], 1)
    return table, refs


@pytest.mark.parametrize("T", [1, 3, 16, 64])
@pytest.mark.parametrize("NB", [40, 700, 5000, 40000])
@pytest.mark.parametrize("S", [1, 7, 130])
def test_a_step_of_single_tokens(T, NB, S):
    g = np.random.default_rng(T * NB + S)
    old = g.integers(0, max(2, 12 * T), S)
    table, refs = state(old[:S], T, max(NB, int((-(-old // T)).sum()) + S), seed=S)
    Step(T, table, refs, old, old + 1, num_rows=S + 3).run().check()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(12))
def test_a_step_of_everything(seed, in_place):
    """Growth, ends, cuts, forks of running, ending and growing sequences, blocks that several name: seeded."""
    g = np.random.default_rng(seed)
    T = int(g.choice([1, 4, 16, 32]))
    S = int(g.choice([5, 40, 300, 1500]))
    old = g.integers(0, 20 * T, S)
    old[g.random(S) < 0.3] = 0
    NB = int((-(-old // T)).sum()) + int(g.choice([S, 8 * S, 30000]))
    table, refs = state(old, T, NB, extra=22, seed=seed)
    for s in range(1, S, 3):  # earlier forks: the first blocks of some are their neighbour's
        k = min(-(-int(old[s]) // T), -(-int(old[s - 1]) // T), int(g.integers(0, 30)))
        refs[table[s, :k]] -= 1
        table[s, :k] = table[s - 1, :k]
        np.add.at(refs, table[s, :k], 1)
    new = old + g.integers(0, 3 * T, S)
    cut = g.random(S) < 0.2
    new[cut] = (old[cut] * g.random(cut.sum())).astype(int)
    parents, shared = np.full(S, -1), np.zeros(S, int)
    for s in np.flatnonzero(old == 0):
        if g.random() < 0.6:
            t = int(g.integers(S))
            parents[s], shared[s] = t, g.integers(0, old[t] + 1)
            new[s] = shared[s] + g.integers(0, 2 * T)
    want = Step(T, table, refs, old, new, parents, shared, num_rows=int((new - old).clip(0).sum()) + 9, first_pos=g.integers(0, 99, S),
                pairs_cap=S, in_place=in_place).run().check()
    assert want["status"] in (0, 4)


def test_the_way_back_frees_what_the_step_took():
    g = np.random.default_rng(1)
    T, S, NB = 16, 200, 9000
    old = g.integers(1, 500, S)
    table, refs = state(old, T, NB, extra=40)
    a = Step(T, table, refs, old, old + g.integers(0, 300, S), num_rows=60000).run()
    want = a.check()
    b = Step(T, want["table"], want["refs"], want["lens"], old).run()
    b.check()
    assert np.array_equal(b.table.cpu().numpy(), table) and np.array_equal(b.refs.cpu().numpy(), refs)


def test_too_few_blocks_rows_or_pairs():
    T, old = 4, np.array([4, 4, 8, 0, 4, 6])
    table, refs = state(old, T, 10)
    new = np.array([5, 4, 2, 9, 5, 7])  # 1 block, none, less, 3, 1, a place in its own
    for NB in range(7, 13):
        t, r = state(old, T, NB)
        Step(T, t, r, old, new, num_rows=20).run().check()
    for rows in (0, 1, 5, 9, 10, 11, 12):
        Step(T, *state(old, T, 20), old, new, num_rows=rows).run().check()
    t, r = state(old, T, 20)
    parents, shared = np.array([-1, -1, -1, 2, -1, -1]), np.array([0, 0, 0, 7, 0, 0])
    r[t[5, 1]] += 1  # somebody else names the last block of sequence 5
    for cap in (0, 1, 2, 3):
        Step(T, t, r, old, new, parents, shared, num_rows=20, pairs_cap=cap).run().check()


def test_bad_sequences_stay_and_the_others_go_on():
    T, old = 4, np.array([5, -1, 5, 5, 0, 0, 0, 0, 5, 0])
    table, refs = state([5] * 10, T, 40, extra=0)
    new = np.array([6, 3, 9, -2, 7, 7, 3, 3, 8, 2])
    parents, shared = np.array([-1, -1, -1, -1, 10, 0, 0, 1, 0, 9]), np.array([0, 0, 0, 0, 1, 6, 4, 0, 0, 0])
    want = Step(T, table, refs, old, new, parents, shared, num_rows=30, pairs_cap=10).run().check()
    assert want["status"] == share.INVALID_ARG
    for n in (2 ** 31 - 1, -2 ** 31, 9):  # two blocks of four have room for eight
        want = Step(T, table[:2], refs, np.array([5, 5]), np.array([n, 7]), num_rows=30).run().check()
        assert want["status"] == share.INVALID_ARG


@pytest.mark.parametrize("bad", [-1, 12, 2 ** 31 - 1, -2 ** 31])
def test_bad_blocks(bad):
    T, old = 4, np.array([7, 8, 0, 6])
    table, refs = state(old, T, 12)
    parents, shared = np.array([-1, -1, 1, -1]), np.array([0, 0, 7, 0])
    for s, j in ((0, 1), (1, 0), (1, 1), (3, 0), (3, 1)):
        t = table.copy()
        t[s, j] = bad
        Step(T, t, refs, old, [9, 8, 12, 1], parents, shared, num_rows=30, pairs_cap=4).run().check()


def test_no_sequences_and_no_blocks():
    for S, NB in ((0, 5), (3, 1)):
        refs = np.zeros(NB, np.int32)
        Step(8, np.full((S, 2), -1, np.int32), refs, np.zeros(S, int), np.zeros(S, int), num_rows=4).run().check()
    Step(8, np.full((2, 2), -1, np.int32), np.ones(1, np.int32), np.zeros(2, int), np.array([1, 0]), num_rows=4).run().check()


# ---------------------------------------------------------------------------------------------------- copies

@pytest.mark.parametrize("order", [0, 1])
@pytest.mark.parametrize("Hkv,D,T,tp,elem", [(4, 64, 16, 1, 2), (8, 128, 16, 4, 2), (2, 128, 5, 2, 2), (6, 64, 1, 2, 4), (1, 16, 8, 1, 1),
                                             (8, 128, 64, 1, 2)])
def test_copies(order, Hkv, D, T, tp, elem):
    L, NB = 3, 23
    layout = A().make_layout(model(Hkv, Hkv, D, L), tp, NB, T, elem_bytes=elem, kv_order=order)
    shape = (L, NB, Hkv // tp, 2, T, D * elem) if order == 0 else (L, 2, NB, T, Hkv // tp, D * elem)
    g = torch.Generator().manual_seed(T)
    pools = [torch.randint(0, 256, shape, generator=g, dtype=torch.uint8) for _ in range(tp)]
    pairs = torch.tensor([[3, 9], [3, 22], [0, 1], [-1, 4], [5, -1], [7, 7], [20, 2], [6, 8]], dtype=torch.int32)
    for n, l0, l1 in ((7, 0, 3), (99, 1, 2), (0, 0, 3), (3, 2, 2), (-4, 0, 3)):
        up = [p.to(DEV) for p in pools]
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        A().amoeba_copy_blocks(layout, up, pairs.to(DEV), dev([n]), l0, l1, status)
        for p, mine in zip(pools, up):
            p = p.clone()
            for a, b in pairs[:max(min(n, 8), 0)].tolist():
                if a >= 0 and b >= 0:
                    if order == 0:
                        p[l0:l1, b] = p[l0:l1, a]
                    else:
                        p[l0:l1, :, b] = p[l0:l1, :, a]
            assert torch.equal(mine.cpu(), p)
        assert int(status.item()) == 0


@pytest.mark.parametrize("pair", [(23, 1), (1, 23), (2 ** 31 - 1, 2)])
def test_copies_of_blocks_outside_the_pool(pair):
    layout = A().make_layout(model(2, 2, 64), 1, 23, 8)
    pool = torch.randn(1, 23, 2, 2, 8, 64, device=DEV).half()
    want, status = pool.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    want[:, 5] = want[:, 4]
    A().amoeba_copy_blocks(layout, [pool], dev([pair, (4, 5)]), dev([2]), 0, 1, status)
    assert torch.equal(pool, want) and int(status.item()) == share.BAD_BLOCK_ID


# ---------------------------------------------------------------------------------------------------- attention

class Case:
    """Groups of sequences whose tables name the same whole blocks for their prefix, and own copies of the block it ends in."""

    def __init__(self, groups, Hq=4, Hkv=2, D=128, tp=1, T=16, order=0, dtype="bf16", lead=(), loose=(), spare=3, L=1, layer=0,
                 extra_rows=0, seed=0):
        """groups: [(prefix, [(own tokens, new tokens), ...]), ...]; lead, loose: sequences in front of and behind the groups."""
        self.m, self.tp, self.T, self.order, self.dtype, self.layer = model(Hq, Hkv, D, L), tp, T, order, dtype, layer
        seqs = [(0, x) for x in lead] + [(p, x) for p, g in groups for x in g] + [(0, x) for x in loose]
        self.lens = np.array([p + own for p, (own, _) in seqs], np.int32)
        self.qlens = np.array([n for _, (_, n) in seqs])
        self.starts = np.concatenate([[0], np.cumsum(self.qlens)]).astype(np.int32)
        self.rows = int(self.starts[-1]) + extra_rows
        self.group_starts = (len(lead) + np.concatenate([[0], np.cumsum([len(g) for _, g in groups])])).astype(np.int32)
        self.prefix = np.array([p for p, _ in groups], np.int32)
        self.NB = int((-(-self.lens // T)).sum()) + spare
        self.cache = ref.Cache(self.m, tp, self.NB, T, order, dtype, seed)
        self.bt = ref.tables(self.lens, T, self.NB, seed, 1)
        for k, (p, g) in enumerate(groups):
            a = self.group_starts[k]
            for s in range(a + 1, self.group_starts[k + 1]):
                self.bt[s, :p // T] = self.bt[a, :p // T]
                for pool in self.cache.pools if p % T else ():
                    x, y, n = int(self.bt[a, p // T]), int(self.bt[s, p // T]), p % T
                    if order == 0:
                        pool[:, y, :, :, :n] = pool[:, x, :, :, :n]
                    else:
                        pool[:, :, y, :n] = pool[:, :, x, :n]
        g = torch.Generator().manual_seed(seed + 1)
        self.q = (torch.randn(self.rows, Hq, D, generator=g) * 2).to(DT[dtype])
        self.scale = D ** -0.5
        self.layout = A().make_layout(self.m, tp, self.NB, T, kv_order=order)

    def up(self, max_group_rows=None):
        a = A()
        self.dpools = [p.to(DEV) for p in self.cache.pools]
        self.dq = [x.contiguous().flatten(1) for x in self.q.to(DEV).chunk(self.tp, 1)]
        self.batch = a.make_batch(dev(self.bt), dev(self.lens), dev(self.starts), self.rows, int(max(1, self.qlens.max(initial=1))))
        gs, S = self.group_starts.clip(0, len(self.lens)), self.starts
        most = int((S[gs[1:]] - S[gs[:-1]]).max(initial=0)) if max_group_rows is None else max_group_rows
        self.prefixes = a.make_prefixes(dev(self.group_starts), dev(self.prefix), most)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = torch.full((a.amoeba_attend_shared_workspace_bytes(self.layout, self.batch, self.prefixes),), 0x7F, dtype=torch.uint8, device=DEV)
        self.out = [torch.full((self.rows, x.shape[1]), 7.0, dtype=DT[self.dtype], device=DEV) for x in self.dq]
        self.lse = torch.full((self.rows, self.m["Hq"]), 7.0, device=DEV)
        return self

    def run(self, stream=None):
        A().amoeba_attend_shared(self.layout, code(self.dtype), self.layer, self.dpools, self.batch, self.prefixes, self.dq, self.scale,
                                 self.out, self.lse, self.status, self.ws, stream)
        return self

    def result(self):
        torch.cuda.synchronize()
        out = torch.cat([o.view(self.rows, -1, self.m["D"]) for o in self.out], 1).double().cpu().numpy()
        return out, self.lse.double().cpu().numpy()

    def check(self, status=0, left_out=()):
        """Against every sequence by itself over its own table; left_out: sequences whose rows keep what they had."""
        want, lse, absv, size = ref.attend(self.cache, self.layer, self.bt, self.lens, self.starts, self.q.double().numpy(), self.scale, 0)
        got, got_lse = self.result()
        assert int(self.status.item()) == status
        n, D = int(self.lens.max(initial=0)) + 1, self.m["D"]
        mine = np.zeros(self.rows, bool)
        for s in range(len(self.lens)):
            mine[self.starts[s]:self.starts[s + 1]] = s not in left_out
        assert (got[~mine] == 7.0).all() and (got_lse[~mine] == 7.0).all()
        empty = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got_lse[mine]), empty[mine]) and (got[mine][empty[mine]] == 0).all()
        vmax = max(float(p.double().abs().nan_to_num(0, 0, 0).max()) for p in self.cache.pools)
        tol = share.tolerance_shared(self.dtype, D, n, want, absv, size, vmax)
        off = np.abs(got - want)[mine]
        assert np.isfinite(got[mine]).all() and (off <= tol[mine]).all(), float((off / tol[mine]).max())
        some = mine[:, None] & ~empty
        assert (np.abs(got_lse - lse)[some] <= share.tolerance_shared_lse(D, n, lse, size)[some]).all()


HEADS = [(4, 4, 64, 1), (4, 2, 128, 2), (12, 4, 64, 2), (8, 1, 128, 1), (16, 1, 64, 1), (20, 1, 128, 1), (40, 1, 128, 1)]


@pytest.mark.parametrize("Hq,Hkv,D,tp", HEADS)
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("order", [0, 1])
def test_single_tokens_behind_a_prefix(Hq, Hkv, D, tp, dtype, order):
    own = [(n, 1) for n in (1, 2, 15, 16, 17, 63, 65, 1)]
    Case([(70, own), (1, own[:2]), (129, own[3:])], Hq, Hkv, D, tp, order=order, dtype=dtype, lead=[(33, 1)], loose=[(5, 1), (90, 1)],
         seed=Hq).up().run().check()


@pytest.mark.parametrize("T", [1, 5, 8, 16, 24, 64, 100, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("order", [0, 1])
def test_block_sizes(T, D, order):
    Case([(64, [(3, 1), (40, 2), (9, 9)]), (131, [(1, 1)] * 20 + [(70, 33)])], 4, 2, D, 2, T=T, order=order, loose=[(8, 3)], seed=T).up().run().check()


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 127, 128, 129, 300, 517])
@pytest.mark.parametrize("members,q", [(2, 1), (9, 1), (40, 1), (3, 5), (2, 70), (5, 130)])
def test_prefix_lengths(prefix, members, q):
    Case([(prefix, [(q + s % 3, q) for s in range(members)])], 8, 2, 128, dtype="fp16", seed=prefix, extra_rows=2).up().run().check()
