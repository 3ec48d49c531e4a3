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


@pytest.mark.parametrize("NB,S", [(65536, 256), (65537, 256), (200001, 50), (8192, 256), (8193, 257), (300, 513)])
def test_sizes_where_the_launch_changes(NB, S):
    g = np.random.default_rng(S)
    old = g.integers(0, max(2, 6 * min(300, NB // S)), S)
    table, refs = state(old, 16, NB, seed=NB)
    Step(16, table, refs, old, old + g.integers(0, 4, S), num_rows=1025).run().check()


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


@pytest.mark.parametrize("T,NB,S", [(4, 60, 8), (4, 12000, 300), (2, 70000, 600)])
def test_blocks_that_are_counted_free(T, NB, S):
    """Named in a table, counted 0: neither shared, copied from, nor given back, and handed out to somebody."""
    g = np.random.default_rng(S)
    old = np.where(np.arange(S) % 4 < 2, 0, g.integers(2, 4 * T, S))
    table, refs = state(old, T, NB, seed=S)
    parents, shared, new = np.full(S, -1), np.zeros(S, int), old + 3
    parents[1::4] = np.arange(2, S, 4)
    shared[1::4] = old[2::4] - g.integers(0, 2, S // 4)
    new[1::4] = shared[1::4] + 2
    new[3::4] = g.integers(0, old[3::4] + 1)
    for s in range(2, S, 8):
        refs[table[s, 0]] = 0
        refs[table[s + 1, -(-old[s + 1] // T) - 1]] = 0
    refs[table[6, (old[6] - 1) // T]] = 0
    want = Step(T, table, refs, old, new, parents, shared, num_rows=12 * S, pairs_cap=S).run().check()
    assert want["status"] == share.BAD_BLOCK_ID


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

    def up(self, always=True, max_group_rows=None):
        a = A()
        self.dpools = [p.to(DEV) for p in self.cache.pools]
        self.dq = [x.contiguous().flatten(1) for x in self.q.to(DEV).chunk(self.tp, 1)]
        self.batch = a.make_batch(dev(self.bt), dev(self.lens), dev(self.starts), self.rows, int(max(1, self.qlens.max(initial=1))))
        gs, S = self.group_starts.clip(0, len(self.lens)), self.starts
        most = int((S[gs[1:]] - S[gs[:-1]]).max(initial=0)) if max_group_rows is None else max_group_rows
        self.prefixes = a.make_prefixes(dev(self.group_starts), dev(self.prefix), most, always)
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
@pytest.mark.parametrize("always", [True, False])
def test_single_tokens_behind_a_prefix(Hq, Hkv, D, tp, dtype, order, always):
    own = [(n, 1) for n in (1, 2, 15, 16, 17, 63, 65, 1)]
    Case([(70, own), (1, own[:2]), (129, own[3:])], Hq, Hkv, D, tp, order=order, dtype=dtype, lead=[(33, 1)], loose=[(5, 1), (90, 1)],
         seed=Hq).up(always).run().check()


@pytest.mark.parametrize("T", [1, 5, 8, 16, 24, 64, 100, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("order", [0, 1])
def test_block_sizes(T, D, order):
    Case([(64, [(3, 1), (40, 2), (9, 9)]), (131, [(1, 1)] * 20 + [(70, 33)])], 4, 2, D, 2, T=T, order=order, loose=[(8, 3)], seed=T).up().run().check()


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 127, 128, 129, 300, 517])
@pytest.mark.parametrize("members,q", [(2, 1), (9, 1), (40, 1), (3, 5), (2, 70), (5, 130)])
def test_prefix_lengths(prefix, members, q):
    Case([(prefix, [(q + s % 3, q) for s in range(members)])], 8, 2, 128, dtype="fp16", seed=prefix, extra_rows=2).up().run().check()


def test_a_group_shares_no_more_than_its_shortest_sequence_has():
    """A prefix that reaches into the new tokens of some sequence, or behind its end."""
    for given in (40, 64, 200, 2 ** 31 - 1):
        c = Case([(40, [(1 + s, 1) for s in range(30)] + [(60, 50)])], 8, 2, 128)
        c.prefix[0] = given
        c.up().run().check()


def test_a_group_through_its_first_sequence_with_rows():
    """Sequences without new tokens, empty ones in front among them, are in the way of nothing."""
    c = Case([(300, [(0, 0), (9, 0)] + [(5 + s % 7, 1) for s in range(50)] + [(2, 0)])], 4, 2, 64)
    c.lens[c.group_starts[0]] = 0
    c.up().run().check()


@pytest.mark.parametrize("members,q", [(40, 1), (3, 70)])
def test_what_nobody_sees_may_be_anything(members, q):
    """NaN in free blocks, behind the last tokens and, as the prefix is read through the first sequence's table, in the others' copies of
    the block that it ends in."""
    c = Case([(150, [(q + 3 + s % 9, q) for s in range(members)])], 8, 4, 128, spare=5, seed=q)
    used = np.zeros((c.NB, c.T), bool)
    for s, n in enumerate(c.lens):
        for i in range(int(n)):
            if i >= 150 or s == 0:  # the first sequence's table is the group's
                used[c.bt[s, i // c.T], i % c.T] = True
    c.up()
    for p, mine in zip(c.cache.pools, c.dpools):
        mine[:] = torch.where(torch.from_numpy(used)[None, :, None, None, :, None], p, float("nan")).to(DEV)
    c.run().check()


@pytest.mark.parametrize("members", [6, 50])
@pytest.mark.parametrize("where", ["prefix", "own"])
@pytest.mark.parametrize("always", [True, False])
def test_bad_blocks_of_a_prefix_and_of_a_sequence(members, where, always):
    c = Case([(600, [(40 + s % 5, 1) for s in range(members)])], 16, 4, 128)
    if where == "prefix":
        c.bt[:, [0, 7, 30]] = [-1, c.NB, 2 ** 31 - 1]
    else:
        c.bt[2, 38], c.bt[5, 39] = -5, c.NB
    c.up(always).run().check(status=share.BAD_BLOCK_ID)


@pytest.mark.parametrize("members", [3, 40])
@pytest.mark.parametrize("always", [True, False])
def test_bad_groups_attend_by_themselves(members, always):
    def case():
        return Case([(150, [(3 + s % 4, 1) for s in range(members)]), (210, [(2, 1)] * members)], 4, 2, 128, lead=[(9, 1)], loose=[(30, 2)])

    n = 2 * members + 2
    for starts in ([1, members + 1, members], [-1, members + 1, n], [1, members + 1, n + 1], [5, 3, n], [2 ** 31 - 1, 0, 1]):
        c = case()
        c.group_starts[:] = starts
        c.up(always, 99).run().check(status=share.INVALID_ARG)
    c = case()
    c.prefix[0] = -1
    c.up(always).run().check(status=share.INVALID_ARG)
    case().up(always, members - 1).run().check(status=share.INVALID_ARG)
    case().up(always, 0).run().check(status=share.INVALID_ARG)


@pytest.mark.parametrize("members,q", [(40, 1), (3, 90)])
@pytest.mark.parametrize("always", [True, False])
def test_bad_sequences_of_a_group_are_left_out(members, q, always):
    c = Case([(500, [(q + s % 4, q) for s in range(members)]), (300, [(q, q)] * members)], 8, 2, 128, extra_rows=1)
    c.up(always)
    lens = c.lens.copy()
    lens[1], lens[members + 2] = -1, c.bt.shape[1] * c.T + 1
    c.batch.keep[1].copy_(dev(lens))
    c.run().check(status=share.INVALID_ARG, left_out=(1, members + 2))


@pytest.mark.parametrize("always", [True, False])
def test_groups_beyond_what_a_block_plans_at_once(always):
    """1100 groups of two."""
    Case([(33, [(2, 1), (1 + k % 3, 1)]) for k in range(1100)], 2, 1, 64, T=8).up(always).run().check()


def test_what_pays_is_shared_and_what_does_not_is_not():
    """One group worth it beside one of two short sequences, by what is read: the others' copies of the block that the prefix ends in
    hold other values."""
    c = Case([(1500, [(2 + s % 5, 1) for s in range(60)]), (40, [(3, 1), (4, 1)])], 8, 8, 128, seed=2)
    for s in range(1, 60):  # (in the oracle's tables too: they name the first sequence's block, as far as the prefix goes)
        for p in c.cache.pools:
            p[:, int(c.bt[s, 93]), :, :, :1500 % 16] = 5.0
    c.up(False).run()
    want = c.bt.copy()
    got, _ = c.result()
    alone = Case([(1500, [(2 + s % 5, 1) for s in range(60)]), (40, [(3, 1), (4, 1)])], 8, 8, 128, seed=2).up(False).run()
    same, _ = alone.result()
    assert np.array_equal(got, same) and np.array_equal(want, c.bt)  # what differs is not read


@pytest.mark.parametrize("members,prefix", [(40, 700), (6, 9000), (120, 150)])
def test_the_same_call_gives_the_same_bits(members, prefix):
    c = Case([(prefix, [(5 + s % 30, 1) for s in range(members)])], 16, 2, 128).up().run()
    first = [x.clone() for x in c.out] + [c.lse.clone()]
    for _ in range(3):
        c.ws.fill_(0x7F)
        c.run()
        assert all(torch.equal(a, b) for a, b in zip(first, c.out + [c.lse]))


def test_without_lse_and_in_wider_rows():
    c = Case([(300, [(4, 1)] * 40)], 8, 4, 128, tp=2).up().run()
    want = [x.clone() for x in c.out]
    wide = [torch.full((c.rows, 1024), 7.0, dtype=DT[c.dtype], device=DEV) for _ in range(2)]
    for w, x in zip(wide, c.dq):
        w[:, :512] = x
    A().amoeba_attend_shared(c.layout, code(c.dtype), 0, c.dpools, c.batch, c.prefixes, [w[:, :512] for w in wide], c.scale,
                             [w[:, 512:] for w in wide], None, c.status, c.ws)
    for w, x, y in zip(wide, c.dq, want):
        assert torch.equal(w[:, 512:], y) and torch.equal(w[:, :512], x)


@pytest.mark.parametrize("always", [True, False])
def test_more_pieces_than_are_dealt(always):
    """300 sequences of 33 new tokens each, in two groups."""
    Case([(40, [(33 + s % 7, 33) for s in range(150)])] * 2, 2, 2, 64, seed=1).up(always).run().check()


def test_units_of_one_and_two_query_tiles_in_turn():
    """Groups of 100, 300, 20, 129, 128 and 513 rows a head, some over a single tile of tokens."""
    groups = [(p, [(2 + s % 3, 1) for s in range(n // 4)] + [(9, n % 4)] * (n % 4 > 0)) for p, n in
              ((300, 100), (100, 300), (700, 20), (128, 129), (129, 128), (64, 513), (500, 60), (90, 44))]
    Case(groups, 4, 1, 128, seed=4).up().run().check()


def test_long_prefix_and_one_long_rest():
    """A rest that is cut into many parts beside short ones."""
    Case([(5000, [(3, 1)] * 20 + [(6000, 1)] + [(1, 1)] * 12)], 8, 1, 128, seed=3).up().run().check()


def test_two_streams_at_once():
    cases = [Case([(400 + 100 * k, [(9, 1)] * 40)], 8, 2, 128, seed=k).up() for k in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, st in zip(cases, streams):
            c.run(st)
    for c in cases:
        c.check()


def test_captured_calls_follow_lengths_and_groups():
    """A step of tables, copies and attention is captured once and replayed as the sequences grow."""
    c = Case([(320, [(8, 1)] * 30), (64, [(8, 1)] * 10)], 8, 2, 128).up().run()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            c.run()
    for own, prefix in ((3, (320, 64)), (8, (17, 0)), (5, (0, 60)), (8, (300, 63))):
        lens = np.concatenate([np.full(30, 320 + own), np.full(10, 64 + own)]).astype(np.int32)
        c.lens[:] = lens
        c.batch.keep[1].copy_(dev(lens))
        c.prefixes.keep[1].copy_(dev(prefix))
        for o in c.out:
            o.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        c.check()


def test_prefixes_of_a_session_are_set_in_place():
    """Step after step without new memory; a captured call reads what was set last; more groups than sequences have room all the same."""
    from paper_2509_19729_b200.session import CacheSession

    s = CacheSession(model(2, 2, 64), 1, 10, 4, 4, scores=False)
    s.set_prefixes([0, 2, 4], [5, 6], 4)
    first, kept, held = s.prefixes, len(s._outgrown), torch.cuda.memory_allocated()
    for n in range(50):
        s.set_prefixes([0, n % 4, 4], [n, 6], 4, always=n % 2 == 1)
    assert len(s._outgrown) == kept and torch.cuda.memory_allocated() == held
    assert (s.prefixes.d_group_starts, s.prefixes.d_prefix_lens) == (first.d_group_starts, first.d_prefix_lens)
    assert first.keep[0].tolist() == [0, 1, 4] and first.keep[1].tolist() == [49, 6]
    s.set_prefixes([0] * 9 + [4], list(range(9)), 4)
    assert s.prefixes.num_groups == 9 and s.prefixes.keep[1].tolist() == list(range(9)) and first.keep[1].tolist() == [49, 6]
    s.set_prefixes([0], [], 4)
    assert s.prefixes.num_groups == 0
    with pytest.raises(ValueError):
        s.set_prefixes([0, 4], [1, 2], 4)


# ---------------------------------------------------------------------------------------------------- a run of them

@pytest.mark.parametrize("order,tp", [(0, 1), (1, 2)])
def test_answers_to_prompts(order, tp):
    """Prompts come in, are forked inside a block, answers grow and end, blocks come back: captured and replayed, the attention by groups
    the same as by sequences, and the same as over a cache that nothing shares."""
    from paper_2509_19729_b200.session import CacheSession

    m, T, S, NB, dt = model(8, 4, 64, 2), 16, 24, 300, torch.bfloat16
    s = CacheSession(m, tp, NB, S, 20, block_tokens=T, kv_order=order)
    flat = CacheSession(m, tp, S * 20, S, 20, block_tokens=T, kv_order=order)  # sequence b has blocks 20 b ...
    flat.block_table.copy_(torch.arange(S * 20, device=DEV).view(S, 20))
    g = torch.Generator(device=DEV).manual_seed(order)
    randn = lambda *n: torch.randn(*n, generator=g, device=DEV).to(dt)  # noqa: E731
    workers = lambda x: list(x.chunk(tp, 1))  # noqa: E731
    keys = [[[None] * 320 for _ in range(S)] for _ in range(2)]  # what every sequence should hold
    lens = np.zeros(S, int)

    def step(new, rows, longest, groups=None, prefix=None, parents=None, shared=None):
        s.advance(new, rows, longest, parents, shared)
        s.copy_forks()
        torch.cuda.synchronize()
        assert int(s.status.item()) == 0
        starts, now = s.q_starts.tolist(), s.seq_lens.tolist()
        assert now == list(new)
        k, v, q = randn(rows, 256), randn(rows, 256), randn(rows, 512)
        for layer in range(2):
            s.append(layer, None, workers(k), workers(v), None, None)
        for b in range(S):
            if parents is not None and parents[b] >= 0:
                for x in keys:
                    x[b][:shared[b]] = x[parents[b]][:shared[b]]
            for j, r in enumerate(range(starts[b], starts[b + 1])):
                i = now[b] - (starts[b + 1] - starts[b]) + j
                keys[0][b][i], keys[1][b][i] = k[r], v[r]
                assert int(s.positions[r]) == i
        if groups is None:
            return
        s.set_prefixes(groups, prefix, rows, always=True)
        shared_out, alone = ([torch.empty(rows, 512 // tp, dtype=dt, device=DEV) for _ in range(tp)] for _ in range(2))
        s.attend_shared(1, workers(q.clone()), shared_out)
        s.attend(1, workers(q.clone()), alone)
        # the flat cache: every sequence's tokens anew
        flat.set_tables(now, flat.block_table.cpu())
        flat.set_rows(np.concatenate([[0], np.cumsum(now)]), int(sum(now)), max(now))
        kk = torch.stack([keys[0][b][i] for b in range(S) for i in range(now[b])])
        vv = torch.stack([keys[1][b][i] for b in range(S) for i in range(now[b])])
        flat.append(1, None, workers(kk), workers(vv), None, None)
        flat.set_rows(starts, rows, longest)
        third = [torch.empty_like(x) for x in alone]
        flat.attend(1, workers(q.clone()), third)
        torch.cuda.synchronize()
        assert int(s.status.item()) == 0 and int(flat.status.item()) == 0
        n = starts[-1]
        for a, b, c in zip(shared_out, alone, third):
            assert torch.equal(b[:n], c[:n])  # the same tokens, read in the same order
            # both are within half a step of bf16 twice (weights and outputs) of the same value, which is an average of the values
            bound = 4 * 2.0 ** -8 * (c[:n].float().abs() + vv.float().abs().max())
            assert ((a[:n].float() - c[:n].float()).abs() <= bound).all()

    new = lens.copy()
    new[[0, 10]] = 200, 77
    step(new, 300, 200)
    parents, shared = np.full(S, -1), np.zeros(S, int)
    parents[1:10], shared[1:10] = 0, 150 + np.arange(9)
    parents[11:20], shared[11:20] = 10, 77
    lens = new.copy()
    new = lens + 1
    new[1:10], new[11:20] = shared[1:10] + 2, 78 + np.arange(9) % 3
    new[20:] = 0
    step(new, 60, 3, [0, 10, 20], [150, 77], parents, shared)
    for k in range(20):
        new = new + (new > 0)
        step(new, 24, 1, [0, 10, 20], [150, 77])
    left = int(s.free_blocks.item())
    held = s.block_refs.clone()
    s.count_blocks()
    assert torch.equal(s.block_refs, held) and left == int((held == 0).sum())
    step(np.zeros(S, int), 0, 1)
    assert int(s.free_blocks.item()) == NB and (s.block_refs == 0).all() and (s.block_table == -1).all()
