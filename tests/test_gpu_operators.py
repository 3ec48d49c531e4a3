"""The serving operators (append, attend, accumulate scores, evict) against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

import cache_reference as ref

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


class Case:
    """A cache, a batch and its rows, on the host and on the device."""

    def __init__(self, Hq=4, Hkv=2, D=128, tp=1, T=16, order=0, dtype="bf16", lens=(5,), qlens=None, L=1, layer=0,
                 extra_rows=0, lead=0, seed=0, spare=3, extra=0):
        self.m, self.tp, self.T, self.order, self.dtype, self.layer = model(Hq, Hkv, D, L), tp, T, order, dtype, layer
        self.lens = np.array(lens, np.int32)
        self.qlens = np.ones(len(lens), int) if qlens is None else np.array(qlens)
        self.starts = (lead + np.concatenate([[0], np.cumsum(self.qlens)])).astype(np.int32)
        self.rows = int(self.starts[-1]) + extra_rows
        self.NB = int(sum(-(-int(n) // T) for n in lens)) + spare
        self.cache = ref.Cache(self.m, tp, self.NB, T, order, dtype, seed)
        self.bt = ref.tables(lens, T, self.NB, seed, extra)
        g = torch.Generator().manual_seed(seed + 1)
        self.q = (torch.randn(self.rows, Hq, D, generator=g) * 2).to(DT[dtype])
        self.layout = A().make_layout(self.m, tp, self.NB, T, kv_order=order)
        self.scale = D ** -0.5

    def up(self):
        a = A()
        dev = lambda x: torch.as_tensor(x).to(DEV)  # noqa: E731
        self.dpools = [p.to(DEV) for p in self.cache.pools]
        self.dbt, self.dlens, self.dstarts = dev(self.bt), dev(self.lens), dev(self.starts)
        self.dq = [x.contiguous().flatten(1) for x in self.q.to(DEV).chunk(self.tp, 1)]
        self.batch = a.make_batch(self.dbt, self.dlens, self.dstarts, self.rows, int(max(1, self.qlens.max(initial=1))))
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.ws = torch.full((a.amoeba_attend_workspace_bytes(self.layout, self.batch),), 0x7F, dtype=torch.uint8, device=DEV)
        self.out = [torch.full((self.rows, x.shape[1]), 7.0, dtype=DT[self.dtype], device=DEV) for x in self.dq]
        self.lse = torch.full((self.rows, self.m["Hq"]), 7.0, device=DEV)
        return self

    def attend(self, window=0, stream=None):
        A().amoeba_attend(self.layout, code(self.dtype), self.layer, self.dpools, self.batch, self.dq, self.scale, window,
                          self.out, self.lse, self.status, self.ws, stream)

    def result(self):
        torch.cuda.synchronize()
        D = self.m["D"]
        out = torch.cat([o.view(self.rows, -1, D) for o in self.out], 1).double().cpu().numpy()
        return out, self.lse.double().cpu().numpy()


def check_attend(c, window=0, status=0):
    want, lse, absv, size = ref.attend(c.cache, c.layer, c.bt, c.lens, c.starts, c.q.double().numpy(), c.scale, window)
    got, got_lse = c.result()
    assert int(c.status.item()) == status
    n = int(c.lens.max(initial=0)) + 1
    mine = np.zeros(c.rows, bool)
    mine[c.starts[0]:c.starts[-1]] = True
    assert (got[~mine] == 7.0).all() and (got_lse[~mine] == 7.0).all()  # rows of no sequence
    empty = np.isneginf(lse)
    assert np.array_equal(np.isneginf(got_lse[mine]), empty[mine]) and (got[empty] == 0).all()
    vmax = max((float(p.double().abs().nan_to_num(0, 0, 0).max()) for p in c.cache.pools), default=0.0)
    tol = ref.tolerance_attend(c.dtype, c.m["D"], n, want, absv, size, vmax)
    off = np.abs(got - want)[mine]
    assert np.isfinite(got[mine]).all() and (off <= tol[mine]).all(), float((off / tol[mine]).max())
    some = mine[:, None] & ~empty
    assert (np.abs(got_lse - lse)[some] <= ref.tolerance_lse(c.m["D"], n, lse, size)[some]).all()


HEADS = [(4, 4, 64, 1), (4, 2, 128, 2), (12, 4, 64, 2), (8, 1, 128, 1), (16, 1, 64, 1), (20, 1, 128, 1), (40, 1, 128, 1)]


@pytest.mark.parametrize("Hq,Hkv,D,tp", HEADS)
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("order", [0, 1])
def test_attend_single_tokens(Hq, Hkv, D, tp, dtype, order):
    c = Case(Hq, Hkv, D, tp, order=order, dtype=dtype, lens=[1, 2, 15, 16, 17, 63, 64, 65, 0, 200, 333], seed=Hq).up()
    c.attend()
    check_attend(c)


@pytest.mark.parametrize("T", [1, 5, 8, 16, 24, 32, 48, 64, 72, 100, 128, 256, 1000])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("order", [0, 1])
def test_attend_block_sizes(T, D, order):
    c = Case(4, 2, D, 2, T=T, order=order, lens=[1, 70, 129, 31, 290], qlens=[1, 3, 40, 0, 60], seed=T).up()
    c.attend()
    check_attend(c)


@pytest.mark.parametrize("window", [0, 1, 2, 15, 16, 17, 64, 100, 1 << 30, 2 ** 31 - 1])
@pytest.mark.parametrize("G", [1, 4])
def test_attend_chunks_and_windows(window, G):
    c = Case(2 * G, 2, 128, lens=[90, 200, 7, 257, 64], qlens=[90, 1, 3, 150, 64], extra_rows=3, lead=2, seed=G).up()
    c.attend(window)
    check_attend(c, window)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,q", [(1, 33), (1, 129), (3, 50), (4, 200), (8, 77), (1, 300)])
def test_attend_long_chunks(dtype, D, G, q):
    c = Case(2 * G, 2, D, 2, dtype=dtype, order=q % 2, lens=[q + 150, q, 40, q + 1], qlens=[q, q, 1, q // 2], seed=q).up()
    c.attend()
    check_attend(c)


@pytest.mark.parametrize("q", [3, 70])
def test_attend_rows_that_see_nothing(q):
    """More new tokens than cached ones, and an empty cache: those rows are 0 with lse -inf."""
    c = Case(8, 2, 128, lens=[2, 0, 1, 30], qlens=[q, q, 2, 2], seed=3).up()
    c.attend()
    check_attend(c)


@pytest.mark.parametrize("q", [2, 65])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attend_ignores_what_no_row_sees(q, window, bad):
    """Infinities and NaN in free blocks, behind the last token and, with a window, before it."""
    c = Case(8, 2, 128, lens=[150, 83], qlens=[q, q - 1], seed=4, spare=5)
    used = {int(b): (s, i) for s in range(2) for i, b in enumerate(c.bt[s]) if b >= 0}
    for b in range(c.NB):
        for t in range(c.T):
            s, i = used.get(b, (None, 0))
            k = i * c.T + t
            hidden = s is None or k >= c.lens[s] or (window and k <= c.lens[s] - c.qlens[s] - window)
            if hidden:
                for h in range(2):
                    c.cache.at(0, b, h, 0, t)[:] = bad
                    c.cache.at(0, b, h, 1, t)[:] = bad
    if window and q > 60:  # only tokens that no row of any tile sees: with many rows a tile's first row sees the most
        pass
    c.up().attend(window)
    check_attend(c, window)


@pytest.mark.parametrize("q", [1, 6, 200])
def test_attend_hands_on_a_nan_key(q):
    """A NaN in a key that a row sees makes that row's outputs NaN, whichever token it is, and no other row's."""
    c = Case(2, 2, 128, lens=[400], qlens=[q], seed=15).up()
    clean = None
    for token in [None, *range(0, 399, 7), 399]:
        if token is not None:
            b, t = int(c.bt[0, token // 16]), token % 16
            keep = c.dpools[0][0, b, 1, 0, t, 5].clone()
            c.dpools[0][0, b, 1, 0, t, 5] = float("nan")
        c.attend()
        got, lse = c.result()
        sees = np.arange(q) + 400 - q >= (400 if token is None else token)
        assert np.isnan(got[sees, 1]).all() and np.isnan(lse[sees, 1]).all() and np.isfinite(got[~sees]).all()
        clean = got if clean is None else clean
        assert np.array_equal(got[:, 0], clean[:, 0]) and np.array_equal(got[~sees], clean[~sees])
        if token is not None:
            c.dpools[0][0, b, 1, 0, t, 5] = keep


def test_attend_large_logits_and_one_hot_rows():
    """Logits of several hundred: the maximum moves, all weight on one token."""
    for dtype in ("fp16", "bf16"):
        c = Case(4, 2, 64, dtype=dtype, lens=[300, 130], qlens=[1, 70], seed=5)
        c.q = (c.q.float() * 40).to(DT[dtype])
        c.up().attend()
        check_attend(c)


def test_attend_bad_block_ids_are_left_out():
    c = Case(8, 2, 128, lens=[100, 60, 40], qlens=[1, 40, 2], seed=6)
    c.bt[0, 2], c.bt[1, 0], c.bt[2, :3] = -1, c.NB, 2 ** 31 - 1
    c.up().attend()
    check_attend(c, status=A().ERR_BAD_BLOCK_ID)


def test_attend_bad_sequences_are_refused_alone():
    """A negative or too long length, decreasing rows, more rows than announced: nothing of that sequence is written."""
    a = A()
    c = Case(4, 2, 64, lens=[20, 30, 40], qlens=[1, 1, 1], seed=7).up()
    good = c.bt.shape[1] * c.T
    for wrong in (-1, good + 1, 2 ** 31 - 1, -2 ** 31):
        for o in c.out:
            o.fill_(7.0)
        c.status.zero_()
        c.dlens.copy_(torch.tensor([20, wrong, 40], dtype=torch.int32))
        c.attend()
        out, _ = c.result()
        assert int(c.status.item()) == a.ERR_INVALID_ARG and (out[1] == 7).all() and (out[[0, 2]] != 7).any(-1).all()
    c.dlens.copy_(torch.from_numpy(c.lens))
    for starts, rows in (([0, 1, 0, 1], 1), ([0, 1, 4, 4], 1), ([-1, 1, 2, 3], 2), ([0, 1, 2, 2 ** 31 - 1], 2)):
        for o in c.out:
            o.fill_(7.0)
        c.status.zero_()
        c.dstarts.copy_(torch.tensor(starts, dtype=torch.int32))
        c.attend()
        out, _ = c.result()
        assert int(c.status.item()) == a.ERR_INVALID_ARG


def test_attend_without_lse_and_row_starts():
    c = Case(4, 2, 128, lens=[20, 0, 300], seed=8).up()
    c.batch = A().make_batch(c.dbt, c.dlens)
    lse, c.lse = c.lse, None
    c.attend()
    c.lse = lse
    plain = [o.clone() for o in c.out]
    c.attend()
    check_attend(c)
    assert all(torch.equal(x, y) for x, y in zip(plain, c.out))


def test_attend_strided_rows_and_three_dimensions():
    a = A()
    c = Case(8, 2, 64, 2, lens=[40, 50], qlens=[3, 2], seed=9).up()
    c.attend()
    want = [o.clone() for o in c.out]
    wide = [torch.zeros(c.rows, x.shape[1] + 128, dtype=x.dtype, device=DEV) for x in c.dq]
    for w, x in zip(wide, c.dq):
        w[:, 64:64 + x.shape[1]] = x
    got = [torch.full_like(w, 3.0) for w in wide]
    n = c.dq[0].shape[1]
    a.amoeba_attend(c.layout, code(c.dtype), 0, c.dpools, c.batch, [w[:, 64:64 + n] for w in wide], c.scale, 0,
                    [g[:, 8:8 + n].view(c.rows, -1, 64) if False else g[:, 8:8 + n] for g in got], None, c.status, c.ws)
    assert all(torch.equal(g[:, 8:8 + n], w) and (g[:, :8] == 3).all() and (g[:, 8 + n:] == 3).all()
               for g, w in zip(got, want))
    three = [torch.empty(c.rows, n // 64, 64, dtype=x.dtype, device=DEV) for x in c.dq]
    a.amoeba_attend(c.layout, code(c.dtype), 0, c.dpools, c.batch, [x.view(c.rows, -1, 64) for x in c.dq], c.scale, 0, three,
                    None, c.status, c.ws)
    assert all(torch.equal(t.flatten(1), w) for t, w in zip(three, want))


def test_attend_layers_and_layer_stride():
    """Layer 1 of two, with room between the layers of the pools."""
    c = Case(4, 2, 64, lens=[33, 20], qlens=[2, 20], L=2, layer=1, seed=10)
    c.up().attend()
    check_attend(c)
    per = c.cache.pools[0][0].numel()
    stride = per + 1024
    c.layout.kv_layer_stride_bytes = stride * 2
    padded = [torch.zeros(2 * stride, dtype=DT[c.dtype], device=DEV) for _ in c.dpools]
    for p, d in zip(padded, c.dpools):
        p[:per], p[stride:stride + per] = d[0].flatten(), d[1].flatten()
    want, c.dpools = [o.clone() for o in c.out], padded
    c.attend()
    assert all(torch.equal(x, y) for x, y in zip(want, c.out))


def test_attend_offsets_past_32_bits():
    """A pool of 5 GiB whose used blocks lie at its end."""
    a = A()
    T, Hkv, D = 16, 8, 128
    block = Hkv * 2 * T * D
    NB = (5 << 30) // (block * 2)
    m = model(32, Hkv, D)
    lens = np.array([100, 40], np.int32)
    small = Case(32, Hkv, D, lens=lens, qlens=[1, 40], seed=11).up()
    small.attend()
    pool = torch.zeros(NB * block, dtype=torch.bfloat16, device=DEV)
    view = pool.view(1, NB, Hkv, 2, T, D)
    view[0, NB - small.NB:] = small.dpools[0][0]
    layout = a.make_layout(m, 1, NB, T)
    bt = torch.where(small.dbt >= 0, small.dbt + NB - small.NB, -1).to(torch.int32)
    batch = a.make_batch(bt, small.dlens, small.dstarts, small.rows, 40)
    out = [torch.empty_like(small.out[0])]
    a.amoeba_attend(layout, a.DTYPE_BF16, 0, [pool], batch, small.dq, small.scale, 0, out, None, small.status, small.ws)
    assert torch.equal(out[0], small.out[0])


def test_attend_long_sequence_beside_short_ones():
    """Split over all CTAs and joined; the definition in 64 bits with torch on the GPU."""
    for q in (1, 40):
        c = Case(8, 2, 128, lens=[17, 20000, 3, 500], qlens=[1, q, 1, min(q, 7)], seed=12).up()
        c.attend()
        out, lse = c.result()
        pool = c.dpools[0][0].double()
        for s, n in enumerate(c.lens):
            i = torch.arange(int(n), device=DEV)
            b, t = c.dbt[s].long()[i // c.T], i % c.T
            lo, hi = c.starts[s], c.starts[s + 1]
            x = c.q[lo:hi].double().to(DEV).view(hi - lo, 2, 4, 128)
            K, V = pool[b, :, 0, t], pool[b, :, 1, t]
            logit = torch.einsum("rhgd,khd->rhgk", x, K) * c.scale
            pos = int(n) - (hi - lo) + torch.arange(int(hi - lo), device=DEV)
            logit.masked_fill_((i[None] > pos[:, None])[:, None, None], -math.inf)
            w = logit.softmax(-1)
            want = torch.einsum("rhgk,khd->rhgd", w, V).reshape(hi - lo, 8, 128).cpu().numpy()
            absv = torch.einsum("rhgk,khd->rhgd", w, V.abs()).reshape(hi - lo, 8, 128).cpu().numpy()
            size = (torch.einsum("rhgd,khd->rhgk", x.abs(), K.abs()) * c.scale).amax(-1).reshape(hi - lo, 8).cpu().numpy()
            tol = ref.tolerance_attend("bf16", 128, int(n), want, absv, size, float(V.abs().max()))
            assert (np.abs(out[lo:hi] - want) <= tol).all()
            L = logit.logsumexp(-1).reshape(hi - lo, 8).cpu().numpy()
            assert (np.abs(lse[lo:hi] - L) <= ref.tolerance_lse(128, int(n), L, size)).all()


@pytest.mark.parametrize("S,Hkv", [(40, 8), (300, 1)])
def test_attend_pieces_of_many_sequences(S, Hkv):
    """Units enough to be dealt out whole before the last are cut; and more sequences than that is kept for."""
    g = np.random.default_rng(S)
    q = g.integers(33, 42, S)
    q[::7] = 1
    c = Case(Hkv, Hkv, 64, lens=q + g.integers(0, 200, S), qlens=q, seed=16).up()
    c.attend()
    check_attend(c)
    first = [o.clone() for o in c.out]
    c.attend()
    assert all(torch.equal(x, y) for x, y in zip(first, c.out))  # the same bits again


def test_attend_many_sequences_and_nothing_to_do():
    a = A()
    n = np.random.default_rng(1).integers(0, 40, 700)
    c = Case(2, 1, 64, lens=n, seed=13).up()
    c.attend()
    check_attend(c)
    e = Case(2, 1, 64, lens=[5], seed=1).up()
    none = a.make_batch(torch.empty(0, 4, dtype=torch.int32, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV))
    a.amoeba_attend(e.layout, code(e.dtype), 0, e.dpools, none, e.dq, 1.0, 0, e.out, None, e.status, e.ws)
    assert all((o == 7).all() for o in e.out)


# ---------------------------------------------------------------------------------------------------------------- append

APPEND = [(4, 4, 64, 1, 16, 0, True, 64, False), (8, 2, 128, 2, 16, 1, True, 128, False), (8, 2, 128, 2, 8, 0, False, 128, True),
          (3, 1, 64, 1, 5, 1, True, 32, True), (5, 5, 128, 5, 48, 0, True, 64, False), (4, 2, 128, 1, 16, 0, True, 0, False),
          (4, 2, 64, 2, 1, 1, False, 16, False), (4, 2, 64, 1, 16, 0, False, 0, False), (8, 8, 128, 8, 16, 1, True, 112, False)]


@pytest.mark.parametrize("Hq,Hkv,D,tp,T,order,norm,rot,inter", APPEND)
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_append(Hq, Hkv, D, tp, T, order, norm, rot, inter, dtype):
    a = A()
    c = Case(Hq, Hkv, D, tp, T, order, dtype, lens=[1, 16, 40, 0, 33, 7], qlens=[1, 1, 37, 0, 2, 7], extra_rows=2, lead=1,
             L=2, layer=1, seed=rot + D).up()
    g = torch.Generator().manual_seed(D)
    wq, wk = Hq // tp * D, Hkv // tp * D
    fused = [torch.randn(c.rows, wq + 2 * wk, generator=g).mul(3).to(DT[dtype]).to(DEV) for _ in range(tp)]
    q, k, v = ([f[:, x:y] for f in fused] for x, y in ((0, wq), (wq, wq + wk), (wq + wk, wq + 2 * wk)))
    nq, nk = (torch.randn(2, D, generator=g).to(DT[dtype]) if norm else (None, None))
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1)) if rot else None
    pos = torch.randint(0, 131072, (c.rows,), generator=g, dtype=torch.int32)
    pos[2], pos[3] = 2 ** 31 - 1, -5
    up = lambda t: None if t is None else t.to(DEV).contiguous()  # noqa: E731
    for positions in (pos, None):
        rotation = a.make_rotation(up(nq), up(nk), 1e-5, up(freq), up(positions), rot, inter)
        for o in c.out:
            o.fill_(7.0)
        pools = [p.clone() for p in c.dpools]
        a.amoeba_append_kv(c.layout, code(dtype), 1, pools, c.batch, q, k, v, rotation, c.out, c.status)
        torch.cuda.synchronize()
        assert int(c.status.item()) == 0
        index = np.zeros(c.rows, np.int64)
        owner = np.full(c.rows, -1)
        for s in range(len(c.lens)):
            lo, hi = c.starts[s], c.starts[s + 1]
            index[lo:hi] = c.lens[s] - (hi - lo) + np.arange(hi - lo)
            owner[lo:hi] = s
        p = index if positions is None else positions.numpy()
        heads = lambda t, n: torch.cat([x.reshape(c.rows, n // tp, D) for x in t], 1).double().cpu().numpy()  # noqa: E731
        f64 = lambda t: None if t is None else t.double().numpy()  # noqa: E731
        eq, zq = ref.turned(heads(q, Hq), f64(nq), 1e-5, f64(freq), p, rot, inter)
        ek, zk = ref.turned(heads(k, Hkv), f64(nk), 1e-5, f64(freq), p, rot, inter)
        mine = owner >= 0
        got = heads(c.out, Hq)
        assert (got[~mine] == 7).all()
        assert (np.abs(got - eq)[mine] <= ref.tolerance_append(dtype, D, eq, zq)[mine]).all()
        host = [x.cpu() for x in pools]
        vv = torch.cat([x.reshape(c.rows, Hkv // tp, D) for x in v], 1).cpu()
        tol = ref.tolerance_append(dtype, D, ek, zk)
        for r in np.flatnonzero(mine):
            b, t = int(c.bt[owner[r], index[r] // T]), int(index[r] % T)
            for h in range(Hkv):
                kk = c.cache.at(1, b, h, 0, t, host)
                assert (np.abs(kk.double().numpy() - ek[r, h]) <= tol[r, h]).all()
                kk[:] = c.cache.at(1, b, h, 0, t)
                assert torch.equal(c.cache.at(1, b, h, 1, t, host), vv[r, h])
                c.cache.at(1, b, h, 1, t, host)[:] = c.cache.at(1, b, h, 1, t)
        assert all(torch.equal(x, y) for x, y in zip(host, c.cache.pools))  # nothing else was written


def test_append_in_place_without_queries_and_without_rotation():
    a = A()
    c = Case(4, 2, 128, 2, lens=[20, 5], qlens=[3, 5], seed=21).up()
    k = [torch.randn(c.rows, 128, device=DEV, dtype=torch.bfloat16) for _ in range(2)]
    freq = (10000.0 ** (-torch.arange(0, 128, 2, dtype=torch.float64) / 128)).to(DEV)
    rotation = a.make_rotation(inv_freq=freq, rot_dim=128)
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, c.dq, k, k, rotation, c.out, c.status)
    first = [p.clone() for p in c.dpools]
    q = [x.clone() for x in c.dq]
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, q, k, k, rotation, q, c.status)
    assert all(torch.equal(x, y) for x, y in zip(q, c.out)) and all(torch.equal(x, y) for x, y in zip(first, c.dpools))
    for p in c.dpools:
        p.zero_()
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, None, k, k, rotation, None, c.status)
    moved = [x.clone() for x in c.dpools]
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, q, k, k, None, c.out, c.status)
    assert all(torch.equal(x, y) for x, y in zip(q, c.out))  # nothing is done to the queries
    for s in range(2):
        for j in range(c.qlens[s]):
            i = c.lens[s] - c.qlens[s] + j
            b, t, r = int(c.bt[s, i // 16]), i % 16, c.starts[s] + j
            for w in range(2):
                assert torch.equal(c.dpools[w][0, b, 0, 0, t], k[w][r]) and torch.equal(c.dpools[w][0, b, 0, 1, t], k[w][r])
                assert torch.equal(moved[w][0, b, 0, 1, t], k[w][r])
    assert int(c.status.item()) == 0


def test_append_bad_blocks_and_sequences():
    a = A()
    c = Case(4, 2, 64, lens=[20, 30, 3], qlens=[2, 2, 4], seed=22)
    c.bt[0, 1] = c.NB
    c.up()
    k = [torch.randn(c.rows, 128, device=DEV, dtype=torch.bfloat16)]
    before = c.dpools[0].clone()
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, c.dq, k, k, None, c.out, c.status)
    torch.cuda.synchronize()
    assert int(c.status.item()) in (a.ERR_BAD_BLOCK_ID, a.ERR_INVALID_ARG)
    assert torch.equal(c.out[0][:4], c.dq[0][:4]) and (c.out[0][4:] == 7).all()  # more new tokens than cached: refused
    changed = (c.dpools[0] != before).flatten(3).any(-1)[0].any(-1).nonzero().flatten().tolist()
    assert changed == [int(c.bt[1, 1])]


# ---------------------------------------------------------------------------------------------------------------- scores

def run_scores(c, window=0, scored=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    shape = (c.m["L"], c.NB, c.m["Hkv"] // c.tp, c.T)
    old = [torch.randn(*shape, generator=g).abs() for _ in range(c.tp)]
    got = [o.to(DEV) for o in old]
    ds = None if scored is None else torch.tensor(scored, dtype=torch.int32, device=DEV)
    A().amoeba_accumulate_scores(c.layout, code(c.dtype), c.layer, c.dpools, c.batch, c.dq, c.scale, window, c.lse, ds, got,
                                 c.status)
    torch.cuda.synchronize()
    return old, got


def check_scores(c, window=0, scored=None, status=0):
    c.attend(window)
    old, got = run_scores(c, window, scored)
    assert int(c.status.item()) == status
    lse = c.lse.double().cpu().numpy()
    Hr = c.m["Hkv"] // c.tp
    at = lambda p, s, h, i: p[h // Hr][c.layer, int(c.bt[s, i // c.T]), h % Hr, i % c.T]  # noqa: E731
    want, tol = ref.scores(c.cache, c.layer, c.bt, c.lens, c.starts, c.q.double().numpy(), c.scale, window, lse, scored,
                           lambda s, h, i: float(at(old, s, h, i)))
    host = [x.cpu() for x in got]
    for (s, h), w in want.items():
        for i in range(len(w)):
            if 0 <= c.bt[s, i // c.T] < c.NB:
                x = at(host, s, h, i)
                assert abs(float(x) - w[i]) <= tol[s, h][i], (s, h, i, float(x), w[i])
                x.copy_(at(old, s, h, i))
    assert all(torch.equal(x, y) for x, y in zip(host, old))  # no other slot was written


@pytest.mark.parametrize("Hq,Hkv,D,tp", HEADS)
@pytest.mark.parametrize("order", [0, 1])
def test_scores_single_tokens(Hq, Hkv, D, tp, order):
    lens = [1, 16, 17, 64, 65, 0, 130]
    check_scores(Case(Hq, Hkv, D, tp, order=order, dtype="fp16" if order else "bf16", lens=lens, seed=30).up(),
                 scored=[n - 1 for n in lens])


@pytest.mark.parametrize("T,window", [(16, 0), (16, 20), (5, 0), (64, 1), (8, 70)])
@pytest.mark.parametrize("G", [1, 4])
def test_scores_chunks(T, window, G):
    c = Case(2 * G, 2, 128, 2, T=T, lens=[90, 150, 7, 64, 20], qlens=[32, 1, 9, 64, 0], L=2, layer=1, extra_rows=1, seed=31).up()
    check_scores(c, window, scored=[58, 200, 0, 0, 13])
    check_scores(c, window)


def test_scores_bad_blocks():
    c = Case(4, 2, 64, lens=[60, 20], qlens=[3, 1], seed=32)
    c.bt[0, 1] = -7
    check_scores(c.up(), status=A().ERR_BAD_BLOCK_ID)


def test_scores_of_long_sequences():
    """Several passes of 128 rows over many tiles, a window, and a share that ends inside a head; against torch in 64 bits."""
    for window in (0, 700):
        c = Case(8, 2, 128, 2, order=1, lens=[2900, 40, 1111], qlens=[100, 40, 1], seed=34).up()
        c.attend(window)
        prior = [2800, 0, 1200]
        old, got = run_scores(c, window, prior)
        for s, n in enumerate(c.lens):
            n = int(n)
            i = torch.arange(n, device=DEV)
            b, t = c.dbt[s].long()[i // 16], i % 16
            lo, hi = int(c.starts[s]), int(c.starts[s + 1])
            pos = n - (hi - lo) + torch.arange(hi - lo, device=DEV)[:, None]
            sees = (i[None] <= pos) & ((i[None] > pos - window) if window else True)
            for h in range(2):
                K = c.dpools[h][0, 0, b, t, 0].double()
                q = c.q[lo:hi, h * 4:h * 4 + 4].double().to(DEV)
                x = torch.einsum("rgd,kd->rgk", q, K) * c.scale
                L = c.lse[lo:hi, h * 4:h * 4 + 4].double()[..., None]
                p = torch.where(sees[:, None], (x - L).exp(), 0.0)
                was = old[h][0].to(DEV)[b, 0, t].double() * (i < prior[s])
                size = torch.einsum("rgd,kd->rgk", q.abs(), K.abs()) * c.scale
                e = (128 + 4) * 2.0 ** -23 * size + 3 * 2.0 ** -23 * (x.abs() + L.abs()) + 2.0 ** -20 + (4 * (hi - lo) + 4) * 2.0 ** -23
                off = (got[h][0][b, 0, t].double() - (was + p.sum((0, 1)))).abs()
                assert (off <= (p * e).sum((0, 1)) + was.abs() * 2.0 ** -22 + 1e-37).all()


def test_scores_sum_to_the_rows():
    """Every row gives away weight 1 for each query head; twice the same call, twice the same bits."""
    c = Case(32, 8, 128, 4, lens=[5000, 333, 64], qlens=[32, 7, 1], seed=33).up()
    c.attend()
    _, a = run_scores(c)
    _, b = run_scores(c)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    for s, n in enumerate(c.lens):
        total = sum(float(a[w][0, c.dbt[s, i].long(), :, :max(0, min(16, n - 16 * i))].double().sum())
                    for w in range(4) for i in range(-(-int(n) // 16)))
        assert abs(total - 32 * c.qlens[s]) <= 32 * c.qlens[s] * 1e-4


# ---------------------------------------------------------------------------------------------------------------- evict

def run_evict(c, scores, budget, recent, in_place, layers=(0, None), dst_blocks=None):
    a = A()
    l0, l1 = layers[0], c.m["L"] if layers[1] is None else layers[1]
    pools, dscores = [p.clone() for p in c.dpools], None if scores is None else [x.to(DEV) for x in scores]
    dst = c.bt if in_place else dst_blocks
    ddst = c.dbt if in_place else torch.from_numpy(dst).to(DEV)
    new = torch.full((len(c.lens),), 99, dtype=torch.int32, device=DEV)
    ws = torch.full((max(16, a.amoeba_evict_workspace_bytes(c.layout, l1 - l0, len(c.lens), budget)),), 0x7F,
                    dtype=torch.uint8, device=DEV)
    a.amoeba_evict_kv(c.layout, l0, l1, pools, dscores, c.dbt, c.dlens, ddst, budget, recent, new, c.status, ws)
    torch.cuda.synchronize()
    return pools, dscores, new, dst


def check_evict(c, scores, budget, recent, in_place, layers=(0, None), dst_blocks=None, status=0, refused=()):
    pools, dscores, new, dst = run_evict(c, scores, budget, recent, in_place, layers, dst_blocks)
    assert int(c.status.item()) == status
    want = [p.clone() for p in c.cache.pools]
    ws = None if scores is None else [x.clone() for x in scores]
    Hr = c.m["Hkv"] // c.tp
    for s, n in enumerate(c.lens):
        if s in refused:
            continue
        for l in range(layers[0], c.m["L"] if layers[1] is None else layers[1]):
            for h in range(c.m["Hkv"]):
                w = h // Hr
                x = None if scores is None else np.array([float(scores[w][l, c.bt[s, i // c.T], h % Hr, i % c.T]) for i in range(n)])
                for j, i in enumerate(ref.kept(x, int(n), budget, recent)):
                    sb, st, db, t = int(c.bt[s, i // c.T]), i % c.T, int(dst[s, j // c.T]), j % c.T
                    for kv in range(2):
                        c.cache.at(l, db, h, kv, t, want)[:] = c.cache.at(l, sb, h, kv, st)
                    if scores is not None:
                        ws[w][l, db, h % Hr, t] = scores[w][l, sb, h % Hr, st]
    bits = lambda t: t.cpu().contiguous().view(torch.int16)  # noqa: E731
    assert all(torch.equal(bits(x), bits(y)) for x, y in zip(pools, want))
    if scores is not None:
        assert all(torch.equal(x.cpu().view(torch.int32), y.view(torch.int32)) for x, y in zip(dscores, ws))
    assert new.tolist() == [-1 if s in refused else min(int(n), budget) for s, n in enumerate(c.lens)]


def draw_scores(c, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(c.tp):
        x = torch.randn(c.m["L"], c.NB, c.m["Hkv"] // c.tp, c.T, generator=g)
        if kind == "ties":
            x = x.mul(2).round() / 2
        elif kind == "equal":
            x = torch.zeros_like(x) * torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)  # 0 and -0 are equal
        elif kind == "special":
            x[x > 1] = math.inf
            x[x < -1] = -math.inf
            x[(x > 0) & (x < 0.4)] = math.nan
            x[(x < 0) & (x > -0.1)] = 1e-42
        out.append(x)
    return out


EVICT = [(4, 4, 64, 1, 16, 0), (4, 2, 128, 2, 8, 1), (8, 2, 64, 1, 5, 0), (3, 3, 128, 3, 32, 1)]


def evict_case(shape, lens, L=2, seed=40):
    Hq, Hkv, D, tp, T, order = shape
    spare = sum(-(-int(n) // T) for n in lens) + 2
    c = Case(Hq, Hkv, D, tp, T, order, "bf16", lens=lens, L=L, seed=seed, spare=spare).up()
    used = set(c.bt[c.bt >= 0].tolist())
    free = np.array([b for b in range(c.NB) if b not in used], np.int32)
    dst, k = np.full_like(c.bt, -1), 0
    for s, n in enumerate(lens):
        m = -(-int(n) // T)
        dst[s, :m] = free[k:k + m]
        k += m
    return c, dst


@pytest.mark.parametrize("shape", EVICT)
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "special"])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(shape, kind, in_place):
    for budget, recent in ((1, 0), (1, 1), (17, 5), (64, 64), (64, 0), (100, 37)):
        c, dst = evict_case(shape, [0, 1, 16, 17, 63, 64, 65, 150, 301])
        check_evict(c, draw_scores(c, kind), budget, recent, in_place, dst_blocks=dst)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_layer_range_and_no_scores(in_place):
    c, dst = evict_case(EVICT[1], [70, 20, 130], L=3)
    check_evict(c, draw_scores(c, "random"), 32, 8, in_place, layers=(1, 2), dst_blocks=dst)
    check_evict(c, None, 24, 24, in_place, dst_blocks=dst)


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_refuses_sequences_one_by_one(in_place):
    a = A()
    c, dst = evict_case(EVICT[0], [70, 90, 130, 40])
    c.bt[1, 5] = c.NB  # a bad id anywhere in the sequence, behind the budget too
    if not in_place:
        dst[2, 0] = -1
    c.dbt.copy_(torch.from_numpy(c.bt))
    check_evict(c, draw_scores(c, "random"), 48, 8, in_place, dst_blocks=dst, status=a.ERR_BAD_BLOCK_ID,
                refused=(1,) if in_place else (1, 2))
    c, dst = evict_case(EVICT[0], [70, 90, 130, 40])
    c.dlens.copy_(torch.tensor([70, -1, 2 ** 31 - 1, 40], dtype=torch.int32))
    check_evict(c, draw_scores(c, "random"), 48, 8, in_place, dst_blocks=dst, status=a.ERR_INVALID_ARG, refused=(1, 2))
    if not in_place:
        c, dst = evict_case(EVICT[0], [70, 20])
        check_evict(c, draw_scores(c, "random"), 48, 8, False, dst_blocks=np.ascontiguousarray(dst[:, :2]), status=a.ERR_INVALID_ARG,
                    refused=(0,))


@pytest.mark.parametrize("elem,D", [(1, 80), (4, 96)])
def test_evict_moves_opaque_elements(elem, D):
    """8- and 32-bit elements and head sizes that the other operators do not take."""
    a = A()
    m = model(2, 2, D)
    NB, T = 20, 16
    layout = a.make_layout(m, 1, NB, T, elem_bytes=elem)
    pool = torch.randint(0, 256, (1, NB, 2, 2, T, D * elem), dtype=torch.uint8, device=DEV)
    scores = torch.rand(1, NB, 2, T, device=DEV)
    bt = torch.randperm(NB, device=DEV).to(torch.int32).view(1, NB)
    lens, new = torch.tensor([NB * T - 3], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(a.amoeba_evict_workspace_bytes(layout, 1, 1, 100), dtype=torch.uint8, device=DEV)
    before, s0 = pool.cpu(), scores.cpu()
    a.amoeba_evict_kv(layout, 0, 1, [pool], [scores], bt, lens, bt, 100, 10, new, status, ws)
    hb, n = bt.cpu().numpy()[0], int(lens.item())
    for h in range(2):
        x = np.array([float(s0[0, hb[i // T], h, i % T]) for i in range(n)])
        for j, i in enumerate(ref.kept(x, n, 100, 10)):
            assert torch.equal(pool[0, hb[j // T], h, :, j % T].cpu(), before[0, hb[i // T], h, :, i % T])
    assert int(new.item()) == 100 and int(status.item()) == 0


def test_evict_long_sequences():
    """Tens of thousands of tokens, in place and out of place, against a stable sort on the GPU."""
    a = A()
    T, D, Hkv = 16, 64, 2
    for n, budget, recent in ((40000, 9000, 100), (70001, 70000, 5), (33333, 200, 0)):
        nb = -(-n // T)
        NB = 2 * nb + 1
        layout = a.make_layout(model(2, Hkv, D), 1, NB, T)
        g = torch.Generator(device=DEV).manual_seed(n)
        pool = torch.randn(1, NB, Hkv, 2, T, D, generator=g, device=DEV).to(torch.bfloat16)
        scores = torch.randn(1, NB, Hkv, T, generator=g, device=DEV).mul(50).round()
        ids = torch.randperm(NB, generator=g, device=DEV).to(torch.int32)
        src, dst = ids[:nb].view(1, nb).contiguous(), ids[nb:2 * nb].view(1, nb).contiguous()
        lens = torch.tensor([n], dtype=torch.int32, device=DEV)
        ws = torch.empty(a.amoeba_evict_workspace_bytes(layout, 1, 1, budget), dtype=torch.uint8, device=DEV)
        i = torch.arange(n, device=DEV)
        x = scores[0, src[0].long()[i // T], :, i % T].T.clone()
        x[:, n - recent:] = math.inf
        best = x.sort(dim=-1, descending=True, stable=True).indices[:, :budget].sort(-1).values
        for to in (dst, src):
            p, sc, new = pool.clone(), scores.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            a.amoeba_evict_kv(layout, 0, 1, [p], [sc], src, lens, to, budget, recent, new, status, ws)
            j = torch.arange(budget, device=DEV)
            for h in range(Hkv):
                f = best[h]
                sb, db = src[0].long()[f // T], to[0].long()[j // T]
                assert torch.equal(p[0, db, h, :, j % T], pool[0, sb, h, :, f % T])
                assert torch.equal(sc[0, db, h, j % T], scores[0, sb, h, f % T])
            assert int(new.item()) == budget and int(status.item()) == 0


def test_evict_more_scores_than_fit_on_chip():
    """Half a million tokens of one small head: the scores are read anew in every pass."""
    a = A()
    T, n, budget = 32, 500001, 70000
    nb = -(-n // T)
    layout = a.make_layout(model(1, 1, 8), 1, nb, T)
    g = torch.Generator(device=DEV).manual_seed(3)
    pool = torch.randn(1, nb, 1, 2, T, 8, generator=g, device=DEV).to(torch.bfloat16)
    scores = torch.randn(1, nb, 1, T, generator=g, device=DEV).mul(1000).round()
    bt = torch.randperm(nb, generator=g, device=DEV).to(torch.int32).view(1, nb)
    lens, new = torch.tensor([n], dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(a.amoeba_evict_workspace_bytes(layout, 1, 1, budget), dtype=torch.uint8, device=DEV)
    i = torch.arange(n, device=DEV)
    x = scores[0, bt[0].long()[i // T], 0, i % T].clone()
    x[n - 100:] = math.inf
    f = x.sort(descending=True, stable=True).indices[:budget].sort().values
    p, sc = pool.clone(), scores.clone()
    a.amoeba_evict_kv(layout, 0, 1, [p], [sc], bt, lens, bt, budget, 100, new, status, ws)
    j = torch.arange(budget, device=DEV)
    sb, db = bt[0].long()[f // T], bt[0].long()[j // T]
    assert torch.equal(p[0, db, 0, :, j % T], pool[0, sb, 0, :, f % T]) and torch.equal(sc[0, db, 0, j % T], scores[0, sb, 0, f % T])
    assert int(new.item()) == budget and int(status.item()) == 0


# ------------------------------------------------------------------------------------------------- streams, graphs, together

def test_other_streams_and_captured_graphs_that_share_a_workspace():
    """A captured call reads the lengths, tables and rows that are there when it is replayed; two graphs use one workspace
    in turn."""
    c = Case(8, 2, 128, 2, lens=[900, 40, 3], seed=50).up()
    d = Case(8, 2, 128, 2, lens=[60, 1500, 30], qlens=[1, 40, 2], seed=51).up()
    d.ws = c.ws if c.ws.numel() >= d.ws.numel() else d.ws
    c.ws = d.ws
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.attend(stream=side)
    side.synchronize()
    check_attend(c)
    graphs = []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.attend()
            run = [torch.zeros(1, x.NB, 2 // x.tp, x.T, device=DEV) for _ in range(x.tp)]
            A().amoeba_accumulate_scores(x.layout, code(x.dtype), 0, x.dpools, x.batch, x.dq, x.scale, 0, x.lse, None, run, x.status)
        graphs.append(g)
    for step in range(3):
        c.lens = np.array([900 - step * 333, 40 + step, 3 - step], np.int32)
        c.dlens.copy_(torch.from_numpy(c.lens))
        for o in c.out + d.out:
            o.fill_(7.0)
        for g in graphs:
            g.replay()
        check_attend(c)
        check_attend(d)


def test_two_calls_at_once():
    """Two streams, two workspaces, the same cache."""
    c = Case(8, 2, 128, 2, lens=[3000, 40, 800], qlens=[1, 1, 1], seed=52).up()
    d = Case(8, 2, 128, 2, lens=[3000, 40, 800], qlens=[90, 30, 1], seed=52).up()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for x, st in zip((c, d), streams):
            x.attend(stream=st)
    torch.cuda.synchronize()
    check_attend(c)
    check_attend(d)


def test_batches_without_rows():
    """No new tokens: nothing to attend or append, and new tokens' scores start at zero."""
    a = A()
    c = Case(4, 2, 64, lens=[40, 20], qlens=[0, 0], seed=53).up()
    assert c.rows == 0
    c.attend()
    a.amoeba_append_kv(c.layout, 1, 0, c.dpools, c.batch, c.dq, [x[:, :128] for x in c.dq], [x[:, :128] for x in c.dq], None, c.out,
                       c.status)
    old, got = run_scores(c, scored=[10, 20])
    torch.cuda.synchronize()
    for s, (n, k) in enumerate(((40, 10), (20, 20))):
        i = torch.arange(n)
        b, t = torch.from_numpy(c.bt[s]).long()[i // 16], i % 16
        want = torch.where(i[:, None] < k, old[0][0][b, :, t], torch.zeros(()))
        assert torch.equal(got[0][0].cpu()[b, :, t], want)
    assert int(c.status.item()) == 0


def test_a_captured_call_outlives_a_larger_workspace():
    """A call captured before the session's workspace grew still has its own to work in."""
    from paper_2509_19729_b200.session import CacheSession

    s = CacheSession(model(4, 2, 64), 1, 80, 2, 40, device=DEV)
    g = torch.Generator().manual_seed(61)
    for pool in s.pools:
        n = pool.numel() // 2
        pool.view(torch.bfloat16).copy_(torch.randn(n, generator=g).to(torch.bfloat16))
    s.set_tables([640, 600], torch.arange(80, dtype=torch.int32).view(2, 40))
    q = torch.randn(2, 256, generator=g).to(torch.bfloat16).to(DEV)
    want, out = torch.empty_like(q), torch.zeros_like(q)
    s.attend(0, [q], [want])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.attend(0, [q], [out])
    before = s.workspace.data_ptr()
    s._room(4 * s.workspace.numel())
    assert s.workspace.data_ptr() != before
    taken = [torch.full((1 << 16,), -1, dtype=torch.int32, device=DEV) for _ in range(64)]
    graph.replay()
    assert torch.equal(out, want) and int(s.status.item()) == 0
    assert all(bool((t == -1).all()) for t in taken)


def test_a_generation_with_eviction_and_a_transformation():
    """Append, attend, accumulate and evict in turn, two layers, as a serving loop calls them; then the instance is split
    TP 1 -> 2 -> its attention is the same to the bit."""
    import workloads  # noqa: F401
    from paper_2509_19729_b200.session import CacheSession, Session

    a = A()
    m = model(8, 4, 64, L=2)
    S, budget, recent = 3, 48, 8
    s = CacheSession(m, 1, 40, S, 8, dtype="bf16", device=DEV)
    g = torch.Generator().manual_seed(60)
    bt = np.random.default_rng(0).permutation(40)[:24].reshape(3, 8).astype(np.int32)
    freq = (10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64)).to(DEV)
    host = {(l, b): [[] for _ in range(4)] for l in range(2) for b in range(S)}  # per head: [key, value, score]
    position = np.zeros(S, np.int64)
    lens = np.zeros(S, np.int64)

    def step(new):
        nonlocal lens
        rows = int(sum(new))
        starts = np.concatenate([[0], np.cumsum(new)])
        lens = lens + new
        s.set_tables(lens, bt)
        pos = np.concatenate([position[b] + np.arange(new[b]) for b in range(S)])
        for b in range(S):
            position[b] += new[b]
        s.set_rows(starts, rows, max(new))
        for l in range(2):
            q, k, v = ((torch.randn(rows, w, generator=g)).to(torch.bfloat16).to(DEV) for w in (512, 256, 256))
            rot = a.make_rotation(inv_freq=freq, positions=torch.from_numpy(pos).to(torch.int32).to(DEV), rot_dim=64)
            q_out, out = torch.empty_like(q), torch.empty_like(q)
            lse = torch.empty(rows, 8, device=DEV)
            s.append(l, [q], [k], [v], rot, [q_out])
            s.attend(l, [q_out], [out], lse)
            prior = lens - new
            s.accumulate(l, [q_out], lse, scored_lens=torch.from_numpy(prior).to(torch.int32).to(DEV))
            kk, _ = ref.turned(k.view(rows, 4, 64).double().cpu().numpy(), None, 0, freq.cpu().numpy(), pos, 64, False)
            for b in range(S):
                for h in range(4):
                    for r in range(starts[b], starts[b + 1]):
                        host[l, b][h].append([kk[r, h], v.view(rows, 4, 64)[r, h].double().cpu().numpy(), 0.0])
                    K = np.array([x[0] for x in host[l, b][h]])
                    V = np.array([x[1] for x in host[l, b][h]])
                    for r in range(starts[b], starts[b + 1]):
                        n = len(K) - (starts[b + 1] - 1 - r)
                        for gq in range(2):
                            x = K[:n] @ q_out.view(rows, 8, 64)[r, h * 2 + gq].double().cpu().numpy() / 8
                            p = np.exp(x - x.max())
                            p /= p.sum()
                            want = p @ V[:n]
                            got = out.view(rows, 8, 64)[r, h * 2 + gq].double().cpu().numpy()
                            # the keys of the cache are rounded once more: a logit moves by up to 2^-8 of sum |q||k|
                            slack = 2 ** -8 * (np.abs(K[:n]) @ np.abs(q_out.view(rows, 8, 64)[r, h * 2 + gq].double().cpu().numpy())).max() / 8
                            bound = (2 * slack + 3 * 2 ** -8) * (p @ np.abs(V[:n])) + 2 ** -8 * np.abs(want)
                            assert (np.abs(got - want) <= bound).all()
                            for i in range(n):
                                host[l, b][h][i][2] += p[i]

    step([70, 20, 1])
    for _ in range(3):
        step([1, 1, 1])
    # cut: the host keeps what the device's own scores say, which are close to the host's sums
    for l in range(2):
        for b in range(S):
            for h in range(4):
                n = int(lens[b])
                dev = np.array([float(s.score_pools[0][l, bt[b, i // 16], h, i % 16]) for i in range(n)])
                want = np.array([x[2] for x in host[l, b][h]])
                assert np.allclose(dev, want, rtol=0.1, atol=0.02)
                host[l, b][h] = [host[l, b][h][i] for i in ref.kept(dev.astype(np.float32), n, budget, recent)]
    s.evict(budget, recent)
    lens = np.minimum(lens, budget)
    assert s.new_lens.tolist() == lens.tolist()
    for _ in range(2):
        step([1, 1, 1])
    step([5, 9, 2])
    assert int(s.status.item()) == 0

    # TP 1 -> 2: the same cache in two pools gives the same attention
    t = Session(m, 1, 2, 40, 40, S, 8, 24, weights=False, device=DEV)
    t.set_tables(lens, np.where(np.arange(8)[None] * 16 < lens[:, None], bt, -1), free_list=np.arange(40)[::-1].copy())
    t.src_pools[0].copy_(s.pools[0])
    t.step()
    q = torch.randn(3, 512, generator=g).to(torch.bfloat16).to(DEV)
    o1, o2 = torch.empty_like(q), [torch.empty(3, 256, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    lse1, lse2 = torch.empty(3, 8, device=DEV), torch.empty(3, 8, device=DEV)
    s.set_tables(lens, bt)
    s.set_rows(None, 3, 1)
    s.attend(1, [q], [o1], lse1)
    batch = a.make_batch(t.dst_bt, t.seq_lens)
    ws = torch.empty(a.amoeba_attend_workspace_bytes(t.dst_layout, batch), dtype=torch.uint8, device=DEV)
    a.amoeba_attend(t.dst_layout, a.DTYPE_BF16, 1, t.dst_pools, batch, [x.contiguous() for x in q.chunk(2, 1)], 64 ** -0.5, 0, o2,
                    lse2, t.status, ws)
    assert torch.equal(torch.cat(o2, 1), o1) and torch.equal(lse1, lse2) and int(t.status.item()) == 0
