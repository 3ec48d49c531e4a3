"""A serving step of sequences that share prompts: what is measured of its operators, in plain torch and through the library.

The cache is paged, one pool per tensor-parallel worker, header-centric [layer][block][header][K/V][token][dim] or token-first
[layer][K/V][block][token][header][dim], with one block table for all workers and a count for every block of the table
entries that name it.  Three operators:

  tables   from the lengths that the sequences have to those that they are to have: free blocks handed out, blocks given back, blocks
           shared with the sequence that one is forked from; the rows of the new tokens, their positions and slots, and the blocks
           to be copied because a fork begins inside them
  copy     those blocks, all layers and workers of them, inside the pools
  shared   attention of new tokens where the sequences of a group have the same first tokens in the cache: these are read
           once for the group, the rest once for every sequence
"""
import math

import numpy as np
import torch

own = False

DT = {"fp16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda"


# ---------------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # one decoding step of a small test model: eight sequences, a handful of blocks; what counts is the call itself
        dict(name="tables_tiny", op="tables", S=8, T=16, lo=16, hi=256, qlo=1, qhi=1, free=25, prompts=0, forks=0),
        # one decoding step of a serving batch of 128 sequences: a token each, a block for one in sixteen
        dict(name="tables_step", op="tables", S=128, T=16, lo=512, hi=8192, qlo=1, qhi=1, free=561, prompts=0, forks=0),
        # a step that takes in new prompts and forks running sequences for several answers beside decoding ones
        dict(name="tables_prompts", op="tables", S=256, T=16, lo=200, hi=4096, qlo=1, qhi=1, free=9000, prompts=24, forks=60),
        # a large instance with small blocks, pieces of prompts for every sequence
        dict(name="tables_pool", op="tables", S=1024, T=8, lo=1, hi=4000, qlo=1, qhi=64, free=500000, prompts=16, forks=100),
        # the half-filled blocks of a few forks of a small model
        dict(name="copy_few", op="copy", Hkv=4, D=64, tp=1, T=16, order=0, dtype="fp16", L=2, pairs=3, cap=8),
        # 64 answers begun from running sequences: one block each, 32 layers, four workers
        dict(name="copy_forks", op="copy", Hkv=8, D=128, tp=4, T=16, order=0, dtype="bf16", L=32, pairs=64, cap=128),
        # token-first pools, as many key heads as query heads, some of the layers
        dict(name="copy_token_first", op="copy", Hkv=32, D=128, tp=2, T=16, order=1, dtype="fp16", L=8, pairs=40, cap=96),
        # eight short answers to one short prompt, a small test model
        dict(name="shared_tiny", op="shared", Hq=4, Hkv=4, D=64, tp=1, T=16, order=0, dtype="fp16", G=1, glo=8, ghi=8, plo=100,
             phi=100, loose=0, lo=8, hi=60, qlo=1, qhi=1),
        # a decoding step of 128 requests behind the same long instructions
        dict(name="shared_step", op="shared", Hq=32, Hkv=8, D=128, tp=4, T=16, order=0, dtype="bf16", G=1, glo=128, ghi=128,
             plo=8192, phi=8192, loose=0, lo=64, hi=2048, qlo=1, qhi=1),
        # several prompts of odd lengths, each shared by a few sequences, others beside them, a few new tokens each, token-first
        dict(name="shared_groups", op="shared", Hq=32, Hkv=32, D=128, tp=2, T=16, order=1, dtype="fp16", G=12, glo=1, ghi=16,
             plo=500, phi=4000, loose=5, lo=30, hi=700, qlo=1, qhi=3),
        # sixteen answers about one very long document
        dict(name="shared_long", op="shared", Hq=64, Hkv=8, D=128, tp=2, T=16, order=0, dtype="bf16", G=1, glo=16, ghi=16,
             plo=131072, phi=131072, loose=0, lo=200, hi=3000, qlo=1, qhi=1),
        # questions of many tokens each about two documents: the matrix products count
        dict(name="shared_chunk", op="shared", Hq=32, Hkv=8, D=128, tp=1, T=16, order=0, dtype="bf16", G=2, glo=6, ghi=8, plo=6000,
             phi=12288, loose=1, lo=64, hi=500, qlo=64, qhi=500),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["tables", "copy", "shared", "shared"])
    T = rng.choice([8, 16, 16, 16, 32, 64])
    if op == "tables":
        S = spread(1, 1024)
        lo = spread(1, 500)
        qlo = spread(1, 32)
        return dict(op=op, S=S, T=T, lo=lo, hi=lo + spread(16, 3500), qlo=qlo, qhi=qlo + rng.choice([0, spread(1, 32)]),
                    free=spread(600, 400000), prompts=rng.choice([0, min(S, spread(1, 16))]), forks=rng.choice([0, S // 2, S // 5]))
    if op == "copy":
        Hkv, D = rng.choice([(4, 64), (8, 128), (32, 128), (40, 128), (1, 128)])
        tp = rng.choice([t for t in (1, 2, 4, 8) if Hkv % t == 0])
        pairs = spread(1, 100)
        L = spread(1, max(1, min(32, 2 ** 27 // (pairs * 4 * T * Hkv * D))))
        return dict(op=op, Hkv=Hkv, D=D, tp=tp, T=T, order=rng.choice([0, 0, 1]), dtype=rng.choice(["fp16", "bf16"]), L=L, pairs=pairs,
                    cap=pairs + rng.choice([0, spread(1, 200)]))
    Hq, Hkv, D = rng.choice([(4, 4, 64), (12, 4, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (16, 1, 128)])
    c = dict(op=op, Hq=Hq, Hkv=Hkv, D=D, tp=rng.choice([t for t in (1, 2, 4, 8) if Hkv % t == 0]), T=T, order=rng.choice([0, 0, 1]),
             dtype=rng.choice(["fp16", "bf16"]))
    c["G"] = spread(1, 12)
    c["ghi"] = spread(1, max(2, 128 // c["G"]))
    c["glo"] = rng.randint(max(1, c["ghi"] // 2), c["ghi"])
    c["loose"] = rng.choice([0, 0, spread(1, 8)])
    if rng.random() < 0.7:  # decoding steps, a few tokens at most
        c["qhi"] = rng.choice([1, 1, 1, 2, 4])
        c["qlo"] = 1
    else:  # pieces of prompts
        c["qhi"] = spread(5, max(6, 2000 * 32 // Hq // (c["G"] * c["ghi"])))
        c["qlo"] = max(1, c["qhi"] // 4)
    c["plo"] = spread(16, max(17, min(8000, 4000 * 8 // Hkv // c["G"])))
    c["phi"] = c["plo"] + spread(1, max(2, min(20000, 50000 * 8 // Hkv // c["G"])))
    c["lo"] = c["qlo"] + spread(1, 64)
    c["hi"] = c["lo"] + spread(1, max(2, min(3000, 100000 * 8 // Hkv // (c["G"] * c["ghi"]))))
    return c


# ---------------------------------------------------------------------------------------------------------- the inputs

def _table_plan(case):
    """Lengths now and after the step, which sequence one is forked from and how much it shares: by the case alone."""
    S, T = case["S"], case["T"]
    g = np.random.RandomState(S * 131 + case["lo"] * 7 + case["hi"] + case["free"])
    old = g.randint(case["lo"], case["hi"] + 1, S)
    new = old + g.randint(case["qlo"], case["qhi"] + 1, S)
    parent, share = np.full(S, -1), np.zeros(S, int)
    order = g.permutation(S)
    fresh, forked = order[:case["prompts"]], order[case["prompts"]:][:case["forks"]]
    running = order[case["prompts"] + len(forked):]
    if len(running) == 0:
        forked = forked[:0]
    old[fresh] = 0
    for s in forked:
        t = running[g.randint(len(running))]
        parent[s], share[s] = t, g.randint(1, old[t] + 1)
        new[s] = share[s] + g.randint(1, 2 * T)
        old[s] = 0
    return old, new, parent, share


def _group_plan(case):
    """Group sizes, prefix lengths, lengths and new tokens of all sequences; the loose ones come last."""
    g = np.random.RandomState(case["G"] * 131 + case["lo"] * 7 + case["hi"] + case["plo"])
    size = g.randint(case["glo"], case["ghi"] + 1, case["G"])
    prefix = g.randint(case["plo"], case["phi"] + 1, case["G"])
    S = int(size.sum()) + case["loose"]
    rest = g.randint(case["lo"], case["hi"] + 1, S)
    q = np.minimum(g.randint(case["qlo"], case["qhi"] + 1, S), rest)
    return size, prefix, rest + np.concatenate([np.repeat(prefix, size), np.zeros(case["loose"], int)]), q


def _pool_shape(case, NB):
    Hr = case["Hkv"] // case["tp"]
    L, T, D = case.get("L", 1), case["T"], case["D"]
    return (L, NB, Hr, 2, T, D) if case["order"] == 0 else (L, 2, NB, T, Hr, D)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    i32 = dict(dtype=torch.int32, device=DEV)
    s = dict(case=case, status=torch.zeros(1, **i32), T=case["T"])
    {"tables": _prepare_tables, "copy": _prepare_copy, "shared": _prepare_shared}[case["op"]](s, case, g, i32)
    if own:
        _handles(s, case)
    return s


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV, torch.int32)


def _prepare_tables(s, c, g, i32):
    old, new, parent, share = _table_plan(c)
    S, T = c["S"], c["T"]
    held = -(-old // T)
    most = int((-(-new // T)).max())
    NB = int(held.sum()) + int(np.maximum(-(-new // T) - held, 0).sum()) + c["free"]
    ids = torch.randperm(NB, generator=g, device=DEV).to(torch.int32)
    n, col = torch.from_numpy(held).to(DEV), torch.arange(most, device=DEV)[None]
    table = torch.where(col < n[:, None], ids[((n.cumsum(0) - n)[:, None] + col).clamp(max=NB - 1)], -1).to(torch.int32).contiguous()
    refs = torch.zeros(NB, **i32)
    refs[ids[:int(held.sum())].long()] = 1
    rows = int(np.where(parent >= 0, new - share, new - old).sum())
    # a few rows more than there are new tokens, as a captured step has
    s.update(table=table, refs=refs, old=_dev(old), new=_dev(new), parent=_dev(parent), share=_dev(share), rows=rows + 5, NB=NB,
             lens=torch.zeros(S, **i32), back=torch.zeros(S, **i32), starts=torch.zeros(S + 1, **i32),
             positions=torch.zeros(rows + 5, **i32), slots=torch.zeros(rows + 5, dtype=torch.int64, device=DEV),
             pairs=torch.full((S, 2), -1, **i32), n_pairs=torch.zeros(1, **i32), left=torch.zeros(2, **i32))


def _prepare_copy(s, c, g, i32):
    n, NB = c["pairs"], 2 * c["pairs"] + 37
    ids = torch.randperm(NB, generator=g, device=DEV)[:2 * n].to(torch.int32)
    pairs = torch.full((c["cap"], 2), -1, **i32)
    pairs[:n] = ids.view(n, 2)
    s.update(pairs=pairs, n_pairs=torch.tensor([n], **i32), NB=NB,
             pools=[torch.randn(*_pool_shape(c, NB), generator=g, device=DEV, dtype=DT[c["dtype"]]) for _ in range(c["tp"])])


def _prepare_shared(s, c, g, i32):
    size, prefix, lens, q = _group_plan(c)
    T, D, tp, dt, S, rows = c["T"], c["D"], c["tp"], DT[c["dtype"]], len(lens), int(q.sum())
    whole = np.concatenate([np.repeat(prefix // T, size), np.zeros(c["loose"], int)])  # blocks that a sequence shares
    nblk = -(-lens // T)
    NB = int((prefix // T).sum() + (nblk - whole).sum()) + 3
    ids = torch.randperm(NB, generator=g, device=DEV).cpu().numpy()
    table, at, first = np.full((S, int(nblk.max())), -1), 0, np.concatenate([[0], np.cumsum(size)])
    copies = []  # blocks in which a prefix ends: every sequence has its own, with the same first tokens
    for k, p in enumerate(prefix):
        table[first[k]:first[k + 1], :p // T] = ids[at:at + p // T]
        at += p // T
    for b in range(S):
        m = int(nblk[b] - whole[b])
        table[b, whole[b]:nblk[b]] = ids[at:at + m]
        at += m
    for k, p in enumerate(prefix):
        if p % T:
            copies += [(table[first[k], p // T], table[b, p // T], p % T) for b in range(first[k] + 1, first[k + 1])]
    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=dt)  # noqa: E731
    pools = [randn(*_pool_shape(c, NB)) for _ in range(tp)]
    for a, b, n in copies:
        for p in pools:
            if c["order"] == 0:
                p[0, int(b), :, :, :n] = p[0, int(a), :, :, :n]
            else:
                p[0, :, int(b), :n] = p[0, :, int(a), :n]
    wq = c["Hq"] // tp * D
    starts = np.concatenate([[0], np.cumsum(q)])
    s.update(table=_dev(table), lens=_dev(lens), starts=_dev(starts), rows=rows, maxq=int(q.max()), pools=pools, NB=NB,
             groups=_dev(first), prefix=_dev(prefix), plan=(size, prefix, lens, q), scale=D ** -0.5,
             most=int((starts[first[1:]] - starts[first[:-1]]).max()),
             q=[randn(rows, wq) * 2 for _ in range(tp)], out=[torch.empty(rows, wq, dtype=dt, device=DEV) for _ in range(tp)],
             lse=torch.empty(rows, c["Hq"], dtype=torch.float32, device=DEV))


def _handles(s, c):
    """What a program keeps between calls: the layout, the batch's and the groups' addresses, the scratch space."""
    import paper_2509_19729_b200 as A

    D, Hkv = c.get("D", 64), c.get("Hkv", 1)
    Hq = c.get("Hq", Hkv)
    s["A"] = A
    s["layout"] = A.make_layout(dict(L=c.get("L", 1), hidden=Hq * D, Hq=Hq, Hkv=Hkv, D=D, I=Hq * D), c.get("tp", 1), s["NB"], c["T"],
                                kv_order=c.get("order", 0))
    if c["op"] == "shared":
        s["dt"] = A.DTYPE_FP16 if c["dtype"] == "fp16" else A.DTYPE_BF16
        s["batch"] = A.make_batch(s["table"], s["lens"], s["starts"], s["rows"], s["maxq"])
        s["prefixes"] = A.make_prefixes(s["groups"], s["prefix"], s["most"])
        s["ws"] = torch.empty(A.amoeba_attend_shared_workspace_bytes(s["layout"], s["batch"], s["prefixes"]), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------------------ one pass of each

def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _tables(s, advance):
    """A step, and the way back to the lengths before it: forks and prompts are finished, the others cut to what they had."""
    advance(s, s["old"], s["new"], True, s["lens"], s["left"][:1])
    advance(s, s["lens"], s["old"], False, s["back"], s["left"][1:])
    return [s[k] for k in ("lens", "starts", "positions", "slots", "pairs", "n_pairs", "table", "refs", "back", "left")]


def _own_advance(s, old, new, step, lens, left):
    if step:
        s["A"].amoeba_advance_tables(s["layout"], s["table"], s["refs"], old, new, s["parent"], s["share"], lens, s["starts"], s["rows"],
                                     None, s["positions"], s["slots"], s["pairs"], s["n_pairs"], left, s["status"])
    else:
        s["A"].amoeba_advance_tables(s["layout"], s["table"], s["refs"], old, new, None, None, lens, None, 0, None, None, None, None,
                                     None, left, s["status"])


def _own_copy(s):
    s["A"].amoeba_copy_blocks(s["layout"], s["pools"], s["pairs"], s["n_pairs"], 0, s["case"]["L"], s["status"])
    return s["pools"]


def _own_shared(s):
    s["A"].amoeba_attend_shared(s["layout"], s["dt"], 0, s["pools"], s["batch"], s["prefixes"], s["q"], s["scale"], s["out"], s["lse"],
                                s["status"], s["ws"])
    return s["out"], s["lse"]


_own = {"tables": lambda s: _tables(s, _own_advance), "copy": _own_copy, "shared": _own_shared}


# ------------------------------------------------------------------------------------------- the plain forms

def _plain_advance(s, old, new, step, lens, left):
    T, table, refs = s["T"], s["table"], s["refs"]
    old, new = old.long(), new.long()
    share = torch.where(s["parent"] >= 0, s["share"].long(), 0) if step else torch.zeros_like(old)
    base = (old + T - 1) // T + share // T  # blocks there already (a fork has none of its own)
    want = (new + T - 1) // T
    grow = (want - base).clamp(min=0)
    before = grow.cumsum(0) - grow
    free = refs == 0
    rank = free.cumsum(0)
    NB = refs.numel()
    ids = torch.zeros(NB + 1, dtype=torch.int64, device=DEV).scatter_(0, torch.where(free, rank - 1, NB), torch.arange(NB, device=DEV))
    col = torch.arange(table.shape[1], device=DEV)[None]
    more = torch.zeros(NB + 1, dtype=torch.int64, device=DEV)
    if step:
        of = table[s["parent"].long().clamp(min=0)]
        shared = col < (share // T)[:, None]
        more.scatter_add_(0, torch.where(shared, of, NB).long().flatten(), shared.long().flatten())
    gone = (col >= want[:, None]) & (col < base[:, None])
    more.scatter_add_(0, torch.where(gone, table, NB).long().flatten(), -gone.long().flatten())
    taken = (col >= base[:, None]) & (col < want[:, None])
    given = ids[(before[:, None] + col - base[:, None]).clamp(0, NB)]
    more.scatter_add_(0, torch.where(taken, given, NB).flatten(), taken.long().flatten())
    if step:
        cut = share % T > 0
        at = (cut.cumsum(0) - 1).clamp(min=0)
        src = of.gather(1, (share // T).clamp(max=table.shape[1] - 1)[:, None])[:, 0]
        pairs = torch.cat([s["pairs"], s["pairs"][:1]])
        pairs[torch.where(cut, at, len(pairs) - 1)] = torch.stack([src.long(), given.gather(1, (share // T).clamp(max=table.shape[1] - 1)[:, None])[:, 0]], 1).int()
        s["pairs"].copy_(pairs[:-1])
        s["n_pairs"].copy_(cut.sum())
        table.copy_(torch.where(shared, of, table))
    table.copy_(torch.where(taken, given, torch.where(gone, -1, table.long())))
    refs.add_(more[:-1].int())
    lens.copy_(new)
    left.copy_((refs == 0).sum())
    if step:
        first = torch.maximum(old, share)
        n = new - first
        s["starts"][1:] = n.cumsum(0)
        row = torch.arange(s["rows"], device=DEV)
        b = torch.searchsorted(s["starts"][1:].contiguous(), row.int(), right=True)
        there = b < len(old)
        b = b.clamp(max=len(old) - 1)
        index = first[b] + row - s["starts"][b]
        s["positions"].copy_(torch.where(there, index, 0))
        block = table[b, (index // T).clamp(max=table.shape[1] - 1)].long()
        s["slots"].copy_(torch.where(there, block * T + index % T, -1))


def _plain_copy(s):
    n = s["case"]["pairs"]
    src, dst = s["pairs"][:n, 0].long(), s["pairs"][:n, 1].long()
    for p in s["pools"]:
        if s["case"]["order"] == 0:
            p[:, dst] = p[:, src]
        else:
            p[:, :, dst] = p[:, :, src]
    return s["pools"]


def _cached(s, row, n, kv):
    """Keys (kv = 0) or values (1) of the cache indices below n of table rows, [..., n, Hkv, D] in 32 bits."""
    i = torch.arange(n, device=DEV)
    block, t = row.long()[..., i // s["T"]].clamp(min=0), i % s["T"]
    if s["case"]["order"] == 0:
        return torch.cat([p[0, block, :, kv, t] for p in s["pools"]], -2).float()
    return torch.cat([p[0, kv, block, t] for p in s["pools"]], -2).float()


def _plain_shared(s):
    c, D = s["case"], s["case"]["D"]
    size, prefix, lens, qn = s["plan"]
    G, dt = c["Hq"] // c["Hkv"], DT[c["dtype"]]
    q = torch.cat(s["q"], 1).view(s["rows"], c["Hkv"], G, D).float()
    out = torch.empty(s["rows"], c["Hq"] * D, dtype=dt, device=DEV)
    first = np.concatenate([[0], np.cumsum(size)])
    sets = [(first[k], first[k + 1], int(prefix[k])) for k in range(len(size))] + [(b, b + 1, 0) for b in range(first[-1], len(lens))]
    starts = np.concatenate([[0], np.cumsum(qn)])
    for a, z, P in sets:
        r0, r1 = int(starts[a]), int(starts[z])
        K, V = _cached(s, s["table"][a], P, 0), _cached(s, s["table"][a], P, 1)
        x = torch.einsum("rhgd,khd->rhgk", q[r0:r1], K).mul_(s["scale"])
        for b in range(a, z):  # each sequence's own tokens behind the prefix
            lo, hi, n = int(starts[b]), int(starts[b + 1]), int(lens[b])
            y = torch.einsum("rhgd,khd->rhgk", q[lo:hi], _cached(s, s["table"][b], n, 0)[P:]).mul_(s["scale"])
            at = torch.arange(n - (hi - lo), n, device=DEV)
            y.masked_fill_((torch.arange(P, n, device=DEV) > at[:, None])[:, None, None], -math.inf)
            own_x = x[lo - r0:hi - r0]
            top = y.amax(-1, keepdim=True)
            if P:
                top = torch.maximum(top, own_x.amax(-1, keepdim=True))
            y = (y - top).exp_()
            own_x.sub_(top).exp_()
            total = y.sum(-1, keepdim=True) + own_x.sum(-1, keepdim=True)
            o = torch.einsum("rhgk,khd->rhgd", y, _cached(s, s["table"][b], n, 1)[P:])
            if P:
                o += torch.einsum("rhgk,khd->rhgd", own_x, V)
            out[lo:hi] = (o / total).flatten(1).to(dt)
            s["lse"][lo:hi] = (total.log() + top).flatten(1)
        del K, V, x
    return list(out.chunk(c["tp"], 1)), s["lse"]


_plain = {"tables": lambda s: _tables(s, _plain_advance), "copy": _plain_copy, "shared": _plain_shared}


# -------------------------------------------------------------------------------------------- the definitions

def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "copy": _exact_copy, "shared": _exact_shared}[case["op"]](s, case)


def _exact_tables(s, c):
    """Sequence by sequence, block by block, on the host."""
    T = c["T"]
    old, new, parent, share = (s[k].tolist() for k in ("old", "new", "parent", "share"))
    table, refs = s["table"].cpu().numpy().copy(), s["refs"].cpu().numpy().copy()
    was = table.copy()
    free = iter(np.flatnonzero(refs == 0).tolist())
    pairs, starts, positions, slots = s["pairs"].cpu().numpy().copy(), [0], [], []
    n_pairs = 0
    for b in range(len(old)):
        have, at = -(-old[b] // T), old[b]
        if parent[b] >= 0:
            have, at = share[b] // T, share[b]
            table[b, :have] = was[parent[b], :have]
            np.add.at(refs, table[b, :have], 1)
        for j in range(have, -(-new[b] // T)):
            table[b, j] = next(free)
            refs[table[b, j]] = 1
        if parent[b] >= 0 and share[b] % T:
            pairs[n_pairs] = was[parent[b], have], table[b, have]
            n_pairs += 1
        positions += list(range(at, new[b]))
        slots += [int(table[b, i // T]) * T + i % T for i in range(at, new[b])]
        starts.append(len(slots))
    pad = s["rows"] - len(slots)
    left = [int((refs == 0).sum())]
    for b in range(len(old)):  # the way back
        for j in range(-(-old[b] // T), -(-new[b] // T)):
            refs[table[b, j]] -= 1
            table[b, j] = -1
    left.append(int((refs == 0).sum()))
    t = lambda x, dt=torch.int32: torch.from_numpy(np.asarray(x)).to(DEV, dt)  # noqa: E731
    return [t(new), t(starts), t(positions + [0] * pad), t(slots + [-1] * pad, torch.int64), t(pairs), t([n_pairs]), t(table), t(refs),
            t(old), t(left)]


def _exact_copy(s, c):
    pools = [p.double() for p in s["pools"]]
    for a, b in s["pairs"][:c["pairs"]].tolist():
        for p in pools:
            if c["order"] == 0:
                p[:, b] = p[:, a]
            else:
                p[:, :, b] = p[:, :, a]
    return pools


def _exact_shared(s, c):
    """Every sequence by itself over its own table row, a key head at a time."""
    G, D, Hr, T = c["Hq"] // c["Hkv"], c["D"], c["Hkv"] // c["tp"], c["T"]
    out = [torch.zeros(s["rows"], c["Hq"] // c["tp"] * D, dtype=torch.float64, device=DEV) for _ in range(c["tp"])]
    lse = torch.zeros(s["rows"], c["Hq"], dtype=torch.float64, device=DEV)
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        i = torch.arange(n, device=DEV)
        block, t = s["table"][b].long()[i // T], i % T
        hidden = i > torch.arange(n - (hi - lo), n, device=DEV)[:, None]
        for head in range(c["Hkv"]):
            r, h = divmod(head, Hr)
            p = s["pools"][r][0]
            K, V = ((p[block, h, kv, t] if c["order"] == 0 else p[kv, block, t, h]).double() for kv in (0, 1))
            q = s["q"][r][lo:hi, h * G * D:(h + 1) * G * D].reshape(hi - lo, G, D).double().transpose(0, 1)
            x = (q @ K.T * s["scale"]).masked_fill(hidden, -math.inf)
            m = x.logsumexp(-1)
            out[r][lo:hi, h * G * D:(h + 1) * G * D] = ((x - m[..., None]).exp() @ V).transpose(0, 1).flatten(1)
            lse[lo:hi, head * G:(head + 1) * G] = m.T
    return out, lse


# ----------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    T = case["T"]
    if case["op"] == "tables":
        old, new, parent, share = _table_plan(case)
        held, want = -(-old // T), -(-new // T)
        NB = int(held.sum() + np.maximum(want - held, 0).sum()) + case["free"]
        touched = int((want - held).sum())  # entries and counts written on the way and on the way back
        rows = int(np.where(parent >= 0, new - share, new - old).sum())
        return dict(bytes=4 * NB + 28 * case["S"] + 12 * (rows + 5) + 20 * touched, flops=0)
    D, Hkv = case["D"], case["Hkv"]
    if case["op"] == "copy":
        return dict(bytes=8 * case["pairs"] + 2 * case["pairs"] * case["L"] * 2 * T * Hkv * D * 2, flops=0)
    size, prefix, lens, q = _group_plan(case)
    shared = np.concatenate([np.repeat(prefix, size), np.zeros(case["loose"], int)])
    keys = int(prefix.sum() + (lens - shared).sum())  # tokens that are read, a prefix once
    pairs = int((q * lens - q * (q - 1) // 2).sum())  # of a row and a token that it sees
    rows, Hq = int(q.sum()), case["Hq"]
    blocks = int((prefix // T).sum() + (-(-lens // T) - shared // T).sum())
    return dict(bytes=4 * blocks + 8 * len(lens) + keys * Hkv * D * 4 + rows * Hq * (4 * D + 4), flops=4 * pairs * Hq * D)
