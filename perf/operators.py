"""The operators on a paged KV cache: what is measured of them, in plain torch and through the library.

An instance's cache is held as the library lays it out: one pool per tensor-parallel worker, header-centric
[layer][block][header][K/V][token][dim] or token-first [layer][K/V][block][token][header][dim], with one block table for
all workers.  Four operators work on it:

  append   norms of the new tokens' queries and keys for each head, the rotation by position, and the write of the new
           keys and values into the cache, in one pass
  attend   attention of a chunk of new tokens (one token or many, ragged over the sequences) over the cache
  scores   the attention weight that every cached token got from a set of queries, summed over the queries and over the
           query heads that share its key
  evict    the cache of long sequences cut to a budget: the most recent tokens and, per layer and key head, those with the
           highest scores, packed into fewer blocks
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
        # one decoding step of a serving batch of 128 (32 query heads on 8 key heads of 128), four workers
        dict(name="append_step", op="append", Hq=32, Hkv=8, D=128, tp=4, T=16, order=0, dtype="bf16", S=128, lo=512,
             hi=8192, qlo=1, qhi=1, norm=True, rot=128, interleaved=False),
        # the prompts of a few new sequences at once, as many key heads as query heads, a token-first pool, pairs of
        # neighbours rotated, no norms
        dict(name="append_prompts", op="append", Hq=32, Hkv=32, D=128, tp=2, T=16, order=1, dtype="fp16", S=7, lo=700,
             hi=3000, qlo=700, qhi=2900, norm=False, rot=128, interleaved=True),
        # the smallest decoding step: eight short sequences of a two-layer test model; what counts is the call itself
        dict(name="attend_tiny", op="attend", Hq=4, Hkv=4, D=64, tp=1, T=16, order=0, dtype="fp16", S=8, lo=16, hi=256,
             long=0, qlo=1, qhi=1, window=0),
        # a decoding step of 128 sequences of 512 to 8192 tokens, grouped heads, four workers: the bytes of the cache
        dict(name="attend_step", op="attend", Hq=32, Hkv=8, D=128, tp=4, T=16, order=0, dtype="bf16", S=128, lo=512,
             hi=8192, long=0, qlo=1, qhi=1, window=0),
        # one very long context beside 31 short ones: the work has to be spread although one sequence holds most of it
        dict(name="attend_long", op="attend", Hq=64, Hkv=8, D=128, tp=2, T=16, order=0, dtype="bf16", S=32, lo=256,
             hi=2048, long=131072, qlo=1, qhi=1, window=0),
        # a chunk of four prompts over what is cached of them: the matrix products count
        dict(name="attend_chunk", op="attend", Hq=32, Hkv=8, D=128, tp=1, T=16, order=0, dtype="bf16", S=4, lo=6000,
             hi=12288, long=0, qlo=1800, qhi=2048, window=0),
        # decoding steps and pieces of prompts in one ragged batch, a sliding window, a token-first pool, odd lengths
        dict(name="attend_mixed", op="attend", Hq=32, Hkv=32, D=128, tp=2, T=16, order=1, dtype="fp16", S=24, lo=300,
             hi=4096, long=0, qlo=1, qhi=300, window=1024),
        # one decoding step's weight on 64 sequences, to drop what the newest token does not look at
        dict(name="scores_step", op="scores", Hq=32, Hkv=8, D=128, tp=4, T=16, order=0, dtype="bf16", S=64, lo=512,
             hi=8192, qlo=1, qhi=1, window=0),
        # the votes of a prompt's last 32 queries on the whole prompt, before it is cut
        dict(name="scores_prompts", op="scores", Hq=32, Hkv=8, D=128, tp=1, T=16, order=0, dtype="bf16", S=6, lo=4000,
             hi=32768, qlo=32, qhi=32, window=0),
        # short sequences of a small model cut to 128 tokens
        dict(name="evict_short", op="evict", Hq=4, Hkv=4, D=64, tp=1, T=16, order=0, dtype="fp16", L=2, S=8, lo=100,
             hi=256, long=0, budget=128, keep=16),
        # a batch of prompts cut to 1024 tokens, some of them shorter than that, two layers at a time
        dict(name="evict_prompts", op="evict", Hq=32, Hkv=8, D=128, tp=2, T=16, order=0, dtype="bf16", L=2, S=32, lo=700,
             hi=8192, long=0, budget=1024, keep=64),
        # one very long context cut to an eighth
        dict(name="evict_long", op="evict", Hq=64, Hkv=8, D=128, tp=2, T=16, order=0, dtype="bf16", L=1, S=1, lo=512,
             hi=1024, long=131072, budget=16384, keep=256),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    Hq, Hkv, D = rng.choice([(4, 4, 64), (12, 4, 64), (32, 32, 128), (32, 8, 128), (40, 40, 128), (64, 8, 128), (16, 1, 128)])
    tp = rng.choice([t for t in (1, 2, 4, 8) if Hkv % t == 0])
    c = dict(op=rng.choice(["append", "attend", "attend", "scores", "evict"]), Hq=Hq, Hkv=Hkv, D=D, tp=tp,
             T=rng.choice([8, 16, 16, 16, 32, 64]), order=rng.choice([0, 0, 1]), dtype=rng.choice(["fp16", "bf16"]))
    if c["op"] == "append":
        S = spread(1, 128)
        q = 1 if rng.random() < 0.4 else spread(2, 12000 // S)
        lo = spread(1, 2000)
        c.update(S=S, lo=lo, hi=lo + spread(1, 4000), qlo=max(1, q // 2), qhi=q, norm=rng.random() < 0.6,
                 rot=rng.choice([D, D, D // 2]), interleaved=rng.random() < 0.3)
    elif c["op"] == "attend":
        if rng.random() < 0.5:  # decoding steps, a few tokens at most
            S = spread(1, 128)
            c.update(S=S, qlo=1, qhi=rng.choice([1, 1, 1, 2, 4]), long=rng.choice([0, 0, spread(4096, 65536)]) if S <= 8 else 0)
            c["lo"] = spread(1, 512)
            c["hi"] = c["lo"] + spread(16, 4096 * 8 // Hkv)
        else:  # pieces of prompts
            S = spread(1, 8)
            q = spread(5, 2048 * 32 // Hq // S)
            c.update(S=S, qlo=max(1, q // 2), qhi=q, long=0)
            c["lo"] = spread(1, 2000)
            c["hi"] = c["lo"] + spread(16, 8000)
        c["window"] = rng.choice([0, 0, 0, spread(16, 4096)])
    elif c["op"] == "scores":
        S = spread(1, 48)
        q = rng.choice([1, 1, spread(2, 64)])
        c.update(S=S, qlo=max(1, q // 2), qhi=q, window=rng.choice([0, 0, spread(16, 4096)]))
        c["lo"] = spread(1, 512)
        c["hi"] = c["lo"] + spread(16, max(17, 65536 // S // q * 8 // Hkv))
    else:
        S = spread(1, 32)
        lo = spread(1, 700)
        hi = lo + spread(16, min(32768, 120000 // S * 8 // Hkv))
        budget = spread(16, max(17, hi))
        c.update(L=rng.choice([1, 1, 2]), S=S, lo=lo, hi=hi, long=0, budget=budget, keep=spread(1, budget))
    return c


# ---------------------------------------------------------------------------------------------------------- the inputs

def _lens(case):
    """Sequence lengths and new tokens of each: by the case alone, so that work() knows them."""
    g = np.random.RandomState(case["S"] * 131 + case["lo"] * 7 + case["hi"])
    n = g.randint(case["lo"], case["hi"] + 1, case["S"])
    if case.get("long"):
        n[case["S"] // 2] = case["long"]
    if "qhi" not in case:
        return n, np.zeros_like(n)
    q = g.randint(case["qlo"], case["qhi"] + 1, case["S"])
    if case["qhi"] >= 100 and case["qlo"] == 1:  # a mixed batch: half the sequences decode
        q[::2] = 1
    return n, np.minimum(n, q)


def _pool_shape(case, L, NB):
    Hr = case["Hkv"] // case["tp"]
    return (L, NB, Hr, 2, case["T"], case["D"]) if case["order"] == 0 else (L, 2, NB, case["T"], Hr, case["D"])


def prepare(case, seed):
    dt, T, tp, D, S = DT[case["dtype"]], case["T"], case["tp"], case["D"], case["S"]
    L = case.get("L", 1)
    g = torch.Generator(device=DEV).manual_seed(seed)
    lens, qlens = _lens(case)
    nblk = -(-lens // T)
    out_len = np.minimum(lens, case["budget"]) if case["op"] == "evict" else lens * 0
    dblk = -(-out_len // T)
    n_live, maxb = int(nblk.sum()), int(nblk.max())
    NB = n_live + int(dblk.sum()) + 3
    ids = torch.randperm(NB, generator=g, device=DEV).to(torch.int32)

    def table(n, at):
        n, width = torch.from_numpy(n).to(DEV), max(1, int(n.max()))
        col = torch.arange(width, device=DEV)[None]
        k = (torch.cumsum(n, 0) - n)[:, None] + col + at
        return torch.where(col < n[:, None], ids[k.clamp(max=NB - 1)], -1).to(torch.int32).contiguous()

    randn = lambda *shape: torch.randn(*shape, generator=g, device=DEV, dtype=dt)  # noqa: E731
    s = dict(case=case, bt=table(nblk, 0), lens=torch.from_numpy(lens).to(DEV, torch.int32), maxb=maxb, NB=NB,
             maxlen=int(lens.max()), status=torch.zeros(1, dtype=torch.int32, device=DEV),
             pools=[randn(*_pool_shape(case, L, NB)) for _ in range(tp)], scale=D ** -0.5, ws=None)
    if case["op"] == "evict":
        s["dbt"] = table(dblk, n_live)
        s["new_lens"] = torch.zeros(S, dtype=torch.int32, device=DEV)
        shape = (L, NB, case["Hkv"] // tp, T)
        # attention weight falls off steeply over the tokens; many get hardly any, and equal values are common
        s["scores"] = [torch.exp(3 * torch.randn(*shape, generator=g, device=DEV)).mul(64).round().div(64) for _ in range(tp)]
    else:
        rows = int(qlens.sum())
        starts = np.concatenate([[0], np.cumsum(qlens)])
        s["starts"] = torch.from_numpy(starts).to(DEV, torch.int32)
        s["rows"], s["maxq"] = rows, int(qlens.max())
        wq, wk = case["Hq"] // tp * D, case["Hkv"] // tp * D
        if case["op"] == "append":  # the workers' fused projections, [q, k, v] a row
            s["qkv"] = [randn(rows, wq + 2 * wk) for _ in range(tp)]
            s["q"], s["k"], s["v"] = ([x[:, a:b] for x in s["qkv"]] for a, b in ((0, wq), (wq, wq + wk), (wq + wk, wq + 2 * wk)))
            s["q_out"] = [torch.empty(rows, wq, dtype=dt, device=DEV) for _ in range(tp)]
            s["wq"] = (1 + 0.1 * randn(D)) if case["norm"] else None
            s["wk"] = (1 + 0.1 * randn(D)) if case["norm"] else None
            s["freq"] = 500000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64, device=DEV) / case["rot"])
            # positions run on from what was once cached: far beyond the cache's own index
            s["pos"] = torch.from_numpy(np.concatenate([np.arange(q) + n - q + 17 * i for i, (n, q) in enumerate(zip(lens, qlens))])).to(DEV, torch.int32)
        else:
            s["q"] = [randn(rows, wq) * 2 for _ in range(tp)]
            s["lse"] = torch.empty(rows, case["Hq"], dtype=torch.float32, device=DEV)
            s["out"] = [torch.empty(rows, wq, dtype=dt, device=DEV) for _ in range(tp)]
        if case["op"] == "scores":
            s["scores"] = [torch.zeros(L, NB, case["Hkv"] // tp, T, device=DEV) for _ in range(tp)]
            s["lse"] = _plain_attend(s, True)[1]
    if own:  # what a program keeps between calls: the layout, the batch's table addresses, the scratch space
        _handles(s, L)
    return s


def _handles(s, L):
    import paper_2509_19729_b200 as A

    c = s["case"]
    model = dict(L=L, hidden=c["Hq"] * c["D"], Hq=c["Hq"], Hkv=c["Hkv"], D=c["D"], I=c["Hq"] * c["D"])
    s["A"] = A
    s["layout"] = A.make_layout(model, c["tp"], s["NB"], c["T"], kv_order=c["order"])
    s["dt"] = A.DTYPE_FP16 if c["dtype"] == "fp16" else A.DTYPE_BF16
    if c["op"] == "evict":
        n = A.amoeba_evict_workspace_bytes(s["layout"], L, c["S"], c["budget"])
    else:
        s["batch"] = A.make_batch(s["bt"], s["lens"], s["starts"], s["rows"], s["maxq"])
        n = A.amoeba_attend_workspace_bytes(s["layout"], s["batch"]) if c["op"] == "attend" else 0
        if c["op"] == "append":
            s["rotation"] = A.make_rotation(s["wq"], s["wk"], 1e-5, s["freq"], s["pos"], c["rot"], c["interleaved"])
    s["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------------------ one pass of each

def run(s):
    return (_own if own else _plain)[s["case"]["op"]](s)


def _own_append(s):
    s["A"].amoeba_append_kv(s["layout"], s["dt"], 0, s["pools"], s["batch"], s["q"], s["k"], s["v"], s["rotation"],
                            s["q_out"], s["status"])
    return s["q_out"], s["pools"]


def _own_attend(s):
    s["A"].amoeba_attend(s["layout"], s["dt"], 0, s["pools"], s["batch"], s["q"], s["scale"], s["case"]["window"],
                         s["out"], s["lse"], s["status"], s["ws"])
    return s["out"], s["lse"]


def _own_scores(s):
    s["A"].amoeba_accumulate_scores(s["layout"], s["dt"], 0, s["pools"], s["batch"], s["q"], s["scale"],
                                    s["case"]["window"], s["lse"], None, s["scores"], s["status"])
    return s["scores"]


def _own_evict(s):
    c = s["case"]
    s["A"].amoeba_evict_kv(s["layout"], 0, c["L"], s["pools"], s["scores"], s["bt"], s["lens"], s["dbt"], c["budget"],
                           c["keep"], s["new_lens"], s["status"], s["ws"])
    return s["pools"], s["scores"], s["new_lens"]


_own = {"append": _own_append, "attend": _own_attend, "scores": _own_scores, "evict": _own_evict}


# ------------------------------------------------------------------------------------------- the plain forms, in 32 bits

def _cached(s, layer, kv):
    """The keys (kv = 0) or values (1) of every sequence, [S, longest, Hkv, D] in 32 bits."""
    T = s["case"]["T"]
    i = torch.arange(s["maxlen"], device=DEV)
    block, t = s["bt"].long()[:, i // T].clamp(min=0), i % T
    if s["case"]["order"] == 0:
        return torch.cat([p[layer, block, :, kv, t] for p in s["pools"]], 2).float()
    return torch.cat([p[layer, kv, block, t] for p in s["pools"]], 2).float()


def _rows(s):
    """The row of every sequence's j-th new token, [S, most], and which of them there are."""
    n = s["starts"].diff()
    j = torch.arange(s["maxq"], device=DEV)
    return (s["starts"][:-1, None] + j).long().clamp(max=s["rows"] - 1), j < n[:, None], n


def _weights(s):
    """Logits [S, Hkv, group, new, keys], -inf where a query does not see a key."""
    c = s["case"]
    G = c["Hq"] // c["Hkv"]
    row, there, n = _rows(s)
    q = torch.cat(s["q"], 1).view(s["rows"], c["Hkv"], G, c["D"])[row].float()
    at = (s["lens"] - n)[:, None, None] + torch.arange(s["maxq"], device=DEV)[None, :, None]
    key = torch.arange(s["maxlen"], device=DEV)
    sees = (key <= at) & there[:, :, None]
    if c["window"]:
        sees &= key > at - c["window"]
    x = torch.einsum("sqhgd,skhd->shgqk", q, _cached(s, 0, 0)).mul_(s["scale"])
    return x.masked_fill_(~sees[:, None, None], -math.inf), row, there


def _plain_attend(s, lse_only=False):
    c = s["case"]
    x, row, there = _weights(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (total.log() + top).squeeze(-1).permute(0, 3, 1, 2).flatten(2)[there]  # rows in order
    if lse_only:
        return None, lse
    o = torch.einsum("shgqk,skhd->sqhgd", x, _cached(s, 0, 1))
    o = (o / total.permute(0, 3, 1, 2, 4).clamp(min=1e-30))[there].flatten(1).to(DT[c["dtype"]])
    return list(o.chunk(c["tp"], 1)), lse


def _plain_scores(s):
    c = s["case"]
    x, row, there = _weights(s)
    lse = s["lse"][row].view(*row.shape, c["Hkv"], -1).permute(0, 2, 3, 1)[..., None]
    w = x.sub_(lse).exp_().sum((2, 3))  # [S, Hkv, keys]
    i = torch.arange(s["maxlen"], device=DEV)
    inside = i < s["lens"][:, None]
    block, t = s["bt"].long()[:, i // c["T"]][inside], i.expand_as(inside)[inside] % c["T"]
    w = w.permute(0, 2, 1)[inside].chunk(c["tp"], 1)
    for p, x in zip(s["scores"], w):
        p[0, block, :, t] = x
    return s["scores"]


def _plain_append(s):
    c, T, D, half = s["case"], s["case"]["T"], s["case"]["D"], s["case"]["rot"] // 2
    row, there, n = _rows(s)
    index = ((s["lens"] - n)[:, None] + torch.arange(s["maxq"], device=DEV))[there].long()
    seq = torch.arange(c["S"], device=DEV)[:, None].expand_as(there)[there]
    block, t = s["bt"].long()[seq, index // T], index % T
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def form(x, w):
        x = x.view(s["rows"], -1, D).float()
        if w is not None:
            x = x * (x.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w.float()
        if c["interleaved"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turned, x[..., 2 * half:]], -1).to(DT[c["dtype"]])

    for r in range(c["tp"]):
        s["q_out"][r].copy_(form(s["q"][r], s["wq"]).flatten(1))
        k, v, p = form(s["k"][r], s["wk"]), s["v"][r].view(s["rows"], -1, D), s["pools"][r]
        if c["order"] == 0:
            p[0, block, :, 0, t], p[0, block, :, 1, t] = k, v
        else:
            p[0, 0, block, t], p[0, 1, block, t] = k, v
    return s["q_out"], s["pools"]


def _plain_evict(s):
    c, T = s["case"], s["case"]["T"]
    lens, i = s["lens"].long(), torch.arange(s["maxlen"], device=DEV)
    new = lens.clamp(max=c["budget"])
    block, t = s["bt"].long()[:, i // T].clamp(min=0), i % T
    j = torch.arange(min(c["budget"], s["maxlen"]), device=DEV)
    dblock, dt = s["dbt"].long()[:, j // T], j % T
    kept = (j < new[:, None])
    seq, rank = kept.nonzero(as_tuple=True)
    for p, sc in zip(s["pools"], s["scores"]):
        for l in range(c["L"]):
            x = sc[l, block, :, t].permute(0, 2, 1)  # [S, heads, tokens]
            x = torch.where(i >= (lens - c["keep"])[:, None, None], math.inf, x)
            x = torch.where(i < lens[:, None, None], x, -math.inf)
            best = x.sort(dim=-1, descending=True, stable=True).indices[..., :j.numel()]
            best = torch.where(kept[:, None], best, s["maxlen"]).sort(-1).values.permute(0, 2, 1)[seq, rank]  # [tokens, heads]
            sb, st = s["bt"].long()[seq[:, None], best // T], best % T
            h = torch.arange(best.shape[1], device=DEV)
            db, d = dblock[seq, rank][:, None], dt[rank][:, None]
            sc[l, db, h, d] = sc[l, sb, h, st]
            if c["order"] == 0:
                p[l, db, h, :, d] = p[l, sb, h, :, st]
            else:
                p[l, :, db, d, h] = p[l, :, sb, st, h]
    s["new_lens"].copy_(new)
    return s["pools"], s["scores"], s["new_lens"]


_plain = {"append": _plain_append, "attend": _plain_attend, "scores": _plain_scores, "evict": _plain_evict}


# -------------------------------------------------------------------------------------------- the definitions, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "scores": _exact_scores, "evict": _exact_evict}[case["op"]](s, case)


def _slots(s, n, i0=0):
    """(block, token in block) of the cache indices i0 .. n-1 of a sequence with table row `n[1]`."""
    i = torch.arange(i0, n[0], device=DEV)
    return s["bt"][n[1]].long()[i // s["case"]["T"]], i % s["case"]["T"]


def _head(s, r, h, kv, at):
    p = s["pools"][r][0]
    return (p[at[0], h, kv, at[1]] if s["case"]["order"] == 0 else p[kv, at[0], at[1], h]).double()


def _exact_walk(s, c):
    """For every sequence and key head: its slots, its logits [group, new, keys] and where its rows are."""
    G, Hr, D = c["Hq"] // c["Hkv"], c["Hkv"] // c["tp"], c["D"]
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    for b, n in enumerate(lens):
        lo, hi = starts[b], starts[b + 1]
        at = _slots(s, (n, b))
        where = torch.arange(n - (hi - lo), n, device=DEV)[:, None]
        key = torch.arange(n, device=DEV)
        hidden = key > where
        if c["window"]:
            hidden = hidden | (key <= where - c["window"])
        for head in range(c["Hkv"]):
            r, h = divmod(head, Hr)
            q = s["q"][r][lo:hi, h * G * D:(h + 1) * G * D].reshape(hi - lo, G, D).double().transpose(0, 1)
            x = (q @ _head(s, r, h, 0, at).T * s["scale"]).masked_fill(hidden, -math.inf)
            yield b, r, h, lo, hi, at, x


def _exact_attend(s, c):
    G, D, Hr = c["Hq"] // c["Hkv"], c["D"], c["Hkv"] // c["tp"]
    out = [torch.zeros(s["rows"], c["Hq"] // c["tp"] * D, dtype=torch.float64, device=DEV) for _ in range(c["tp"])]
    lse = torch.full((s["rows"], c["Hq"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, r, h, lo, hi, at, x in _exact_walk(s, c):
        m = x.logsumexp(-1)
        out[r][lo:hi, h * G * D:(h + 1) * G * D] = ((x - m[..., None]).exp() @ _head(s, r, h, 1, at)).transpose(0, 1).flatten(1)
        lse[lo:hi, (r * Hr + h) * G:(r * Hr + h + 1) * G] = m.T
    return out, lse


def _exact_scores(s, c):
    G, Hr = c["Hq"] // c["Hkv"], c["Hkv"] // c["tp"]
    got = [p.double() for p in s["scores"]]
    for b, r, h, lo, hi, at, x in _exact_walk(s, c):
        lse = s["lse"][lo:hi, (r * Hr + h) * G:(r * Hr + h + 1) * G].double().T[..., None]
        got[r][0, at[0], h, at[1]] = (x - lse).exp().sum((0, 1))
    return got


def _exact_append(s, c):
    D, T, rot = c["D"], c["T"], c["rot"]
    pools = [p.double() for p in s["pools"]]
    first = torch.arange(0, rot, 2, device=DEV) if c["interleaved"] else torch.arange(rot // 2, device=DEV)
    second = first + (1 if c["interleaved"] else rot // 2)
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), s["pos"].double()[:, None, None] * s["freq"])

    def turn(x, w):
        x = x.reshape(s["rows"], -1, D).double()
        if w is not None:
            x = x / torch.sqrt((x ** 2).mean(-1, keepdim=True) + 1e-5) * w.double()
        y = torch.complex(x[..., first], x[..., second]) * z
        x = x.clone()
        x[..., first], x[..., second] = y.real, y.imag
        return x

    q_out = [turn(q, s["wq"]).flatten(1) for q in s["q"]]
    lens, starts = s["lens"].tolist(), s["starts"].tolist()
    for r in range(c["tp"]):
        k, v = turn(s["k"][r], s["wk"]), s["v"][r].reshape(s["rows"], -1, D).double()
        for b, n in enumerate(lens):
            lo, hi = starts[b], starts[b + 1]
            block, t = _slots(s, (n, b), n - (hi - lo))
            if c["order"] == 0:
                pools[r][0, block, :, 0, t], pools[r][0, block, :, 1, t] = k[lo:hi], v[lo:hi]
            else:
                pools[r][0, 0, block, t], pools[r][0, 1, block, t] = k[lo:hi], v[lo:hi]
    return q_out, pools


def _exact_evict(s, c):
    """Moved values have no rounding; which ones are kept is decided here on the host, token by token."""
    T, B, keep = c["T"], c["budget"], c["keep"]
    bt, dbt, lens = s["bt"].cpu().numpy(), s["dbt"].cpu().numpy(), s["lens"].tolist()
    pools, scores = [p.clone() for p in s["pools"]], [x.clone() for x in s["scores"]]
    for r in range(c["tp"]):
        host = s["scores"][r].cpu().numpy()
        for b, n in enumerate(lens):
            m = min(n, B)
            i = np.arange(n)
            to = np.arange(m)
            tb, tt = dbt[b][to // T], to % T
            for l in range(c["L"]):
                for h in range(c["Hkv"] // c["tp"]):
                    x = host[l, bt[b][i // T], h, i % T]
                    free = max(n - keep, 0)
                    order = np.lexsort((i[:free], -x[:free]))[: max(m - (n - free), 0)]
                    kept = np.concatenate([np.sort(order), i[free:]]) if n > B else i
                    fb, ft = bt[b][kept // T], kept % T
                    scores[r][l, tb, h, tt] = s["scores"][r][l, fb, h, ft]
                    if c["order"] == 0:
                        pools[r][l, tb, h, :, tt] = s["pools"][r][l, fb, h, :, ft]
                    else:
                        pools[r][l, :, tb, tt, h] = s["pools"][r][l, :, fb, ft, h]
    return [p.double() for p in pools], [x.double() for x in scores], None


# ----------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    lens, qlens = (x.astype(np.int64) for x in _lens(case))
    D, Hq, Hkv, T = case["D"], case["Hq"], case["Hkv"], case["T"]
    rows = int(qlens.sum())
    tables = int((-(-lens // T)).sum()) * 4 + 8 * case["S"]
    if case["op"] == "append":  # q, k and v are read, the turned q, k and v written
        values = rows * (Hq + 2 * Hkv) * D
        return dict(bytes=tables + 4 * values, flops=rows * (Hq + Hkv) * D * (7 if case["norm"] else 3))
    if case["op"] == "evict":
        m = np.minimum(lens, case["budget"])
        cut = int(lens[lens > case["budget"]].sum())
        return dict(bytes=tables + case["L"] * Hkv * (4 * cut + int(m.sum()) * (2 * 2 * D * 2 + 8)), flops=case["L"] * Hkv * cut)
    # pairs of a query and a key that it sees; keys that any query sees
    pairs, keys = 0, 0
    for n, q in zip(lens.tolist(), qlens.tolist()):
        seen = np.arange(n - q + 1, n + 1)
        pairs += int(np.minimum(seen, case["window"]).sum() if case["window"] else seen.sum())
        keys += min(n, case["window"] + q - 1) if case["window"] else n
    if case["op"] == "attend":
        return dict(bytes=tables + keys * Hkv * D * 4 + rows * Hq * (4 * D + 4), flops=4 * pairs * Hq * D)
    return dict(bytes=tables + keys * Hkv * D * 2 + int(lens.sum()) * Hkv * 4 + rows * Hq * (2 * D + 4), flops=2 * pairs * Hq * D)
