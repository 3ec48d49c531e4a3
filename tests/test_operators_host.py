"""What the serving operators refuse before anything reaches a GPU, and their structs as C sees them."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import cache_reference as ref
import paper_2509_19729_b200 as A
from paper_2509_19729_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
M = dict(L=2, hidden=512, Hq=8, Hkv=4, D=64, I=512)
PTR = 1 << 20  # an address that nothing reads: every call here is refused on the host


def ptrs(n, at=PTR):
    return (C.c_void_p * n)(*[at + 4096 * i for i in range(n)])


def batch(**kw):
    b = B.Batch(PTR, PTR, PTR, 3, 4, 10, 5)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def call(name, layout=None, **kw):
    """The C call with arguments that are in order but for kw."""
    l = layout or A.make_layout(M, 2, 10)
    tp = l.tp
    # (the row buffers of in-order arguments are distinct)
    a = dict(layout=C.byref(l), dtype=0, layer=0, pools=ptrs(tp), batch=C.byref(kw.pop("batch", None) or batch()), q=ptrs(tp, 2 * PTR),
             qs=0, k=ptrs(tp), ks=0, v=ptrs(tp), vs=0, rotation=None, out=ptrs(tp, 3 * PTR), outs=0, status=PTR, scale=1.0,
             window=0, lse=PTR, ws=PTR, ws_bytes=1 << 40, scored=None, scores=ptrs(tp), l0=0, l1=1, src=PTR, lens=PTR,
             S=3, maxb=4, dst=2 * PTR, dmaxb=4, budget=10, recent=2, new=3 * PTR)
    a.update(kw)
    lib = B._load()
    if name == "append":
        return lib.amoeba_append_kv(a["layout"], a["dtype"], a["layer"], a["pools"], a["batch"], a["q"], a["qs"], a["k"], a["ks"],
                                    a["v"], a["vs"], a["rotation"], a["out"], a["outs"], a["status"], None)
    if name == "attend":
        return lib.amoeba_attend(a["layout"], a["dtype"], a["layer"], a["pools"], a["batch"], a["q"], a["qs"], a["scale"],
                                 a["window"], a["out"], a["outs"], a["lse"], a["status"], a["ws"], a["ws_bytes"], None)
    if name == "scores":
        return lib.amoeba_accumulate_scores(a["layout"], a["dtype"], a["layer"], a["pools"], a["batch"], a["q"], a["qs"],
                                            a["scale"], a["window"], a["lse"], a["scored"], a["scores"], a["status"], None)
    return lib.amoeba_evict_kv(a["layout"], a["l0"], a["l1"], a["pools"], a["scores"], a["src"], a["lens"], a["S"], a["maxb"],
                               a["dst"], a["dmaxb"], a["budget"], a["recent"], a["new"], a["status"], a["ws"], a["ws_bytes"],
                               None)


INV, UNS, ALI = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED, A.ERR_ALIGNMENT
ROWS = ["append", "attend", "scores"]


@pytest.mark.parametrize("name", ROWS)
def test_row_operators_refuse(name):
    odd = ptrs(2, PTR + 8)
    null = (C.c_void_p * 2)(PTR, None)
    assert call(name, layout=A.make_layout(dict(M, D=96), 2, 10)) == UNS
    assert call(name, layout=A.make_layout(dict(M, D=32), 2, 10)) == UNS
    assert call(name, layout=A.make_layout(M, 2, 10, elem_bytes=1)) == UNS
    assert call(name, layout=A.make_layout(M, 3, 10)) == UNS
    assert call(name, layout=A.make_layout(M, 2, 0)) == INV
    assert call(name, dtype=2) == UNS and call(name, dtype=-1) == UNS
    assert call(name, layer=-1) == INV and call(name, layer=2) == INV
    assert call(name, pools=null) == INV and call(name, pools=odd) == ALI and call(name, pools=None) == INV
    assert call(name, q=null) == INV and call(name, q=odd) == ALI
    assert call(name, qs=255) == INV and call(name, qs=260) == ALI
    assert call(name, status=None) == INV
    for bad in (dict(num_seqs=-1), dict(max_blocks_per_seq=-1), dict(num_rows=-1), dict(max_q_len=-1), dict(d_seq_lens=None),
                dict(d_block_table=None), dict(d_q_starts=None, num_rows=2), dict(d_q_starts=None, max_q_len=0)):
        assert call(name, batch=batch(**bad)) == INV, bad
    assert call(name, layout=A.make_layout(M, 2, 10, kv_layer_stride_bytes=16)) == INV
    assert call(name, layout=A.make_layout(M, 2, 10, kv_layer_stride_bytes=(1 << 20) + 8)) == ALI


def test_append_refuses():
    odd, null = ptrs(2, PTR + 2), (C.c_void_p * 2)(PTR, None)
    for which in ("k", "v", "out"):
        assert call("append", **{which: null}) == INV and call("append", **{which: odd}) == ALI
    assert call("append", q=None) == INV and call("append", out=None) == INV and call("append", k=None) == INV
    q = ptrs(2, 2 * PTR)
    assert call("append", q=q, out=q, qs=256, outs=512) == INV  # in place at another stride

    def rot(**kw):
        r = B.Rotation(PTR, PTR, PTR, PTR, 1e-6, 64, 0, 0)
        for k, v in kw.items():
            setattr(r, k, v)
        return C.byref(r)

    for bad in (dict(rot_dim=0), dict(rot_dim=80), dict(rot_dim=24), dict(rot_dim=-16), dict(interleaved=2)):
        assert call("append", rotation=rot(**bad)) == INV, bad
    assert call("append", rotation=rot(d_q_norm=PTR + 8)) == ALI


def test_attend_and_scores_refuse():
    q = ptrs(2, 2 * PTR)
    assert call("attend", q=q, out=q) == INV and call("attend", out=None) == INV and call("attend", outs=8) == INV
    assert call("attend", window=-1) == INV and call("scores", window=-1) == INV
    assert call("attend", ws=None) == INV and call("attend", ws=PTR + 8) == ALI
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert call("attend", scale=scale) == INV and call("scores", scale=scale) == INV
    need = C.c_int64()
    assert B._load().amoeba_attend_workspace_bytes(C.byref(A.make_layout(M, 2, 10)), C.byref(batch()), C.byref(need)) == 0
    assert call("attend", ws_bytes=need.value - 1) == INV
    assert call("scores", lse=None) == INV and call("scores", scores=None) == INV
    assert call("scores", scores=(C.c_void_p * 2)(PTR, None)) == INV and call("scores", scores=ptrs(2, PTR + 4)) == ALI


def test_evict_refuses():
    for bad in (dict(budget=0), dict(budget=-3), dict(recent=-1), dict(recent=11), dict(S=-1), dict(maxb=-1), dict(dmaxb=-1),
                dict(l0=-1), dict(l0=2, l1=1), dict(l1=3), dict(status=None), dict(src=None), dict(dst=None), dict(lens=None),
                dict(new=None), dict(new=PTR), dict(ws=None), dict(ws_bytes=2 * 3 * 4 * 10 * 2 - 16), dict(scores=None),
                dict(scores=(C.c_void_p * 2)(PTR, None)), dict(pools=None), dict(dst=PTR, dmaxb=5)):
        assert call("evict", **bad) == INV, bad
    assert call("evict", ws=PTR + 4) == ALI and call("evict", scores=ptrs(2, PTR + 8)) == ALI
    assert call("evict", layout=A.make_layout(dict(M, D=20), 2, 10)) == ALI
    assert call("evict", S=0) == 0 and call("evict", l0=1, l1=1) == 0  # nothing to do


def test_binding_refuses_tensors_that_do_not_fit():
    """Types, shapes, strides and devices, before a call is made."""
    i32 = dict(dtype=torch.int32)
    bt, lens = torch.zeros(3, 4, **i32), torch.zeros(3, **i32)
    for args in ((bt[:2], lens), (bt.long(), lens), (bt, lens.long()), (bt.t(), lens[:4]), (bt, lens, torch.zeros(3, **i32), 3),
                 (bt, lens, torch.zeros(4, **i32))):
        with pytest.raises(A.AmoebaError):
            A.make_batch(*args)
    with pytest.raises(A.AmoebaError):
        A.make_rotation(inv_freq=torch.zeros(32), rot_dim=64)
    with pytest.raises(A.AmoebaError):
        A.make_rotation(inv_freq=torch.zeros(31, dtype=torch.float64), rot_dim=64)
    layout = A.make_layout(M, 2, 10)
    b = A.make_batch(bt, lens)
    pools = [torch.zeros(2, 10, 2, 2, 16, 64, dtype=torch.float16) for _ in range(2)]
    q = [torch.zeros(3, 256, dtype=torch.float16) for _ in range(2)]
    out = [torch.zeros(3, 256, dtype=torch.float16) for _ in range(2)]
    st, ws = torch.zeros(1, **i32), torch.zeros(1 << 26, dtype=torch.uint8)
    good = dict(pools=pools, q=q, out=out, lse=torch.zeros(3, 8), status=st, ws=ws)

    def attend(**kw):
        a = dict(good, **kw)
        A.amoeba_attend(layout, A.DTYPE_FP16, 0, a["pools"], b, a["q"], 1.0, 0, a["out"], a["lse"], a["status"], a["ws"])

    for bad in (dict(), dict(pools=pools[:1]), dict(pools=[p[:, :9] for p in pools]), dict(q=q[:1]), dict(q=[x[:2] for x in q]),
                dict(q=[x[:, :128] for x in q]), dict(q=[x.float() for x in q]), dict(q=[x.t().contiguous().t() for x in q]),
                dict(q=[q[0], torch.zeros(3, 512, dtype=torch.float16)[:, :256]]), dict(lse=torch.zeros(3, 7)),
                dict(lse=torch.zeros(3, 8, dtype=torch.float64)), dict(status=torch.zeros(1)), dict(ws=ws.view(torch.int32))):
        with pytest.raises(A.AmoebaError):  # the first: tensors that are not on a GPU
            attend(**bad)


def test_structs_match_the_binding(tmp_path):
    lib = str(A.library_path())
    exe = str(tmp_path / "operators_check")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "c_abi", "operators_check.c"), "-o", exe, lib,
                    f"-Wl,-rpath,{os.path.dirname(lib)}"], check=True)
    got = dict(line.split(" ", 1) for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    for name, cls in (("amoeba_batch", B.Batch), ("amoeba_rotation", B.Rotation)):
        assert int(got[f"sizeof.{name}"]) == C.sizeof(cls)
        for field, _ in cls._fields_:
            assert int(got[f"offsetof.{name}.{field}"]) == getattr(cls, field).offset
    assert int(got["attend_ws"]) == 0 and int(got["attend_ws_bytes"]) % 16 == 0 and int(got["evict_ws"]) == 0
    assert int(got["evict_ws_bytes"]) == A.amoeba_evict_workspace_bytes(A.make_layout(dict(M, Hq=16, Hkv=8, D=128), 2, 10), 2, 3, 100)
    assert int(got["evict_ws_budget"]) == INV


def test_reference_on_a_case_worked_by_hand():
    """Two tokens, one head: weights 1/(1+e) and e/(1+e); the newest of three and the best of the others stay."""
    m = dict(L=1, hidden=1, Hq=1, Hkv=1, D=2, I=1)
    c = ref.Cache(m, 1, 2, 2, 0, "fp16", fill=0.0)
    bt = np.array([[1]], np.int32)
    c.at(0, 1, 0, 0, 1)[0] = 1.0
    c.at(0, 1, 0, 1, 0)[:] = torch.tensor([1.0, 0.0])
    c.at(0, 1, 0, 1, 1)[:] = torch.tensor([0.0, 1.0])
    out, lse, _, _ = ref.attend(c, 0, bt, [2], [0, 1], np.array([[[2.0, 5.0]]]), 0.5, 0)
    e = np.e
    assert np.allclose(out[0, 0], [1 / (1 + e), e / (1 + e)]) and np.isclose(lse[0, 0], np.log(1 + e))
    assert ref.kept([3.0, 5.0, 5.0, 1.0], 4, 2, 1).tolist() == [1, 3]
    assert ref.kept([np.nan, -np.inf, 1.0], 3, 2, 0).tolist() == [1, 2]
    y, _ = ref.turned(np.array([[[1.0, 0.0]]]), None, 0, np.array([np.pi / 2]), np.array([1]), 2, False)
    assert np.allclose(y, [[[0.0, 1.0]]])


@pytest.mark.parametrize("name", ROWS + ["evict"])
def test_blocks_longer_than_any_sequence_are_refused(name):
    layout = A.make_layout(dict(M, D=64), 2, 1, (1 << 30) + 16)
    assert call(name, layout=layout) == UNS


# ---- the Python calls' own checks, each refused for its own reason.  Tensors on the host are checked like those on a GPU and
# refused last, so that none of this needs one.

class Calls:
    """The four Python calls with host tensors that are in order but for their device, and arguments in their place."""

    def __init__(self):
        i32, f16 = dict(dtype=torch.int32), dict(dtype=torch.float16)
        self.layout = A.make_layout(M, 2, 10)
        self.pools = [torch.zeros(2, 10, 2, 2, 16, 64, **f16) for _ in range(2)]
        self.scores = [torch.zeros(2, 10, 2, 16) for _ in range(2)]
        self.bt, self.lens = torch.zeros(3, 4, **i32), torch.zeros(3, **i32)
        self.batch = A.make_batch(self.bt, self.lens)
        self.wide = [torch.zeros(3, 256, **f16) for _ in range(2)]  # rows of 4 query heads of 64
        self.slim = [torch.zeros(3, 128, **f16) for _ in range(2)]  # of 2 key heads
        self.status, self.ws = torch.zeros(1, **i32), torch.zeros(1 << 26, dtype=torch.uint8)
        self.lse = torch.zeros(3, 8)

    def __call__(self, name, **kw):
        g = lambda k, d: kw.get(k, d)  # noqa: E731
        pools, q, st = g("pools", self.pools), g("q", self.wide), g("status", self.status)
        dtype, layer, batch = g("dtype", A.DTYPE_FP16), g("layer", 0), g("batch", self.batch)
        out, scores, scale, stream = g("out", [x.clone() for x in self.wide]), g("scores", self.scores), g("scale", 1.0), g("stream", None)
        if name == "append":
            A.amoeba_append_kv(self.layout, dtype, layer, pools, batch, q, g("k", self.slim), g("v", self.slim), g("rotation", None),
                               out, st, stream)
        elif name == "attend":
            A.amoeba_attend(self.layout, dtype, layer, pools, batch, q, scale, g("window", 0), out, g("lse", self.lse), st,
                            g("ws", self.ws), stream)
        elif name == "scores":
            A.amoeba_accumulate_scores(self.layout, dtype, layer, pools, batch, q, scale, g("window", 0), g("lse", self.lse),
                                       g("scored", None), scores, st, stream)
        else:
            A.amoeba_evict_kv(self.layout, g("l0", 0), g("l1", 2), pools, scores, g("src", self.bt), g("lens", self.lens),
                              g("dst", self.bt), g("budget", 10), 2, g("new", self.lens.clone()), st, g("ws", self.ws), stream)


ALL = ROWS + ["evict"]
POOL, ROW, LSE = "a pool is on another device, strided or too small", "row buffers are", "lse is float32"


@pytest.mark.parametrize("name", ALL)
def test_calls_in_order_are_refused_for_the_device_alone(name):
    with pytest.raises(A.AmoebaError, match="not on a GPU"):
        Calls()(name)


@pytest.mark.parametrize("names,bad,why", [
    (ALL, lambda c: dict(pools=c.pools[:1]), "pool count != tp"),
    (ALL, lambda c: dict(pools=c.pools[0]), "as a list or tuple"),
    (ALL, lambda c: dict(pools=[None, None]), "a tensor is needed"),
    (ALL, lambda c: dict(pools=[p[:, :9] for p in c.pools]), POOL),
    (ALL, lambda c: dict(pools=[p.transpose(3, 4) for p in c.pools]), POOL),
    (ALL, lambda c: dict(pools=[p.to("meta") for p in c.pools]), POOL),
    (ROWS, lambda c: dict(pools=[p[:1] for p in c.pools], layer=1), POOL),
    (["evict"], lambda c: dict(pools=[p[:1] for p in c.pools]), POOL),
    (ROWS, lambda c: dict(dtype=2), "dtype is"),
    (ROWS, lambda c: dict(layer=1 << 40), "does not fit 32 bits"),
    (ROWS, lambda c: dict(q=c.wide[:1]), "row buffer count != tp"),
    (ROWS, lambda c: dict(q=[x[:2] for x in c.wide]), ROW),
    (ROWS, lambda c: dict(q=c.slim), ROW),
    (ROWS, lambda c: dict(q=[x.float() for x in c.wide]), ROW),
    (ROWS, lambda c: dict(q=[x.t().contiguous().t() for x in c.wide]), ROW),
    (ROWS, lambda c: dict(q=[x.view(3, 4, 64).transpose(1, 2).reshape(3, 4, 64).transpose(1, 2) for x in c.wide]), ROW),
    (ROWS, lambda c: dict(q=[torch.zeros(3, 8, 64, dtype=torch.float16)[:, ::2] for _ in c.wide]), ROW),
    (ROWS, lambda c: dict(q=[c.wide[0], torch.zeros(3, 512, dtype=torch.float16)[:, :256]]), ROW),
    (ROWS, lambda c: dict(q=[x.flatten() for x in c.wide]), ROW),
    (["append"], lambda c: dict(k=c.wide), ROW), (["append"], lambda c: dict(v=[x[:2] for x in c.slim]), ROW),
    (["append", "attend"], lambda c: dict(out=c.slim), ROW),
    (["attend", "scores"], lambda c: dict(lse=torch.zeros(3, 7)), LSE),
    (["attend", "scores"], lambda c: dict(lse=torch.zeros(3, 8, dtype=torch.float64)), LSE),
    (["attend", "scores"], lambda c: dict(lse=torch.zeros(8, 3).t()), LSE),
    (["attend", "scores"], lambda c: dict(window=1 << 31), "does not fit 32 bits"),
    (["scores"], lambda c: dict(scored=torch.zeros(2, dtype=torch.int32)), "scored_lens is int32"),
    (["scores"], lambda c: dict(scored=torch.zeros(3, dtype=torch.int64)), "scored_lens is int32"),
    (["scores", "evict"], lambda c: dict(scores=[x.double() for x in c.scores]), "score pools are float32"),
    (["scores", "evict"], lambda c: dict(scores=[x[:, :9] for x in c.scores]), POOL),
    (["scores", "evict"], lambda c: dict(scores=c.scores[:1]), "score pool count != tp"),
    (["scores"], lambda c: dict(scores=None), "as a list or tuple"),
    (["evict"], lambda c: dict(src=c.bt[:2]), "block tables are"), (["evict"], lambda c: dict(dst=c.bt.long()), "block tables are int32"),
    (["evict"], lambda c: dict(src=c.bt.t().contiguous().t()), "block tables are int32"),
    (["evict"], lambda c: dict(dst=c.bt[0]), "block tables are"),
    (["evict"], lambda c: dict(new=c.lens[:2]), "lengths are int32"), (["evict"], lambda c: dict(new=c.lens.long()), "lengths are int32"),
    (["evict"], lambda c: dict(lens=c.lens.long()), "lengths are int32"),
    (ALL, lambda c: dict(status=torch.zeros(1)), "status is int32"), (ALL, lambda c: dict(status=c.status[:0]), "status is int32"),
    (["attend", "evict"], lambda c: dict(ws=c.ws.view(torch.int32)), "the workspace is uint8"),
])
def test_calls_say_which_tensor_does_not_fit(names, bad, why):
    c = Calls()
    for name in names:
        with pytest.raises(A.AmoebaError, match=why):
            c(name, **bad(c))


@pytest.mark.parametrize("name", ROWS)
def test_rows_that_share_storage_are_refused(name):
    """A broadcast row, or rows that overlap: the kernels would read and write behind the storage, or on other rows."""
    c = Calls()
    one = torch.zeros(1, 256, dtype=torch.float16)
    flat = torch.zeros(4096, dtype=torch.float16)
    for q in (one.expand(3, 256), flat.as_strided((3, 256), (128, 1)), one.view(1, 4, 64).expand(3, 4, 64)):
        with pytest.raises(A.AmoebaError, match=ROW):
            c(name, q=[q, q])
        if name != "scores":
            with pytest.raises(A.AmoebaError, match=ROW):
                c(name, out=[q, q])
    if name == "append":
        with pytest.raises(A.AmoebaError, match=ROW):
            c(name, v=[one[:, :128].expand(3, 128)] * 2)


def test_a_tensor_of_one_row_fits_beside_any_stride():
    """Its row stride says nothing: one worker's row may be a tensor of its own, another's part of a wider one."""
    c = Calls()
    c.batch = A.make_batch(c.bt[:1], c.lens[:1])
    alone, part = torch.zeros(1, 256, dtype=torch.float16), torch.zeros(3, 512, dtype=torch.float16)[:, :256]
    for q in ([alone, part], [part, alone], [alone, part[:1]], [alone, alone]):
        with pytest.raises(A.AmoebaError, match="not on a GPU"):
            c("attend", q=q)


class NoStream:
    cuda_stream = "7"


@pytest.mark.parametrize("names,bad", [
    (["attend", "scores"], dict(scale="1")), (["attend", "scores"], dict(scale=None)), (["attend", "scores"], dict(window=1.5)),
    (ROWS, dict(dtype="fp16")), (ROWS, dict(layer=None)), (["evict"], dict(l0=0.0)), (["evict"], dict(budget="10")),
    (ALL, dict(stream=NoStream())), (ALL, dict(stream=NoStream)),
])
def test_what_is_no_number_is_a_type_error(names, bad):
    for name in names:
        with pytest.raises(TypeError):
            Calls()(name, **bad)


def test_the_largest_numbers_are_refused():
    c = Calls()
    for bad in (dict(layer=2 ** 31 - 1), dict(layer=-1), dict(layer=-2 ** 31)):
        for name in ROWS:
            with pytest.raises(A.AmoebaError):
                c(name, **bad)
    for bad in (dict(l1=2 ** 31 - 1), dict(l0=-1), dict(budget=2 ** 31)):
        with pytest.raises(A.AmoebaError):
            c("evict", **bad)


def test_another_torch_does_not_load_this_one_s_module(monkeypatch):
    """The module that reads tensors by their C++ layout is built anew for another version of torch or of Python's interface."""
    import sys

    from paper_2509_19729_b200 import build

    here = build.torch_calls_path()
    assert here.exists() and not build.torch_calls_stale()
    for target, name, value in ((torch, "__version__", "0.0.1"), (sys.implementation, "cache_tag", "cpython-300"),
                                (torch._C, "_GLIBCXX_USE_CXX11_ABI", not torch._C._GLIBCXX_USE_CXX11_ABI)):
        with monkeypatch.context() as m:
            m.setattr(target, name, value)
            assert build.torch_calls_path() != here and build.torch_calls_stale()
