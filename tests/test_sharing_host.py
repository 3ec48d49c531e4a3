"""What the calls for sequences that share blocks refuse before anything reaches a GPU, and their structs as C sees them."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2509_19729_b200 as A
import sharing_reference as share
from paper_2509_19729_b200 import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
M = dict(L=2, hidden=512, Hq=8, Hkv=4, D=64, I=512)
PTR = 1 << 20  # an address that nothing reads: every call here is refused on the host
INV, UNS, ALI = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED, A.ERR_ALIGNMENT


def ptrs(n, at=PTR):
    return (C.c_void_p * n)(*[at + 4096 * i for i in range(n)])


def changed(struct, **kw):
    for k, v in kw.items():
        setattr(struct, k, v)
    return struct


def prefixes(**kw):
    return changed(B.Prefixes(PTR, PTR, 2, 5, 0, 0), **kw)


def batch(**kw):
    return changed(B.Batch(PTR, PTR, PTR, 3, 4, 10, 5), **kw)


def attend(layout=None, **kw):
    l = layout or A.make_layout(M, 2, 10)
    a = dict(dtype=0, layer=0, pools=ptrs(2), batch=batch(), prefixes=prefixes(), q=ptrs(2, 2 * PTR), qs=0, scale=1.0, out=ptrs(2, 3 * PTR),
             outs=0, lse=PTR, status=PTR, ws=PTR, n=1 << 40)
    a.update(kw)
    by = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return B._load().amoeba_attend_shared(C.byref(l), a["dtype"], a["layer"], a["pools"], by(a["batch"]), by(a["prefixes"]), a["q"], a["qs"],
                                          a["scale"], a["out"], a["outs"], a["lse"], a["status"], a["ws"], a["n"], None)


def test_attend_shared_refuses():
    odd, null = ptrs(2, PTR + 8), (C.c_void_p * 2)(PTR, None)
    assert attend(layout=A.make_layout(dict(M, D=96), 2, 10)) == UNS and attend(layout=A.make_layout(M, 2, 10, elem_bytes=1)) == UNS
    assert attend(dtype=2) == UNS and attend(layer=-1) == INV and attend(layer=2) == INV
    for name in ("pools", "q", "out"):
        assert attend(**{name: null}) == INV and attend(**{name: odd}) == ALI and attend(**{name: None}) == INV
    assert attend(qs=255) == INV and attend(qs=260) == ALI and attend(outs=8) == INV
    assert attend(status=None) == INV and attend(ws=None) == INV and attend(ws=PTR + 8) == ALI
    assert attend(batch=None) == INV and attend(prefixes=None) == INV
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert attend(scale=scale) == INV
    q = ptrs(2, 2 * PTR)
    assert attend(q=q, out=q) == INV
    for bad in (dict(num_seqs=-1), dict(num_rows=-1), dict(max_q_len=-1), dict(d_seq_lens=None), dict(d_block_table=None),
                dict(d_q_starts=None, num_rows=2)):
        assert attend(batch=batch(**bad)) == INV, bad
    for bad in (dict(d_group_starts=None), dict(d_prefix_lens=None), dict(num_groups=-1), dict(max_group_rows=-1), dict(always=2),
                dict(always=-1)):
        assert attend(prefixes=prefixes(**bad)) == INV, bad
    need = A.amoeba_attend_shared_workspace_bytes(A.make_layout(M, 2, 10), batch(), prefixes())
    assert attend(n=need - 1) == INV
    assert attend(batch=batch(max_q_len=2 ** 31 - 1)) == UNS  # pieces of work are numbered in 32 bits
    assert attend(batch=batch(num_rows=2 ** 30), prefixes=prefixes(max_group_rows=2 ** 30, num_groups=4096)) in (UNS, INV)


def test_the_workspace_grows_with_rows_and_groups():
    l = A.make_layout(M, 2, 10)
    size = lambda b={}, x={}: A.amoeba_attend_shared_workspace_bytes(l, batch(**b), prefixes(**x))  # noqa: E731
    assert size() % 16 == 0 and size(dict(num_rows=20)) >= size() + 8 * (64 + 2) * 10 * 8
    assert size(x=dict(num_groups=102)) > size() and size(x=dict(max_group_rows=5000)) >= size()
    with pytest.raises(A.AmoebaError):
        size(x=dict(num_groups=-1))


def step(layout=None, status=PTR, **kw):
    s = B.TableStep(*[PTR + 16 * i for i in range(14)], 3, 4, 10, 2)
    l = layout or A.make_layout(M, 2, 10)
    return B._load().amoeba_advance_tables(C.byref(l), C.byref(changed(s, **kw)), status, None)


def test_advance_tables_refuses():
    lib = B._load()
    assert lib.amoeba_advance_tables(None, C.byref(B.TableStep()), PTR, None) == INV
    assert lib.amoeba_advance_tables(C.byref(A.make_layout(M, 2, 10)), None, PTR, None) == INV
    assert step(status=None) == INV and step(layout=A.make_layout(M, 2, 0)) == INV
    for bad in (dict(num_seqs=-1), dict(max_blocks_per_seq=-1), dict(num_rows=-1), dict(pairs_cap=-1), dict(d_block_table=None),
                dict(d_block_refs=None), dict(d_seq_lens=None), dict(d_new_lens=None), dict(d_lens_out=None), dict(d_parents=None),
                dict(d_shared_lens=None), dict(d_q_starts=None), dict(d_positions=None), dict(d_pairs=None), dict(d_num_pairs=None),
                dict(d_q_starts=None, d_positions=None, d_slots=None, d_first_positions=None)):
        assert step(**bad) == INV, bad
    assert step(d_pairs=PTR + 4) == ALI and step(d_slots=PTR + 4) == ALI
    assert step(num_seqs=1 << 16, max_blocks_per_seq=(1 << 14) + 1) == UNS and step(num_rows=(1 << 30) + 1) == UNS


def test_copy_blocks_refuses():
    l = A.make_layout(M, 2, 10)

    def call(layout=l, pools=ptrs(2), pairs=PTR, n=PTR, cap=4, l0=0, l1=2, status=PTR):
        return B._load().amoeba_copy_blocks(None if layout is None else C.byref(layout), pools, pairs, n, cap, l0, l1, status, None)

    for bad in (dict(layout=None), dict(pools=None), dict(pools=(C.c_void_p * 2)(PTR, None)), dict(pairs=None), dict(n=None), dict(cap=-1),
                dict(l0=-1), dict(l0=2, l1=1), dict(l1=3), dict(status=None), dict(layout=A.make_layout(M, 2, 0))):
        assert call(**bad) == INV, bad
    assert call(pools=ptrs(2, PTR + 8)) == ALI and call(pairs=PTR + 4) == ALI and call(layout=A.make_layout(M, 3, 10)) == UNS
    assert call(cap=0, pairs=None, n=None) == 0 and call(l0=1, l1=1) == 0  # nothing to do


def test_structs_match_the_header(tmp_path):
    lib = str(A.library_path())
    exe = str(tmp_path / "sharing_check")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "c_abi", "sharing_check.c"), "-o", exe, lib, f"-Wl,-rpath,{os.path.dirname(lib)}"], check=True)
    got = dict(line.split(" ", 1) for line in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.splitlines())
    fields = 0
    for cname, cls in {"amoeba_prefixes": B.Prefixes, "amoeba_table_step": B.TableStep}.items():
        assert int(got[f"sizeof.{cname}"]) == C.sizeof(cls)
        for field, _ in cls._fields_:
            assert int(got[f"offsetof.{cname}.{field}"]) == getattr(cls, field).offset, (cname, field)
            fields += 1
    assert fields == sum(k.startswith("offsetof.") for k in got)
    m = dict(L=2, hidden=512, Hq=16, Hkv=8, D=128, I=1792)
    want = A.amoeba_attend_shared_workspace_bytes(A.make_layout(m, 2, 10), B.Batch(None, None, None, 3, 4, 3, 1), B.Prefixes(None, None, 2, 2, 0, 0))
    assert int(got["ws"]) == 0 and int(got["ws_bytes"]) == want and int(got["ws_groups"]) == INV


class Calls:
    """The Python calls with host tensors that are in order but for their device."""

    def __init__(self):
        i32 = dict(dtype=torch.int32)
        z = lambda *n: torch.zeros(*n, **i32)  # noqa: E731
        self.layout = A.make_layout(M, 2, 10)
        self.pools = [torch.zeros(2, 10, 2, 2, 16, 64, dtype=torch.float16) for _ in range(2)]
        self.t = dict(table=z(3, 4), refs=z(10), old=z(3), new=z(3), parents=z(3), shared=z(3), out=z(3), starts=z(4), first=z(3),
                      positions=z(5), slots=torch.zeros(5, dtype=torch.int64), pairs=z(2, 2), n=z(1), free=z(1), status=z(1))
        self.batch = A.make_batch(self.t["table"], self.t["old"])
        self.prefixes = A.make_prefixes(z(3), z(2), 4)
        self.rows = [torch.zeros(3, 256, dtype=torch.float16) for _ in range(2)]

    def advance(self, rows=5, stream=None, **kw):
        t = dict(self.t, **kw)
        A.amoeba_advance_tables(self.layout, t["table"], t["refs"], t["old"], t["new"], t["parents"], t["shared"], t["out"], t["starts"], rows,
                                t["first"], t["positions"], t["slots"], t["pairs"], t["n"], t["free"], t["status"], stream)

    def copy(self, pools=None, l0=0, l1=2, stream=None, **kw):
        t = dict(self.t, **kw)
        A.amoeba_copy_blocks(self.layout, pools or self.pools, t["pairs"], t["n"], l0, l1, t["status"], stream)

    def attend(self, q=None, out=None, lse=None, ws=None, scale=1.0, stream=None, **kw):
        t = dict(self.t, **kw)
        A.amoeba_attend_shared(self.layout, A.DTYPE_FP16, 0, self.pools, kw.get("batch", self.batch), kw.get("prefixes", self.prefixes),
                               q or self.rows, scale, out or [x.clone() for x in self.rows], lse,
                               t["status"], torch.zeros(1 << 26, dtype=torch.uint8) if ws is None else ws, stream)


@pytest.mark.parametrize("name", ["advance", "copy", "attend"])
def test_calls_in_order_are_refused_for_the_device_alone(name):
    with pytest.raises(A.AmoebaError, match="not on a GPU"):
        getattr(Calls(), name)()


@pytest.mark.parametrize("name,bad,why", [
    ("advance", lambda c: dict(table=c.t["table"][0]), "block tables are"), ("advance", lambda c: dict(table=c.t["table"][:2]), "block tables are"),
    ("advance", lambda c: dict(table=c.t["table"].long()), "block tables are int32"),
    ("advance", lambda c: dict(table=c.t["table"].t().contiguous().t()), "block tables are int32"),
    ("advance", lambda c: dict(refs=c.t["refs"][:9]), "block counts are"), ("advance", lambda c: dict(refs=c.t["refs"].to("meta")), "block counts are"),
    ("advance", lambda c: dict(new=c.t["new"][:2]), "lengths are"), ("advance", lambda c: dict(old=c.t["old"].long()), "lengths are"),
    ("advance", lambda c: dict(out=c.t["out"].float()), "lengths are"), ("advance", lambda c: dict(old=None), "a tensor is needed"),
    ("advance", lambda c: dict(parents=c.t["parents"][:1]), "parents are"), ("advance", lambda c: dict(shared=c.t["shared"].short()), "shared lengths are"),
    ("advance", lambda c: dict(starts=c.t["starts"][:3]), "row starts are"), ("advance", lambda c: dict(first=c.t["first"][:2]), "first positions are"),
    ("advance", lambda c: dict(positions=c.t["positions"][:4]), "positions are"), ("advance", lambda c: dict(slots=c.t["positions"]), "slots are int64"),
    ("advance", lambda c: dict(slots=c.t["slots"][:4]), "slots are int64"), ("advance", lambda c: dict(pairs=c.t["pairs"].flatten()), "pairs are int32"),
    ("advance", lambda c: dict(pairs=torch.zeros(2, 3, dtype=torch.int32)), "pairs are int32"), ("advance", lambda c: dict(n=c.t["n"][:0]), "number of pairs"),
    ("advance", lambda c: dict(free=c.t["free"].long()), "free count"), ("advance", lambda c: dict(status=c.t["status"][:0]), "status is int32"),
    ("advance", lambda c: dict(rows=1 << 40), "does not fit 32 bits"),
    ("copy", lambda c: dict(pools=c.pools[:1]), "pool count"), ("copy", lambda c: dict(pools=[p[:, :9] for p in c.pools]), "a pool is on another"),
    ("copy", lambda c: dict(pools=[p[:1] for p in c.pools]), "a pool is on another"), ("copy", lambda c: dict(pairs=c.t["pairs"].long()), "pairs are int32"),
    ("copy", lambda c: dict(pairs=c.t["pairs"].t()[:, :1]), "pairs are int32"), ("copy", lambda c: dict(n=c.t["n"].float()), "number of pairs"),
    ("copy", lambda c: dict(l1=1 << 33), "does not fit 32 bits"), ("copy", lambda c: dict(status=c.t["status"].long()), "status is int32"),
    ("attend", lambda c: dict(q=[x[:2] for x in c.rows]), "row buffers are"), ("attend", lambda c: dict(out=[x.float() for x in c.rows]), "row buffers are"),
    ("attend", lambda c: dict(lse=torch.zeros(3, 7)), "lse is float32"), ("attend", lambda c: dict(ws=torch.zeros(9)), "the workspace is uint8"),
    ("attend", lambda c: dict(q=[c.rows[0][:1].expand(3, 256)] * 2), "row buffers are"),
])
def test_calls_say_which_tensor_does_not_fit(name, bad, why):
    c = Calls()
    with pytest.raises(A.AmoebaError, match=why):
        getattr(c, name)(**bad(c))


@pytest.mark.parametrize("name,bad", [("advance", dict(rows="5")), ("advance", dict(stream="7")), ("copy", dict(l0=None)), ("copy", dict(l1=1.5)),
                                      ("attend", dict(scale="1")), ("attend", dict(stream="7"))])
def test_what_is_no_number_is_a_type_error(name, bad):
    with pytest.raises((TypeError, AttributeError)):
        getattr(Calls(), name)(**bad)


def test_prefixes_are_checked_when_they_are_made():
    i32 = torch.zeros(3, dtype=torch.int32)
    for starts, lens in ((i32[:2], i32[:2]), (i32.long(), i32[:2]), (i32, i32[:2].float())):
        with pytest.raises(A.AmoebaError):
            A.make_prefixes(starts, lens, 3)


def test_the_oracle_by_hand():
    """Sequence 0 of six tokens grows by one into its second block, which sequence 1 also names; 2 is forked from it inside a block; 3 ends."""
    T = 4
    table = np.array([[5, 1, -1], [5, 1, -1], [-1, -1, -1], [2, -1, -1]], np.int32)
    refs = np.array([0, 2, 1, 0, 0, 2, 0], np.int32)
    got = share.advance(T, table, refs, [6, 6, 0, 3], [7, 6, 6, 0], [-1, -1, 0, -1], [0, 0, 5, 0], num_rows=4, pairs_cap=4)
    assert got["table"].tolist() == [[5, 0, -1], [5, 1, -1], [5, 3, -1], [-1, -1, -1]]
    assert got["refs"].tolist() == [1, 1, 0, 1, 0, 3, 0] and got["pairs"].tolist() == [[1, 0], [1, 3]]
    assert got["starts"].tolist() == [0, 1, 1, 2, 2] and got["positions"].tolist() == [6, 5, 0, 0]
    assert got["slots"].tolist() == [0 * 4 + 2, 3 * 4 + 1, -1, -1] and got["free"] == 3 and got["status"] == 0
    short = share.advance(T, table, np.where(refs == 0, 9, refs), [6, 6, 0, 3], [7, 6, 6, 0], [-1, -1, 0, -1], [0, 0, 5, 0], num_rows=4, pairs_cap=4)
    assert short["status"] == share.NO_FREE_BLOCKS and short["lens"].tolist() == [6, 6, 0, 0]
