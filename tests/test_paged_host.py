"""The paged cache without a GPU: refusals before any launch, and the arithmetic of rows and pages (csrc/paged.h) on the host."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2312_04985_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2312_04985_amd", "csrc")
FAKE = 0x7F0000001000      # 16-byte aligned, never dereferenced: validation fails first
ROOM = 1 << 30


def shape(**kw):
    d = dict(B=2, H=4, H_kv=2, d_h=128, page_size=16, n_pages=8, max_pages=4, dtype=0, page_type=0, flags=0, window=0, S_bound=0)
    d.update(kw)
    return B.SparqPagedShape(*[d[f] for f, _ in B.SparqPagedShape._fields_])


def cache(**kw):
    d = {f: FAKE for f, _ in B.SparqPagedCache._fields_}
    d.update(kw)
    return B.SparqPagedCache(*[d[f] for f, _ in B.SparqPagedCache._fields_])


def rows(n=1, n_rows=0, n_per_seq=None, row_start=None):
    return B.SparqRows(n, n_rows, n_per_seq, row_start)


def strides(seq=1024, head=128, row=512):
    return B.SparqStrides(seq, head, row)


def calls(sh=None, c=None, r=None, s=None, so=None, x=FAKE, y=FAKE, ws=FAKE, ws_bytes=ROOM, skip=()):
    """The statuses of the three calls."""
    L, ref = B.load(), ctypes.byref
    sh, c, r, s = sh or shape(), c or cache(), r or rows(), s or strides()
    so = so or s
    got = {}
    if "append" not in skip:
        got["append"] = L.sparq_paged_append(ref(sh), ref(c), ref(r), x, y, ref(s), ws, ws_bytes, None)
    if "read" not in skip:
        got["read"] = L.sparq_paged_read(ref(sh), ref(c), ref(r), None, x, y, ref(so), ws, ws_bytes, None)
    if "attend" not in skip:
        got["attend"] = L.sparq_paged_attention(ref(sh), ref(c), ref(r), x, ref(s), y, ref(so), None, ws, ws_bytes, None)
    return set(got.values())


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), B.SPARQ_EINVAL), (dict(H=5), B.SPARQ_EINVAL), (dict(H_kv=0), B.SPARQ_EINVAL), (dict(d_h=0), B.SPARQ_EINVAL), (dict(page_size=0), B.SPARQ_EINVAL),
    (dict(page_size=24), B.SPARQ_EINVAL), (dict(page_size=8), B.SPARQ_EINVAL), (dict(n_pages=0), B.SPARQ_EINVAL), (dict(max_pages=0), B.SPARQ_EINVAL),
    (dict(max_pages=1 << 27), B.SPARQ_EINVAL), (dict(dtype=2), B.SPARQ_EINVAL), (dict(page_type=3), B.SPARQ_EINVAL), (dict(page_type=-1), B.SPARQ_EINVAL),
    (dict(flags=2), B.SPARQ_EINVAL), (dict(window=-1), B.SPARQ_EINVAL), (dict(S_bound=-1), B.SPARQ_EINVAL), (dict(S_bound=65), B.SPARQ_EINVAL),
    (dict(d_h=96), B.SPARQ_EUNSUPPORTED), (dict(B=1 << 20, H=1 << 12, H_kv=1 << 12), B.SPARQ_EUNSUPPORTED)])
def test_shapes(bad, code):
    assert calls(shape(**bad)) == {code}
    with pytest.raises(B.SparqError) as e:
        B.sparq_paged_workspace_bytes(shape(**bad), 1)
    assert e.value.status == code


def test_pointers_rows_strides_and_workspaces():
    E = B.SPARQ_EINVAL
    for f in ("K", "V", "page_table", "seq_lens"):
        assert calls(c=cache(**{f: None})) == {E}
    assert calls(c=cache(K=FAKE + 8)) == {E} and calls(c=cache(V=FAKE + 2)) == {E}
    for t in (B.SPARQ_PAGES_I8, B.SPARQ_PAGES_E4M3):
        assert calls(shape(page_type=t), cache(K_scale=None)) == {E} and calls(shape(page_type=t), cache(V_scale=FAKE + 4)) == {E}
    assert calls(x=None) == {E} and calls(y=None) == {E} and calls(x=FAKE + 8) == {E} and calls(y=FAKE + 2) == {E}
    assert calls(r=rows(0)) == {E} and calls(r=rows(-1)) == {E} and calls(r=rows(2, 5, FAKE, FAKE)) == {E} and calls(r=rows(2, 0, None, FAKE)) == {E}
    assert calls(r=rows(1 << 29)) == {B.SPARQ_EUNSUPPORTED}
    for s in (strides(seq=-8), strides(head=-128), strides(row=-8), strides(seq=1020), strides(head=130), strides(row=4)):
        assert calls(r=rows(2), s=s) == {E}
    # what is written must not lie on top of itself; what is read may
    for s in (strides(seq=0), strides(head=0), strides(head=64)):
        assert calls(so=s, skip=("append",)) == {E}
    assert calls(r=rows(2), so=strides(row=0), skip=("append",)) == {E} and calls(r=rows(1, 2, None, FAKE), so=strides(row=64), skip=("append",)) == {E}
    W = B.SPARQ_EWORKSPACE
    assert calls(ws=None) == {W} and calls(ws=FAKE + 4) == {W} and calls(ws_bytes=65535) == {W}
    L = B.load()
    assert L.sparq_paged_workspace_bytes(ctypes.byref(shape()), 0, ctypes.byref(ctypes.c_size_t())) == E
    assert L.sparq_paged_workspace_bytes(ctypes.byref(shape()), 1, None) == E
    assert L.sparq_paged_workspace_bytes(None, 1, ctypes.byref(ctypes.c_size_t())) == E
    assert L.sparq_paged_append(ctypes.byref(shape()), None, ctypes.byref(rows()), FAKE, FAKE, ctypes.byref(strides()), FAKE, ROOM, None) == E
    assert L.sparq_paged_append(ctypes.byref(shape()), ctypes.byref(cache()), None, FAKE, FAKE, ctypes.byref(strides()), FAKE, ROOM, None) == E
    assert L.sparq_paged_append(ctypes.byref(shape()), ctypes.byref(cache()), ctypes.byref(rows()), FAKE, FAKE, None, FAKE, ROOM, None) == E


@pytest.mark.parametrize("d_h,n", [(64, 1 << 25), (128, 1 << 24), (256, 1 << 23)])
def test_rows_beyond_a_launch(d_h, n):
    """A thread moves 8 channels: B n H_kv d_h / 8 threads of one launch count in 32 bits."""
    sh = shape(B=16, H=1, H_kv=1, d_h=d_h)
    st = strides(seq=n * d_h, head=d_h, row=d_h)
    assert 16 * n * (d_h // 8) == 1 << 32 and 16 * n < 1 << 31
    assert calls(sh, r=rows(n), s=st, skip=("attend",), ws_bytes=1 << 60) == {B.SPARQ_EUNSUPPORTED}



def test_a_workspace_serves_calls_of_fewer_rows():
    for kw in (dict(), dict(max_pages=2048, page_size=16), dict(B=64, H=32, H_kv=8, max_pages=512), dict(B=1, H=32, H_kv=1, max_pages=4096, d_h=256)):
        sizes = [B.sparq_paged_workspace_bytes(shape(**kw), n) for n in (1, 2, 7, 8, 15, 16, 17, 64, 65, 500, 4096)]
        assert sizes == sorted(sizes) and sizes[0] >= 65536


def test_host_tensors_are_refused():
    from paper_2312_04985_amd.paged import PagedCache
    z = torch.zeros
    with pytest.raises(ValueError):
        B.make_paged_cache(z(4), z(4), None, None, z(4, dtype=torch.int32), z(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        PagedCache.over(z((4, 2, 16, 64), dtype=torch.float16), z((4, 2, 16, 64), dtype=torch.float16), z((2, 2), dtype=torch.int32), z(2, dtype=torch.int32), 4, torch.float16)
    with pytest.raises(ValueError):          # (pools that are not the rows' type)
        PagedCache.over(z((4, 2, 16, 64)), z((4, 2, 16, 64)), z((2, 2), dtype=torch.int32), z(2, dtype=torch.int32), 4, torch.float16)
    with pytest.raises(ValueError):
        PagedCache(1, 1, 1, 64, 16, 1, 1, torch.float16, pages="i4", device="cpu")
    with pytest.raises(ValueError):
        B._rows_dev(z((2, 2, 1, 64)), "q", False)


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    src, lib = str(d / "paged.cpp"), str(d / "paged.so")
    with open(src, "w") as f:
        f.write('''#include "paged.h"
using namespace sparq;
extern "C" void rows(int len, int bound, int n, const int* per, const int* start, int n_rows, int b, int* out) {
  const SeqRows r = seq_rows(len, bound, n, per, start, n_rows, b);
  out[0] = r.S; out[1] = r.n; out[2] = r.row0; out[3] = r.err;
}
extern "C" long long offset(long long seq, long long head, long long row, int packed, int b, int row0, int h, int t) {
  return row_offset(RowStrides{seq, head, row}, packed, b, row0, h, t);
}
extern "C" long long place(const int* table, int max_pages, int n_pages, int page_size, int H_kv, int b, int head, int pos) {
  PagedArgs a{};
  a.page_table = table; a.max_pages = max_pages; a.n_pages = n_pages; a.page_size = page_size; a.H_kv = H_kv;
  a.by_page = make_divider(page_size);
  const int index = divided(pos, a.by_page), page = page_at(a, b, index);
  return page < 0 ? -1 : pool_row(a, page, head, pos - index * page_size);
}
''')
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", CSRC, "-I", rocm + "/include", src, "-o", lib], check=True)
    m = ctypes.CDLL(lib)
    m.offset.restype = m.place.restype = ctypes.c_longlong
    m.offset.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int] * 5
    return m


def seq_rows(host, length, bound, n, per=None, start=None, n_rows=0, b=0):
    arr = lambda x: None if x is None else (ctypes.c_int * len(x))(*x)   # noqa: E731
    out = (ctypes.c_int * 4)()
    host.rows(length, bound, n, arr(per), arr(start), n_rows, b, out)
    return list(out)


def test_rows_of_a_sequence(host):
    big = 2 ** 31 - 1
    assert seq_rows(host, 50, 64, 3) == [50, 3, 0, 0] and seq_rows(host, 0, 64, 3) == [0, 3, 0, 0] and seq_rows(host, 64, 64, 3) == [64, 3, 0, 0]
    for length in (-1, 65, big, -big - 1):
        assert seq_rows(host, length, 64, 3) == [0, 3, 0, B.SPARQ_ERR_BAD_SEQ_LEN]
    assert seq_rows(host, 50, 64, 3, per=[9, 0], b=1) == [50, 0, 0, 0] and seq_rows(host, 50, 64, 3, per=[3]) == [50, 3, 0, 0]
    for k in (4, -1, big, -big - 1):
        assert seq_rows(host, 50, 64, 3, per=[k]) == [50, 0, 0, B.SPARQ_ERR_BAD_ROWS]
    assert seq_rows(host, 50, 64, 3, start=[0, 2, 5, 5], n_rows=5, b=1) == [50, 3, 2, 0]
    assert seq_rows(host, 50, 64, 3, start=[0, 2, 5, 5], n_rows=5, b=2) == [50, 0, 5, 0]
    for a, z in ((-1, 1), (3, 2), (4, 6), (0, 4), (big, -big), (-big - 1, big), (0, big), (-1, -1)):
        assert seq_rows(host, 50, 64, 3, start=[a, z], n_rows=5) == [50, 0, 0, B.SPARQ_ERR_BAD_ROWS]
    assert seq_rows(host, -5, 64, 3, start=[3, 2], n_rows=5) == [0, 0, 0, B.SPARQ_ERR_BAD_ROWS | B.SPARQ_ERR_BAD_SEQ_LEN]


def test_places(host):
    table = (ctypes.c_int * 6)(3, 0, 4, 7, -1, 8)
    at = lambda b, head, pos: host.place(table, 3, 8, 48, 5, b, head, pos)   # noqa: E731
    assert at(0, 2, 0) == (3 * 5 + 2) * 48 and at(0, 0, 47) == 3 * 5 * 48 + 47 and at(0, 4, 48) == 4 * 48 and at(0, 1, 143) == (4 * 5 + 1) * 48 + 47
    assert at(1, 0, 0) == 7 * 5 * 48 and at(1, 0, 48) == -1 and at(1, 0, 96) == -1           # pages -1 and 8 of 8 are none
    far = (ctypes.c_int * 1)(2 ** 20)
    assert host.place(far, 1, 2 ** 20 + 1, 256, 32, 0, 31, 255) == (2 ** 20 * 32 + 31) * 256 + 255   # beyond 32 bits


def test_row_offsets(host):
    assert host.offset(1000, 64, 256, 0, 3, 7, 2, 5) == 3000 + 128 + (7 + 5) * 256           # (row0 is 0 where rows are not packed)
    assert host.offset(1000, 64, 256, 1, 3, 7, 2, 5) == 128 + 12 * 256
    assert host.offset(2 ** 33, 2 ** 34, 2 ** 32, 0, 2, 0, 3, 4) == 2 ** 34 + 3 * 2 ** 34 + 4 * 2 ** 32
