"""sparq_paged_append and sparq_paged_read: codes, scales and places exactly; what they leave alone."""
import pytest
import torch

from paper_2312_04985_amd import binding as B

import paged_harness as P

pytestmark = pytest.mark.gpu


def pool_of(built, name):
    """The pool as the append of all of the call's rows must leave it, on the host (bytes, scales)."""
    c = built.c
    pool, scale = getattr(c, name).cpu().clone(), getattr(c, name + "_scale")
    return pool, None if scale is None else scale.cpu().clone()


def same(got, want):
    return torch.equal(got.contiguous().view(torch.uint8).cpu(), want.contiguous().view(torch.uint8))


def expect(built, n_rows):
    want = {}
    table = built.c.page_table.cpu().tolist()
    for name in ("K", "V"):
        pool, scale = pool_of(built, name)
        for b, n in enumerate(n_rows):
            s = built.lens[b]
            for t in range(s - n, s):
                page, slot = table[b][t // built.page], t % built.page
                row = getattr(built, name)[b][t]
                if scale is None:
                    pool[page, :, slot] = row
                else:
                    codes, sc = P.quantised(row, built.pages)
                    pool.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
                    scale[page, :, slot] = sc
        want[name] = (pool, scale)
    return want


def new_rows(built, n_rows, n, name, layout):
    """The last rows of every sequence as the call takes them, the rest poison."""
    x = torch.full((built.Bn, n, built.H_kv, built.d_h), float("nan"), dtype=built.dtype)
    for b, k in enumerate(n_rows):
        if k:
            x[b, :k] = getattr(built, name)[b][built.lens[b] - k:]
    if layout == "tokens":
        return x.cuda().transpose(1, 2)
    if layout == "heads":
        return x.cuda().transpose(1, 2).contiguous()
    wide = torch.full((built.Bn, n, built.H_kv + 3, built.d_h + 8), float("nan"), dtype=built.dtype, device="cuda")   # a slice of a wider product
    wide[:, :, 1:1 + built.H_kv, :built.d_h] = x.cuda()
    return wide[:, :, 1:1 + built.H_kv, :built.d_h].transpose(1, 2)


CASES = [
    # lens, rows: single tokens at every place of a page; a sequence of one; nothing; whole pages; odd ends
    ((1, 16, 17, 40), (1, 1, 1, 1)),
    ((5, 31, 100, 64), (5, 0, 33, 64)),
    ((129,), (129,)),
]


@pytest.mark.parametrize("pages", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("dtype,d_h,h_kv,page", [("f16", 128, 2, 16), ("bf16", 64, 5, 48), ("bf16", 256, 1, 64), ("f16", 64, 3, 32), ("bf16", 128, 8, 16)])
@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("layout", ["tokens", "heads", "wide", "packed"])
def test_append_and_read(pages, dtype, d_h, h_kv, page, case, layout):
    lens, n_rows = CASES[case]
    built = P.Built(lens, h_kv, h_kv, d_h, dtype, pages, page, 100 + case + d_h)
    for b in range(built.Bn):              # rows that an average one is not: zeros, one value alone, tiny, huge, ties of the rounding
        for rows in (built.K[b], built.V[b]):
            rows[-1] = 0
            if rows.shape[0] > 1:
                rows[-2, :, 1:] = 0
            if rows.shape[0] > 3:
                rows[-3] = rows[-3] * (2.0 ** -14 if dtype == "f16" else 2.0 ** -100)
                rows[-4] = rows[-4] * (2.0 ** 12 if dtype == "f16" else 2.0 ** 90)
    n = max(n_rows)
    want = expect(built, n_rows)
    if layout == "packed":
        starts = [sum(n_rows[:b]) for b in range(built.Bn + 1)]
        pack = lambda name: torch.cat([getattr(built, name)[b][built.lens[b] - k:] for b, k in enumerate(n_rows)] + [torch.full((3, h_kv, d_h), float("nan"), dtype=built.dtype)]).cuda()   # noqa: E731
        kw = dict(row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), n_new=n)
        k, v = pack("K"), pack("V")
    else:
        kw = {} if min(n_rows) == n else dict(n_new_per_seq=torch.tensor(n_rows, dtype=torch.int32, device="cuda"))
        k, v = new_rows(built, n_rows, n, "K", layout), new_rows(built, n_rows, n, "V", layout)
    for _ in range(2):                     # the second time over itself: the same
        built.c.append(k, v, **kw)
        for name in ("K", "V"):
            assert same(getattr(built.c, name), want[name][0]), name
            if pages != "16":
                assert torch.equal(getattr(built.c, name + "_scale").cpu().view(torch.int32), want[name][1].view(torch.int32)), name
    # back again: the rows that were written, and not those around them
    first = torch.tensor([s - k for s, k in zip(lens, n_rows)], dtype=torch.int32, device="cuda")
    if layout == "packed":
        ko, vo = (torch.full_like(k, 7.0) for _ in range(2))
        built.c.read(ko, vo, first=first, **kw)
        assert (ko[starts[-1]:] == 7).all() and (vo[starts[-1]:] == 7).all()
        got = lambda o, b, kk: o[starts[b]:starts[b] + kk]   # noqa: E731
    else:
        mk = lambda: torch.full((built.Bn, n + 2, h_kv + 1, d_h + 8), 7.0, dtype=built.dtype, device="cuda")   # noqa: E731
        wide = mk(), mk()
        ko, vo = (w[:, :n, :h_kv, :d_h].transpose(1, 2) for w in wide)
        built.c.read(ko, vo, first=first, n_per_seq=kw.get("n_new_per_seq"))
        for w in wide:
            assert (w[:, n:] == 7).all() and (w[:, :, h_kv:] == 7).all() and (w[..., d_h:] == 7).all()
            assert all((w[b, k:] == 7).all() for b, k in enumerate(n_rows))
        got = lambda o, b, kk: o[b, :, :kk].transpose(0, 1)   # noqa: E731
    for b, kk in enumerate(n_rows):
        for o, name in ((ko, "K"), (vo, "V")):
            exact = built.stored(name, b)[lens[b] - kk:]
            y = exact.to(built.dtype) if pages == "16" else exact.float().to(built.dtype)
            # (a code times an fp32 scale, rounded to fp32 and then to 16 bits: the same two roundings)
            assert torch.equal(got(o, b, kk).cpu(), y)
            if pages != "16" and kk:       # what quantisation may cost
                src = getattr(built, name)[b][lens[b] - kk:].double()
                a = src.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -60)
                step = a / 254 if pages == "i8" else torch.maximum(src.abs() / 16, a / 448 / 1024)
                # half a step; x (q / a) has two fp32 roundings and the scale one: 3 x 2^-24 of up to 254 half steps < 2^-14
                assert ((exact - src).abs() <= step * (1 + 2.0 ** -14)).all()
    assert built.c.error_flags() == 0


@pytest.mark.parametrize("pages", ["i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_rows_with_infinities_and_nan_are_nan_whole(pages, dtype):
    built = P.Built((20, 4), 4, 2, 128, dtype, pages, 16, 5)
    built.K[0][3, 0, 5], built.V[0][7, 1, 0], built.K[1][2, 1, 127] = float("inf"), float("nan"), -float("inf")
    want = expect(built, (20, 4))
    n = torch.tensor([20, 4], dtype=torch.int32, device="cuda")
    built.c.append(new_rows(built, (20, 4), 20, "K", "tokens"), new_rows(built, (20, 4), 20, "V", "tokens"), n)
    for name in ("K", "V"):
        assert same(getattr(built.c, name), want[name][0])
        got, ref = getattr(built.c, name + "_scale").cpu(), want[name][1]
        assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(), ref.nan_to_num())
    k, v = (torch.zeros((2, 2, 20, 128), dtype=built.dtype, device="cuda") for _ in range(2))
    built.c.read(k, v, n_per_seq=n)
    assert k[0, 0, 3].isnan().all() and v[0, 1, 7].isnan().all() and k[1, 1, 2].isnan().all()
    assert k.isnan().any(-1).sum() == 2 and v.isnan().any(-1).sum() == 1


def test_what_cannot_be_written_is_left_alone_and_reported():
    """A length beyond the table, more rows than positions, row counts that are none, a page that is none."""
    lens = (10, 20, 30, 40, 50, 33)
    built = P.Built(lens, 2, 2, 64, "f16", "i8", 16, 6)
    n_rows = [3, 21, 5, 4, 2, 20]
    n = 21
    rows = lambda name: new_rows(built, [min(k, s) for k, s in zip(n_rows, lens)], n, name, "tokens")   # noqa: E731
    k, v = rows("K"), rows("V")
    built.c.seq_lens[2] = built.c.max_pages * 16 + 1
    built.c.seq_lens[4] = -1
    built.c.page_table[5, 1] = built.c.n_pages          # positions 16 .. 31 of the last one
    counts = torch.tensor(n_rows, dtype=torch.int32, device="cuda")
    counts[3] = n + 1
    keep = {x: getattr(built.c, x).cpu().clone() for x in ("K", "V")}
    built.c.append(k, v, counts)
    assert built.c.error_flags() == B.SPARQ_ERR_BAD_SEQ_LEN | B.SPARQ_ERR_BAD_ROWS | B.SPARQ_ERR_BAD_PAGE
    assert built.c.error_flags() == 0
    table = built.c.page_table.cpu().tolist()
    written = [(0, t) for t in range(7, 10)] + [(5, t) for t in (13, 14, 15, 32)]
    for name in ("K", "V"):
        want = keep[name]
        for b, t in written:
            want[table[b][t // 16], :, t % 16] = P.quantised(getattr(built, name)[b][t], "i8")[0]
        assert same(getattr(built.c, name), want)
    ko, vo = (torch.full((6, 2, 40, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    built.c.read(ko, vo, first=torch.tensor([5, 0, 0, 0, 0, -2], dtype=torch.int32, device="cuda"))
    assert built.c.error_flags() == B.SPARQ_ERR_BAD_SEQ_LEN | B.SPARQ_ERR_BAD_PAGE
    assert (ko[0, :, 5:] == 7).all() and (ko[0, :, :5] != 7).any() and (ko[2] == 7).all() and (ko[4] == 7).all() and (ko[5, :, :2] == 7).all()
    assert (ko[5, :, 18:34] == 7).all() and (vo[5, :, 35:] == 7).all()
    # packed rows that start before the buffer, run backwards, end behind it
    for starts in ([-1, 2, 4, 6, 8, 10, 12], [0, 2, 1, 3, 5, 7, 9], [0, 2, 4, 6, 8, 10, 23]):
        built.c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        p = torch.zeros((22, 2, 64), dtype=torch.float16, device="cuda")
        built.c.append(p, p.clone(), row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), n_new=12)
        assert built.c.error_flags() & B.SPARQ_ERR_BAD_ROWS


@pytest.mark.parametrize("pages", ["16", "i8"])
def test_rows_beyond_4_gib_of_a_pool(pages):
    """The pages that count lie more than 2^32 bytes behind the pool's first one."""
    d_h, h_kv, page = 256, 8, 256
    each = h_kv * page * d_h * (2 if pages == "16" else 1)
    n_pages = (1 << 32) // each + 3
    built = P.Built((2 * page,), h_kv, h_kv, d_h, "bf16", pages, page, 8, extra=n_pages - 2)
    built.c.page_table[0, :2] = torch.tensor([n_pages - 1, n_pages - 3], dtype=torch.int32)
    k, v = (getattr(built, x)[0].cuda().transpose(0, 1)[None] for x in ("K", "V"))
    built.c.append(k, v)
    ko, vo = (torch.zeros((1, h_kv, 2 * page, d_h), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    built.c.read(ko, vo)
    for o, name in ((ko, "K"), (vo, "V")):
        assert torch.equal(o[0].transpose(0, 1).cpu(), built.stored(name, 0).float().to(torch.bfloat16))
    assert built.c.error_flags() == 0
