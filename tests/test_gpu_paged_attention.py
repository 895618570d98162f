"""sparq_paged_attention against the formulas in 64 bits: lengths, groups, page types, masks, strides, poison."""
import pytest
import torch

from paper_2312_04985_amd import binding as B

import paged_harness as P

pytestmark = pytest.mark.gpu


def attend(built, q, n_rows=None, lse=True, layout="tokens", **kw):
    """out [B, n, H, d_h] and lse [B, H, n], 7 where nothing is written."""
    Bn, n, H, d = q.shape
    counts = None if n_rows is None else torch.tensor(n_rows, dtype=torch.int32, device="cuda")
    x = q.cuda()
    l = torch.full((Bn, H, n), 7.0, device="cuda") if lse else None
    if layout == "heads":
        x = x.transpose(1, 2).contiguous()
        out = torch.full_like(x, 7.0)
    elif layout == "wide":
        w = torch.full((Bn, n, H + 2, d + 16), float("nan"), dtype=q.dtype, device="cuda")
        w[:, :, 2:, 8:8 + d] = x
        x = w[:, :, 2:, 8:8 + d].transpose(1, 2)
        out = torch.full((n, Bn, H, d + 8), 7.0, dtype=q.dtype, device="cuda")[..., :d].permute(1, 2, 0, 3)
    else:
        x = x.transpose(1, 2)
        out = torch.full((Bn, n, H, d), 7.0, dtype=q.dtype, device="cuda").transpose(1, 2)
    got = built.c.attend(x, counts, out=out, lse=l, **kw)
    assert got is out
    return out.transpose(1, 2), l


SHAPES = [   # d_h, H_kv, g, dtype, pages, page
    (128, 2, 1, "f16", "16", 16), (128, 2, 4, "bf16", "16", 64), (64, 1, 8, "f16", "16", 32), (64, 3, 2, "bf16", "16", 48), (256, 2, 1, "bf16", "16", 16),
    (256, 1, 3, "f16", "16", 128), (128, 2, 4, "f16", "i8", 16), (128, 1, 7, "bf16", "i8", 64), (64, 2, 1, "bf16", "i8", 48), (256, 1, 2, "f16", "i8", 32),
    (256, 2, 5, "bf16", "i8", 16), (128, 1, 16, "f16", "e4m3", 32), (128, 2, 2, "bf16", "e4m3", 16), (64, 1, 4, "f16", "e4m3", 64), (256, 1, 1, "bf16", "e4m3", 48),
]


@pytest.mark.parametrize("d_h,h_kv,g,dtype,pages,page", SHAPES)
@pytest.mark.parametrize("lens,n_rows", [
    ((1, 2, 16, 17, 64, 65), None),                            # one token each: around the tiles' edges
    ((700, 1, 129, 0, 333), (1, 1, 1, 1, 1)),                  # ... an empty sequence among them
    ((3, 9, 200, 64), (3, 0, 2, 1)),                           # a few rows: from the start, none, in the middle of a cache
    ((70, 140, 33), (70, 37, 33)),                             # chunks, whole prompts
    ((400, 5, 261), (130, 5, 259)),                            # row tiles that are full and not
])
def test_lengths(d_h, h_kv, g, dtype, pages, page, lens, n_rows):
    print("[case]", d_h, h_kv, g, dtype, pages, page, lens, n_rows, flush=True)
    built = P.Built(lens, h_kv * g, h_kv, d_h, dtype, pages, page, 40 + d_h + g).fill()
    n = max(n_rows) if n_rows else 1
    q = built.queries(n)
    for layout in ("tokens", "heads"):
        out, lse = attend(built, q, n_rows, layout=layout)
        P.check_attention(built, q, out, n_rows or [n] * built.Bn, lse)
    assert built.c.error_flags() == 0


@pytest.mark.parametrize("d_h,g,dtype,pages", [(128, 4, "bf16", "16"), (64, 2, "f16", "i8"), (256, 1, "bf16", "e4m3")])
@pytest.mark.parametrize("window,causal", [(1, True), (5, True), (64, True), (100, True), (1000, True), (0, False), (70, False)])
def test_masks(d_h, g, dtype, pages, window, causal):
    lens, n_rows = (500, 64, 65, 2, 131), (150, 64, 1, 2, 131)
    built = P.Built(lens, 2 * g, 2, d_h, dtype, pages, 32, 60 + window, causal=causal, window=window).fill()
    q = built.queries(max(n_rows))
    out, lse = attend(built, q, n_rows, layout="wide")
    P.check_attention(built, q, out, n_rows, lse, causal, window)
    q = built.queries(1)
    out, lse = attend(built, q, None, layout="wide")
    P.check_attention(built, q, out, [1] * 5, lse, causal, window)


@pytest.mark.parametrize("d_h,h_kv,g,dtype,pages", [(128, 2, 4, "bf16", "e4m3"), (64, 1, 3, "f16", "16"), (256, 2, 2, "bf16", "i8")])
def test_packed_rows(d_h, h_kv, g, dtype, pages):
    """Sequences one behind the other; rows behind the last one, and those of a sequence without rows, stay as they are."""
    lens, n_rows = (300, 20, 7, 150, 4000), (90, 1, 0, 150, 1)
    built = P.Built(lens, h_kv * g, h_kv, d_h, dtype, pages, 16, 70).fill()
    n = max(n_rows)
    q = built.queries(n)
    starts = [sum(n_rows[:b]) for b in range(6)]
    flat = torch.cat([q[b, :k] for b, k in enumerate(n_rows)] + [torch.full((5, h_kv * g, d_h), float("nan"), dtype=built.dtype)]).cuda()
    out = torch.full_like(flat, 7.0)
    lse = torch.full((h_kv * g, flat.shape[0]), 7.0, device="cuda")
    built.c.attend(flat, row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), n_new=n, out=out, lse=lse)
    full = torch.full((5, n, h_kv * g, d_h), 7.0, dtype=built.dtype, device="cuda")
    l = torch.full((5, h_kv * g, n), 7.0, device="cuda")
    for b, k in enumerate(n_rows):
        full[b, :k], l[b, :, :k] = out[starts[b]:starts[b] + k], lse[:, starts[b]:starts[b] + k]
    P.check_attention(built, q, full, n_rows, l)
    assert (out[starts[-1]:] == 7).all() and (lse[:, starts[-1]:] == 7).all()
    assert built.c.error_flags() == 0


@pytest.mark.parametrize("pages", ["16", "i8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n", [1, 40, 200])
def test_infinities_and_nan_that_a_row_does_not_see(pages, dtype, n):
    """Values of later positions, of positions before the window and of unused pages do not reach a row; seen ones do."""
    S, window = 300, 90
    for w in (0, window):
        built = P.Built((S, S), 4, 2, 128, dtype, pages, 16, 80 + n, window=w)
        clean = [x.clone() for x in built.V]
        bad = {S - 2: float("inf"), S - 15: float("nan"), S - n - 95: float("nan")} if w else {S - 2: float("inf"), S - 15: float("nan")}
        for j, x in bad.items():
            if j >= 0:
                built.V[0][j, 0, 17], built.K[0][j, 1, 3] = x, x
        built.fill()
        q = built.queries(n)
        out, _ = attend(built, q)
        y, tol, _, _ = P.reference(built, 0, q[0], n, True, w)
        # 16-bit pages: the value's own channel; 8-bit pages: the row whole
        for i in range(n):
            p = S - n + i
            seen = [j for j in bad if j <= p and (not w or j > p - w)]
            if not seen:
                P.check(out[0, i:i + 1], y[i:i + 1], tol[i:i + 1], f"row {i}")
            else:
                assert not torch.isfinite(out[0, i, :2, 17]).any() and torch.isnan(out[0, i, 2:]).all()
                if pages == "16":
                    rest = torch.arange(128, device="cuda") != 17
                    P.check(out[0, i:i + 1, :2][..., rest], y[i:i + 1, :2][..., rest], tol[i:i + 1, :2][..., rest], f"row {i}")
        built.V = clean
        y, tol, _, _ = P.reference(built, 1, q[1], n, True, w)
        P.check(out[1], y, tol, "the other sequence")


@pytest.mark.parametrize("dtype,pages", [("f16", "16"), ("bf16", "16"), ("bf16", "i8"), ("f16", "e4m3")])
@pytest.mark.parametrize("scale", [0.0, 1e-4, 20.0])
def test_logits_flat_and_peaked(dtype, pages, scale):
    """All weights alike; one position takes all, wherever it stands (the running maximum rises late)."""
    built = P.Built((1000, 190), 8, 2, 128, dtype, pages, 64, 90).fill()
    for n in (1, 100):
        q = built.queries(n, scale)
        out, lse = attend(built, q)
        P.check_attention(built, q, out, [n, n], lse)


def test_values_of_very_different_sizes():
    """8-bit pages: value scales over a hundred binary orders, rows of zeros between them."""
    built = P.Built((200,), 2, 1, 64, "bf16", "i8", 16, 91)
    for j in range(200):
        built.V[0][j] = built.V[0][j] * 2.0 ** ((j * 7) % 100 - 50) if j % 5 else 0 * built.V[0][j]
    built.fill()
    for n in (1, 66):
        q = built.queries(n)
        out, lse = attend(built, q)
        P.check_attention(built, q, out, [n], lse)
    built.V[0][:] = 0
    built.fill()
    out, _ = attend(built, q)
    assert (out == 0).all()


def test_queries_of_very_different_sizes():
    """8-bit pages with bf16 rows: heads whose queries are far outside fp16's range, beside ordinary ones and infinite ones."""
    built = P.Built((150,), 8, 1, 128, "bf16", "e4m3", 16, 92).fill()
    for n in (1, 40):
        q = built.queries(n)
        for h, s in enumerate((2.0 ** -100, 2.0 ** -20, 1.0, 2.0 ** 3, 0.0)):
            q[:, :, h] = q[:, :, h] * s
        q[:, :, 5, 3:] *= 2.0 ** -30
        q[:, :, 7, 9] = float("inf")
        out, lse = attend(built, q)
        y, tol, l, ltol = P.reference(built, 0, q[0], n)
        for h in range(7):
            P.check(out[0, :, h], y[:, h], tol[:, h], f"head {h}")
            P.check(lse[0, h], l[:, h], ltol[:, h], f"lse of head {h}")
        assert out[0, :, 7].isnan().all()


@pytest.mark.parametrize("n", [1, 90])
def test_bad_descriptions(n):
    """Lengths, counts and pages that are none: zeros or nothing for that sequence, the error bit, the others as ever."""
    lens = (200, 150, 120, 100, 130, 95)
    built = P.Built(lens, 4, 2, 64, "f16", "16", 16, 93, room=20).fill()
    q = built.queries(n)

    def as_ever(b, out, l=None):           # (the order of its sums goes by the lengths of the whole batch)
        y, tol, lse, ltol = P.reference(built, b, q[b], n)
        P.check(out[b], y, tol, f"sequence {b}")
        assert l is None or P.check(l[b].T, lse, ltol, f"lse of sequence {b}") is None
    counts = torch.tensor([n, n, n, n + 1, -1, n], dtype=torch.int32, device="cuda")
    built.c.seq_lens[1], built.c.seq_lens[2] = 20 * 16 + 1, -3
    out = torch.full((6, n, 4, 64), 7.0, dtype=torch.float16, device="cuda").transpose(1, 2)
    l = torch.full((6, 4, n), 7.0, device="cuda")
    built.c.attend(q.cuda().transpose(1, 2), counts, out=out, lse=l)
    assert built.c.error_flags() == B.SPARQ_ERR_BAD_SEQ_LEN | B.SPARQ_ERR_BAD_ROWS
    out = out.transpose(1, 2)
    for b in (0, 5):
        as_ever(b, out, l)
    for b in (1, 2):
        assert (out[b] == 0).all() and (l[b] == -float("inf")).all()
    for b in (3, 4):
        assert (out[b] == 7).all() and (l[b] == 7).all()
    built.c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
    built.c.page_table[3, 2] = built.c.n_pages
    built.c.page_table[4, 0] = -1
    out, _ = attend(built, q, [n] * 6)
    assert built.c.error_flags() == B.SPARQ_ERR_BAD_PAGE
    for b in (0, 1, 2, 5):
        as_ever(b, out)
    # more rows than positions: those before position 0 see nothing
    if n > 1:
        built.c.seq_lens[0] = 5
        out, l = attend(built, q)
        assert (out[0, :n - 5] == 0).all() and (l[0, :, :n - 5] == -float("inf")).all() and (out[0, n - 5:] != 0).any()


def test_a_bound_on_the_lengths():
    built = P.Built((400, 90), 4, 1, 128, "bf16", "16", 16, 94, room=4000).fill()
    q = built.queries(1)
    for bound in (0, 400, 4096):
        built.c.with_bound(bound)
        out, lse = attend(built, q)
        P.check_attention(built, q, out, [1, 1], lse)
        assert built.c.error_flags() == 0
    built.c.with_bound(399)
    out, _ = attend(built, q)
    assert (out[0] == 0).all() and built.c.error_flags() == B.SPARQ_ERR_BAD_SEQ_LEN


@pytest.mark.parametrize("pages,n", [("16", 1), ("i8", 1), ("16", 70)])
def test_pages_beyond_4_gib_of_a_pool(pages, n):
    d_h, h_kv, page = 256, 8, 256
    each = h_kv * page * d_h * (2 if pages == "16" else 1)
    n_pages = (1 << 32) // each + 3
    built = P.Built((2 * page - 9,), h_kv, h_kv, d_h, "bf16", pages, page, 95, extra=n_pages - 2)
    built.c.page_table[0, :2] = torch.tensor([n_pages - 1, n_pages - 3], dtype=torch.int32)
    built.fill()
    q = built.queries(n)
    out, lse = attend(built, q)
    P.check_attention(built, q, out, [n], lse)


def test_broadcast_queries():
    """One row of queries for all heads (a head stride of 0)."""
    built = P.Built((77, 300), 6, 2, 64, "f16", "16", 16, 96).fill()
    for n in (1, 50):
        q = built.queries(n)[:, :, :1]
        x = q.cuda().transpose(1, 2).expand(2, 6, n, 64)
        out = torch.empty((2, 6, n, 64), dtype=torch.float16, device="cuda")
        built.c.attend(x, out=out)
        P.check_attention(built, q.expand(2, n, 6, 64), out.transpose(1, 2), [n, n])


@pytest.mark.parametrize("d_h,b,h_kv,g,n,dtype,pages", [
    (128, 43, 9, 1, 40, "f16", "16"),          # one row tile per KV head, not a multiple of eight of them
    (64, 8, 8, 3, 390, "bf16", "i8"),          # ten each, the last of them not full
    (256, 10, 10, 2, 140, "bf16", "e4m3"),
])
def test_a_workgroup_for_every_row_tile(d_h, b, h_kv, g, n, dtype, pages):
    """The same number of rows everywhere, so many that no row tile is divided; lengths all different, one sequence of fewer positions than rows."""
    lens = [n + (i * 37) % 211 for i in range(b)]
    lens[1], lens[2] = n // 2, 0
    built = P.Built(lens, h_kv * g, h_kv, d_h, dtype, pages, 16, 97).fill()
    q = built.queries(n)
    out, lse = attend(built, q)
    P.check_attention(built, q, out, [n] * b, lse)
    assert built.c.error_flags() == 0
