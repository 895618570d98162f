"""The paged calls as a program runs them: prompts in chunks beside single tokens, into a SparQ cache, captured, on other streams, twice."""
import math

import pytest
import torch

from paper_2312_04985_amd import binding as B
from paper_2312_04985_amd import workloads as W
from paper_2312_04985_amd.cache import DecodeCache
from paper_2312_04985_amd.paged import PagedCache

import harness as Hn
import paged_harness as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages,dtype,d_h,h_kv,g,page", [("16", "f16", 128, 2, 2, 64), ("i8", "bf16", 128, 2, 4, 16), ("e4m3", "f16", 64, 3, 1, 48), ("i8", "f16", 256, 1, 2, 32)])
def test_a_serving_program(pages, dtype, d_h, h_kv, g, page):
    """Three prompts arrive at different times and are taken in chunks while the others decode; every output is the formula's over
    what the pages stand for; the caches then go on as SparQ caches."""
    final = (150, 77, 213)
    built = P.Built(final, h_kv * g, h_kv, d_h, dtype, pages, page, 300 + d_h)
    q_all = [(0.3 * torch.randn((s, h_kv * g, d_h), generator=built.gen)).to(built.dtype) for s in final]
    done = [0, 0, 0]
    steps = [(64, 0, 40), (64, 10, 40), (1, 61, 100), (1, 1, 1), (15, 1, 31), (5, 4, 1)]
    for counts in steps:
        n = max(counts)
        lens = [a + k for a, k in zip(done, counts)]
        built.c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        starts = [sum(counts[:b]) for b in range(4)]
        pack = lambda rows: torch.cat([rows[b][done[b]:lens[b]] for b in range(3)]).cuda()   # noqa: E731
        kw = dict(row_start=torch.tensor(starts, dtype=torch.int32, device="cuda"), n_new=n)
        built.c.append(pack(built.K), pack(built.V), **kw)
        out, lse = built.c.attend(pack(q_all), lse=True, **kw)
        for b in range(3):
            if counts[b] == 0:
                continue
            part = P.Built.__new__(P.Built)
            part.__dict__.update(built.__dict__)
            part.lens = lens
            part.K, part.V = [x[:k] for x, k in zip(built.K, lens)], [x[:k] for x, k in zip(built.V, lens)]
            y, tol, l, ltol = P.reference(part, b, q_all[b][done[b]:lens[b]], counts[b])
            P.check(out[starts[b]:starts[b + 1]], y, tol, f"{counts}, sequence {b}")
            P.check(lse[:, starts[b]:starts[b + 1]].T, l, ltol, f"{counts}, lse of sequence {b}")
        done = lens
    assert tuple(done) == final and built.c.error_flags() == 0
    # on as SparQ caches: with r = d_h and k = S a step is dense attention over what the pages stood for and the new row
    c = built.c.to_decode_cache(max(final), 256, d_h, 256)
    assert c.seq_lens.tolist() == list(final)
    kn, vn, q = ((0.5 * torch.randn((3, heads, d_h), generator=built.gen)).to(built.dtype).cuda() for heads in (h_kv, h_kv, h_kv * g))
    y = c.step(kn, vn, q)
    for b in range(3):
        K = torch.cat([built.stored("K", b).float().to(built.dtype).double().cuda(), kn[b][None].double()])
        V = torch.cat([built.stored("V", b).float().to(built.dtype).double().cuda(), vn[b][None].double()])
        for h in range(h_kv * g):
            w = torch.softmax(K[:, h // g] @ q[b, h].double() / math.sqrt(d_h), 0)
            Hn.check_output(y[b, h].float().cpu().numpy(), (w @ V[:, h // g]).cpu().numpy(), 0 if dtype == "f16" else 1)
    assert c.error_flags() == 0


@pytest.mark.parametrize("dtype,d_h,h,h_kv,flags", [("f16", 128, 4, 2, 0), ("bf16", 64, 6, 2, B.SPARQ_FLAG_SINGLE_K)])
def test_prefill_of_a_sparq_cache(dtype, d_h, h, h_kv, flags):
    """DecodeCache.prefill in two chunks, then a dense decode and a step; against the formulas and against decode over the same rows."""
    w = W.Workload("prefill", 2, h, h_kv, d_h, 200, 16, 64, dtype, seed=310)
    K, V = W.draw_kv(w, "cuda", v_offset=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = (0.2 * torch.randn((2, 200, h, d_h), generator=gen, device="cuda")).to(w.torch_dtype).transpose(1, 2)
    c = DecodeCache(2, h, h_kv, 256, d_h, 16, 64, w.torch_dtype, flags=flags, poison=6e4)
    n = torch.tensor([130, 70], dtype=torch.int32, device="cuda")
    a = c.prefill(q[:, :, :130], K[:, :, :130].contiguous(), V[:, :, :130].contiguous(), n)
    rest = [K[0, :, 130:200], K[1, :, 70:140]], [V[0, :, 130:200], V[1, :, 70:140]]
    q2 = torch.stack([q[0, :, 130:200], q[1, :, 70:140]])
    z = c.prefill(q2, torch.stack(rest[0]).contiguous(), torch.stack(rest[1]).contiguous())
    assert c.seq_lens.tolist() == [200, 140]
    built = P.Built((200, 140), h, h_kv, d_h, dtype, "16", 64, 311)
    built.K, built.V = ([x[b, :, :s].transpose(0, 1).cpu() for b, s in enumerate((200, 140))] for x in (K, V))
    for b, (s, first) in enumerate(((200, 130), (140, 70))):
        y, tol, _, _ = P.reference(built, b, q[b, :, :s].transpose(0, 1).cpu(), s)
        P.check(a[b, :, :first].transpose(0, 1), y[:first], tol[:first], f"first chunk of {b}")
        P.check(z[b].transpose(0, 1), y[first:], tol[first:], f"second chunk of {b}")
    last = torch.stack([q[0, :, 199], q[1, :, 139]]).contiguous()
    d = c.dense(last)
    for b, s in enumerate((200, 140)):
        y, _, _, _ = P.reference(built, b, q[b, :, s - 1:s].transpose(0, 1).cpu(), 1)
        Hn.check_output(d[b].float().cpu().numpy(), y[0].cpu().numpy(), w.dtype_code)
    out = c.step(K[:, :, 0].contiguous(), V[:, :, 0].contiguous(), last)
    assert torch.isfinite(out).all() and c.error_flags() == 0
    m = c.prefill(q[:, :, :3], K[:, :, :3].contiguous(), V[:, :, :3].contiguous())      # the lengths' tensor has changed places in the step
    assert c.seq_lens.tolist() == [204, 144] and torch.isfinite(m).all()


def test_prefill_refuses_the_tiled_layout():
    c = DecodeCache(1, 1, 1, 64, 64, 8, 8, torch.float16, flags=B.SPARQ_FLAG_TILED_K)
    x = torch.zeros((1, 1, 2, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(ValueError):
        c.prefill(x, x, x)


@pytest.mark.parametrize("pages,counts", [("16", (1, 1, 1)), ("i8", (90, 1, 200)), ("e4m3", (300, 300, 300)), ("16", (40, 40, 40))])
def test_captured_and_replayed(pages, counts):
    """Append and attention in a graph, replayed over changed rows, lengths and pages, with eager calls between."""
    built = P.Built((700, 330, 2000), 8, 2, 128, "bf16", pages, 16, 320, room=140).fill()
    n = max(counts)
    c = built.c
    q = built.queries(n).cuda().transpose(1, 2).contiguous()
    k = torch.randn((3, 2, n, 128), device="cuda").to(torch.bfloat16)
    v = torch.randn((3, 2, n, 128), device="cuda").to(torch.bfloat16)
    per = None if len(set(counts)) == 1 else torch.tensor(counts, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((3, 8, n), device="cuda")
    other = PagedCache.over(c.K, c.V, c.page_table, c.seq_lens, 8, torch.bfloat16, K_scale=c.K_scale, V_scale=c.V_scale)   # a workspace of its own for eager calls

    def call(cache, out, lse):
        cache.append(k, v, per)
        cache.attend(q, per, out=out, lse=lse)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        call(c, out, lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(c, out, lse)
    lens = c.seq_lens.clone()
    for i in range(4):
        q.copy_(torch.randn(q.shape, device="cuda") * 0.3)
        k.copy_(torch.randn(k.shape, device="cuda"))
        v.copy_(torch.randn(v.shape, device="cuda"))
        c.seq_lens.copy_(lens - i * 13)
        c.page_table[0, :5] = c.page_table[0, :5].flip(0)
        out.fill_(7), lse.fill_(7)
        want, wl = out.clone(), lse.clone()
        g.replay()
        torch.cuda.synchronize()
        K, V = c.K.clone(), c.V.clone()
        call(other, want, wl)
        assert torch.equal(out, want) and torch.equal(lse, wl), i
        assert torch.equal(K.view(torch.uint8), c.K.view(torch.uint8)) and torch.equal(V.view(torch.uint8), c.V.view(torch.uint8))
    # (291 positions, 300 rows: such an append leaves that sequence alone and says so)
    want = B.SPARQ_ERR_BAD_SEQ_LEN if counts[1] > 330 - 39 else 0
    assert c.error_flags() == want and other.error_flags() == want


def test_two_streams_with_a_workspace_each():
    """Calls on two streams at once over the same pages, each cache with a workspace of its own."""
    built = P.Built((9000, 300, 4100), 8, 2, 128, "f16", "i8", 16, 330).fill()
    c = built.c
    other = PagedCache.over(c.K, c.V, c.page_table, c.seq_lens, 8, torch.float16, K_scale=c.K_scale, V_scale=c.V_scale)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for n in (1, 60):
        q = built.queries(n).cuda().transpose(1, 2)
        want = c.attend(q)
        outs = [[torch.empty_like(q) for _ in range(10)] for _ in range(2)]
        torch.cuda.synchronize()
        for i in range(10):
            for cache, s, o in zip((c, other), streams, outs):
                cache.attend(q, out=o[i], stream=s)
        torch.cuda.synchronize()
        for o in outs[0] + outs[1]:
            assert torch.equal(o, want)


@pytest.mark.parametrize("d_h,g,n,dtype,pages", [(128, 1, 40, "f16", "16"), (128, 5, 7, "bf16", "e4m3"), (64, 2, 33, "bf16", "i8"), (256, 1, 20, "f16", "16"), (128, 4, 1, "bf16", "i8"), (64, 8, 1, "f16", "16")])
def test_few_rows_over_a_long_cache(d_h, g, n, dtype, pages):
    """Row tiles and units that very many workgroups share, put together in two levels; the same bits every time."""
    built = P.Built((20011,), g, 1, d_h, dtype, pages, 64, 340).fill()
    q = built.queries(n)
    x = q.cuda().transpose(1, 2)
    out, lse = built.c.attend(x, lse=True)
    full, l = out.transpose(1, 2), lse
    P.check_attention(built, q, full, [n], l)
    for _ in range(3):
        again, lse2 = built.c.attend(x, lse=True)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("d_h,h_kv,g,dtype,pages,lens,counts,window", [
    (128, 2, 4, "f16", "16", (20011,), (500,), 0),            # 16 row tiles per KV head, 15 parts each
    (128, 2, 4, "bf16", "e4m3", (20011, 9007), (300, 200), 0),   # ... of different lengths
    (256, 1, 2, "f16", "16", (20011,), (1500,), 8000),
    (64, 3, 4, "bf16", "i8", (20011,), (440,), 0)])
def test_row_tiles_in_parts_of_their_own(d_h, h_kv, g, dtype, pages, lens, counts, window):
    """Chunks over long caches whose row tiles the workgroups are dealt out to in equal parts; the same bits every time."""
    built = P.Built(lens, h_kv * g, h_kv, d_h, dtype, pages, 64, 345, window=window).fill()
    n = max(counts)
    q = built.queries(n)
    x = q.cuda().transpose(1, 2)
    kw = {} if len(lens) == 1 else dict(n_new_per_seq=torch.tensor(counts, dtype=torch.int32, device="cuda"))
    out, lse = torch.full_like(x, 7), torch.full(x.shape[:3], 7.0, device="cuda")       # (rows behind a sequence's last stay as they are)
    built.c.attend(x, out=out, lse=lse, **kw)
    P.check_attention(built, q, out.transpose(1, 2), list(counts), lse, window=window)
    for _ in range(3):
        again, lse2 = torch.full_like(x, 7), torch.full(x.shape[:3], 7.0, device="cuda")
        built.c.attend(x, out=again, lse=lse2, **kw)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    assert built.c.error_flags() == 0


def test_a_workspace_that_serves_calls_of_every_size():
    """Calls of few, many and few rows on one workspace: every call leaves its counters as it found them."""
    built = P.Built((3000, 900), 8, 2, 128, "bf16", "16", 64, 350).fill()
    for n in (1, 500, 2, 17, 64, 1, 300, 8):
        q = built.queries(n)
        out = built.c.attend(q.cuda().transpose(1, 2))
        P.check_attention(built, q, out.transpose(1, 2), [n, n])
    assert built.c.error_flags() == 0


def test_a_workspace_outgrown():
    """The errors of calls before it was replaced are told too; it is not replaced during a capture."""
    built = P.Built((900,), 8, 2, 128, "bf16", "16", 64, 360).fill()
    c = built.c
    keep = c.page_table[0, 3].item()
    c.page_table[0, 3] = -1
    c.attend(built.queries(1).cuda().transpose(1, 2))
    c.page_table[0, 3] = keep
    small = c.workspace.numel()
    q = built.queries(200)
    x = q.cuda().transpose(1, 2)
    with pytest.raises(RuntimeError, match="capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            c.attend(x)
    torch.cuda.synchronize()
    out = c.attend(x)
    assert c.workspace.numel() > small and c.error_flags() == B.SPARQ_ERR_BAD_PAGE and c.error_flags() == 0
    P.check_attention(built, q, out.transpose(1, 2), [200])


@pytest.mark.parametrize("packed", [False, True])
def test_results_that_a_call_makes_belong_to_its_stream(packed):
    """Outputs and logarithms made by the call on another stream are filled there, before its kernels, however busy the current one is."""
    built = P.Built((200, 131), 4, 2, 64, "f16", "16", 16, 370).fill()
    n = (5, 40)
    q = built.queries(40).cuda().transpose(1, 2)
    if packed:
        x = torch.cat([q[b, :, :n[b]].transpose(0, 1) for b in range(2)]).contiguous()
        kw = dict(row_start=torch.tensor([0, 5, 45], dtype=torch.int32, device="cuda"), n_new=40)
    else:
        x, kw = q, dict(n_new_per_seq=torch.tensor(n, dtype=torch.int32, device="cuda"))
    want, want_lse = built.c.attend(x, lse=True, **kw)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn((4096, 4096), device="cuda")
    for _ in range(20):
        busy = busy @ busy * 1e-3
    out, lse = built.c.attend(x, lse=True, stream=other, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_a_first_prefill_is_not_captured():
    """It makes a workspace, which is initialised outside of a graph; after a prefill the next one may be captured."""
    c = DecodeCache(1, 2, 2, 64, 64, 16, 16, torch.float16)
    x = torch.randn((1, 2, 8, 64), device="cuda", dtype=torch.float16)
    with pytest.raises(RuntimeError, match="capture"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            c.prefill(x, x, x)
    torch.cuda.synchronize()
    c.seq_lens.zero_()
    a = c.prefill(x, x, x)
    out, graph = torch.empty_like(x), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.prefill(x, x, x, out=out)
    for _ in range(3):
        c.seq_lens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, a) and c.error_flags() == 0
