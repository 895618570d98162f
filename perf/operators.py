"""The paged cache's operators: rows written into pages (16 bits, or quantised to 8), pages read back, attention of new tokens over pages.

A case is a dict of plain values:
  call     "append"  write the new rows of every sequence into its pages
           "read"    read rows of every sequence back as 16-bit rows
           "attend"  attention of the new rows' queries over the pages
           "serve"   append, then attend: one step of a serving program
  B, H, H_kv, d_h, dtype   as in the library's shapes
  pages    "16" the rows' own type, "i8" or "e4m3" with a scale per row and KV head
  page     positions per page
  S, lo    positions per sequence, the new ones included (the most and the least of them)
  n        rows per sequence in this call (the most of them)
  rows     "same" n rows everywhere; "ragged" 1 to n; "mixed" single tokens, and chunks of up to n in a quarter of the sequences
  packed   rows of all sequences one behind the other, with unused rows behind the last; otherwise [B, n, heads, d_h] in memory
  window   0, or how many positions a query sees
  lse      the logarithms of the softmax denominators are asked for too

Lengths go by the case, values by the seed.  Pages lie scattered over the pool.
"""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
QMAX = {"i8": 127.0, "e4m3": 448.0}
LEAST, MOST = 2.0 ** -60, 2.0 ** 100       # what a row's largest magnitude is taken as, at least and at most


def make(call, heads, d_h, dtype, pages, page, S, n, *, lo=0, rows="same", packed=False, window=0, lse=False):
    b, h, h_kv = heads
    return {"call": call, "B": b, "H": h, "H_kv": h_kv, "d_h": d_h, "dtype": dtype, "pages": pages, "page": page, "S": S, "lo": lo or S,
            "n": n, "rows": rows, "packed": packed, "window": window, "lse": lse}


def listed():
    cases = {
        # the smallest call: the new token of every sequence of an ordinary batch (c2_llama2_7b's heads), latency only
        "append_token_i8": make("append", (16, 32, 32), 128, "f16", "i8", 64, 4096, 1),
        # chunked prefill under continuous batching: up to 512 rows of each sequence, packed
        "append_chunks_e4m3": make("append", (16, 32, 8), 128, "bf16", "e4m3", 32, 4001, 512, lo=512, rows="ragged", packed=True),
        # the tail of a short conversation, read back for the step kernels
        "read_short_i8": make("read", (1, 32, 8), 128, "f16", "i8", 16, 701, 701),
        # a prompt read back for cache construction (31 777 rows, as the bulk append's)
        "read_prompt_e4m3": make("read", (1, 32, 8), 128, "bf16", "e4m3", 64, 31777, 31777),
        # one user, one token, an odd length: latency
        "attend_token_one": make("attend", (1, 32, 8), 128, "f16", "16", 16, 3981, 1),
        # the large serving batch (c4_large_batch's lengths, grouped heads) over int8 pages
        "attend_token_batch_i8": make("attend", (64, 32, 8), 128, "f16", "i8", 64, 8192, 1),
        # one long document (c3_llama3_8b_gqa) over e4m3 pages: few heads, a long axis
        "attend_token_long_e4m3": make("attend", (1, 32, 8), 128, "bf16", "e4m3", 128, 32768, 1, lse=True),
        # wide heads, lengths over 16x, 16-bit pages (c5_gemma_7b_ragged)
        "attend_token_ragged": make("attend", (32, 16, 16), 256, "bf16", "16", 32, 16384, 1, lo=1024),
        # a whole prompt at once into an empty cache
        "attend_prompt": make("attend", (1, 32, 32), 128, "f16", "16", 64, 8192, 8192),
        # the last chunk of a long document on grouped heads
        "attend_chunk_long": make("attend", (1, 32, 8), 128, "bf16", "16", 64, 32768, 512),
        # odd ragged chunks, narrow heads, a sliding window, int8 pages, packed rows
        "attend_chunk_window_i8": make("attend", (8, 16, 2), 64, "bf16", "i8", 48, 4999, 301, lo=301, rows="ragged", packed=True, window=1000, lse=True),
        # a serving step: chunks of some sequences beside single tokens of the others, written and attended
        "serve_mixed_e4m3": make("serve", (16, 32, 8), 128, "bf16", "e4m3", 64, 8192, 512, lo=600, rows="mixed", packed=True),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(costs(c)[0] for c in listed()), max(costs(c)[1] for c in listed())
    while True:
        call = rng.choice(["append", "append", "read", "read", "attend", "attend", "attend", "attend", "attend", "serve"])
        d_h = rng.choice([64, 128, 128, 256])
        h_kv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32])
        g = rng.choice([1, 1, 2, 3, 4, 4, 7, 8])
        b = log_uniform(rng, 1, 64)
        S = log_uniform(rng, 1, 32768)
        if call == "read":
            n = S
        elif call == "append":
            n = log_uniform(rng, 1, S)
        else:
            n = rng.choice([1, 1, log_uniform(rng, 1, 16), log_uniform(rng, 16, 8192)])
        n = min(n, S)
        rows = "same" if n == 1 or call == "read" else rng.choice(["same", "ragged", "mixed"])
        window = log_uniform(rng, 1, 8192) if call == "attend" and rng.random() < 0.2 else 0
        c = make(call, (b, g * h_kv, h_kv), d_h, rng.choice(["f16", "bf16"]), rng.choice(["16", "i8", "e4m3"]),
                 rng.choice([16, 32, 48, 64, 64, 128, 256]), S, n, lo=max(n, S // rng.choice([1, 1, 4, 16])), rows=rows,
                 packed=call != "read" and rng.random() < 0.5, window=window, lse=call == "attend" and rng.random() < 0.3)
        w = work(c)
        if w["bytes"] <= 5e9 and w["flops"] <= 6e11 and all(x <= m for x, m in zip(costs(c), most)):
            return c


def costs(c):
    """(elements of the logits, elements of the cache as rows): what a plain form holds in 32 bits."""
    attends = c["call"] in ("attend", "serve")
    return c["B"] * c["H"] * c["n"] * c["S"] if attends else 0, c["B"] * c["H_kv"] * c["S"] * c["d_h"]


def lengths(c):
    """(S_b, n_b) of every sequence."""
    rng = random.Random(c["S"] * 1009 + c["B"] * 31 + c["n"])
    S = [c["S"]] + [rng.randint(c["lo"], c["S"]) for _ in range(c["B"] - 1)]
    if c["rows"] == "same":
        n = [min(c["n"], s) for s in S]
    elif c["rows"] == "ragged":
        n = [min(c["n"], S[0])] + [rng.randint(1, min(c["n"], s)) for s in S[1:]]
    else:
        n = [min(c["n"], S[0])] + [rng.randint(1, min(c["n"], s)) if i % 4 == 0 else 1 for i, s in enumerate(S[1:], 1)]
    return S, n


def visible_pairs(c, s, n):
    """Pairs (row, visible position) of n rows at the end of s positions."""
    w = c["window"] or s
    return sum(min(p + 1, w) for p in range(s - n, s))


def work(c):
    S, n = lengths(c)
    d, hk, h = c["d_h"], c["H_kv"], c["H"]
    row16, stored = 2 * d, 2 * d if c["pages"] == "16" else d + 4
    table = sum(4 * -(-s // c["page"]) for s in S) + 4 * c["B"]
    moved = 2 * hk * sum(n) * (row16 + stored) + table
    if c["call"] in ("append", "read"):
        return {"bytes": moved, "flops": 0 if c["pages"] == "16" else 4 * hk * d * sum(n)}
    seen = sum(min(s, c["window"] + k - 1) if c["window"] else s for s, k in zip(S, n))
    pairs = sum(visible_pairs(c, s, k) for s, k in zip(S, n))
    b = 2 * hk * seen * stored + 2 * h * sum(n) * row16 + table + (4 * h * sum(n) if c["lse"] else 0)
    return {"bytes": b + (moved if c["call"] == "serve" else 0), "flops": 4 * h * d * pairs}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def quantised(x, pages):
    """(codes, scales) of rows x [..., d_h] in fp32: the definition."""
    a = x.abs().amax(-1).clamp(LEAST, MOST)
    q = torch.full_like(a, QMAX[pages])
    y = (x * torch.div(q, a).unsqueeze(-1)).clamp(-QMAX[pages], QMAX[pages])
    return (y.round() if pages == "i8" else y).to(CODES[pages]), torch.div(a, q)


def prepare(c, seed):
    """Heavy-tailed channels in the keys, an offset per channel in the values; a query is a part of one cached key and noise."""
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + c["S"] + c["n"])
    dt, d, hk, h, page = DTYPES[c["dtype"]], c["d_h"], c["H_kv"], c["H"], c["page"]
    S, n = lengths(c)
    need = [-(-s // page) for s in S]
    per, n_pages = max(need), sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=dev)
    first = torch.tensor([sum(need[:b]) for b in range(c["B"])], device=dev)[:, None]
    at = torch.arange(per, device=dev)[None, :]
    used = at < torch.tensor(need, device=dev)[:, None]
    table = torch.where(used, order[(first + at).clamp(max=n_pages - 1)], 0).to(torch.int32)

    scale = torch.exp(torch.randn((hk, 1, d), generator=gen, device=dev))
    shift = torch.randn((hk, 1, d), generator=gen, device=dev)
    keys = lambda k: torch.randn((k, hk, page, d), generator=gen, device=dev) * scale      # noqa: E731
    values = lambda k: torch.randn((k, hk, page, d), generator=gen, device=dev) + shift    # noqa: E731
    pool_type = dt if c["pages"] == "16" else CODES[c["pages"]]
    s = {"case": c, "page_table": table, "seq_lens": torch.tensor(S, dtype=torch.int32, device=dev), "K_scale": None, "V_scale": None}
    for name, rows in (("K", keys), ("V", values)):
        pool = torch.empty((n_pages, hk, page, d), dtype=pool_type, device=dev)
        scales = torch.empty((n_pages, hk, page), device=dev)
        step = max(1, (1 << 28) // (hk * page * d))
        for i in range(0, n_pages, step):
            x = rows(min(step, n_pages - i)).to(dt)
            if c["pages"] == "16":
                pool[i:i + step] = x
            else:
                pool[i:i + step], scales[i:i + step] = quantised(x.float(), c["pages"])
        s[name] = pool
        if c["pages"] != "16":
            s[name + "_scale"] = scales

    starts = [sum(n[:b]) for b in range(c["B"] + 1)]
    total = starts[-1] + 5 if c["packed"] else c["B"] * c["n"]
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device=dev) if c["packed"] else None
    s["n_per_seq"] = torch.tensor(n, dtype=torch.int32, device=dev)
    if c["call"] in ("append", "serve"):
        pick = lambda x: rows_view(x.permute(0, 2, 1, 3).reshape(-1, hk, d)[:total].to(dt), c)   # noqa: E731
        s["k_new"], s["v_new"] = pick(keys(-(-total // page))), pick(values(-(-total // page)))
    if c["call"] in ("attend", "serve"):
        b_of = (torch.arange(total, device=dev) // c["n"]).clamp(max=c["B"] - 1)
        if c["packed"]:
            b_of = (torch.searchsorted(s["row_start"].long(), torch.arange(total, device=dev), right=True) - 1).clamp(max=c["B"] - 1)
        p = (torch.rand((total, h), generator=gen, device=dev) * s["seq_lens"][b_of][:, None]).long()
        head = (torch.arange(h, device=dev) // (h // hk))[None, :]
        where = (table[b_of[:, None], p // page].long(), head, p % page)
        near = s["K"][where].float()
        if c["pages"] != "16":
            near = near * s["K_scale"][where].unsqueeze(-1)
        noise = torch.randn((total, h, d), generator=gen, device=dev)
        s["q"] = rows_view((0.05 * (near + 0.5 * noise)).to(dt), c)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.full((h, total) if c["packed"] else (c["B"], h, c["n"]), -math.inf, device=dev) if c["lse"] else None
    if c["call"] == "read":
        s["K_out"] = torch.zeros((c["B"], hk, c["n"], d), dtype=dt, device=dev)
        s["V_out"] = torch.zeros_like(s["K_out"])
    return s


def rows_view(x, c):
    """[rows, heads, d_h] as the call takes it: packed as it is, otherwise seen as [B, heads, n, d_h]."""
    return x if c["packed"] else x.view(c["B"], c["n"], *x.shape[1:]).transpose(1, 2)


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(s):
    return run_own(s) if own else run_plain(s)


def run_own(s):
    from paper_2312_04985_amd.paged import PagedCache
    c = s["case"]
    if "cache" not in s:                      # the handle that a program keeps: shape and workspace
        s["cache"] = PagedCache.over(s["K"], s["V"], s["page_table"], s["seq_lens"], c["H"], DTYPES[c["dtype"]],
                                     K_scale=s["K_scale"], V_scale=s["V_scale"], window=c["window"])
    cache = s["cache"]
    rows = {"n_new": c["n"]}
    if c["packed"]:
        rows["row_start"] = s["row_start"]
    elif c["rows"] != "same" or c["call"] == "read":
        rows["n_new_per_seq"] = s["n_per_seq"]
    if c["call"] == "read":
        return dict(zip(("K_out", "V_out"), cache.read(s["K_out"], s["V_out"], n_per_seq=s["n_per_seq"])))
    got = {}
    if c["call"] in ("append", "serve"):
        cache.append(s["k_new"], s["v_new"], **rows)
        got = written(s)
    if c["call"] in ("attend", "serve"):
        got["out"] = cache.attend(s["q"], out=s["out"], lse=s["lse"], **rows)
        if c["lse"]:
            got["lse"] = s["lse"]
    return got


def written(s):
    return {k: s[k] for k in ("K", "V", "K_scale", "V_scale") if s[k] is not None}


def run_plain(s):
    c = s["case"]
    if c["call"] == "read":
        return plain_read(s)
    got = plain_append(s) if c["call"] in ("append", "serve") else {}
    return {**got, **plain_attend(s)} if c["call"] in ("attend", "serve") else got


def row_places(s):
    """Of every row of the call: its sequence, its number there, and whether it belongs to one."""
    c = s["case"]
    dev = s["n_per_seq"].device
    if c["packed"]:
        at = torch.arange((s["q"] if "q" in s else s["k_new"]).shape[0], device=dev)
        b = torch.searchsorted(s["row_start"].long(), at, right=True) - 1
        ok = b < c["B"]
        b = b.clamp(max=c["B"] - 1)
        return b, at - s["row_start"].long()[b], ok
    b = torch.arange(c["B"], device=dev).repeat_interleave(c["n"])
    t = torch.arange(c["n"], device=dev).repeat(c["B"])
    return b, t, t < s["n_per_seq"][b]


def plain_append(s):
    c = s["case"]
    b, t, ok = row_places(s)
    p = torch.where(ok, s["seq_lens"].long()[b] - s["n_per_seq"].long()[b] + t, 0)
    # a row that belongs to no sequence writes what the first one writes
    i = torch.where(ok, torch.arange(b.numel(), device=b.device), 0)
    b, p = b[i], p[i]
    page, slot = s["page_table"].long()[b, p // c["page"]], p % c["page"]
    heads = torch.arange(c["H_kv"], device=b.device)[None, :]
    for name, new in (("K", s["k_new"]), ("V", s["v_new"])):
        x = new if c["packed"] else new.transpose(1, 2).reshape(-1, c["H_kv"], c["d_h"])
        x = x[i]
        if c["pages"] == "16":
            s[name][page[:, None], heads, slot[:, None]] = x
        else:
            codes, scales = quantised(x.float(), c["pages"])
            s[name].view(torch.int8)[page[:, None], heads, slot[:, None]] = codes.view(torch.int8)
            s[name + "_scale"][page[:, None], heads, slot[:, None]] = scales
    return written(s)


def plain_rows(s, name):
    """The cache as rows [B, H_kv, positions, d_h] in fp32."""
    c = s["case"]
    table = s["page_table"].long()
    x = s[name][table].float()
    if c["pages"] != "16":
        x = x * s[name + "_scale"][table].unsqueeze(-1)
    return x.transpose(1, 2).reshape(c["B"], c["H_kv"], -1, c["d_h"])


def plain_read(s):
    c = s["case"]
    got = {}
    ok = (torch.arange(c["n"], device=s["seq_lens"].device)[None, :] < s["n_per_seq"][:, None])[:, None, :, None]
    for name in ("K", "V"):
        got[name + "_out"] = torch.where(ok, plain_rows(s, name)[:, :, :c["n"]], 0.0).to(DTYPES[c["dtype"]])
    return got


def plain_attend(s):
    c = s["case"]
    B, H, hk, n, d = c["B"], c["H"], c["H_kv"], c["n"], c["d_h"]
    S, k = s["seq_lens"].long(), s["n_per_seq"].long()
    if c["packed"]:
        at = (s["row_start"].long()[:-1, None] + torch.arange(n, device=S.device)).clamp(max=s["q"].shape[0] - 1)
        q = s["q"][at].float().transpose(1, 2)                        # [B, H, n, d_h]
    else:
        q = s["q"].float()
    K, V = plain_rows(s, "K"), plain_rows(s, "V")
    j = torch.arange(K.shape[2], device=S.device)[None, None, :]
    p = (S - k)[:, None, None] + torch.arange(n, device=S.device)[None, :, None]
    seen = (j <= p) & (j < S[:, None, None]) & (p < S[:, None, None])
    if c["window"]:
        seen &= j > p - c["window"]
    seen = seen[:, None, None]                                        # [B, 1, 1, n, positions]
    V = torch.where((j[:, 0] < S[:, None])[:, None, :, None], V, 0.0)
    z = (q.reshape(B, hk, (H // hk) * n, d) @ K.transpose(2, 3)).view(B, hk, H // hk, n, -1)
    z = torch.where(seen, z / math.sqrt(d), -math.inf)
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(m > -math.inf, m, 0.0))
    del z
    total = e.sum(-1, keepdim=True)
    y = (e.view(B, hk, -1, e.shape[-1]) @ V).view(B, hk, H // hk, n, d)
    y = torch.where(total > 0, y / total, 0.0).reshape(B, H, n, d)
    lse = (m + torch.log(total)).reshape(B, H, n)
    if c["packed"]:
        b, t, ok = row_places(s)
        t = t.clamp(max=n - 1)
        y = torch.where(ok[:, None, None], y[b, :, t], 0.0)
        lse = torch.where(ok[None, :], lse[b, :, t].T, -math.inf)
    else:
        ok = (torch.arange(n, device=S.device)[None, :] < k[:, None])[:, None, :, None]
        y = torch.where(ok, y, 0.0)
        lse = torch.where(ok[..., 0], lse, -math.inf)
    got = {"out": y.to(DTYPES[c["dtype"]])}
    if c["lse"]:
        got["lse"] = lse
    return got


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    S, n = lengths(c)
    d, hk, page, g = c["d_h"], c["H_kv"], c["page"], c["H"] // c["H_kv"]
    table = s["page_table"].tolist()
    starts = [sum(n[:b]) if c["packed"] else 0 for b in range(c["B"])]

    def rows_of(x, b):                        # [n_b, heads, d_h]
        return x[starts[b]:starts[b] + n[b]] if c["packed"] else x[b].transpose(0, 1)[:n[b]]

    def cached(name, b, head, count):
        ids = table[b][:-(-count // page)]
        x = s[name][ids, head].double()
        if c["pages"] != "16":
            x = x * s[name + "_scale"][ids, head].double().unsqueeze(-1)
        return x.reshape(-1, d)[:count]

    if c["call"] == "read":
        got = {}
        for name in ("K", "V"):
            y = torch.zeros((c["B"], hk, c["n"], d), dtype=torch.float64, device="cuda")
            for b in range(c["B"]):
                for head in range(hk):
                    y[b, head, :n[b]] = cached(name, b, head, n[b])
            got[name + "_out"] = y
        return got

    got = {}
    new = {}
    if c["call"] in ("append", "serve"):
        for name, x in (("K", s["k_new"]), ("V", s["v_new"])):
            if c["pages"] == "16":
                pool = s[name].double()
            else:
                scales = s[name + "_scale"].double()
            for b in range(c["B"]):
                r = rows_of(x, b).double()
                at = range(S[b] - n[b], S[b])
                ids, slots = [table[b][p // page] for p in at], [p % page for p in at]
                if c["pages"] == "16":
                    pool[ids, :, slots] = r
                    new[name, b] = r
                else:
                    a = r.abs().amax(-1).clamp(LEAST, MOST)
                    scales[ids, :, slots] = a / QMAX[c["pages"]]
                    code = r * (QMAX[c["pages"]] / a).unsqueeze(-1)
                    code = code.round() if c["pages"] == "i8" else code.float().to(torch.float8_e4m3fn).double()
                    new[name, b] = code * (a / QMAX[c["pages"]]).unsqueeze(-1)
            got[name] = pool if c["pages"] == "16" else None       # (codes are whole steps: they have no other value)
            if c["pages"] != "16":
                got[name + "_scale"] = scales
    if c["call"] == "append":
        return got

    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = s["lse"].double() if c["lse"] else None
    for b in range(c["B"]):
        q = rows_of(s["q"], b)
        p = torch.arange(S[b] - n[b], S[b], device="cuda")[:, None]
        j = torch.arange(S[b], device="cuda")[None, :]
        hidden = j > p
        if c["window"]:
            hidden = hidden | (j <= p - c["window"])
        for head in range(hk):
            K, V = cached("K", b, head, S[b]), cached("V", b, head, S[b])
            if c["call"] == "serve":
                K[S[b] - n[b]:], V[S[b] - n[b]:] = new["K", b][:, head], new["V", b][:, head]
            for h in range(head * g, head * g + g):
                z = ((q[:, h].double() @ K.T) / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                top = z.amax(1, keepdim=True)
                e = z.sub_(top).exp_()
                total = e.sum(1, keepdim=True)
                y = (e @ V) / total
                at = (slice(starts[b], starts[b] + n[b]), h) if c["packed"] else (b, h, slice(0, n[b]))
                out[at] = y
                if c["lse"]:
                    lse[at[::-1] if c["packed"] else at] = (top + total.log())[:, 0]
    got["out"] = out
    if c["lse"]:
        got["lse"] = lse
    return got
