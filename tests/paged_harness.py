"""Paged caches for the tests and what the calls must give, in 64 bits, from plain formulas."""
import math

import numpy as np
import torch

from paper_2312_04985_amd import binding as B
from paper_2312_04985_amd.paged import PagedCache

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
QMAX = {"i8": 127.0, "e4m3": 448.0}


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def quantised(x: torch.Tensor, pages: str):
    """Codes and scales of rows [.., d_h] (float32 on the host): the three operations of the definition."""
    x = x.float()
    a = x.abs().amax(-1).clamp(2.0 ** -60, 2.0 ** 100).numpy()
    q = np.float32(QMAX[pages])
    scale, inv = a / q, q / a                     # float32 by float32: rounded once
    y = np.clip(x.numpy() * inv[..., None], -q, q)
    t = torch.from_numpy(y)
    codes = torch.from_numpy(np.rint(y)).to(torch.int8) if pages == "i8" else t.to(torch.float8_e4m3fn)
    special = ~torch.isfinite(x).all(-1)
    scale = torch.from_numpy(scale).masked_fill(special, float("nan"))
    return torch.where(special[..., None], torch.zeros((), dtype=torch.uint8), codes.view(torch.uint8)).view(codes.dtype), scale


def values(codes: torch.Tensor, scales) -> torch.Tensor:
    return codes.double() if scales is None else codes.float().double() * scales.double()[..., None]


class Built:
    """A cache whose pool is NaN wherever nothing was written, with rows K, V [B][S_b, H_kv, d_h] on the host."""

    def __init__(self, lens, H, H_kv, d_h, dtype, pages, page, seed, *, causal=True, window=0, extra=2, room=None, v_shift=1.0):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.dtype, self.pages, self.page = list(lens), DT[dtype], pages, page
        self.Bn, self.H, self.H_kv, self.d_h = len(lens), H, H_kv, d_h
        need = [-(-s // page) for s in lens]
        per = room or max(max(need), 1)
        n_pages = sum(need) + extra
        self.ids = torch.randperm(n_pages, generator=g)[:sum(need)].tolist()
        table = torch.full((self.Bn, per), -7, dtype=torch.int32)     # entries behind the length are never looked at
        at = 0
        for b, k in enumerate(need):
            table[b, :k] = torch.tensor(self.ids[at:at + k], dtype=torch.int32)
            at += k
        self.c = PagedCache(self.Bn, H, H_kv, d_h, page, n_pages, per, self.dtype, pages=pages, causal=causal, window=window)
        scale = torch.exp(0.7 * torch.randn((H_kv, d_h), generator=g))
        shift = v_shift * torch.randn((H_kv, d_h), generator=g)
        self.K = [(torch.randn((s, H_kv, d_h), generator=g) * scale).to(self.dtype) for s in lens]
        self.V = [(torch.randn((s, H_kv, d_h), generator=g) + shift).to(self.dtype) for s in lens]
        self.gen = g
        self.poison()
        self.c.page_table.copy_(table)
        self.c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))

    def poison(self):
        if self.pages == "16":
            self.c.K.fill_(float("nan")), self.c.V.fill_(float("nan"))
        else:
            for t in (self.c.K, self.c.V):
                t.view(torch.uint8).fill_(0x55)
            self.c.K_scale.fill_(float("nan")), self.c.V_scale.fill_(float("nan"))

    def fill(self):
        """All rows into their pages, by torch (the append has tests of its own)."""
        table = self.c.page_table.cpu().tolist()
        for name, rows in (("K", self.K), ("V", self.V)):
            pool = getattr(self.c, name)
            for b, s in enumerate(self.lens):
                if s <= 0:
                    continue
                p = torch.arange(s)
                page, slot = torch.tensor(table[b])[p // self.page].long().cuda(), (p % self.page).cuda()
                if self.pages == "16":
                    pool[page, :, slot] = rows[b].cuda()
                else:
                    codes, scales = quantised(rows[b], self.pages)
                    pool.view(torch.uint8)[page, :, slot] = codes.view(torch.uint8).cuda()
                    getattr(self.c, name + "_scale")[page, :, slot] = scales.cuda()
        return self

    def stored(self, name, b):
        """What the pages of sequence b stand for, in 64 bits [S_b, H_kv, d_h]."""
        rows = getattr(self, name)[b]
        return rows.double() if self.pages == "16" else values(*quantised(rows, self.pages))

    def queries(self, n, scale=0.3):
        """[B, n, H, d_h] on the host."""
        return (scale * torch.randn((self.Bn, n, self.H, self.d_h), generator=self.gen)).to(self.dtype)


def reference(built, b, q, n_b, causal=True, window=0):
    """(y, bound on |got - y|, lse, bound) [n_b, H, ..] of the last n_b rows of sequence b with queries q [n_b, H, d_h].

    The bound counts, for a result of fp32 sums over weights rounded to 16 bits: u_out |y| for the last rounding; u_w sum p |v| for the
    weights' (their fp16 subnormals: 2^-25 of the largest weight each); the exponent's error e, which changes a weight by the factor
    exp(+-e) and numerator and denominator each: 2 e sum p |v|; an fp32 sum of N terms, N 2^-24 of their magnitudes, twice."""
    S, d, g = built.lens[b], built.d_h, built.H // built.H_kv
    K, V = built.stored("K", b).cuda(), built.stored("V", b).cuda()
    q = q.double().cuda()
    u_out = half_step(built.dtype)
    u_w = half_step(built.dtype) if built.pages == "16" else half_step(torch.float16)
    p = torch.arange(S - n_b, S, device="cuda")[:, None]
    j = torch.arange(max(S, 0), device="cuda")[None, :]
    seen = torch.ones((n_b, max(S, 0)), dtype=torch.bool, device="cuda")
    if causal:
        seen &= j <= p
    if window:
        seen &= j > p - window
    y = torch.zeros((n_b, built.H, d), dtype=torch.float64, device="cuda")
    tol, lse, ltol = torch.zeros_like(y), torch.full((n_b, built.H), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros((n_b, built.H), dtype=torch.float64, device="cuda")
    some = seen.any(1)
    if not some.any():
        return y, tol, lse, ltol
    N = int(seen.sum(1).max())
    for h in range(built.H):
        Kh, Vh = K[:, h // g], V[:, h // g]
        z = (q[:, h] @ Kh.T) / math.sqrt(d)
        # magnitudes of what a score is summed of; d + 8 roundings of them (products, sums, scales, the way to the exponent)
        size = ((q[:, h].abs() @ Kh.abs().T) / math.sqrt(d)).masked_fill(~seen, 0.0)
        z = z.masked_fill(~seen, -math.inf)
        top = z.amax(1, keepdim=True)
        e = torch.where(seen, torch.exp(z - torch.where(some[:, None], top, 0.0)), 0.0)
        tot = e.sum(1, keepdim=True)
        w = e / tot.clamp(min=1e-300)
        Vz = Vh
        if not torch.isfinite(Vh).all():           # what a row does not see has no part in it
            yy = torch.stack([(w[i, seen[i]][:, None] * Vh[seen[i]]).sum(0) for i in range(n_b)])
            Vz = torch.where(torch.isfinite(Vh), Vh, 0.0)
        else:
            yy = w @ Vh
        mag = w @ Vz.abs()
        err = (d + 8) * 2.0 ** -24 * (size.amax(1) + z.abs().masked_fill(~seen, 0.0).amax(1)) + 2.0 ** -22
        y[:, h] = torch.where(some[:, None], yy, 0.0)
        # weights below fp16's normal range: 2^-25 of the largest one each, at most
        sub = 2.0 ** -25 * N * Vz.abs().amax() / tot if u_w == 2.0 ** -11 else 0.0
        tol[:, h] = u_out * yy.abs() + (u_w + 2 * err[:, None] + 2 * N * 2.0 ** -24) * mag + sub + 2.0 ** -25
        lse[:, h] = torch.where(some, (top + torch.log(tot))[:, 0], -math.inf)
        ltol[:, h] = err + N * 2.0 ** -24 + 2.0 ** -22 * (1 + lse[:, h].abs().nan_to_num(posinf=0.0))
    return y, tol, lse, ltol


def check(got, y, tol, what):
    got = got.double()
    ok = ((got - y).abs() <= tol) | (got == y) | (torch.isnan(y) & torch.isnan(got))
    if not bool(ok.all()):
        i = (~ok).nonzero()[0].tolist()
        d = (got - y).abs()
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} outside, first at {i}: got {got[tuple(i)].item()}, want {y[tuple(i)].item()}, "
                             f"bound {tol[tuple(i)].item()}, largest difference {d[torch.isfinite(d)].max().item() if torch.isfinite(d).any() else 'nan'}")


def check_attention(built, q, out, n_rows, lse=None, causal=True, window=0, what=""):
    """out [B, n, H, d_h] against the formulas; rows behind n_b hold 7 (the caller's filling), in lse too."""
    for b in range(built.Bn):
        n = n_rows[b]
        if n:
            y, tol, l, ltol = reference(built, b, q[b, :n], n, causal, window)
            check(out[b, :n], y, tol, f"{what} sequence {b}")
            if lse is not None:
                check(lse[b, :, :n].T, l, ltol, f"{what} lse of sequence {b}")
        assert (out[b, n:] == 7).all(), "rows behind the sequence's last"
        assert lse is None or (lse[b, :, n:] == 7).all()
