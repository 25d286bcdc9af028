"""Plain 64-bit model of the 8-bit paged cache (test infrastructure): what appends leave in codes and scales, and what
they stand for.  Pools are kept as float64 values of the codes and int64 exponents."""
from __future__ import annotations

import torch

E_MIN, E_MAX, BIAS, TOP = -64, 50, 127, 448.0
F64 = torch.float64


def two_to(e):
    """2^e, exactly, for an integer tensor or number."""
    return torch.tensor([2.0 ** int(x) for x in torch.as_tensor(e).flatten()], dtype=F64).view(torch.as_tensor(e).shape)


def nearest(v):
    """Values to the nearest e4m3 value, ties to even; beyond 448 to 448, not finite to NaN."""
    v = v.to(F64)
    a = v.abs()
    fine = torch.isfinite(v)
    b = torch.where(fine, a, torch.zeros_like(a)).clamp(max=TOP)
    e = torch.full_like(b, -6)
    for x in range(-5, 9):  # the binade, by comparison
        e = torch.where(b >= 2.0 ** x, torch.full_like(b, x), e)
    step = torch.pow(torch.full_like(b, 2.0), e - 3)
    r = torch.round(b / step) * step
    return torch.where(fine, torch.copysign(r, v), torch.full_like(r, float("nan")))


def exponent(most):
    """The smallest e of [-64, 50] with most <= 448 * 2^e, by trying each."""
    for e in range(E_MIN, E_MAX):
        if most <= TOP * 2.0 ** e:
            return e
    return E_MAX


def most(x):
    """Largest finite magnitude of x (0 if there is none)."""
    x = x.to(F64).abs()
    x = x[torch.isfinite(x)]
    return float(x.max()) if x.numel() else 0.0


class Cache:
    """One pool: codes [pages][Hkv][P][n][Dh] (their values), exponents [pages][Hkv][P/T]."""

    def __init__(self, pages, P, n, Hkv, Dh, T, codes=None, scales=None):
        self.P, self.n, self.T = P, n, T
        self.codes = torch.zeros(pages, Hkv, P, n, Dh, dtype=F64) if codes is None else \
            codes.float().to(F64).view(pages, Hkv, P, n, Dh).clone()
        self.e = torch.zeros(pages, Hkv, P // T, dtype=torch.int64) if scales is None else scales.long() - BIAS

    def clone(self):
        c = Cache.__new__(Cache)
        c.P, c.n, c.T, c.codes, c.e = self.P, self.n, self.T, self.codes.clone(), self.e.clone()
        return c

    def append(self, rows, table_row, first):
        """rows [tokens][n][Hkv][Dh] become tokens first ... of the sequence."""
        x = rows.to(F64).transpose(1, 2)  # [tokens][Hkv][n][Dh]
        t = first
        while t < first + x.shape[0]:
            start = t // self.T * self.T
            end = min(start + self.T, first + x.shape[0])
            page, slot = int(table_row[start // self.P]), start % self.P
            j = slot // self.T
            for h in range(x.shape[1]):
                new = x[t - first:end - first, h]
                e = exponent(most(new))
                if t > start:
                    had = min(max(int(self.e[page, h, j]), E_MIN), E_MAX)
                    e = max(e, had)
                    if e > had:
                        old = self.codes[page, h, slot:slot + t - start]
                        self.codes[page, h, slot:slot + t - start] = nearest(old * 2.0 ** (had - e))
                self.codes[page, h, slot + t - start:slot + end - start] = nearest(new * 2.0 ** -e)
                self.e[page, h, j] = e
            t = end

    def rows(self, table_row, tokens):
        """The values of the first tokens, [tokens * n][Hkv][Dh]."""
        ids = torch.as_tensor(table_row)[:-(-tokens // self.P)].long()
        v = self.codes[ids] * two_to(self.e[ids].clamp(E_MIN, E_MAX)).repeat_interleave(self.T, 2)[..., None, None]
        return v.permute(0, 2, 3, 1, 4).flatten(0, 2)[:tokens * self.n]

    def same(self, codes, scales):
        got = codes.cpu().float().to(F64).view(self.codes.shape)
        assert torch.equal(torch.isnan(got), torch.isnan(self.codes))
        assert torch.equal(got.nan_to_num(0.0), self.codes.nan_to_num(0.0))
        assert torch.equal(scales.cpu().long() - BIAS, self.e)


def quantised(cache, lens, P, T, n, seed, spare=3, width=None, fill=0x7F, scale_fill=255):
    """A contiguous bf16 cache [B][Lcap*n][Hkv][Dh] as an 8-bit paged one: (codes, scales, table, values), values
    [B][Lcap*n][Hkv][Dh] bf16 being what the codes stand for.  Codes of rows that no sequence holds are `fill` (NaN),
    scales of blocks that none holds `scale_fill`."""
    B, rows, Hkv, Dh = cache.shape
    held = [-(-int(x) // P) for x in lens]
    pages = sum(held) + spare
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    codes = torch.full((pages, Hkv, P, n, Dh), fill, dtype=torch.uint8)
    scales = torch.full((pages, Hkv, P // T), scale_fill, dtype=torch.uint8)
    table = torch.full((B, width or max(1, max(held))), -1, dtype=torch.int32)
    values = torch.zeros_like(cache)
    for b, L in enumerate(int(x) for x in lens):
        for i in range(held[b]):
            table[b, i] = perm.pop()
        x = cache[b, :L * n].view(L, n, Hkv, Dh).transpose(1, 2).to(F64)  # [L][Hkv][n][Dh]
        blocks = -(-L // T)
        pad = torch.cat([x, x.new_zeros(blocks * T - L, Hkv, n, Dh)]).view(blocks, T, Hkv, n * Dh) if L else x
        if not L:
            continue
        a = pad.abs().nan_to_num(0.0, posinf=0.0).amax((1, 3))  # [blocks][Hkv]
        e = torch.full_like(a, E_MIN)
        for y in range(E_MIN, E_MAX):
            e = torch.where(a > TOP * 2.0 ** y, torch.full_like(a, y + 1), e)
        f = torch.pow(torch.full_like(e, 2.0), e)
        f = f.repeat_interleave(T, 0)[:L, :, None, None]
        c = nearest(x / f)
        values[b, :L * n] = (c * f).transpose(1, 2).reshape(L * n, Hkv, Dh).to(torch.bfloat16)
        tok = torch.arange(L)
        page, slot = table[b].long()[tok // P], tok % P
        codes[page, :, slot] = c.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
        at = torch.arange(blocks) * T
        scales[table[b].long()[at // P], :, at % P // T] = (e + BIAS).to(torch.uint8)
    return codes.view(pages, Hkv, P * n, Dh).view(torch.float8_e4m3fn), scales, table, values
