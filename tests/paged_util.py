"""A paged cache for the tests and what the operators on it compute, in 64 bits and by plain loops over the sequences."""
import math

import torch

BF16_STEP = 2.0 ** -8      # half a step of bf16, relative
F32_STEP = 2.0 ** -24


def power(k):
    """2 ** k in 64 bits, exactly."""
    return (torch.as_tensor(k).long() + 1023 << 52).view(torch.float64)


def quantised(x):
    """(e4m3 codes, scale bytes) of rows x [..., D]: the definition, in 64 bits."""
    x = x.double()
    a = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(a)
    k = torch.where(a == 0, 0, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126))
    y = x * power(-k).unsqueeze(-1)
    step = power(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    y = torch.where(x.isfinite(), torch.round(y / step) * step, float("nan"))
    return y.float().to(torch.float8_e4m3fn), (k + 127).to(torch.uint8)


class Cache:
    """Pages in a shuffled order, tables, lengths; every slot holds something, slots and table entries that no sequence uses hold the worst."""

    def __init__(self, kv, q, Hkv=2, D=128, page=16, f8=False, layout="head", seed=0, device="cuda", poison=True, spare=2, std=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.q, self.Hkv, self.D, self.page, self.f8 = kv, q, Hkv, D, page, f8
        used = [-(-n // page) for n in kv]
        self.n_pages, width = sum(used) + spare, max(used + [1])
        ids = torch.randperm(self.n_pages, generator=g).tolist()
        table = torch.full((len(kv), width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(used):
            table[b, :n] = torch.tensor(ids[at:at + n], dtype=torch.int32)
            at += n
        shape = (self.n_pages, Hkv, page) if layout == "head" else (self.n_pages, page, Hkv)
        self.values, self.pages, self.scales = {}, {}, {}
        for name in "kv":
            x = (torch.randn(*shape, D, generator=g) * std).bfloat16()
            if poison:
                live = torch.zeros(self.n_pages, page, dtype=torch.bool)
                for b, n in enumerate(kv):
                    for i in range(used[b]):
                        live[table[b, i], :max(0, min(page, n - i * page))] = True
                dead = ~(live[:, None] if layout == "head" else live[:, :, None]).expand(*shape)
                x[dead] = float("nan")
            if f8:
                codes, e = quantised(x)
                e = torch.where(x.isnan().all(-1), 255, e)
                codes, e = codes.view(torch.uint8), e.to(torch.uint8)
                if layout == "token":
                    codes, e = codes.transpose(1, 2), e.transpose(1, 2)
                dense = lambda t: t.to(device) if layout == "head" else t.transpose(1, 2).contiguous().to(device).transpose(1, 2)   # noqa: E731
                self.pages[name] = dense(codes).view(torch.float8_e4m3fn)
                self.scales[name] = e.contiguous().to(device).view(torch.float8_e8m0fnu)
            else:
                self.pages[name] = (x if layout == "head" else x.transpose(1, 2)).to(device) if layout == "head" else x.to(device).transpose(1, 2)
                self.scales[name] = None
        self.table = table.to(device)
        self.kv_len = torch.tensor(kv, dtype=torch.int32, device=device)
        starts = [0]
        for n in q:
            starts.append(starts[-1] + n)
        self.tokens = starts[-1]
        self.q_start = torch.tensor(starts, dtype=torch.int32, device=device)
        self.starts = starts

    def args(self):
        return self.pages["k"], self.pages["v"], self.table, self.kv_len

    def scale_args(self):
        return self.scales["k"], self.scales["v"]

    def rows(self, name, b, n=None):
        """Keys 0 .. n - 1 of sequence b in 64 bits: [n, Hkv, D]; and which of them lie on a page."""
        n = self.kv[b] if n is None else n
        c = torch.arange(n, device=self.table.device)
        page = self.table[b].long()[c // self.page]
        ok = (page >= 0) & (page < self.n_pages)
        page = torch.where(ok, page, 0)
        codes = self.pages[name]
        raw = codes.view(torch.uint8) if self.f8 else codes
        x = raw[page, :, c % self.page]
        if self.f8:
            e = self.scales[name].view(torch.uint8)[page, :, c % self.page].long()
            x = x.view(torch.float8_e4m3fn).double() * torch.where(e == 255, float("nan"), power(e - 127)).unsqueeze(-1)
        return x.double(), ok


def attention(cache, q, scale, causal, pos=None):
    """out, lse of tr_paged_attn in 64 bits, and bounds on what rounding may add: a list of (rows, out, lse, out bound, lse bound) by sequence.

    Rounding: a weight to bf16 (half a step of itself) and the result likewise; scores, weights and sums in 32 bits."""
    found = []
    gq = q.shape[1] // cache.Hkv
    for b, n in enumerate(cache.q):
        if n == 0:
            continue
        lo = cache.starts[b]
        K, ok = cache.rows("k", b)
        V, _ = cache.rows("v", b)
        kv = cache.kv[b]
        t, c = torch.arange(n, device=q.device), torch.arange(kv, device=q.device)
        seen = ok.expand(n, kv)
        if causal:
            p0 = kv - n if pos is None else pos[b]
            seen = seen & (c <= (p0 + t)[:, None])
        qs = q[0, :, lo:lo + n].double().view(cache.Hkv, gq, n, cache.D)
        K = torch.where(ok[:, None, None], K, 0.0).permute(1, 0, 2)[:, None]   # [Hkv, 1, kv, D]
        V = V.permute(1, 0, 2)[:, None]
        K = torch.where(seen.any(0)[:, None], K, 0.0)      # a key that no row sees may hold anything
        x = (qs @ K.transpose(2, 3) * scale).masked_fill(~seen, -math.inf)
        size = (qs.abs() @ K.abs().transpose(2, 3) * scale).masked_fill(~seen, 0.0).amax(-1) if kv else torch.zeros_like(qs[..., 0])
        lse = torch.logsumexp(x, -1) if kv else torch.full_like(qs[..., 0], -math.inf)
        p = torch.exp(x - lse.clamp(min=-1e300).unsqueeze(-1))
        clean = torch.where(V.isfinite(), V, 0.0).expand(cache.Hkv, gq, kv, cache.D)
        out, mean = p @ clean, p @ clean.abs()
        out = torch.where(torch.isnan(lse).unsqueeze(-1), float("nan"), out)
        for h, j, d in (~V.isfinite())[:, 0].nonzero().tolist():      # one value at a time: 0 times an infinity is NaN
            out[h, :, :, d] += torch.where(p[h, :, :, j] > 0, V[h, 0, j, d], 0.0)
        d_lse = (cache.D + 16) * F32_STEP * size + (kv + 16) * F32_STEP + 2.0 ** -20 + 2 * F32_STEP * lse.abs().nan_to_num(0, 0, 0)
        d_out = (BF16_STEP + 2 * d_lse.unsqueeze(-1)) * mean + 2.0 ** -126
        shape = (1, q.shape[1], n)
        found.append((slice(lo, lo + n), out.reshape(*shape, cache.D), lse.reshape(shape), d_out.reshape(*shape, cache.D), d_lse.reshape(shape)))
    return found


def check(found, out, lse):
    """Compares with what attention() found; returns the worst shares of the bounds that were used up."""
    worst = [0.0, 0.0]
    for rows, ref_o, ref_l, d_o, d_l in found:
        o, l = out[:, :, rows].double(), lse[:, :, rows].double()
        if out.dtype == torch.bfloat16:
            d_o = d_o + BF16_STEP * (ref_o.abs() + d_o)
        for at, (x, y, d) in enumerate(((o, ref_o, d_o), (l, ref_l, d_l))):
            fine = y.isfinite()
            assert torch.equal(x.isnan(), y.isnan()), "NaN in other places"
            assert torch.equal(x[~fine & ~y.isnan()], y[~fine & ~y.isnan()]), "infinities in other places"
            assert x[fine].isfinite().all()
            share = ((x - y).abs() / d)[fine]
            if share.numel():
                worst[at] = max(worst[at], float(share.max()))
    assert worst[0] <= 1 and worst[1] <= 1, worst
    return worst
