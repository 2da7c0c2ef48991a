"""A plain 64-bit model of the 4-bit cache, byte by byte, for the cache's tests (any device; no code of the package)."""
import math

import torch

HALF_STEP = 2.0 ** -8  # bf16: half a step, relative to the value


def token_bytes(d, group):
    return d + 8 * (d // group)


MOST_KEY, MOST_VALUE = 16384.0, 2.0 ** 100


def quantise(x, group, most=math.inf):
    """x bf16 [..., d], values up to most -> codes (int64, as x), scale, minimum (fp32 values that are bf16, [..., groups])"""
    g = x.double().reshape(*x.shape[:-1], -1, group)
    bad = ~(torch.isfinite(g) & (g.abs() <= most)).all(-1)
    g = torch.where(bad[..., None], torch.zeros_like(g), g)
    low, high = g.amin(-1), g.amax(-1)
    s = ((high - low) / 15).float().bfloat16().float()
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    one = torch.where(s == 0, torch.ones_like(s), s).double()[..., None]
    c = torch.round((g - low[..., None]) / one).clamp(0, 15)
    c = torch.where((s == 0)[..., None], torch.zeros_like(c), c).long().reshape(x.shape)
    nan = torch.full_like(s, math.nan)
    return c, torch.where(bad, nan, s), torch.where(bad, nan, low.float() + 0.0)


def bf16_bytes(x):
    """fp32 [...] -> uint8 [..., 2], little end first (NaN: 0x7fc0)"""
    b = x.bfloat16().view(torch.int16).int() & 0xffff
    b = torch.where(torch.isnan(x), torch.full_like(b, 0x7fc0), b)
    return torch.stack([b & 255, b >> 8], dim=-1).to(torch.uint8)


class Model:
    """pool bytes plus the description they follow"""

    def __init__(self, pool, H_kv, d, group, page, n_pages, max_pages):
        self.pool, self.H_kv, self.d, self.group, self.page, self.n_pages, self.max_pages = pool, H_kv, d, group, page, n_pages, max_pages
        self.head_bytes = page * token_bytes(d, group)

    def run(self, page, h):
        at = (page * self.H_kv + h) * self.head_bytes
        return self.pool[at:at + self.head_bytes]

    def places(self, pages_row, first, rows):
        """(row, page of the pool, slot) of the rows that have a place"""
        out = []
        for i in range(rows):
            pos = first + i
            if 0 <= pos < self.max_pages * self.page:
                pg = int(pages_row[pos // self.page])
                if 0 <= pg < self.n_pages:
                    out.append((i, pg, pos % self.page))
        return out

    def code_place(self, is_key):
        """byte and shift of every channel inside a token's codes"""
        ch = torch.arange(self.d)
        word = (ch % 32) // 8 * (self.d // 32) + ch // 32 if is_key else ch // 8
        return 4 * word + ch % 8 // 2, ch % 2 * 4

    def write(self, k, v, pages, length, n_new):
        d, page, groups = self.d, self.page, self.d // self.group
        for b in range(k.shape[0]):
            new = max(0, min(int(n_new[b]), k.shape[2]))
            for i, pg, slot in self.places(pages[b], max(0, int(length[b])) - new, new):
                for h in range(self.H_kv):
                    run = self.run(pg, h)
                    for is_key, x in ((True, k), (False, v)):
                        c, s, m = quantise(x[b, h, i], self.group, MOST_KEY if is_key else MOST_VALUE)
                        byte, shift = self.code_place(is_key)
                        code = torch.zeros(d // 2, dtype=torch.long).index_add_(0, byte, c.cpu() << shift)
                        at = (0 if is_key else page * d // 2) + slot * (d // 2)
                        run[at:at + d // 2] = code.to(torch.uint8)
                        at = page * d + (0 if is_key else page * groups * 4) + slot * groups * 4
                        run[at:at + groups * 4] = torch.cat([bf16_bytes(s), bf16_bytes(m)], dim=-1).flatten().cpu()

    def tokens(self, pages_row, h, length, is_key):
        """fp64 [length, d] and which of them lie in a page that is followed"""
        length = max(0, min(length, self.max_pages * self.page))
        d, page, groups, dev = self.d, self.page, self.d // self.group, self.pool.device
        pos = torch.arange(length, device=dev)
        pg = pages_row.to(dev).long()[pos // page]
        ok = (pg >= 0) & (pg < self.n_pages)
        base = (torch.where(ok, pg, torch.zeros_like(pg)) * self.H_kv + h) * self.head_bytes
        byte, shift = (t.to(dev) for t in self.code_place(is_key))
        at = base + (0 if is_key else page * d // 2) + pos % page * (d // 2)
        code = (self.pool[at[:, None] + byte].long() >> shift) & 15
        at = base + page * d + (0 if is_key else page * groups * 4) + pos % page * (groups * 4)
        at = at[:, None] + 4 * (torch.arange(d, device=dev) // self.group)

        def number(at):
            return ((self.pool[at].int() | (self.pool[at + 1].int() << 8)) << 16).view(torch.float32)
        return number(at).double() * code + number(at + 2).double(), ok

    def attention(self, q, pages, length, n_new, causal, scale):
        """-> out, lse in 64 bits and what they may be off by (zero rows where nothing was to be written).

        Tolerance, per output value.  o = sum_t p_t v_t.  Roundings: the output to bf16, half a step of |o|; every weight, scaled or not,
        to bf16, and every value to bf16 where the values are formed: each relative error up to u = 2^-8, independent, of terms no larger
        than the group's largest |v| (g); keys to bf16 where they are formed, which moves logit t by sum_c q_c k_c e_c, standard deviation at most
        u / sqrt(3) scale sqrt(sum_c q_c^2 k_c^2) =: z_t, and o by sum_t p_t (v_t - o) times that.  Six standard deviations of the sum
        of all of these (which covers the worst case of up to a dozen terms), and 2^-16 of sum p g for what binary32 sums lose."""
        B, H, n, d = q.shape
        share = H // self.H_kv
        out = torch.zeros((B, H, n, d), dtype=torch.float64, device=q.device)
        tol, lse, lse_tol = torch.zeros_like(out), torch.zeros_like(out[..., 0]), torch.zeros_like(out[..., 0])
        u = HALF_STEP
        for b in range(B):
            new = max(0, min(int(n_new[b]), n))
            L = max(0, int(length[b]))
            for hk in range(self.H_kv if new else 0):
                k, ok = self.tokens(pages[b], hk, L, True)
                v, _ = self.tokens(pages[b], hk, L, False)
                g = v.abs().unflatten(1, (self.d // self.group, self.group)).amax(-1).repeat_interleave(self.group, dim=1)
                pos = torch.arange(v.shape[0], device=q.device)
                for h in range(hk * share, (hk + 1) * share):
                    qr = q[b, h, :new].double()
                    z = qr @ k.T * scale
                    hide = ~ok[None, :].expand(new, -1)
                    if causal:
                        hide = hide | (pos[None, :] > (L - new + torch.arange(new, device=q.device))[:, None])
                    z = z.masked_fill(hide, -math.inf)
                    empty = hide.all(1)
                    l = torch.logsumexp(z, 1) if z.shape[1] else torch.full((new,), -math.inf, dtype=torch.float64, device=q.device)
                    p = torch.exp(z - torch.where(empty, torch.zeros_like(l), l)[:, None])
                    seen = ~hide.all(0)  # what no row sees may be anything
                    vv, gg, kk = (torch.where(seen[:, None], t, torch.zeros_like(t)) for t in (v, g, k))
                    o = p @ vv
                    zt = (u / math.sqrt(3)) ** 2 * scale ** 2 * (qr ** 2 @ (kk ** 2).T)
                    var = (p ** 2) @ (gg ** 2) * (3 * u ** 2 / 3) + (p ** 2 * zt) @ vv ** 2 - 2 * o * ((p ** 2 * zt) @ vv) + o ** 2 * (p ** 2 * zt).sum(1, keepdim=True)
                    out[b, h, :new], lse[b, h, :new] = o, l
                    tol[b, h, :new] = u * o.abs() + 6 * var.clamp_min(0).sqrt() + 2.0 ** -16 * (p @ gg)
                    lse_tol[b, h, :new] = 6 * ((p ** 2 * zt).sum(1)).sqrt() + (p * zt).sum(1) + 2.0 ** -16 * (1 + l.abs().nan_to_num(posinf=0.0))
        return out, lse, tol, lse_tol
