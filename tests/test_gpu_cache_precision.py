"""Attention over the 4-bit cache where the logits' precision decides: both kernels against the 64-bit model, with a bound that holds keys to
what binary32 leaves of them, at every magnitude that a cache holds."""
import math

import pytest
import torch

from _cache_util import HALF_STEP
from test_gpu_cache import DEV, FORMATS, P, Setup  # noqa: F401  (P is the fixture)
from test_gpu_cache_many_rows import Wide

pytestmark = pytest.mark.gpu
# rows of a key/value head: one and twelve (4 and 16 of them a workgroup), 140 (256 a workgroup)
ROWS = [1, 12, 140]


def setup(P, lens, n, **kw):
    return (Wide if n > 16 else Setup)(P, lens, [min(n, max(length, 1)) for length in lens], n=n, **kw)


def bounds(s, causal, scale, q, pool):
    """-> out, lse in 64 bits and what they may be off by.

    Logits.  With X = sum over the groups of (sum of |q| in it) * (largest |k| of the token in it): S = sum_g s sum q c + m sum q has a scale of at
    most 2/15 (1 + 2^-8) of a group's largest |k| and a minimum of at most that.  The few-row kernel sums q (16 + c) - 16 q in binary32, up to 132
    roundings a group, each of at most 2^-24 of a partial sum whose standard deviation (signs of q are random) is at most 24 |q| sqrt(32): a random walk of them is
    good to six standard deviations of 2^-24 / sqrt(3) * sqrt(132) * 24 / sqrt(32) * s sum |q| = 2^-24 * 169 * s sum |q|, which is 2^-19.4 of the
    group's part of X; the minimum's part, three roundings, 2^-22 of it.  The many-row kernel has K exact, the sums of q and m + 8 s to 2^-22 each and up to 9 * 32
    roundings of sums of s |c - 8| q: less.  Together 2^-18 X.  It rounds K and q, where they are 2^30 and 2^24 below the largest, to 2^-38 and 2^-32
    of the largest product of a group; six standard deviations of d such roundings are 6 sqrt(d / 3) (2^-32 + 2^-38) < 2^-26 of it.  A weight's exponent in log2 units, m and lse are binary32: 2^-22 of the
    logit itself, taken as 2^-22 (1 + |z|).

    lse moves by at most sum p dz (and its own roundings 2^-20 (1 + |lse|)), o by sum p |v - o| dz; weights and values are rounded to bf16 (u = 2^-8, six
    standard deviations, as in the model), the output by half a step."""
    m = s.model(pool)
    c = s.cache
    B, H, n, d = q.shape
    share, u = H // c.H_kv, HALF_STEP
    out = torch.zeros((B, H, n, d), dtype=torch.float64, device=q.device)
    tol, lse, lse_tol = torch.zeros_like(out), torch.zeros_like(out[..., 0]), torch.zeros_like(out[..., 0])
    for b in range(B):
        new, L = max(0, min(s.news[b], n)), max(0, s.lens[b])
        if L == 0:
            lse[b] = -math.inf
        for h in range(H if new and L else 0):
            k, ok = m.tokens(s.pages[b], h // share, L, True)
            v, _ = m.tokens(s.pages[b], h // share, L, False)
            groups = (d // c.group, c.group)
            top_k = k.abs().unflatten(1, groups).amax(-1)
            g = v.abs().unflatten(1, groups).amax(-1).repeat_interleave(c.group, dim=1)
            qr = q[b, h, :new].double()
            z = qr @ k.T * scale
            x = qr.abs().unflatten(1, groups).sum(-1) @ top_k.T
            most = (qr.abs().unflatten(1, groups).amax(-1) * top_k.amax(0)).amax(-1, keepdim=True)
            dz = scale * (2.0 ** -18 * x + 2.0 ** -26 * most) + 2.0 ** -22 * (1 + z.abs())
            hide = ~ok[None, :].expand(new, -1)
            if causal:
                pos = torch.arange(L, device=q.device)
                hide = hide | (pos[None, :] > (L - new + torch.arange(new, device=q.device))[:, None])
            z = z.masked_fill(hide, -math.inf)
            l = torch.logsumexp(z, 1)
            p = torch.exp(z - torch.where(torch.isinf(l), torch.zeros_like(l), l)[:, None])
            o = p @ v
            move = torch.stack([(p[i, :, None] * dz[i, :, None] * (v - o[i]).abs()).sum(0) for i in range(new)])
            out[b, h, :new], lse[b, h, :new] = o, l
            tol[b, h, :new] = u * o.abs() + 6 * u * ((p ** 2) @ (g ** 2)).sqrt() + move + 2.0 ** -16 * (p @ g)
            lse_tol[b, h, :new] = (p * dz).sum(1) + 2.0 ** -20 * (1 + l.abs().nan_to_num(posinf=0.0))
    return out, lse, tol, lse_tol


def check(s, causal=False, scale=0.0):
    if isinstance(s, Wide):
        assert s.planned_for_256_rows()
    q, pool = s.q.to(DEV), s.pool.to(DEV)
    out, lse = s.attend(causal, scale)
    want, wl, tol, lt = bounds(s, causal, scale or s.cache.d ** -0.5, q, pool)
    for b, new in enumerate(s.news):
        rows = slice(0, max(0, min(new, s.q.shape[2])))
        got, ref = lse[b, :, rows].double(), wl[b, :, rows]
        fin = torch.isfinite(ref)
        assert (got[~fin] == ref[~fin]).all(), f"sequence {b}: lse of rows that see nothing"
        err = (got - ref).abs()
        assert (err <= lt[b, :, rows])[fin].all(), f"sequence {b}: lse off by {err[fin].max():.3e}, {(err / lt[b, :, rows])[fin].max():.2f} of what is allowed"
        err = (out[b, :, rows].double() - want[b, :, rows]).abs()
        assert (err <= tol[b, :, rows]).all(), f"sequence {b}: off by {err.max():.3e}, {(err / tol[b, :, rows]).nan_to_num().max():.2f} of what is allowed"


def written(s):
    """K and V as they stand, through the model's quantiser"""
    m = s.model(s.pool)
    m.write(s.k, s.v, s.pages, s.lens, s.news)
    return s


def setup_written(P, lens, n, k_by=1.0, q_by=1.0, offset=0.0, **kw):
    """tokens of all sequences written with K and q times powers of two (per channel or one), the last n rows attend"""
    by = Setup(P, lens, lens, n=max(lens), **kw)
    by.k, by.q = ((by.k.float() + offset) * k_by).bfloat16(), (by.q.float() * q_by).bfloat16()
    written(by)
    s = setup(P, lens, n, **kw)
    q = torch.zeros_like(s.q)
    for b, new in enumerate(s.news):
        q[b, :, :new] = by.q[b, :, :new]
    s.pool, s.q = by.pool, q
    s.pages[:, :by.pages.shape[1]] = by.pages
    return s


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("d, group", FORMATS)
def test_keys_are_not_rounded(P, d, group, n):
    """logits of single tokens as they are (lse), keys with and without an offset"""
    for offset in (0.0, 8.0):
        check(setup_written(P, [1, 2, 3, 150], n, offset=offset, H=2, H_kv=1, d=d, group=group, page=64))


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("d, group", [(128, 32), (64, 64), (128, 128)])
@pytest.mark.parametrize("k", [-10, 15, 16, 18, 20, 24, 40, 90, 118])
def test_small_keys_with_large_queries(P, d, group, n, k):
    """ordinary logits from keys of 2^-k and queries of 2^k"""
    kw = dict(k_by=2.0 ** -k, H=2, H_kv=1, d=d, group=group, page=64)
    if k < 100:
        check(setup_written(P, [1, 200, 70], n, q_by=2.0 ** k, **kw))
    check(setup_written(P, [1, 200, 70], n, **kw), scale=2.0 ** k * d ** -0.5)  # and where the scale makes up for it
    check(setup_written(P, [130, 70], n, q_by=2.0 ** (k // 2), **kw), causal=True, scale=2.0 ** (k - k // 2) * d ** -0.5)


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("powers", [(10, -30, 0, -60), (-20, 10, -19, -21), (-90, -90, 5, -4), (0, 0, -25, -100)])
def test_groups_of_different_magnitudes(P, powers, n):
    """every group has the same share in the logits"""
    by = 2.0 ** torch.tensor(powers, dtype=torch.float64).repeat_interleave(32)
    check(setup_written(P, [1, 190, 64], n, k_by=by.float(), q_by=(1 / by).float(), H=2, H_kv=2, page=64))


@pytest.mark.parametrize("n", ROWS)
def test_a_group_of_large_keys_and_queries_that_hardly_look_at_it(P, n):
    for small in (-14, -16, -20, -26):
        by, q_by = torch.ones(128), torch.ones(128)
        by[32:64], q_by[32:64] = 2.0 ** 10, 2.0 ** small
        check(setup_written(P, [1, 2, 190], n, k_by=by, q_by=q_by, H=2, H_kv=1, page=64))


@pytest.mark.parametrize("n", ROWS)
def test_small_keys_beside_large_ones(P, n):
    """tokens 2^-20 of others, whose logits are large and negative: the small ones decide"""
    s = Setup(P, [180], [180], n=180, H=1, H_kv=1, page=64)
    s.q = s.q.abs()
    s.k[0, 0, ::3] = -s.k[0, 0, ::3].abs() * 16
    s.k[0, 0, 1::3] *= 2.0 ** -16
    s.k[0, 0, 2::3] *= 2.0 ** -16
    written(s)
    t = setup(P, [180], n, H=1, H_kv=1, page=64)
    t.pool, t.q = s.pool, s.q[:, :, :n] * 2.0 ** 16
    t.pages[:, :s.pages.shape[1]] = s.pages
    check(t)


@pytest.mark.parametrize("n", ROWS)
def test_groups_of_zeros_and_of_nan(P, n):
    """keys of a group that are all zero (whatever q is there), all alike, or NaN in a token that nobody sees"""
    kw = dict(H=1, H_kv=1, page=64)
    by, q_by = torch.ones(128), torch.ones(128)
    by[:32], q_by[:32] = 0.0, 2.0 ** 90
    by[64:96] = 2.0 ** -110
    s = setup_written(P, [170], n, k_by=by, q_by=q_by, **kw)
    run = s.model(s.pool).run(int(s.pages[0, 2]), 0)
    run[64 * 128:].view(2, 64, 16)[:, 42:] = 0xff  # slots behind the last token
    check(s)
    check(setup_written(P, [130], n, k_by=0.0, **kw))
    s = setup_written(P, [130], n, **kw)
    s.q[:] = 0.0
    check(s)


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("length", [1, 37, 64, 150])
@pytest.mark.parametrize("scale", [1e-3, 1e-9, 1e-30, 1e-45])
def test_small_scales(P, n, length, scale):
    """rows of zeros and of small numbers in tiles with tokens that are not seen, rows that see nothing"""
    for causal in (False, True):
        s = setup_written(P, [length, 0], n, H=1, H_kv=1, page=64) if not causal else setup_written(P, [length, 1], n, H=1, H_kv=1, page=64)
        s.q[0, 0, 0] = 0.0
        if n > 2:
            s.q[0, 0, 2] *= 2.0 ** -100
        check(s, causal, scale)


def test_rows_ahead_of_the_first_token_with_a_small_scale(P):
    s = Wide(P, [5, 90], [140, 140], n=140, H=1, H_kv=1, page=64).fill()
    s.q[:, :, ::2] = 0.0
    out, lse = s.attend(causal=True, scale=1e-9)
    assert torch.isinf(lse[0, 0, :135]).all() and not out[0, 0, :135].any()
    assert torch.isinf(lse[1, 0, :50]).all() and not out[1, 0, :50].any()
    seen = torch.cat([lse[0, 0, 135:], lse[1, 0, 50:]])
    assert torch.isfinite(seen).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("n", ROWS)
@pytest.mark.parametrize("v", [-126, -118, -110, -60, 60, 95])
def test_values_at_every_magnitude(P, n, v):
    """values of 2^v (and a group of zeros); the smallest are bf16 numbers of few bits, whose scale is 0 in the cache"""
    kw = dict(H=2, H_kv=1, page=64)
    s = Setup(P, [200, 3], [200, 3], n=200, **kw)
    s.v = (s.v.double() * 2.0 ** v).float().bfloat16()
    s.v[..., 32:64] = 0.0
    written(s)
    t = setup(P, [200, 3], n, **kw)
    t.pool, t.q = s.pool, torch.nn.functional.pad(s.q[:, :, :n], (0, 0, 0, max(0, t.q.shape[2] - 200)))
    t.pages[:, :s.pages.shape[1]] = s.pages
    check(t)


def test_either_way_gives_the_same_logits(P):
    """small keys and large queries, the same call planned for short sequences (16-row workgroups) and for long ones"""
    s = setup_written(P, [150, 100], 140, k_by=2.0 ** -24, q_by=2.0 ** 24, H=2, H_kv=2)
    _, wl, _, lt = bounds(s, False, 128 ** -0.5, s.q.to(DEV), s.pool.to(DEV))
    for n_max in (0, 150):
        lse = s.attend(n_max=n_max)[1]
        for b, new in enumerate(s.news):
            assert ((lse.double() - wl).abs() <= lt)[b, :, :new].all()


@pytest.mark.parametrize("k", [0, 30])
def test_more_sequences_than_a_part_has_room_for_the_magnitudes_of(P, k):
    """16,500 sequences of 1 to 100 tokens in two pages: sequences of one length have one result, and that is the model's"""
    B, n, d, page = 16500, 140, 64, 65536
    cache = P.Cache(H_kv=1, d=d, group=32, page=page, n_pages=2, max_pages=16)
    s = setup_written(P, [100], 100, H=1, H_kv=1, d=d, page=128, k_by=2.0 ** -k)
    pool = torch.zeros(P.cache_bytes(cache), dtype=torch.uint8)
    small = s.model(s.pool).run(int(s.pages[0, 0]), 0)
    big = pool[pool.numel() // 2:]  # page 1
    for part, at in ((128 * 32, 0), (128 * 32, 128 * 32), (128 * 8, 128 * 64), (128 * 8, 128 * 72)):
        big[at // 128 * page:][:part] = small[at:at + part]
    pages = torch.full((B, 16), -1, dtype=torch.int32)
    pages[:, 0] = 1
    lens = torch.arange(B, dtype=torch.int32) % 100 + 1
    q = (torch.randn(1, 1, n, d, generator=torch.Generator().manual_seed(1)) * 2.0 ** k).bfloat16().to(DEV).repeat(B, 1, 1, 1)
    shape = P.Shape.of(q)
    need = P.cache_attn_workspace_bytes(shape, cache, 0)
    assert need > 2 * 256 * 256 * (d + 2) * 4 + B * 4  # planned for 256 rows, with the magnitudes behind everything else
    out, lse = P.cache_attn(q, shape, cache, pool.to(DEV), pages.to(DEV), lens.to(DEV), want_lse=True)
    lse = lse.view(B, n)
    keys, _ = s.model(s.pool).tokens(s.pages[0], 0, 100, True)
    z = q[0, 0].double() @ keys.to(DEV).T * d ** -0.5
    want = torch.logcumsumexp(z, 1).T[(lens - 1).long().to(DEV)]
    # as in bounds(), with the largest |k| of all for every group of every token
    x = q[0, 0].double().abs().sum(1) * keys.abs().max().item()
    tol = d ** -0.5 * (2.0 ** -18 + 2.0 ** -26) * x + 2.0 ** -22 * (1 + z.abs().amax(1)) + 2.0 ** -20 * (1 + want.abs())
    assert ((lse.double() - want).abs() <= tol).all() and torch.isfinite(out).all()
