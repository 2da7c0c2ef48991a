"""The 4-bit key/value cache against a 64-bit model of it (tests/_cache_util.py): bytes written, values read back, attention."""
import math

import pytest
import torch

from _cache_util import Model, token_bytes

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def P():
    import paper_2604_12219_amd as P
    P.load_library()
    return P


class Setup:
    """a pool of random bytes, pages dealt out in any order, rows of q, k, v"""

    def __init__(self, P, lens, news, n=None, H=2, H_kv=2, d=128, group=32, page=64, token_major=False, seed=0, spare=2, max_pages=None, n_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.P, self.lens, self.news, self.H = P, list(lens), list(news), H
        B, n = len(lens), n if n is not None else max(max(news), 1)
        need = [max(0, -(-l // page)) for l in lens]
        max_pages = max_pages or max(max(need), 1) + 1
        n_pages = n_pages or sum(need) + spare
        self.cache = P.Cache(H_kv=H_kv, d=d, group=group, page=page, n_pages=n_pages, max_pages=max_pages)
        order = torch.randperm(n_pages, generator=g)
        self.pages = torch.full((B, max_pages), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            m = min(m, max_pages)
            self.pages[b, :m] = order[at:at + m].int()
            at += m
        # bytes of earlier users: any codes, any parameters, NaN and infinities among them
        self.pool = torch.randint(0, 256, (P.cache_bytes(self.cache),), generator=g, dtype=torch.uint8)

        def rows(heads, offset):
            size = (B, n, heads, d) if token_major else (B, heads, n, d)
            x = torch.randn(size, generator=g) * (0.5 + torch.rand(d, generator=g)) + offset * torch.randn(d, generator=g)
            x = x.bfloat16()
            return x.transpose(1, 2) if token_major else x
        self.q, self.k, self.v = rows(H, 0.0) * 1.5, rows(H_kv, 0.5), rows(H_kv, 0.3)
        self.gen = g

    def model(self, pool=None):
        c = self.cache
        return Model(self.pool.clone() if pool is None else pool, c.H_kv, c.d, c.group, c.page, c.n_pages, c.max_pages)

    def fill(self):
        """sensible contents for every page in use (random rows through the model's quantiser, a page at a time)"""
        from _cache_util import bf16_bytes, quantise
        c = self.cache
        m = self.model(self.pool)
        groups = c.d // c.group
        for row in self.pages.tolist():
            for pg in row:
                for h in range(c.H_kv if 0 <= pg < c.n_pages else 0):
                    run = m.run(pg, h)
                    run[:c.page * c.d] = torch.randint(0, 256, (c.page * c.d,), generator=self.gen, dtype=torch.uint8)
                    x = torch.randn((2 * c.page, c.d), generator=self.gen).bfloat16()
                    _, s, low = quantise(x, c.group)
                    run[c.page * c.d:] = torch.cat([bf16_bytes(s), bf16_bytes(low)], dim=-1).flatten()
        return self

    def dev(self, x):
        return x.to(DEV)

    def where(self, n_new=True):
        t = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
        return self.pages.to(DEV), t(self.lens), t(self.news) if n_new else None

    def attend(self, causal=False, scale=0.0, n_max=0, q=None, pool=None):
        P, q = self.P, self.q.to(DEV) if q is None else q
        shape = P.Shape.of(q, scale=scale)
        out, lse = torch.full_like(q, 7.0), torch.full((q.shape[0] * self.H, q.shape[2]), 7.0, device=DEV)
        pool = self.pool.to(DEV) if pool is None else pool
        P.cache_attn(q, shape, self.cache, pool, *self.where(), causal=causal, n_max=n_max, out=out, lse=lse, want_lse=True)
        return out, lse.view(q.shape[:3])

    def check(self, causal=False, scale=0.0, n_max=0, on=DEV):
        out, lse = self.attend(causal, scale, n_max)
        m = self.model(self.pool.to(on))
        want, wl, tol, lt = m.attention(self.q.to(on), self.pages, self.lens, self.news, causal, scale or self.cache.d ** -0.5)
        for b, new in enumerate(self.news):
            new = max(0, min(new, self.q.shape[2]))
            err = (out[b, :, :new].double().to(on) - want[b, :, :new]).abs()
            assert (err <= tol[b, :, :new]).all(), f"sequence {b}: off by {err.max():.3e}, {(err / tol[b, :, :new]).nan_to_num().max():.2f} of what is allowed"
            got, ref = lse[b, :, :new].double().to(on), wl[b, :, :new]
            fin = torch.isfinite(ref)
            assert (got[~fin] == ref[~fin]).all() and ((got - ref).abs()[fin] <= lt[b, :, :new][fin]).all(), f"sequence {b}: lse"
            assert (out[b, :, new:] == 7.0).all() and (lse[b, :, new:] == 7.0).all(), f"sequence {b}: padding was written"


FORMATS = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


# ---- writing -----------------------------------------------------------------------------------------
def written(s, P, n_new=True):
    pool = s.pool.to(DEV)
    k, v = s.k.to(DEV), s.v.to(DEV)
    P.cache_write(k, v, P.Shape.of(k), s.cache, pool, *s.where(n_new))
    m = s.model()
    m.write(s.k, s.v, s.pages, s.lens, s.news)
    return pool.cpu(), m.pool


@pytest.mark.parametrize("d, group", FORMATS)
@pytest.mark.parametrize("page, lens, news, token_major", [(16, [37, 5], [37, 1], False), (64, [130, 64, 1], [67, 64, 1], True), (512, [40], [33], False)])
def test_written_bytes(P, d, group, page, lens, news, token_major):
    got, want = written(Setup(P, lens, news, d=d, group=group, page=page, token_major=token_major), P)
    assert torch.equal(got, want)


def test_written_bytes_without_row_counts(P):
    s = Setup(P, [50, 20], [20, 20])
    got, want = written(s, P, n_new=False)
    assert torch.equal(got, want)


@pytest.mark.parametrize("lens, news", [([0, 9], [0, 3]), ([3, 40], [10, 40]), ([-5, 17], [2, 5]), ([40, 0], [-3, 40]), ([30, 30], [99, 7])])
def test_rows_without_a_place_are_not_written(P, lens, news):
    """idle slots, more rows than tokens (their positions are negative), negative counts, counts beyond the tensor"""
    got, want = written(Setup(P, lens, news, n=40, page=16), P)
    assert torch.equal(got, want)


def test_pages_that_are_not_followed_and_tokens_beyond_the_table(P):
    s = Setup(P, [100, 100], [100, 100], page=16, max_pages=5, n_pages=20)
    s.pages[0, 1], s.pages[0, 3], s.pages[1, 0] = -1, 20, 2 ** 31 - 1
    got, want = written(s, P)
    assert torch.equal(got, want)


def test_values_at_the_edges_of_the_type(P):
    s = Setup(P, [64], [64], H_kv=1, page=64)
    x = s.k[0, 0]
    big, tiny = 3.3895e38, 2.0 ** -133
    x[0] = 0.0
    x[1] = -0.0
    x[2] = 1.5
    x[3, :32], x[3, 32:64] = torch.linspace(-big, big, 32).bfloat16(), tiny
    x[3, 64], x[3, 96:] = tiny, -tiny
    x[4] = (torch.randn(128, generator=s.gen) * 2.0 ** -126).bfloat16()
    x[5] = (torch.randn(128, generator=s.gen) * 2.0 ** -121).bfloat16()
    x[6, 5], x[6, 40], x[6, 70], x[6, 127] = math.inf, -math.inf, math.nan, -math.nan
    x[7, :] = 1.0
    x[7, 3], x[7, 40] = -2.0 ** -40, 2.0 ** -70
    x[8] = torch.arange(128).bfloat16() % 31 / 2  # scale 1, every other value in the middle between two codes
    x[9] = (torch.arange(128) % 31 - 15).bfloat16()
    x[10] = torch.tensor([2.0 ** (i % 32 - 16) for i in range(128)]).bfloat16()
    x[11], x[11, ::32] = 29.0, -1.0
    x[11, 1::32] = 2.0 ** -70
    for i in range(12, 64):  # few mantissa bits: many quotients exactly in the middle
        x[i] = (torch.randint(-40, 41, (128,), generator=s.gen) * 2.0 ** int(torch.randint(-20, 20, (1,), generator=s.gen))).bfloat16()
    s.v[0, 0] = x.flip(0)
    got, want = written(s, P)
    assert torch.equal(got, want)


def test_long_random_rows_round_as_in_64_bits(P):
    """half a million quotients: codes at the border between two integers included"""
    s = Setup(P, [2100], [2100], H_kv=1, page=128)
    got, want = written(s, P)
    assert torch.equal(got, want)


def test_ties_with_the_smallest_scales(P):
    """scales of 2^-126 to 2^-120, whose products leave binary32's normal range; quotients in the middle between two codes wherever bf16 has them"""
    s = Setup(P, [192], [192], H_kv=1, page=64)
    scale = (torch.arange(0x80, 0x380, dtype=torch.int32) << 16).view(torch.float32).double()  # 768 groups, 192 rows of four
    high = (15 * scale).float().bfloat16()
    scale = (high.double() / 15).float().bfloat16().double()
    x = torch.zeros(768, 32, dtype=torch.bfloat16)
    x[:, 0] = high
    x[:, 1:16] = ((torch.arange(15) + 0.5) * scale[:, None]).float().bfloat16()
    x[:, 17:32] = ((torch.arange(15) + 0.5) * scale[:, None] * 0.99).float().bfloat16()
    s.k[0, 0], s.v[0, 0] = x.view(192, 128), (x - high[:, None]).view(192, 128)
    got, want = written(s, P)
    assert torch.equal(got, want)


# ---- reading back ------------------------------------------------------------------------------------
@pytest.mark.parametrize("d, group", FORMATS)
@pytest.mark.parametrize("token_major", [False, True])
def test_values_read_back(P, d, group, token_major):
    s = Setup(P, [75, 0, 33, 200], [75, 0, 2, 40], d=d, group=group, page=16, token_major=token_major, H_kv=3, H=3).fill()
    s.pages[3, 10] = -1
    k, v = torch.full_like(s.k, 7.0).to(DEV), torch.full_like(s.v, 7.0).to(DEV)
    gk, gv = P.cache_read(P.Shape.of(k), s.cache, s.pool.to(DEV), *s.where(), k=k, v=v)
    assert gk is k and gv is v
    m = s.model()
    for is_key, got in ((True, k.cpu()), (False, v.cpu())):
        for b, (length, new) in enumerate(zip(s.lens, s.news)):
            for h in range(3):
                want = torch.full((got.shape[2], d), 7.0, dtype=torch.float64)
                val, ok = m.tokens(s.pages[b], h, length, is_key)
                rows = torch.arange(length - new, length)
                want[:new][ok[rows]] = val[rows][ok[rows]]
                # rounded to binary32 (2^-24), then to bf16
                assert ((got[b, h].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -24) * want.abs()).all(), (is_key, b, h)


def test_read_back_into_new_tensors_and_nan_groups(P):
    s = Setup(P, [20], [20], H_kv=1, page=16)
    s.k[0, 0, 4, 40] = math.nan
    s.v[0, 0, 5, 3] = math.inf
    pool = s.pool.to(DEV)
    kd, vd = s.k.to(DEV), s.v.to(DEV)
    P.cache_write(kd, vd, P.Shape.of(kd), s.cache, pool, *s.where())
    k, v = P.cache_read(P.Shape.of(kd), s.cache, pool, *s.where())
    nan_k, nan_v = torch.isnan(k[0, 0]).cpu(), torch.isnan(v[0, 0]).cpu()
    want_k, want_v = torch.zeros(20, 128, dtype=torch.bool), torch.zeros(20, 128, dtype=torch.bool)
    want_k[4, 32:64], want_v[5, :32] = True, True
    assert torch.equal(nan_k, want_k) and torch.equal(nan_v, want_v)
    # a value lies within half a step of the grid of its group, the step rounded to bf16 (2^-8 of it, 15 steps away), and bf16 itself
    ok = ~want_k
    x, y = s.k[0, 0].double(), k[0, 0].cpu().double()
    g = x.reshape(20, 4, 32)
    step = ((g.amax(-1) - g.amin(-1)) / 15)[..., None].expand(-1, -1, 32).reshape(20, 128)
    assert ((x - y).abs()[ok] <= (step * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -8 * y.abs())[ok]).all()


# ---- attention ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("d, group", FORMATS)
@pytest.mark.parametrize("lens", [[1, 2, 15], [16, 17, 63], [64, 65, 127], [128, 200, 1000]])
def test_single_tokens(P, d, group, lens):
    Setup(P, lens, [1] * 3, d=d, group=group, page=16).fill().check()


@pytest.mark.parametrize("share", [1, 2, 3, 4, 5, 8, 12, 16, 24])
@pytest.mark.parametrize("d, group", [(128, 32), (64, 64)])
def test_shared_heads(P, d, group, share):
    Setup(P, [333, 40], [1, 1], H=2 * share, H_kv=2, d=d, group=group, page=32).fill().check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n, H, H_kv, d, group, page", [
    (2, 2, 2, 128, 32, 16), (3, 6, 2, 64, 32, 64), (5, 8, 1, 128, 128, 16), (16, 1, 1, 64, 64, 32), (17, 2, 2, 128, 64, 64),
    (31, 4, 4, 128, 32, 128), (33, 6, 3, 64, 64, 16), (64, 2, 1, 128, 32, 64), (100, 3, 1, 128, 128, 32), (129, 2, 2, 64, 32, 64),
    (257, 2, 2, 128, 32, 64), (300, 4, 2, 128, 64, 16)])
def test_several_rows(P, n, H, H_kv, d, group, page, causal):
    lens = [n, n + 1, n + 63, n + 500, n + 130]
    news = [n, n, max(1, n - 1), max(1, n // 2), 0]
    Setup(P, lens, news, n=n, H=H, H_kv=H_kv, d=d, group=group, page=page).fill().check(causal)


@pytest.mark.parametrize("n, share", [(1, 1), (6, 2), (40, 1), (150, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_rows_that_see_nothing(P, n, share, causal):
    """empty sequences, rows ahead of the first token (causal), sequences whose pages are not followed at all"""
    s = Setup(P, [0, 1, n // 2, 70, 0, -4], [n, n, n, n, 0, n], H=2 * share, H_kv=2, page=16, n_pages=30, max_pages=12).fill()
    s.pages[3] = -1
    s.check(causal)


@pytest.mark.parametrize("n", [1, 20, 200])
def test_pages_that_are_not_followed_are_seen_by_no_query(P, n):
    s = Setup(P, [300, 90], [n, min(n, 90)], n=n, page=16, n_pages=40).fill()
    s.pages[0, 2], s.pages[0, 7], s.pages[1, 5], s.pages[1, 0] = -1, 40, -2 ** 31, 1 << 30
    s.check()
    s.check(causal=True)


@pytest.mark.parametrize("n", [1, 30, 130])
def test_tokens_beyond_the_page_table_are_not_seen(P, n):
    Setup(P, [500, 160], [n, n], n=n, page=32, max_pages=5, n_pages=12).fill().check()


@pytest.mark.parametrize("n", [1, 4, 40, 140])
def test_what_a_row_does_not_see_does_not_matter(P, n):
    """NaN and infinite parameters in tokens behind the sequence and, for causal rows, in later tokens of it"""
    s = Setup(P, [64 * 3 + 36], [n], H=1, H_kv=1, page=64, n=n).fill()
    m = s.model(s.pool)
    run = m.run(int(s.pages[0, 3]), 0)
    par = run[64 * 128:].view(2, 64, 16)
    par[:, 36:] = 0xff  # slots behind the last token
    s.check()
    if n > 4:
        late = min(n // 2, 36)
        par[:, 36 - late:36] = torch.tensor([0x80, 0x7f] * 8, dtype=torch.uint8)  # infinite scale and minimum
        out, lse = s.attend(causal=True)
        par[:, 36 - late:36] = 0
        out2, lse2 = s.attend(causal=True)
        keep = n - late
        assert torch.equal(out[:, :, :keep], out2[:, :, :keep]) and torch.equal(lse[:, :, :keep], lse2[:, :, :keep])
        assert torch.isnan(out[:, :, keep:]).all() and torch.isfinite(out2).all()


@pytest.mark.parametrize("n, H", [(1, 4), (33, 2)])
@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_scale_of_the_caller_and_peaked_rows(P, n, H, scale):
    Setup(P, [700], [n], H=H, H_kv=2, page=64).fill().check(scale=scale)


@pytest.mark.parametrize("n, H, H_kv, length, d, group", [(1, 1, 1, 20011, 128, 32), (1, 16, 2, 9000, 64, 32), (4, 8, 1, 12345, 128, 128),
                                                         (60, 1, 1, 15000, 128, 64), (500, 2, 1, 6100, 64, 64)])
def test_long_sequences(P, n, H, H_kv, length, d, group):
    """divided among workgroups; n_max right, too small and not given"""
    s = Setup(P, [length, length // 7], [n, n], H=H, H_kv=H_kv, d=d, group=group, page=256).fill()
    for n_max in (length, 100, 0):
        s.check(causal=n > 1, n_max=n_max)


@pytest.mark.parametrize("n", [1, 40])
def test_strides_of_a_fused_projection(P, n):
    """q, k, v and out as slices of wider rows"""
    s = Setup(P, [90], [n], n=n, page=32).fill()
    wide = torch.zeros(1, n, 2, 3 * 128, dtype=torch.bfloat16, device=DEV)
    q, k, v = (wide[..., 128 * i:128 * (i + 1)].transpose(1, 2) for i in range(3))
    q.copy_(s.q), k.copy_(s.k), v.copy_(s.v)
    before = wide.clone()
    pool = s.pool.to(DEV)
    P.cache_write(k, v, P.Shape.of(k), s.cache, pool, *s.where())
    m = s.model()
    m.write(s.k, s.v, s.pages, s.lens, s.news)
    assert torch.equal(pool.cpu(), m.pool) and torch.equal(wide, before)
    out = torch.zeros_like(wide)[..., 128:256].transpose(1, 2)
    P.cache_attn(q, P.Shape.of(q), s.cache, pool, *s.where(), out=out)
    s.pool = pool.cpu()
    plain, _ = s.attend()
    assert torch.equal(out, plain)
    with pytest.raises(ValueError, match="strides"):  # out of another layout than q
        P.cache_attn(q, P.Shape.of(q), s.cache, pool, *s.where())


def test_a_pool_beyond_4_gib(P):
    """the last pages of a pool of 5 GB: offsets past 32 bits"""
    n_pages = 270_000
    s = Setup(P, [300, 129], [130, 1], n=130, H_kv=2, page=64, max_pages=6).fill()
    cache = P.Cache(H_kv=2, d=128, group=32, page=64, n_pages=n_pages, max_pages=6)
    assert P.cache_bytes(cache) > 5 << 30
    small = s.pool.to(DEV)
    where = s.where()
    far = (where[0] + (n_pages - s.cache.n_pages) * (where[0] >= 0)).int()
    pool = torch.zeros(P.cache_bytes(cache), dtype=torch.uint8, device=DEV)
    k, v, q = s.k.to(DEV), s.v.to(DEV), s.q.to(DEV)
    pool[-small.numel():] = small
    outs = []
    for c, p, pg in ((s.cache, small, where[0]), (cache, pool, far)):
        P.cache_write(k, v, P.Shape.of(k), c, p, pg, *where[1:])
        outs.append((*P.cache_read(P.Shape.of(k), c, p, pg, *where[1:]), P.cache_attn(q, P.Shape.of(q), c, p, pg, *where[1:])))
    assert torch.equal(pool[-small.numel():], small) and not pool[:-small.numel()].any()
    for a, b in zip(*outs):
        assert torch.equal(a, b)


# ---- together ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("d, group, chunk, causal", [(128, 32, 1, False), (64, 64, 5, True), (128, 128, 40, True), (128, 32, 150, False)])
def test_generation_step_by_step(P, d, group, chunk, causal):
    """chunks written and attended over one after the other, two sequences that grow at different speeds"""
    steps, H, H_kv, page = 4, 4, 2, 32
    total = steps * chunk
    s = Setup(P, [total, total], [chunk, chunk], H=H, H_kv=H_kv, d=d, group=group, page=page)
    pool, where = s.pool.to(DEV), s.where()
    length = torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    model_pool = s.pool.clone()
    for step in range(steps):
        news = [chunk, chunk if step % 2 == 0 else max(0, chunk - 1)]
        n_new = torch.tensor(news, dtype=torch.int32, device=DEV)
        length += n_new
        part = Setup(P, length.tolist(), news, n=chunk, H=H, H_kv=H_kv, d=d, group=group, page=page, seed=10 + step)
        k, v, q = part.k.to(DEV), part.v.to(DEV), part.q.to(DEV)
        P.cache_write(k, v, P.Shape.of(k), s.cache, pool, where[0], length, n_new)
        out, lse = P.cache_attn(q, P.Shape.of(q), s.cache, pool, where[0], length, n_new, causal=causal, want_lse=True)
        m = s.model(model_pool)
        m.write(part.k, part.v, s.pages, length.tolist(), news)
        want, _, tol, _ = m.attention(part.q, s.pages, length.tolist(), news, causal, d ** -0.5)
        for b, new in enumerate(news):
            assert ((out[b, :, :new].double().cpu() - want[b, :, :new]).abs() <= tol[b, :, :new]).all(), (step, b)
    assert torch.equal(pool.cpu(), model_pool)


@pytest.mark.parametrize("n", [1, 70])
def test_a_captured_step_is_replayed_while_the_sequences_grow(P, n):
    s = Setup(P, [3000, 1200], [n, n], n=n, H=4, H_kv=2, page=64).fill()
    pool, (pages, length, n_new) = s.pool.to(DEV), s.where()
    k, v, q = s.k.to(DEV), s.v.to(DEV), s.q.to(DEV)
    ks, qs = P.Shape.of(k), P.Shape.of(q)
    ws = torch.empty(P.cache_attn_workspace_bytes(qs, s.cache, 3000), dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros_like(q), torch.zeros((2 * 4, n), device=DEV)

    def step(out, lse, ws, pool):
        P.cache_write(k, v, ks, s.cache, pool, pages, length, n_new)
        P.cache_attn(q, qs, s.cache, pool, pages, length, n_new, causal=True, n_max=3000, out=out, lse=lse, ws=ws, want_lse=True)
    step(out, lse, ws, pool.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse, ws, pool)
    for i in range(4):
        length.copy_(torch.tensor([3000 - 300 * i, 1200 + 400 * i]))
        q.normal_(), k.normal_()
        eager_pool, eo, el = pool.clone(), torch.zeros_like(out), torch.zeros_like(lse)
        step(eo, el, torch.empty_like(ws), eager_pool)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, eager_pool) and torch.equal(out, eo) and torch.equal(lse, el), i


def test_two_graphs_that_share_a_workspace(P):
    a = Setup(P, [2500], [1], H=2, H_kv=1, page=64).fill()
    b = Setup(P, [1800], [1], H=2, H_kv=1, page=64, seed=5).fill()
    ws, graphs = None, []
    for s in (a, b):
        q = s.q.to(DEV)
        shape, pool, where, out = P.Shape.of(q), s.pool.to(DEV), s.where(), torch.zeros_like(q)
        if ws is None:
            ws = torch.empty(P.cache_attn_workspace_bytes(shape, s.cache, 2500), dtype=torch.uint8, device=DEV)
        want = P.cache_attn(q, shape, s.cache, pool, *where, n_max=2500)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            P.cache_attn(q, shape, s.cache, pool, *where, n_max=2500, out=out, ws=ws)
        graphs.append((g, out, want, q, pool, where))
    for _ in range(3):
        for g, out, want, *_ in graphs:
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_two_streams_at_once(P):
    s = Setup(P, [5000], [1], H=8, H_kv=2, page=64).fill()
    pool, where, q = s.pool.to(DEV), s.where(), s.q.to(DEV)
    shape = P.Shape.of(q)
    want = P.cache_attn(q, shape, s.cache, pool, *where)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(P.cache_attn(q, shape, s.cache, pool, *where))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


@pytest.mark.parametrize("n, H", [(1, 6), (9, 2), (150, 2)])
def test_same_bits_every_time(P, n, H):
    s = Setup(P, [4000, 700], [n, n], H=H, H_kv=2, page=64).fill()
    a, al = s.attend(causal=True)
    b, bl = s.attend(causal=True)
    assert torch.equal(a, b) and torch.equal(al, bl)


def test_a_batch_gives_what_its_sequences_give_alone(P):
    """the same sequence on either end of a ragged batch"""
    s = Setup(P, [400, 3, 400], [2, 2, 2], H=4, H_kv=2, page=32).fill()
    s.pages[2], s.q[2] = s.pages[0], s.q[0]
    out, _ = s.attend(causal=True)
    assert torch.equal(out[0], out[2])


def test_against_attention_over_bf16(P):
    """the dense kernel on the values read back sees what the cache holds"""
    n, H = 320, 2
    s = Setup(P, [n], [n], H=H, H_kv=H, page=64)
    k, v, q, pool, where = s.k.to(DEV), s.v.to(DEV), s.q.to(DEV), s.pool.to(DEV), s.where()
    shape = P.Shape.of(q)
    P.cache_write(k, v, shape, s.cache, pool, *where)
    kb, vb = P.cache_read(shape, s.cache, pool, *where)
    dense = P.attn_dense_ref(q, kb, vb, shape).double()
    got = P.cache_attn(q, shape, s.cache, pool, *where).double()
    m = s.model(pool.cpu())
    _, _, tol, _ = m.attention(s.q, s.pages, s.lens, s.news, False, 128 ** -0.5)
    assert ((got - dense).abs().cpu() <= 2 * tol).all()  # both are within tol of the model
    assert token_bytes(128, 32) == 160
