"""Attention over the 4-bit cache by 256-row workgroups, against the 64-bit model.  A page table wide enough for a million tokens and no hint of the
length make the call plan for that many, so that short sequences take the way of long ones."""
import math

import pytest
import torch

from test_gpu_cache import DEV, FORMATS, P, Setup  # noqa: F401  (P is the fixture)

pytestmark = pytest.mark.gpu
TOKENS = 1 << 20


class Wide(Setup):
    def __init__(self, P, lens, news, page=64, **kw):
        super().__init__(P, lens, news, page=page, **kw)
        c = self.cache
        self.pages = torch.nn.functional.pad(self.pages, (0, TOKENS // page - c.max_pages), value=-1)
        self.cache = P.Cache(H_kv=c.H_kv, d=c.d, group=c.group, page=page, n_pages=c.n_pages, max_pages=TOKENS // page)

    def planned_for_256_rows(self):
        """the workspace holds two parts of 256 rows for every workgroup"""
        P, c, (B, H, n, d) = self.P, self.cache, self.q.shape
        wgs = min(256, 64 * B * c.H_kv * -(-(H // c.H_kv * n) // 256))
        room = 2 * wgs * 256 * (d + 2) * 4
        return room < P.cache_attn_workspace_bytes(P.Shape.of(self.q), c, 0) <= room + 16 * wgs + 1024

    def check(self, *a, **kw):
        assert self.planned_for_256_rows()
        super().check(*a, **kw)


@pytest.mark.parametrize("d, group", FORMATS)
@pytest.mark.parametrize("tiles", [(0, 1, 2, 3), (4, 5, 6, 7), (8, 9, 10, 17)])
@pytest.mark.parametrize("rest", [0, 1, 63])
def test_every_number_of_tiles(P, d, group, tiles, rest):
    """shared items: parts of two tiles, the last of one or two, whole and not"""
    lens = [64 * t + rest for t in tiles]
    Wide(P, lens, [130] * 4, n=130, H=2, H_kv=1, d=d, group=group).fill().check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n, H, H_kv, d, group, page", [(257, 2, 2, 128, 32, 64), (300, 6, 2, 64, 64, 16), (129, 5, 1, 128, 64, 32), (512, 1, 1, 128, 128, 256),
                                                        (700, 3, 3, 64, 32, 128)])
def test_several_runs_of_rows(P, n, H, H_kv, d, group, page, causal):
    """the last run incomplete, heads that share a run, causal runs that see less than others"""
    lens = [n, n + 1, n + 63, n + 500, n + 130, n // 3]
    Wide(P, lens, [n, n, n - 1, n // 2, 0, n], n=n, H=H, H_kv=H_kv, d=d, group=group, page=page).fill().check(causal)


@pytest.mark.parametrize("causal", [False, True])
def test_more_items_than_workgroups(P, causal):
    """320 items of 0 to 20 tiles: items alone in a workgroup, several in one, and shared ones"""
    lens = [(37 * b * b) % 1290 for b in range(80)]
    Wide(P, lens, [(53 * b) % 141 for b in range(80)], n=140, H=4, H_kv=4, d=64, group=64).fill().check(causal)


def test_few_sequences_among_many_idle_ones(P):
    lens, news = [0] * 400, [0] * 400
    for b, length in ((3, 700), (4, 130), (70, 64), (255, 1290), (398, 5)):
        lens[b], news[b] = length, min(length, 140)
    lens[200] = 900  # tokens, no rows
    Wide(P, lens, news, n=140, H=2, H_kv=2, d=64, group=32, page=1024).fill().check()


@pytest.mark.parametrize("length, n, H, d, group", [(9000, 130, 1, 128, 32), (20011, 100, 2, 128, 64), (30000, 140, 1, 64, 32), (2900, 400, 1, 128, 128)])
def test_one_sequence_in_many_parts(P, length, n, H, d, group):
    s = Wide(P, [length], [n], H=H, H_kv=H, d=d, group=group, page=256).fill()
    s.check()
    s.check(causal=True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n, share", [(130, 1), (150, 2)])
def test_rows_that_see_nothing(P, n, share, causal):
    s = Wide(P, [0, 1, n // 2, 190, 0, -4], [n, n, n, n, 0, n], H=2 * share, H_kv=2, page=16, n_pages=50).fill()
    s.pages[3] = -1
    s.check(causal)


def test_pages_that_are_not_followed(P):
    s = Wide(P, [600, 190], [200, 190], n=200, page=16, n_pages=60).fill()
    s.pages[0, 2], s.pages[0, 7], s.pages[1, 5], s.pages[1, 0] = -1, 60, -2 ** 31, 1 << 30
    s.pages[0, 12:24] = -1  # three tiles in a row
    s.check()
    s.check(causal=True)


@pytest.mark.parametrize("token", [0, 63, 64, 130, 191, 192, 383, 384, 399])
@pytest.mark.parametrize("d, group", [(128, 32), (64, 64)])
def test_a_value_that_is_not_finite_reaches_the_rows_that_see_it(P, d, group, token):
    """in tiles that every row sees and in others: NaN in that group's channels (all channels may be) of the rows that see the token, nothing elsewhere"""
    n, length = 140, 400
    s = Wide(P, [length], [n], H=1, H_kv=1, d=d, group=group).fill()
    m = s.model(s.pool)
    assert s.planned_for_256_rows()
    run = m.run(int(s.pages[0, token // 64]), 0)
    at = 64 * d + 64 * (d // group) * 4 + token % 64 * (d // group) * 4
    clean, _ = s.attend(causal=True)
    run[at:at + 4] = torch.tensor([0xc0, 0x7f, 0xc0, 0x7f], dtype=torch.uint8)  # the value's first group reads back as NaN
    out, lse = s.attend(causal=True)
    sees = torch.arange(n) + length - n >= token
    assert torch.isnan(out[0, 0, sees][:, :group]).all() and torch.isfinite(lse).all()
    assert torch.equal(out[0, 0, ~sees], clean[0, 0, ~sees])


def test_what_a_row_does_not_see_does_not_matter(P):
    n = 200
    s = Wide(P, [64 * 5 + 36], [n], H=1, H_kv=1, n=n).fill()
    run = s.model(s.pool).run(int(s.pages[0, 5]), 0)
    par = run[64 * 128:].view(2, 64, 16)
    par[:, 36:] = 0xff
    s.check()
    par[:, 10:36] = torch.tensor([0x80, 0x7f] * 8, dtype=torch.uint8)
    out, lse = s.attend(causal=True)
    par[:, 10:36] = 0
    out2, lse2 = s.attend(causal=True)
    assert torch.equal(out[:, :, :n - 26], out2[:, :, :n - 26]) and torch.equal(lse[:, :, :n - 26], lse2[:, :, :n - 26])
    assert torch.isnan(out[:, :, n - 26:]).all() and torch.isfinite(out2).all()


def test_keys_and_values_at_the_ends_of_their_range(P):
    """keys of +-16384 and values of +-2^100 in one group with small ones, and the smallest that exist"""
    n = 200
    s = Wide(P, [n], [n], H=1, H_kv=1)
    s.k[0, 0, ::3, 5], s.k[0, 0, 1::3, 5], s.q[0, 0, :, 5] = 16384.0, -16384.0, 2.0 ** -10
    s.k[0, 0, :, 64:] *= 2.0 ** -120
    s.v[0, 0, ::2, 7], s.v[0, 0, 1::2, 40], s.v[0, 0, :, 96:] = 2.0 ** 100, -2.0 ** 100, 2.0 ** -126
    s.model(s.pool).write(s.k, s.v, s.pages, s.lens, s.news)
    s.check()
    assert torch.isfinite(s.attend()[0]).all()


@pytest.mark.parametrize("scale", [0.0, 0.02, 1.0])
def test_large_queries_and_scales(P, scale):
    s = Wide(P, [500], [150], H=1, H_kv=1).fill()
    # |q k| stays below 2^24 * 4 * 2 * 128 * 3 and the logits below 2^30 (their weights are good to there: with spacing a, exp2 gets up to a / 2 above 0 instead
    # of 0, which out and lse both allow for, and overflows at 128; a factor of 2^40 gives a = 2^19)
    s.q[0, 0, 3], s.q[0, 0, 4] = 0.0, s.q[0, 0, 4] * (2.0 ** 24 if scale < 1 else 2.0 ** 17)
    s.q[0, 0, 5] *= 2.0 ** -100
    s.q[0, 0, 6:8] *= 1e4
    out, lse = s.attend(scale=scale)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    keep = [r for r in range(150) if r not in (4, 6, 7)]  # (rows with one weight that is not zero: the model's tolerance does not hold for logits of 1e7 and more)
    m = s.model(s.pool.to(DEV))
    want, wl, tol, lt = m.attention(s.q.to(DEV), s.pages, s.lens, s.news, False, scale or 128 ** -0.5)
    assert ((out.double() - want).abs() <= tol)[0, 0, keep].all() and ((lse.double() - wl).abs() <= lt)[0, 0, keep].all()


@pytest.mark.parametrize("n_max", [1, 5000, 100000])
def test_a_hint_that_is_wrong(P, n_max):
    s = Setup(P, [5000, 800], [300, 300], H=4, H_kv=2, page=64).fill()
    s.check(causal=True, n_max=n_max)


def test_strides_of_a_fused_projection(P):
    n = 150
    s = Wide(P, [290], [n], n=n, page=32).fill()
    wide = torch.zeros(1, n, 2, 3 * 128, dtype=torch.bfloat16, device=DEV)
    q = wide[..., :128].transpose(1, 2)
    q.copy_(s.q)
    out = torch.zeros_like(wide)
    P.cache_attn(q, P.Shape.of(q), s.cache, s.pool.to(DEV), *s.where(), out=out[..., 128:256].transpose(1, 2))
    assert torch.equal(out[..., 128:256].transpose(1, 2), s.attend()[0]) and not out[..., :128].any() and not out[..., 256:].any()


def test_replayed_while_the_sequences_grow_and_with_a_used_workspace(P):
    n = 140
    s = Wide(P, [3000, 1200], [n, n], n=n, H=4, H_kv=2).fill()
    assert s.planned_for_256_rows()
    pool, (pages, length, n_new), q = s.pool.to(DEV), s.where(), s.q.to(DEV)
    shape = P.Shape.of(q)
    ws = torch.full((P.cache_attn_workspace_bytes(shape, s.cache, 0),), 255, dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros_like(q), torch.zeros((2 * 4, n), device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.cache_attn(q, shape, s.cache, pool, pages, length, n_new, causal=True, out=out, lse=lse, ws=ws, want_lse=True)
    for i in range(5):
        length.copy_(torch.tensor([[3000, 1200], [10, 0], [2999, 64], [1, 1279], [128, 3000]][i]))
        n_new.copy_(torch.tensor([n, n - 30 * i]))
        q.normal_(), out.fill_(7.0), lse.fill_(7.0)
        eo, el = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
        P.cache_attn(q, shape, s.cache, pool, pages, length, n_new, causal=True, out=eo, lse=el, want_lse=True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eo) and torch.equal(lse, el), i


def test_two_streams_at_once(P):
    s = Wide(P, [2000, 900], [200, 150], n=200, H=8, H_kv=4).fill()
    pool, where, q = s.pool.to(DEV), s.where(), s.q.to(DEV)
    shape, outs = P.Shape.of(q), []
    want = torch.zeros_like(q)
    P.cache_attn(q, shape, s.cache, pool, *where, out=want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            outs.append(P.cache_attn(q, shape, s.cache, pool, *where, out=torch.zeros_like(q)))
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_either_way_gives_the_same_within_what_is_allowed(P):
    """the same call planned for short sequences (16-row workgroups) and for long ones"""
    s = Wide(P, [700, 300], [150, 100], n=150, H=2, H_kv=2, d=128, group=64).fill()
    a, al = s.attend(causal=True)
    b, bl = s.attend(causal=True, n_max=700)
    m = s.model(s.pool)
    _, _, tol, lt = m.attention(s.q, s.pages, s.lens, s.news, True, 128 ** -0.5)
    for i, new in enumerate(s.news):
        assert ((a - b)[i, :, :new].double().abs().cpu() <= 2 * tol[i, :, :new]).all()
        fin = torch.isfinite(al[i, :, :new]).cpu()
        assert ((al - bl)[i, :, :new].double().abs().cpu() <= 2 * lt[i, :, :new])[fin].all()
    assert math.isfinite(al.nan_to_num(neginf=0.0).sum().item())
