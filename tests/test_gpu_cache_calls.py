"""Calls of attention over the 4-bit cache as a generation makes them: one workspace for every length."""
import pytest
import torch

from test_gpu_cache import DEV, P, Setup  # noqa: F401  (P is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B, H, n", [(4, 8, 40), (8, 32, 1), (1, 8, 12)])
@pytest.mark.parametrize("longest", [0, 128000])
def test_a_workspace_for_the_longest_sequences_serves_all(P, B, H, n, longest):
    """n_max follows the sequences, the workspace is that of the largest one (whose call needs less of it than some others would take)"""
    lens = [1 + 1500 * (b + 1) for b in range(B)]
    s = Setup(P, lens, [n] * B, n=n, H=H, H_kv=8, page=64).fill()
    columns = 131072 // 64
    s.pages = torch.nn.functional.pad(s.pages, (0, columns - s.pages.shape[1]), value=-1)
    s.cache = P.Cache(H_kv=8, d=128, group=32, page=64, n_pages=s.cache.n_pages, max_pages=columns)
    q, pool, where = s.q.to(DEV), s.pool.to(DEV), s.where()
    shape = P.Shape.of(q)
    ws = torch.empty(P.cache_attn_workspace_bytes(shape, s.cache, longest), dtype=torch.uint8, device=DEV)
    asks = []
    want, wl, tol, lt = s.model(pool).attention(q, s.pages, lens, s.news, True, 128 ** -0.5)
    for n_max in (131072, 130560, 126976, 123904, 60000, 20000, max(lens), 512, 1):
        if longest and n_max > longest:
            continue
        asks.append(P.cache_attn_workspace_bytes(shape, s.cache, n_max))
        out, lse = P.cache_attn(q, shape, s.cache, pool, *where, causal=True, n_max=n_max, ws=ws, want_lse=True)
        assert ((out.double() - want).abs() <= tol).all(), n_max
        assert ((lse.view(B, H, n).double() - wl).abs() <= lt).all(), n_max
    if longest == 0 and B > 1:
        assert max(asks) > ws.numel()  # of the calls above some would have taken more
    with pytest.raises(P.PasaError):
        P.cache_attn(q, shape, s.cache, pool, *where, causal=True, ws=ws[:255])
