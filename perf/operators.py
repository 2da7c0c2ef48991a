"""Performance cases of the 4-bit key/value cache: writing it, reading it back and attending over it.

A streaming generation keeps the keys and values of everything it has produced and adds a chunk of frames (or, in a
language model, a token) at a time.  The cache is a pool of pages; a page holds `page` tokens of one sequence, and in
it, per key/value head, one run of bytes:

  K codes   [page][d/2]     the four bits of 8 channels in a 32-bit word, channel c of the 8 in bits 4c..4c+3;
                            word q * (d/32) + j holds channels 32 j + 8 q .. + 7   (q = 0..3)
  V codes   [page][d/2]     word w holds channels 8 w .. 8 w + 7
  K params  [page][d/G][2]  bf16 scale s and minimum m of every group of G channels
  V params  [page][d/G][2]

and a code c stands for s c + m.  Row i of sequence b is token len[b] - new[b] + i of that sequence.

``path`` of a case:
  write  cache_write of new rows, then cache_read of the same rows       -> k, v as the cache holds them
  read   cache_read of every sequence                                    -> k, v
  attn   cache_attn of new rows over the cached tokens                   -> out, lse
Rows at and behind new[b] are padding: nobody writes them.
"""
import math

import torch

own = False


def _case(path, batch, heads, kv_heads, n, length, d=128, group=32, page=64, ragged=False, causal=False, token_major=False):
    return {"path": path, "batch": batch, "heads": heads, "kv_heads": kv_heads, "n": n, "length": length, "d": d, "group": group,
            "page": page, "ragged": ragged, "causal": causal, "token_major": token_major}


def listed():
    cases = {
        # a decoding step of a few conversations writes one token each: launches and host work count
        "write-token": _case("write", 8, 8, 8, 1, 1024, page=16, ragged=True),
        # a chunk of three latent frames at 480p (30 x 52 patches), 12 heads, appended behind 18 frames, stored token by token
        "write-chunk-480p": _case("write", 1, 12, 12, 4680, 32760, token_major=True),
        # the same of a 720p generation with 40 heads (45 x 80 patches), groups of 64
        "write-chunk-720p": _case("write", 1, 40, 40, 10800, 75600, group=64, page=256),
        # a short clip read back whole: two prompts of different length, head dimension 64, pages that end inside a tile
        "read-clip": _case("read", 2, 3, 3, 1365, 1365, d=64, page=16, ragged=True),
        # the 720p cache read back whole, as a step with full-precision attention would
        "read-720p": _case("read", 1, 40, 40, 75600, 75600, page=256),
        # one token over a short context: nothing but latency
        "token-short": _case("attn", 1, 12, 12, 1, 333, d=64, page=16),
        # a batch of conversations of 800 to 8000 tokens and an idle slot, four query heads to a key/value head
        "token-batch": _case("attn", 32, 32, 8, 1, 8000, page=16, ragged=True),
        # one token over the whole 720p cache
        "token-720p": _case("attn", 1, 40, 40, 1, 75600, page=256),
        # four drafted tokens to be checked at once, eight query heads to a key/value head
        "draft-tokens": _case("attn", 4, 24, 3, 4, 20011, d=128, group=128, page=64, ragged=True, causal=True),
        # prompts of up to 2048 tokens being read in behind what was there, padded batch, head dimension 64
        "prompt-batch": _case("attn", 4, 16, 4, 2048, 6000, d=64, group=64, page=32, ragged=True, causal=True, token_major=True),
        # a chunk of three frames at 480p over the cache of all 21
        "chunk-480p": _case("attn", 1, 12, 12, 4680, 32760, token_major=True),
        # one frame at 720p over the cache of all 21, 40 heads
        "frame-720p": _case("attn", 1, 40, 40, 3600, 75600, page=256),
    }
    return [dict(c, name=n) for n, c in cases.items()]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {p: {x: max(work(c)[x] for c in listed() if c["path"] == p) for x in ("bytes", "flops")} for p in ("write", "read", "attn")}
    path = rng.choice(["attn", "attn", "attn", "write", "read"])
    while True:
        kv_heads = _log_uniform(rng, 1, 40)
        heads = kv_heads * (rng.choice([1, 1, 2, 3, 4, 8, 16]) if path == "attn" else 1)
        batch, length = _log_uniform(rng, 1, 32), _log_uniform(rng, 16, 120000)
        if path == "attn":
            n = rng.choice([1, 1, rng.randint(2, 8), _log_uniform(rng, 9, 5000)])
        else:
            n = length if path == "read" else rng.choice([1, _log_uniform(rng, 2, 12000)])
        d = rng.choice([64, 128, 128])
        c = _case(path, batch, heads, kv_heads, n, length, d, rng.choice([32, 32, 64, 128]), rng.choice([16, 32, 64, 128, 512]),
                  batch > 1 and rng.random() < 0.7, path == "attn" and n > 1 and rng.random() < 0.5, rng.random() < 0.4)
        if n > length or c["group"] > d or heads > 64 or batch * kv_heads * length > 4_000_000:
            continue
        if any(work(c)[x] > most[path][x] for x in most[path]):
            continue
        return c


def _lengths(c):
    """(length, new rows) of every sequence.  Ragged: from the full length down to a tenth of it, new rows alike but never
    more than there are tokens; the last of four or more slots is idle."""
    lens, news = [], []
    for b in range(c["batch"]):
        part = 1 - 0.9 * b / c["batch"] if c["ragged"] else 1
        lens.append(max(1, int(c["length"] * part)))
        if c["path"] == "read":
            news.append(lens[-1])
        else:
            news.append(min(lens[-1], max(1, int(c["n"] * (1 - 0.7 * (b % 5) / 5 if c["ragged"] else 1)))))
    if c["ragged"] and c["batch"] >= 4:
        lens[-1] = news[-1] = 0
    return lens, news


def _token_bytes(c):
    return c["d"] + 8 * (c["d"] // c["group"])


def _quantise(x, group):
    """codes (uint8, as x), scale and minimum (bf16 [..., groups]) of bf16 x [..., d].  The quotients in 64 bits: a value in the middle
    between two codes must not go by a rounding before it"""
    x = x.double().unflatten(-1, (-1, group))
    low, high = x.amin(-1), x.amax(-1)
    s = ((high - low) / 15).float().bfloat16()
    s = torch.where(s.float() < 2.0 ** -126, torch.zeros_like(s), s)
    d = torch.where(s == 0, torch.ones_like(s), s).double()[..., None]
    c = ((x - low[..., None]) / d).round().clamp(0, 15) * (s != 0)[..., None]
    return c.to(torch.uint8).flatten(-2), s, low.bfloat16()


def _fields(pool, c):
    """views of a pool: K codes, V codes [pages, heads, page, d/2] uint8, K params, V params [pages, heads, page, groups, 2] bf16"""
    page, d, groups = c["page"], c["d"], c["d"] // c["group"]
    p = pool.view(-1, c["kv_heads"], page * _token_bytes(c))
    code, par = page * d // 2, page * groups * 4
    kc, vc, kp, vp = p.split([code, code, par, par], dim=2)
    return (kc.unflatten(2, (page, d // 2)), vc.unflatten(2, (page, d // 2)),
            kp.view(torch.bfloat16).unflatten(2, (page, groups, 2)), vp.view(torch.bfloat16).unflatten(2, (page, groups, 2)))


def _pack(codes, is_key):
    if is_key:  # channel 32 j + 8 q + c -> place (q, j, c)
        codes = codes.unflatten(-1, (-1, 4, 8)).transpose(-3, -2).flatten(-3)
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _unpack(packed, par, is_key):
    """fp32 values [..., d] of codes [..., d/2] and parameters [..., groups, 2]"""
    codes = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2)
    if is_key:
        codes = codes.unflatten(-1, (4, -1, 8)).transpose(-3, -2).flatten(-3)
    par = par.float()
    return (codes.unflatten(-1, (par.shape[-2], -1)).float() * par[..., 0:1] + par[..., 1:2]).flatten(-2)


def _places(s):
    """(sequence, row, page of the pool, slot in it) of every new row, as index tensors"""
    c, dev = s["case"], s["pages"].device
    b = torch.cat([torch.full((m,), i, device=dev) for i, m in enumerate(s["news"])])
    row = torch.cat([torch.arange(m, device=dev) for m in s["news"]])
    pos = torch.cat([torch.arange(l - m, l, device=dev) for l, m in zip(s["lens"], s["news"])])
    return b, row, s["pages"][b, pos // c["page"]].long(), pos % c["page"]


def _tokens(s, b):
    """fp32 K and V [kv_heads, length, d] of sequence b"""
    c, length = s["case"], s["lens"][b]
    of = s["pages"][b, :-(-length // c["page"])].long()
    kc, vc, kp, vp = (f[of].transpose(0, 1).flatten(1, 2)[:, :length] for f in _fields(s["pool"], c))
    return _unpack(kc, kp, True), _unpack(vc, vp, False)


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    B, n, d = c["batch"], c["n"], c["d"]
    lens, news = _lengths(c)

    def rows(heads, spread, offset):
        """[B, heads, n, d] (token-major storage: a view of [B, n, heads, d]); channels differ in scale and offset, as they do in
        trained models"""
        size = (B, n, heads, d) if c["token_major"] else (B, heads, n, d)
        x = torch.randn(size, generator=g, device=dev) * spread
        x = x * (0.5 + torch.rand(d, generator=g, device=dev)) + offset * torch.randn(d, generator=g, device=dev)
        x = x.bfloat16()
        return x.transpose(1, 2) if c["token_major"] else x

    # the pool: a few pages more than are in use, dealt out in any order, bytes of earlier users in what is not written
    need = [-(-l // c["page"]) for l in lens]
    n_pages, columns = sum(need) + 3, max(need) + 1
    order = torch.randperm(n_pages, generator=g, device=dev).int()
    pages = torch.zeros((B, columns), dtype=torch.int32, device=dev)
    at = 0
    for b, m in enumerate(need):
        pages[b, :m] = order[at:at + m]
        at += m
    pool = torch.randint(0, 256, (n_pages * c["kv_heads"] * c["page"] * _token_bytes(c),), generator=g, device=dev, dtype=torch.uint8)
    s = {"case": c, "pool": pool, "pages": pages, "lens": lens, "news": news, "n_pages": n_pages, "columns": columns,
         "len": torch.tensor(lens, dtype=torch.int32, device=dev), "new": torch.tensor(news, dtype=torch.int32, device=dev)}
    if c["path"] == "write":
        s["k"], s["v"] = rows(c["kv_heads"], 1.0, 1.0), rows(c["kv_heads"], 1.0, 0.3)
    else:  # what earlier steps left in the cache
        kc, vc, kp, vp = _fields(pool, c)
        for b, length in enumerate(lens):
            of = pages[b, :need[b]].long()
            for h in range(c["kv_heads"]):
                for codes, par, offset in ((kc, kp, 1.0), (vc, vp, 0.3)):
                    x = torch.randn((need[b], c["page"], d), generator=g, device=dev)
                    x = x * (0.5 + torch.rand(d, generator=g, device=dev)) + offset * torch.randn(d, generator=g, device=dev)
                    q, scale, low = _quantise(x.bfloat16(), c["group"])
                    codes[of, h] = _pack(q, codes is kc)
                    par[of, h] = torch.stack([scale, low], dim=-1)
    if c["path"] == "attn":
        s["q"] = rows(c["heads"], 1.5, 0.0)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B * c["heads"], n), device=dev)
    else:
        like = s["k"] if c["path"] == "write" else rows(c["kv_heads"], 0.0, 0.0)
        s["k_back"], s["v_back"] = torch.zeros_like(like), torch.zeros_like(like)
    if own:
        _handle(s)
    return s


def _handle(s):
    """what a program that uses the framework keeps beside its tensors: the cache's description, shapes, a workspace"""
    import paper_2604_12219_amd as P
    c = s["case"]
    s["P"] = P
    s["cache"] = P.Cache(H_kv=c["kv_heads"], d=c["d"], group=c["group"], page=c["page"], n_pages=s["n_pages"], max_pages=s["columns"])
    s["shape"] = P.Shape.of(s["q"] if c["path"] == "attn" else s["k_back"])
    if c["path"] == "attn":
        s["ws"] = torch.empty(P.cache_attn_workspace_bytes(s["shape"], s["cache"], c["length"]), dtype=torch.uint8, device="cuda")


def run(state):
    s, path = state, state["case"]["path"]
    if not own:
        return _run_plain(s)
    if "P" not in s:
        _handle(s)
    P, shape, cache = s["P"], s["shape"], s["cache"]
    where = (s["pool"], s["pages"], s["len"], s["new"])
    if path == "attn":
        return P.cache_attn(s["q"], shape, cache, *where, causal=s["case"]["causal"], n_max=s["case"]["length"], out=s["out"], lse=s["lse"],
                            ws=s["ws"], want_lse=True)
    if path == "write":
        P.cache_write(s["k"], s["v"], shape, cache, *where)
    return P.cache_read(shape, cache, *where, k=s["k_back"], v=s["v_back"])


def _run_plain(s):
    c, path = s["case"], s["case"]["path"]
    if path != "attn":
        b, row, page, slot = _places(s)
        kc, vc, kp, vp = _fields(s["pool"], c)
        if path == "write":
            for x, codes, par in ((s["k"], kc, kp), (s["v"], vc, vp)):
                q, scale, low = _quantise(x[b, :, row], c["group"])
                codes[page, :, slot] = _pack(q, codes is kc)
                par[page, :, slot] = torch.stack([scale, low], dim=-1)
        for back, codes, par in ((s["k_back"], kc, kp), (s["v_back"], vc, vp)):
            back[b, :, row] = _unpack(codes[page, :, slot], par[page, :, slot], codes is kc).bfloat16()
        return s["k_back"], s["v_back"]
    share, scale = c["heads"] // c["kv_heads"], c["d"] ** -0.5
    lse = s["lse"].view(c["batch"], c["heads"], c["n"])
    for b, (length, new) in enumerate(zip(s["lens"], s["news"])):
        if new == 0:
            continue
        k, v = _tokens(s, b)
        key = torch.arange(length, device=k.device)
        step = max(1, 2 ** 29 // (c["heads"] * length))
        for r in range(0, new, step):
            e = min(r + step, new)
            q = s["q"][b, :, r:e].float().unflatten(0, (-1, share)).flatten(1, 2)  # [kv_heads, share * rows, d]
            z = (q @ k.transpose(1, 2)) * scale
            if c["causal"]:
                last = (length - new + torch.arange(r, e, device=k.device)).repeat(share)
                z = z.masked_fill(key > last[:, None], -math.inf)
            top = z.amax(-1, keepdim=True)
            p = torch.exp(z - top)
            total = p.sum(-1, keepdim=True)
            s["out"][b, :, r:e] = ((p @ v) / total).unflatten(1, (share, -1)).flatten(0, 1).bfloat16()
            lse[b, :, r:e] = (top + torch.log(total)).squeeze(-1).unflatten(1, (share, -1)).flatten(0, 1)
    return s["out"], s["lse"]


def work(case):
    c = case
    lens, news = _lengths(c)
    rows, tokens = sum(news) * c["heads"], sum(lens) * c["kv_heads"]
    if c["path"] == "write":
        return {"bytes": rows * (8 * c["d"] + _token_bytes(c)), "flops": 16 * rows * c["d"]}
    if c["path"] == "read":
        return {"bytes": rows * (4 * c["d"] + _token_bytes(c)), "flops": 4 * rows * c["d"]}
    pairs = sum(new * length - (new * (new - 1) // 2 if c["causal"] else 0) for length, new in zip(lens, news)) * c["heads"]
    return {"bytes": tokens * _token_bytes(c) + rows * (4 * c["d"] + 4), "flops": 4 * pairs * c["d"]}


def exact(case, seed):
    """What run() returns, in 64 bits, from the definition of the cache and of attention."""
    c = case
    s = prepare(c, seed)
    dev, d, group, page = s["pool"].device, c["d"], c["group"], c["page"]
    ch = torch.arange(d, device=dev)
    groups, head_bytes = d // group, page * _token_bytes(c)

    def values(b, h, first, last, is_key):
        """tokens first..last-1 of sequence b, head h, straight from the bytes"""
        pos = torch.arange(first, last, device=dev)
        base = (s["pages"][b, pos // page].long() * c["kv_heads"] + h) * head_bytes
        slot = pos % page
        word = (ch % 32 // 8) * (d // 32) + ch // 32 if is_key else ch // 8
        at = base + slot * (d // 2) + (0 if is_key else page * d // 2)
        byte = s["pool"][at[:, None] + (4 * word + ch % 8 // 2)]
        code = torch.where(ch % 2 == 1, byte >> 4, byte & 15).double()
        at = base + page * d + (0 if is_key else page * groups * 4) + slot * (groups * 4)
        at = at[:, None] + 4 * (ch // group)

        def number(at):  # two bytes of a bf16
            return ((s["pool"][at].int() | (s["pool"][at + 1].int() << 8)) << 16).view(torch.float32).double()
        return number(at) * code + number(at + 2)

    def held(x):
        """what rows x [new, d] become"""
        out = torch.empty_like(x, dtype=torch.float64)
        for g in range(groups):
            part = x[:, g * group:(g + 1) * group].double()
            low, high = part.min(1, keepdim=True).values, part.max(1, keepdim=True).values
            scale = ((high - low) / 15).float().bfloat16().double()
            scale[scale < 2.0 ** -126] = 0
            code = torch.nan_to_num((part - low) / scale, nan=0.0, posinf=0.0).round().clamp(0, 15)
            out[:, g * group:(g + 1) * group] = scale * code + low
        return out

    if c["path"] != "attn":
        outs = []
        for is_key in (True, False):
            back = torch.zeros((c["batch"], c["kv_heads"], c["n"], d), dtype=torch.float64, device=dev)
            for b, (length, new) in enumerate(zip(s["lens"], s["news"])):
                for h in range(c["kv_heads"] if new else 0):
                    if c["path"] == "write":
                        back[b, h, :new] = held((s["k"] if is_key else s["v"])[b, h, :new])
                    else:
                        back[b, h, :new] = values(b, h, length - new, length, is_key)
            outs.append(back)
        return tuple(outs)
    out = torch.zeros((c["batch"], c["heads"], c["n"], d), dtype=torch.float64, device=dev)
    lse = torch.zeros((c["batch"], c["heads"], c["n"]), dtype=torch.float64, device=dev)
    share = c["heads"] // c["kv_heads"]
    for b, (length, new) in enumerate(zip(s["lens"], s["news"])):
        for h in range(c["kv_heads"] if new else 0):
            k, v = values(b, h, 0, length, True), values(b, h, 0, length, False)
            step = max(1, 2 ** 28 // length)
            for head in range(h * share, (h + 1) * share):
                for r in range(0, new, step):
                    e = min(r + step, new)
                    z = s["q"][b, head, r:e].double() @ k.T / math.sqrt(d)
                    if c["causal"]:
                        seen = length - new + torch.arange(r, e, device=dev)
                        z[torch.arange(length, device=dev)[None, :] > seen[:, None]] = -math.inf
                    lse[b, head, r:e] = torch.logsumexp(z, dim=1)
                    out[b, head, r:e] = torch.softmax(z, dim=1) @ v
    return out, lse.flatten(0, 1)
