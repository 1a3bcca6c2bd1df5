"""The operators that a server of topic-routed adapters runs in four bits, as cases that can be measured.

Such a server's memory goes to its adapters, so the base weights and the cache of keys and values are held in MXFP4: blocks
of 32 values of E2M1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives) that share a power of two 2^(E - 127).

``listed()`` names twelve cases, ``draw()`` gives more of the same ranges.  A case's ``kind`` says which operator it measures:

* ``tables``  block tables, slot maps and offsets of a step from the requests' lengths;
* ``append``  keys and values of new tokens into the paged cache, and the values that it then holds;
* ``attend``  attention of the step's tokens over the cache: single tokens, chunks behind a prefix, whole prompts;
* ``linear``  a product with 4-bit weights, with the adapters of the tokens' experts or without.

The cache holds, for a page and a kv head, ``page / 64`` records of 64 tokens x D channels, 68 D bytes each; token
``16 i + m`` of a record (i < 4, m < 16) has its
  keys     at [i][D / 32][m][16 bytes],   channels 32 b .. 32 b + 31 of block b, the even one of a pair in the low nibble,
  values   at [i][D / 8][m][4 bytes],     channels 8 c .. 8 c + 7 of word c, likewise,
  scales   at [D / 32][m][i], first all of the keys', then all of the values'.
A 4-bit weight [d_out, d_in] is held in records of 16 rows x 512 columns, 4352 bytes each, padded with zeros: row m, column
128 j + 32 g + c at byte [j][g][m][c / 2], then the scale bytes at [g][m][j].
"""
import math

import torch

own = False

BF16, F32 = torch.bfloat16, torch.float32
# d_in -> d_out of the projections of a 2048-wide layer, and of larger ones
PROJECTIONS = [(2048, 2048), (2048, 256), (2048, 5632), (5632, 2048), (1024, 1416), (2048, 2000), (1000, 2048), (4096, 4096),
               (8192, 8192)]
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ------------------------------------------------------------------------------------------

def listed():
    return [
        # A decode step of 64 requests: one new token each, few of which need a new page. All latency.
        dict(name="tables_decode", kind="tables", S=64, kv_lo=1, kv_hi=4096, new_lo=1, new_hi=1, page=64, max_pages=72, tight=False),
        # A step that admits many prompts of uneven length beside requests that are under way.
        dict(name="tables_prompts", kind="tables", S=1000, kv_lo=0, kv_hi=2000, new_lo=0, new_hi=700, page=64, max_pages=64,
             tight=False),
        # The decode batch of 256 tokens, four kv heads of 64: what every layer adds in a step.
        dict(name="append_decode", kind="append", T=256, H=4, D=64, page=64),
        # A prefill batch of 32 x 2048 tokens, eight kv heads of 128.
        dict(name="append_prompts", kind="append", T=65536, H=8, D=128, page=128),
        # One user at a thousand tokens: the latency of a single request's step.
        dict(name="attend_one", kind="attend", S=1, kv_lo=1000, kv_hi=1000, new_lo=1, new_hi=1, heads=32, H=4, D=64, page=64, window=0,
             y="bf16"),
        # A full decode batch at uneven lengths.
        dict(name="attend_batch", kind="attend", S=256, kv_lo=64, kv_hi=4096, new_lo=1, new_hi=1, heads=32, H=4, D=64, page=64,
             window=0, y="bf16"),
        # Two users with very long documents behind them, wider heads: few rows, a long axis.
        dict(name="attend_long", kind="attend", S=2, kv_lo=99999, kv_hi=131072, new_lo=1, new_hi=1, heads=64, H=8, D=128, page=128,
             window=0, y="f32"),
        # Eight prompts of 2048 tokens, nothing cached before.
        dict(name="attend_prompts", kind="attend", S=8, kv_lo=0, kv_hi=0, new_lo=2048, new_hi=2048, heads=32, H=4, D=64, page=64,
             window=0, y="bf16"),
        # Chunks of prompts behind long prefixes, a head of keys for each of queries, a sliding window.
        dict(name="attend_chunks", kind="attend", S=4, kv_lo=1500, kv_hi=8000, new_lo=400, new_hi=512, heads=16, H=16, D=128, page=64,
             window=4096, y="bf16"),
        # One token through an up projection: the smallest product.
        dict(name="linear_one", kind="linear", T=1, d_in=2048, d_out=5632, r=0, E=0, y="bf16"),
        # A few tokens through a large projection: the weights' bytes are what counts.
        dict(name="linear_large", kind="linear", T=24, d_in=8192, d_out=28672, r=0, E=0, y="f32"),
        # A decode batch of 256 requests, each with its own rank-128 adapter.
        dict(name="linear_adapters", kind="linear", T=256, d_in=2048, d_out=5632, r=128, E=2000, y="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tables", "append", "attend", "attend", "attend", "linear", "linear"])
    if kind == "tables":
        S, page = _log(rng, 1, 4000), rng.choice([64, 128, 256])
        kv, new = rng.choice([0, _log(rng, 1, 5000)]), min(350000 // S, rng.choice([1, 1, _log(rng, 1, 700)]))
        return dict(kind=kind, S=S, kv_lo=kv // 20, kv_hi=kv, new_lo=rng.choice([0, new]), new_hi=new, page=page,
                    max_pages=(kv + new) // page + rng.randint(1, 9), tight=rng.random() < 0.2)
    if kind == "append":
        H, D = rng.choice([(4, 64), (8, 128), (1, 64), (2, 256), (5, 128)])
        return dict(kind=kind, T=_log(rng, 1, 32768), H=H, D=D, page=rng.choice([64, 128, 256]))
    if kind == "attend":
        heads, H, D = rng.choice([(32, 4, 64), (32, 4, 64), (64, 8, 128), (16, 16, 128), (12, 4, 64), (7, 1, 64), (8, 2, 256)])
        page, window = rng.choice([64, 64, 128, 256]), rng.choice([0, 0, 0, _log(rng, 1, 5000)])
        y = rng.choice(["bf16", "bf16", "f32"])
        form = rng.choice(["one", "one", "few", "prompt", "mixed"])
        if form == "one":     # single tokens: about the same cache in all, many requests or long ones
            S = _log(rng, 1, 300)
            kv = _log(rng, 16, min(131072, (1 << 24) // (S * H * D // 16)))
            return dict(kind=kind, S=S, kv_lo=kv // rng.choice([1, 2, 50]), kv_hi=kv, new_lo=1, new_hi=1, heads=heads, H=H, D=D,
                        page=page, window=window, y=y)
        if form == "few":     # a handful of tokens each, as a draft's checks take
            S, new = _log(rng, 1, 64), rng.randint(2, 9)
            kv = _log(rng, 16, min(32768, (1 << 23) // (S * H * D // 16)))
            return dict(kind=kind, S=S, kv_lo=kv // rng.choice([1, 3]), kv_hi=kv, new_lo=rng.choice([0, new]), new_hi=new, heads=heads,
                        H=H, D=D, page=page, window=window, y=y)
        S, new = _log(rng, 1, 12), _log(rng, 10, 1500)
        kv = rng.choice([0, _log(rng, 1, 4000)])
        while S * new * (kv + new) * heads * D > 1 << 35:   # (the listed prompts: twice that, half of it masked)
            S, new = (S + 1) // 2, (new + 1) // 2
        return dict(kind=kind, S=S, kv_lo=kv // 3, kv_hi=kv, new_lo=1 if form == "mixed" else new, new_hi=new, heads=heads, H=H, D=D,
                    page=page, window=window, y=y)
    d_in, d_out = rng.choice(PROJECTIONS)
    r = rng.choice([0, 0, 16, 64, 128])
    return dict(kind=kind, T=_log(rng, 1, min(1024, (1 << 34) // (d_in * d_out))), d_in=d_in, d_out=d_out, r=r, E=_log(rng, 8, 400) if r else 0,
                y=rng.choice(["bf16", "bf16", "f32"]))


# ---- lengths: a property of the case, the same for every seed -------------------------------------------

def _lens(c):
    """Tokens that each request has in the cache before the step, and tokens that the step adds."""
    g = torch.Generator()
    g.manual_seed(c["S"] * 1009 + c["kv_hi"] * 31 + c["new_hi"])

    def some(lo, hi):
        return torch.randint(lo, hi + 1, (c["S"],), generator=g).to(torch.int32)

    kv, new = some(c["kv_lo"], c["kv_hi"]), some(c["new_lo"], c["new_hi"])
    if int(new.sum()) == 0:
        new[0] = 1
    return kv, new


def _ceil(a, b):
    return (a + b - 1) // b


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _normal(g, shape, std=1.0, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _to_codes(v):
    """Codes and scale bytes of [..., 32] fp32 blocks."""
    bits = v.abs().amax(-1, keepdim=True).view(torch.int32)
    E = (((bits + 0x200000) >> 23) - 2).clamp(min=2)
    E = torch.where(bits == 0, 127, torch.where(bits >= 0x7F800000, 255, E))
    a = v.abs() * ((254 - E).clamp(min=1) << 23).view(F32)
    # midpoints between neighbours: those above an even code go down, those above an odd one up
    c = sum((a > m).to(torch.uint8) for m in (0.25, 1.25, 2.5, 5.0)) + sum((a >= m).to(torch.uint8) for m in (0.75, 1.75, 3.5))
    return c + (v < 0).to(torch.uint8) * 8, E.squeeze(-1).to(torch.uint8)


def _from_codes(c, E):
    """fp32 values of codes [..., n] with scale bytes [..., 1] or wider."""
    a = (c & 7).to(F32)
    mag = torch.where(a < 4, a * 0.5, torch.where(a < 6, a - 2.0, a * 2.0 - 8.0))
    return torch.where(c >= 8, -mag, mag) * torch.exp2(E.to(F32) - 127.0)


def _keys_like(g, shape):
    """bf16 keys or values as a projection gives them: channels of uneven strength, some with an offset."""
    D = shape[-1]
    strength = torch.exp(0.5 * _normal(g, shape[-2:], dtype=F32))
    offset = _normal(g, shape[-2:], dtype=F32) * (torch.arange(D, device="cuda") % 7 == 0)
    return (_normal(g, shape, dtype=F32) * strength + offset).to(BF16)


def _pairs(c):
    """Bytes of codes [..., 2 n]: the even one of a pair in the low nibble."""
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _records(k, v):
    """[n, 64, H, D] keys and values as records [n, H, 68 D]."""
    n, _, H, D = k.shape

    def coded(x):
        c, E = _to_codes(x.to(F32).view(n, 4, 16, H, D // 32, 32))
        return c, E.permute(0, 3, 4, 2, 1).reshape(n, H, 2 * D)    # [b][m][i]

    (ck, Ek), (cv, Ev) = coded(k), coded(v)
    bk = _pairs(ck).permute(0, 3, 1, 4, 2, 5).reshape(n, H, 32 * D)
    bv = _pairs(cv.reshape(n, 4, 16, H, D // 8, 8)).permute(0, 3, 1, 4, 2, 5).reshape(n, H, 32 * D)
    return torch.cat([bk, bv, Ek, Ev], -1)


def _weight(W):
    """A bf16 weight [d_out, d_in] as records [row tiles, column tiles, 4352]."""
    d_out, d_in = W.shape
    R, C = _ceil(d_out, 16), _ceil(d_in, 512)
    full = torch.zeros((R * 16, C * 512), dtype=F32, device=W.device)
    full[:d_out, :d_in] = W
    c, E = _to_codes(full.view(R, 16, C, 4, 4, 32))                # [R][m][C][j][g][32]
    b = _pairs(c).permute(0, 2, 3, 4, 1, 5).reshape(R, C, 4096)
    return torch.cat([b, E.permute(0, 2, 4, 1, 3).reshape(R, C, 256)], -1)


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if c["kind"] in ("tables", "attend"):
        kv, new = _lens(c)
        P = c["page"]
        have, all_ = _ceil(kv, P), _ceil(kv + new, P)
        max_pages = c.get("max_pages") or int(all_.max()) + 1
        held, total = int(have.sum()), int(all_.sum())
        # pages of a pool that has been in use: in no order.  The requests hold the first, the rest is free
        n_pages = total + 3 if not c.get("tight") else held + (total - held) * 2 // 3
        order = torch.randperm(max(n_pages, 1), generator=_gen(seed, "cpu")).to(torch.int32)
        grid = torch.arange(max_pages)
        table = torch.full((c["S"], max_pages), -1, dtype=torch.int32)
        table[grid < have[:, None]] = order[:held]
        st.update(T=int(new.sum()), max_new=int(new.max()), n_pages=max(n_pages, 1), kv=kv.cuda(), new=new.cuda())
        if c["kind"] == "tables":
            st.update(free=order[held:].cuda() if n_pages > held else torch.zeros(1, dtype=torch.int32, device="cuda"),
                      n_free=torch.tensor([n_pages - held], dtype=torch.int32, device="cuda"), table=table.cuda())
            if own:   # the step's plan, kept by the server
                from paper_2410_09687_amd import moin
                st["ctx"] = moin.Context(torch.cuda.current_device())
                st["plan"] = moin.KVPlan(st["ctx"])
            return st
        before = dict(kv=st["kv"], new=st["new"], table=table.cuda(), free=order[held:].cuda(),
                      n_free=torch.tensor([n_pages - held], dtype=torch.int32, device="cuda"))
        table[(grid >= have[:, None]) & (grid < all_[:, None])] = order[held:total]
        H, D, B = c["H"], c["D"], P // 64
        # what the pool held before stays in the tokens beyond a request's end
        data = torch.randint(0, 256, (st["n_pages"], H, B, 68 * D), dtype=torch.uint8, device="cuda", generator=g)
        used = order[:total].long().cuda()
        step = max(1, (1 << 27) // (P * H * D))
        for lo in range(0, total, step):
            n = min(total, lo + step) - lo
            rec = _records(_keys_like(g, (n * B, 64, H, D)), _keys_like(g, (n * B, 64, H, D)))
            data[used[lo:lo + n]] = rec.view(n, B, H, 68 * D).transpose(1, 2)
        # tokens of the last pages that no request has reached: scale bytes that stand for NaN
        tail = data.view(st["n_pages"], H, B, 68 * D)[..., 64 * D:].view(st["n_pages"], H, B, D // 16, 16, 4)
        end, last = (kv + new), table[torch.arange(c["S"]), (all_ - 1).clamp(min=0)].long()
        tok = torch.arange(P).view(B, 4, 16)
        beyond = ((all_ - 1) * P)[:, None, None, None] + tok >= end[:, None, None, None]
        beyond = beyond & (all_ > 0)[:, None, None, None]
        mask = torch.zeros((st["n_pages"], B, 4, 16), dtype=torch.bool)
        mask[last.clamp(min=0)] |= beyond
        tail.masked_fill_(mask.permute(0, 1, 3, 2).cuda()[:, None, :, None], 255)
        off = torch.zeros(c["S"] + 1, dtype=torch.int32)
        off[1:] = new.cumsum(0)
        st.update(data=data, table=table.cuda(), off=off.cuda(), len=end.to(torch.int32).cuda(), max_len=int(end.max()),
                  q=_normal(g, (st["T"], c["heads"], D)))
        if own:   # the step's plan: one for all layers
            from paper_2410_09687_amd import moin
            st["ctx"] = moin.Context(torch.cuda.current_device())
            st["pages"] = moin.KVPages(data, H, D, P)
            st["plan"] = moin.KVPlan(st["ctx"])
            # (the pages were dealt in this order above, so the plan deals them as the table has them)
            free = before["free"].clone()
            free[:total - held] = before["free"][:total - held].flip(0)
            k = total - held
            stack = torch.cat([before["free"][k:], free[:k]])
            st["plan"].build(before["kv"], before["new"], st["T"], before["table"], stack, before["n_free"], n_pages=st["n_pages"],
                             page_tokens=P, n_heads=c["heads"], n_kv=H, max_new=st["max_new"])
        return st
    if c["kind"] == "append":
        T, H, D, P = c["T"], c["H"], c["D"], c["page"]
        n_pages = _ceil(T, P) + 2
        order = torch.randperm(n_pages, generator=_gen(seed, "cpu")).cuda()
        t = torch.arange(T, device="cuda") + P // 3     # a run of requests' tokens that begins and ends inside pages
        st["slots"] = (order[t // P] * P + t % P).to(torch.int32)
        # q, k and v of a token are one row of the projections' output
        st["kv"] = torch.cat([_keys_like(g, (T, H, D)), _keys_like(g, (T, H, D))], 1)
        st["data"] = torch.randint(0, 256, (n_pages, H, P // 64, 68 * D), dtype=torch.uint8, device="cuda", generator=g)
        if own:
            from paper_2410_09687_amd import moin
            st["ctx"] = moin.Context(torch.cuda.current_device())
            st["pages"] = moin.KVPages(st["data"], H, D, P)
        return st
    T, d_in, d_out, r, E = c["T"], c["d_in"], c["d_out"], c["r"], c["E"]
    st["x"] = _normal(g, (T, d_in))
    st["W"] = _weight(_normal(g, (d_out, d_in), d_in ** -0.5))
    if r:
        p = torch.arange(1, E + 1, dtype=torch.float64) ** -1.1     # few experts serve most requests
        ids = torch.multinomial(p, T, replacement=True, generator=_gen(seed, "cpu"))
        st["ids"] = torch.randperm(E, generator=_gen(seed + 1, "cpu"))[ids].to(torch.int32).cuda()
        st["A"], st["B"] = _normal(g, (E, r, d_in), d_in ** -0.5), _normal(g, (E, d_out, r), r ** -0.5)
    if own:
        from paper_2410_09687_amd import moin
        st["ctx"] = moin.Context(torch.cuda.current_device())
        st["w4"] = moin.MX4Weight(st["W"], d_out, d_in)
        if r:   # the batch's grouping: one for all projections of all layers
            st["plan"] = moin.Plan(st["ctx"])
            st["plan"].build(torch.arange(T + 1, dtype=torch.int32, device="cuda"), st["ids"], T, E)
    return st


# ---- one pass -------------------------------------------------------------------------------------------

SCALE = 2.0     # of the adapters, as everywhere here


def _dtype(c):
    return BF16 if c["y"] == "bf16" else F32


def run(st):
    c = st["case"]
    if own:
        return _run_own(c, st)
    return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend, "linear": _plain_linear}[c["kind"]](c, st)


def _run_own(c, st):
    from paper_2410_09687_amd import moin
    ctx = st["ctx"]
    if c["kind"] == "tables":
        off, lens, slots, n_free = st["plan"].build(st["kv"], st["new"], st["T"], st["table"], st["free"], st["n_free"],
                                                    n_pages=st["n_pages"], page_tokens=c["page"], n_heads=32, n_kv=4,
                                                    max_new=st["max_new"])
        return dict(table=st["table"], offsets=off, lens=lens, slots=slots, n_free=n_free)
    if c["kind"] == "append":
        H = c["H"]
        moin.moin_kv_append(ctx, st["pages"], st["kv"][:, :H], st["kv"][:, H:], st["slots"])
        k, v = moin.moin_kv_gather(ctx, st["pages"], st["slots"])
        return dict(k=k, v=v)
    if c["kind"] == "attend":
        y, lse = moin.moin_kv_attention(ctx, st["plan"], st["pages"], st["q"], st["table"], window=c["window"], y_dtype=_dtype(c),
                                        want_lse=True)
        return dict(y=y, lse=lse)
    if c["r"]:
        return moin.moin_lora_linear_mx4_planned(ctx, st["plan"], st["x"], st["w4"], st["A"], st["B"], SCALE, y_dtype=_dtype(c))
    return moin.moin_mx4_linear(ctx, st["x"], st["w4"], y_dtype=_dtype(c))


def _plain_tables(c, st):
    P, kv, new, T, max_pages = c["page"], st["kv"].long(), st["new"].long(), st["T"], c["max_pages"]
    n_free = st["n_free"].long()
    have, all_ = _ceil(kv, P), _ceil(kv + new, P)
    fits = all_ <= max_pages
    need = torch.where(fits, all_ - have, 0)
    upto = need.cumsum(0)
    served = fits & ((need == 0) | (upto <= n_free))      # all of a request's pages, or none
    base = upto - need
    off = torch.nn.functional.pad(new.cumsum(0), (1, 0))
    j = torch.arange(max_pages, device=kv.device) - have[:, None]
    at = (n_free - 1 - (base[:, None] + j)).clamp(0, st["free"].numel() - 1)
    table = torch.where(served[:, None] & (j >= 0) & (j < need[:, None]), st["free"][at], st["table"])
    t = torch.arange(T, device=kv.device)
    s = torch.searchsorted(off[1:], t, right=True)
    pos = kv[s] + t - off[s]
    page = table[s, (pos // P).clamp(max=max_pages - 1)].long()
    slots = torch.where(served[s], page * P + pos % P, -1)
    i32 = torch.int32
    return dict(table=table, offsets=off.to(i32), lens=torch.where(served, kv + new, kv).to(i32), slots=slots.to(i32),
                n_free=(n_free - torch.where(served, need, 0).sum()).to(i32))


def _plain_append(c, st):
    T, H, D = c["T"], c["H"], c["D"]
    codes, E = _to_codes(st["kv"].to(F32).view(T, 2 * H, D // 32, 32))
    held = _from_codes(codes, E[..., None]).view(T, 2 * H, D).to(BF16)
    return dict(k=held[:, :H], v=held[:, H:])


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _cached(st, c, nb):
    """Keys and values [S, H, 64 nb, D] in fp32 that the requests' first nb records hold."""
    S, H, D, B = c["S"], c["H"], c["D"], c["page"] // 64
    blk = torch.arange(nb, device="cuda")
    page = st["table"][:, blk // B].long().clamp(min=0)
    rec = st["data"][page, :, blk % B]                                        # [S, nb, H, 68 D]
    E = rec[..., 64 * D:].view(S, nb, H, 2, D // 32, 16, 4).permute(3, 0, 2, 1, 6, 5, 4)[..., None]   # [2][S][H][nb][i][m][b][1]
    ck = _nibbles(rec[..., :32 * D].reshape(S, nb, H, 4, D // 32, 16, 16)).permute(0, 2, 1, 3, 5, 4, 6)
    k = _from_codes(ck, E[0]).reshape(S, H, nb * 64, D)
    cv = _nibbles(rec[..., 32 * D:64 * D].reshape(S, nb, H, 4, D // 8, 16, 4)).permute(0, 2, 1, 3, 5, 4, 6)
    v = _from_codes(cv.reshape(S, H, nb, 4, 16, D // 32, 32), E[1]).reshape(S, H, nb * 64, D)
    return k, v


def _plain_attend(c, st):
    S, H, D, n, T = c["S"], c["H"], c["D"], st["max_new"], st["T"]
    G = c["heads"] // H
    k, v = _cached(st, c, _ceil(st["max_len"], 64))
    L = k.shape[2]
    off, lens = st["off"].long(), st["len"].long()
    new = off[1:] - off[:-1]
    row = torch.arange(n, device="cuda")
    tok = (off[:-1, None] + row).clamp(max=T - 1)                              # [S, n]
    q = st["q"][tok].to(F32).view(S, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, n * G, D)
    key = torch.arange(L, device="cuda")
    held = key < lens[:, None]
    k, v = (torch.where(held[:, None, :, None], x, 0.0) for x in (k, v))       # no key is read beyond a request's end
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
    pos = (lens - new)[:, None] + row                                          # [S, n]
    seen = (key <= pos[..., None]) & (pos[..., None] >= 0)
    if c["window"]:
        seen = seen & (key > pos[..., None] - c["window"])
    s = s.view(S, H, n, G, L).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = (s - torch.where(m == -math.inf, 0.0, m)).exp_()
    sums = p.sum(-1, keepdim=True)
    y = torch.matmul(p.view(S, H, n * G, L), v).view(S, H, n, G, D) / torch.where(sums == 0, 1.0, sums)
    lse = (m + sums.log()).squeeze(-1)
    real = row < new[:, None]                                                  # [S, n], in the order of the tokens
    return dict(y=y.permute(0, 2, 1, 3, 4).reshape(S, n, H * G, D)[real].to(_dtype(c)),
                lse=lse.permute(0, 2, 1, 3).reshape(S, n, H * G)[real])


def _plain_linear(c, st):
    x, T = st["x"].to(F32), c["T"]
    rec = st["W"]
    R, C = rec.shape[:2]
    codes = _nibbles(rec[..., :4096].reshape(R, C, 4, 4, 16, 16))              # [R][C][j][g][m][32]
    E = rec[..., 4096:].view(R, C, 4, 16, 4).permute(0, 1, 4, 2, 3)[..., None]
    W = _from_codes(codes, E).permute(0, 4, 1, 2, 3, 5).reshape(R * 16, C * 512)[:c["d_out"], :c["d_in"]]
    y = x @ W.t()
    if c["r"]:
        A, B = st["A"], st["B"]
        used, at = torch.unique(st["ids"].long(), return_inverse=True)
        # the tokens of each adapter side by side, padded to the most that one has
        order = at.argsort(stable=True)
        count = torch.bincount(at, minlength=used.numel())
        place = torch.arange(T, device="cuda") - (count.cumsum(0) - count)[at[order]]
        xs = torch.zeros((used.numel(), int(count.max()), c["d_in"]), dtype=F32, device="cuda")
        xs[at[order], place] = x[order]
        u = torch.bmm(xs, A[used].to(F32).transpose(1, 2).contiguous())
        z = torch.bmm(u, B[used].to(F32).transpose(1, 2).contiguous())
        y[order] += SCALE * z[at[order], place]
    return y.to(_dtype(c))


# ---- from the definitions, in 64 bits -------------------------------------------------------------------

F64 = torch.float64


def _level(code):
    mag = torch.tensor(LEVELS, dtype=F64, device=code.device)[(code & 7).long()]
    return torch.where(code > 7, -mag, mag)


def _power(E):
    p = torch.ldexp(torch.ones_like(E, dtype=F64), E.to(torch.int32) - 127)
    return torch.where(E == 255, math.nan, p)


def exact(case, seed):
    c = case
    if c["kind"] == "tables":
        return None
    st = _plain_state(case, seed)
    if c["kind"] == "append":
        T, H, D = c["T"], c["H"], c["D"]
        x = st["kv"].to(F64).view(T * 2 * H * D // 32, 32)
        top = x.abs().amax(1)
        # the smallest power of two in whose units the block's largest value rounds to 6 or less
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -200))) - 2
        e = torch.where(top / torch.exp2(e) >= 7, e + 1, e).clamp(min=-125)
        unit = torch.exp2(e)[:, None]
        lv = torch.tensor(LEVELS, dtype=F64, device="cuda")
        far = (x.abs() / unit)[..., None] - lv                                  # distance to every level
        far = far.abs() - torch.tensor([1e-12, 0, 1e-12, 0, 1e-12, 0, 1e-12, 0], dtype=F64, device="cuda")   # ties: the even code
        held = (lv[far.argmin(-1)] * unit * x.sign()).view(T, 2 * H, D)
        return dict(k=held[:, :H], v=held[:, H:])
    if c["kind"] == "linear":
        d_in, d_out = c["d_in"], c["d_out"]
        b = st["W"][..., :4096]
        R, C = b.shape[:2]
        W = torch.empty((R, 16, C, 4, 4, 16, 2), dtype=F64, device="cuda")
        for nib in range(2):
            W[..., nib] = _level((b >> (4 * nib)) & 15).view(R, C, 4, 4, 16, 16).permute(0, 4, 1, 2, 3, 5)
        E = _power(st["W"][..., 4096:]).view(R, C, 4, 16, 4)
        W *= E.permute(0, 3, 1, 4, 2)[..., None, None]
        W = W.view(R * 16, C * 512)[:d_out, :d_in]
        x = st["x"].to(F64)
        y = x @ W.t()
        if c["r"]:
            for e in st["ids"].unique().tolist():
                rows = (st["ids"] == e).nonzero().squeeze(1)
                y[rows] += SCALE * (x[rows] @ st["A"][e].to(F64).t() @ st["B"][e].to(F64).t())
        return y
    H, D, P, G = c["H"], c["D"], c["page"], c["heads"] // c["H"]
    y = torch.zeros((st["T"], c["heads"], D), dtype=F64, device="cuda")
    lse = torch.full((st["T"], c["heads"]), -math.inf, dtype=F64, device="cuda")
    off, lens, table = st["off"].tolist(), st["len"].tolist(), st["table"].tolist()
    t64 = torch.arange(64, device="cuda")
    i, m = t64 // 16, t64 % 16
    for s in range(c["S"]):
        n, L = off[s + 1] - off[s], lens[s]
        if not n or not L:
            continue
        pages = torch.tensor(table[s][:_ceil(L, P)], device="cuda")
        rec = st["data"][pages].transpose(1, 2).reshape(-1, H, 68 * D)          # [records][H][bytes]
        N = rec.shape[0]
        kb = rec[..., :32 * D].reshape(N, H, 4, D // 32, 16, 16)[:, :, i, :, m]         # [64][N][H][D / 32][16]
        vb = rec[..., 32 * D:64 * D].reshape(N, H, 4, D // 8, 16, 4)[:, :, i, :, m]     # [64][N][H][D / 8][4]
        sb = rec[..., 64 * D:].reshape(N, H, 2, D // 32, 16, 4)[..., m, i]              # [N][H][2][D / 32][64]

        def values(b, E):
            x = torch.stack([_level(b & 15), _level(b >> 4)], -1).reshape(64, N, H, D // 32, 32)
            x = x * _power(E).permute(3, 0, 1, 2)[..., None]
            return x.reshape(64, N, H, D).permute(2, 1, 0, 3).reshape(H, N * 64, D)[:, :L]

        k, v = values(kb, sb[:, :, 0]), values(vb, sb[:, :, 1])
        pos = L - n + torch.arange(n, device="cuda")
        lo, hi = (pos - c["window"] + 1 if c["window"] else pos * 0).clamp(min=0), pos + 1
        key = torch.arange(L, device="cuda")
        out = (key < lo[:, None]) | (key >= hi[:, None])                        # [n, L]
        for h in range(H):
            q = st["q"][off[s]:off[s + 1], h * G:(h + 1) * G].to(F64)           # [n, G, D]
            z = (q.reshape(n * G, D) @ k[h].t().contiguous()).view(n, G, L) / math.sqrt(D)
            z.masked_fill_(out[:, None], -math.inf)
            a = torch.logsumexp(z, -1)
            w = torch.where(a[..., None] == -math.inf, 0.0, (z - a[..., None]).exp())
            lse[off[s]:off[s + 1], h * G:(h + 1) * G] = a
            y[off[s]:off[s + 1], h * G:(h + 1) * G] = (w.view(n * G, L) @ v[h]).view(n, G, D)
    return dict(y=y, lse=lse)


def _plain_state(case, seed):
    """The inputs alone, without the framework's handles."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


# ---- what a pass cannot do without ----------------------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "tables":
        kv, new = _lens(c)
        pages = int((_ceil(kv + new, c["page"]) - _ceil(kv, c["page"])).sum())
        return dict(bytes=4.0 * (2 * c["S"] + 2 * pages + 3 * c["S"] + 2 + int(new.sum())), flops=0.0)
    if c["kind"] == "append":
        n = 2.0 * c["T"] * c["H"] * c["D"]
        return dict(bytes=n * (2 + 17 / 32 + 2) + 4 * c["T"], flops=0.0)
    if c["kind"] == "attend":
        kv, new = _lens(c)
        pairs, keys = 0.0, 0
        for L0, n in zip(kv.tolist(), new.tolist()):
            if not n:
                continue
            L, w = L0 + n, c["window"]
            keys += min(L, n + w - 1) if w else L
            if not w or w >= L:
                pairs += n * L0 + n * (n + 1) / 2
            else:
                pairs += sum(min(w, L0 + i + 1) for i in range(n))
        T = int(new.sum())
        return dict(bytes=keys * c["H"] * c["D"] * 2 * 17 / 32 + T * c["heads"] * (c["D"] * (2 + (2 if c["y"] == "bf16" else 4)) + 4),
                    flops=4.0 * pairs * c["heads"] * c["D"])
    T, d_in, d_out, r = c["T"], c["d_in"], c["d_out"], c["r"]
    b = d_in * d_out * 17 / 32 + T * (2 * d_in + (2 if c["y"] == "bf16" else 4) * d_out)
    f = 2.0 * T * d_in * d_out
    if r:
        p = torch.arange(1, c["E"] + 1, dtype=torch.float64) ** -1.1
        distinct = float((1 - (1 - p / p.sum()) ** T).sum())
        b += 2 * distinct * r * (d_in + d_out)
        f += 2.0 * T * r * (d_in + d_out)
    return dict(bytes=b, flops=f)
