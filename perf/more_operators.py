"""The operators that a server of topic-routed adapters runs in eight bits, as cases that can be measured.

Where four bits lose too much, base weights are held as 8-bit integers with a scale for each output channel, and keys and values
as E4M3 with a power of two 2^(E - 127) for each block of 64 tokens and head.

``listed()`` names twelve cases, ``draw()`` gives more of the same ranges.  A case's ``kind`` says which operator it measures:

* ``rotate``  norms of queries and keys for each head and the rotation by their positions, in one pass;
* ``append``  keys and values of new tokens into the paged cache, and what the blocks that they touch hold afterwards;
* ``attend``  attention of the step's tokens over the cache: single tokens, chunks behind a prefix, whole prompts;
* ``linear``  a product in 8-bit integers, with the adapters of the tokens' experts or without.

The cache holds, for a page and a kv head, ``page / 64`` records of 64 tokens x D channels, 128 D bytes each:
  keys    channel 64 l + c of token 16 i + m at byte [i][l][m][c]                                   (i < 4, m < 16, c < 64),
  values  channel 16 j + m of token 32 h + 16 u + 4 g + e at byte [j][m][g][h][u][e], from byte 64 D on,
then, behind a page's records, the bytes E: [kv heads][page / 64][2], the keys' and the values', padded to a multiple of 128.
A block's E is the largest that its tokens have asked for: the smallest, 10 to 246, in whose unit the largest magnitude is below 464.
Tokens that the block held before are rounded again where E grows.
An integer weight [d_out, d_in] is held as rows of codes padded with zeros to a multiple of 128 bytes, 256 at least, with a
scale of fp32 for each row: s = max(amax / 127, 2^-126), code = x / s to the nearest.  So are the tokens, by the call itself.
"""
import math

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
E4M3 = torch.float8_e4m3fn
EPS = 1e-6       # of the norms
THETA = 10000.0  # of the rotation
SCALE = 2.0      # of the adapters, as everywhere here
# d_in -> d_out of the projections of a 2048-wide layer, and of larger and odd ones
PROJECTIONS = [(2048, 2048), (2048, 256), (2048, 5632), (5632, 2048), (1024, 1416), (2048, 2000), (1000, 2048), (4096, 4096),
               (8192, 8192)]


# ---- the cases ------------------------------------------------------------------------------------------

def listed():
    return [
        # One user's token: all latency.
        dict(name="rotate_one", kind="rotate", T=1, heads=32, H=4, D=64, rot=64, pairs="halves", norm=True, x="bf16", pos_hi=4096),
        # A prefill batch of 8 x 2048 tokens, heads of 128 channels.
        dict(name="rotate_prompts", kind="rotate", T=16384, heads=32, H=8, D=128, rot=128, pairs="halves", norm=True, x="bf16",
             pos_hi=131072),
        # The decode batch of 256 tokens, four kv heads of 64: what every layer adds in a step, into blocks begun before.
        dict(name="append_decode", kind="append", S=256, kv_lo=1, kv_hi=4096, new_lo=1, new_hi=1, H=4, D=64, page=64),
        # A prefill batch of 32 x 2048 tokens, eight kv heads of 128, behind prefixes that end inside a block.
        dict(name="append_prompts", kind="append", S=32, kv_lo=0, kv_hi=100, new_lo=2048, new_hi=2048, H=8, D=128, page=128),
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
        # One token through an up projection: the smallest product.
        dict(name="linear_one", kind="linear", S=1, len_lo=1, len_hi=1, d_in=2048, d_out=5632, r=0, E=0, y="bf16"),
        # A few tokens through a large projection: the weights' bytes are what counts.
        dict(name="linear_large", kind="linear", S=24, len_lo=1, len_hi=1, d_in=8192, d_out=28672, r=0, E=0, y="f32"),
        # A decode batch of 256 requests, each with the rank-128 adapter of its own topic.
        dict(name="linear_adapters", kind="linear", S=256, len_lo=1, len_hi=1, d_in=2048, d_out=5632, r=128, E=2000, y="bf16"),
        # Prompts of uneven length through an up projection with their adapters: the matrix cores are what counts.
        dict(name="linear_prompts", kind="linear", S=32, len_lo=300, len_hi=700, d_in=2048, d_out=5632, r=64, E=500, y="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "attend", "attend", "linear", "linear"])
    if kind == "rotate":
        heads, H, D = rng.choice([(32, 4, 64), (32, 8, 128), (16, 16, 128), (7, 1, 64), (8, 2, 256), (5, 5, 128)])
        return dict(kind=kind, T=_log(rng, 1, 16384 * 40 * 128 // ((heads + H) * D)), heads=heads, H=H, D=D, rot=rng.choice([D, D, D // 2, 32]),
                    pairs=rng.choice(["halves", "neighbours"]), norm=rng.random() < 0.8, x=rng.choice(["bf16", "bf16", "f32"]),
                    pos_hi=_log(rng, 10, 1000000))
    if kind == "append":
        H, D = rng.choice([(4, 64), (8, 128), (1, 64), (2, 256), (5, 128)])
        S = _log(rng, 1, 600)
        new = rng.choice([1, 1, _log(rng, 2, 70), min(4000, 32768 // S + 1)])
        return dict(kind=kind, S=S, kv_lo=0, kv_hi=rng.choice([0, _log(rng, 1, min(4000, 300000 // S + 1))]), new_lo=rng.choice([0, new]), new_hi=new, H=H,
                    D=D, page=rng.choice([64, 128, 256]))
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
    r = rng.choice([0, 0, 64, 128])
    most = (1 << 36) // (d_in * d_out)
    if rng.random() < 0.6:    # single tokens
        S, lo, hi = _log(rng, 1, min(1000, most)), 1, 1
    else:
        hi = _log(rng, 2, min(2000, most))
        S, lo = _log(rng, 1, max(1, min(64, most // hi))), rng.choice([hi, 1 + hi // 3])
    return dict(kind=kind, S=S, len_lo=lo, len_hi=hi, d_in=d_in, d_out=d_out, r=r, E=_log(rng, 8, 400) if r else 0,
                y=rng.choice(["bf16", "bf16", "f32"]))


# ---- lengths: a property of the case, the same for every seed -------------------------------------------

def _some(c, lo, hi, salt):
    g = torch.Generator()
    g.manual_seed(c["S"] * 1009 + lo * 101 + hi * 31 + salt)
    return torch.randint(lo, hi + 1, (c["S"],), generator=g).to(I32)


def _lens(c):
    """Tokens that each request has in the cache before the step, and tokens that the step adds."""
    kv, new = _some(c, c["kv_lo"], c["kv_hi"], 1), _some(c, c["new_lo"], c["new_hi"], 2)
    if int(new.sum()) == 0:
        new[0] = 1
    return kv, new


def _ceil(a, b):
    return (a + b - 1) // b


def _offsets(n):
    return torch.nn.functional.pad(n.cumsum(0), (1, 0)).to(I32)


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _normal(g, shape, std=1.0, dtype=BF16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _keys_like(g, shape):
    """bf16 keys or values as a projection gives them: channels of uneven strength, some with an offset."""
    D = shape[-1]
    strength = torch.exp(0.5 * _normal(g, shape[-2:], dtype=F32))
    offset = _normal(g, shape[-2:], dtype=F32) * (torch.arange(D, device="cuda") % 7 == 0)
    return (_normal(g, shape, dtype=F32) * strength + offset).to(BF16)


def _unit(E):
    """2^(E - 127) in fp32, E 1 to 254."""
    return (E.to(I32) << 23).view(F32)


def _scale_byte(amax):
    """E of blocks whose largest magnitudes these fp32 are."""
    return (((amax.view(I32) + 0x180000) >> 23) - 8).clamp(10, 246)


def _to_e4m3(x):
    return x.clamp(-448.0, 448.0).to(E4M3)


def _layout(ck, cv):
    """Codes [n, 64, H, D] of keys and values as records [n, H, 128 D]."""
    n, _, H, D = ck.shape
    k = ck.view(n, 4, 16, H, D // 64, 64).permute(0, 3, 1, 4, 2, 5).reshape(n, H, 64 * D)
    v = cv.view(n, 2, 2, 4, 4, H, D // 16, 16).permute(0, 5, 6, 7, 3, 1, 2, 4).reshape(n, H, 64 * D)   # [h][u][g][e] -> [j][m][g][h][u][e]
    return torch.cat([k, v], -1)


def _unlayout(rec, D):
    """Records [n, H, 128 D] as codes [n, 64, H, D] of keys and of values."""
    n, H = rec.shape[:2]
    k = rec[..., :64 * D].reshape(n, H, 4, D // 64, 16, 64).permute(0, 2, 4, 1, 3, 5).reshape(n, 64, H, D)
    v = rec[..., 64 * D:].reshape(n, H, D // 16, 16, 4, 2, 2, 4).permute(0, 5, 6, 4, 7, 1, 2, 3).reshape(n, 64, H, D)
    return k, v


def _page_bytes(c):
    B = c["page"] // 64
    return _ceil(c["H"] * B * (128 * c["D"]) + 2 * c["H"] * B, 128) * 128


def _records_of(data, c):
    """Records [n_pages, H, B, 128 D] and bytes E [n_pages, H, B, 2] of a cache, as views."""
    n, H, D, B = data.shape[0], c["H"], c["D"], c["page"] // 64
    size = H * B * 128 * D
    return data[:, :size].view(n, H, B, 128 * D), data[:, size:size + 2 * H * B].view(n, H, B, 2)


def _cache(c, st, g, seed):
    """A pool that has been in use, the requests' pages in no order, filled up to their lengths before the step (append) or after it
    (attend); whatever its other bytes are stays in them."""
    kv, new = _lens(c)
    P, H, D, B = c["page"], c["H"], c["D"], c["page"] // 64
    end = kv + new
    have, all_ = _ceil(kv, P), _ceil(end, P)
    max_pages, held, total = int(all_.max()) + 1, int(have.sum()), int(all_.sum())
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=_gen(seed, "cpu")).to(I32)
    grid = torch.arange(max_pages)
    before = torch.full((c["S"], max_pages), -1, dtype=I32)
    before[grid < have[:, None]] = order[:held]
    table = before.clone()
    table[(grid >= have[:, None]) & (grid < all_[:, None])] = order[held:total]
    data = torch.empty((n_pages, _page_bytes(c)), dtype=torch.uint8, device="cuda")
    data.random_(0, 256, generator=g)
    rec, E = _records_of(data, c)
    # blocks of the requests' tokens: whole ones of keys and values like a projection's
    full = kv if c["kind"] == "append" else end
    n_blocks = _ceil(full, 64)
    b = torch.arange(max_pages * B)
    s_of, b_of = (b < n_blocks[:, None]).nonzero(as_tuple=True)
    page, blk = table[s_of, b_of // B].long().cuda(), (b_of % B).cuda()
    valid = (b_of[:, None] * 64 + torch.arange(64) < full[s_of][:, None]).cuda()
    step = max(1, (1 << 27) // (64 * H * D))
    for lo in range(0, page.numel(), step):
        p, q = page[lo:lo + step], blk[lo:lo + step]
        n, codes, bytes_ = p.numel(), [], []
        old = _unlayout(rec[p, :, q], D)
        for i in range(2):
            x = _keys_like(g, (n, 64, H, D)).to(F32)
            there = valid[lo:lo + step, :, None, None]
            e = _scale_byte(torch.where(there, x.abs(), 0.0).amax((1, 3)))            # [n, H]
            z = _to_e4m3(x * _unit(254 - e)[:, None, :, None]).view(torch.uint8)
            codes.append(torch.where(there, z, old[i]))
            bytes_.append(e.to(torch.uint8))
        rec[p, :, q] = _layout(*codes)
        E[p, :, q] = torch.stack(bytes_, -1)
    st.update(T=int(new.sum()), max_new=int(new.max()), n_pages=n_pages, table=table.cuda(), data=data, off=_offsets(new).cuda(),
              len=end.to(I32).cuda(), max_len=int(end.max()))
    return kv, new, order, before, held, total


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if own:
        from paper_2410_09687_amd import moin
        st["ctx"] = moin.Context(torch.cuda.current_device())
    if c["kind"] == "rotate":
        T, D, h, H = c["T"], c["D"], c["heads"], c["H"]
        # q, k and v of a token are one row of the projections' output
        st["qkv"] = _keys_like(g, (T, h + 2 * H, D)).to(BF16 if c["x"] == "bf16" else F32)
        st["pos"] = torch.randint(0, c["pos_hi"], (T,), generator=g, device="cuda", dtype=I32)
        st["gain_q"], st["gain_k"] = (1.0 + _normal(g, (D,), 0.2, F32)).to(BF16), (1.0 + _normal(g, (D,), 0.2, F32)).to(BF16)
        st["freqs"] = THETA ** (torch.arange(c["rot"] // 2, dtype=F64, device="cuda") * (-2.0 / c["rot"]))
        return st
    if c["kind"] in ("append", "attend"):
        kv, new, order, before, held, total = _cache(c, st, g, seed)
        P, H, D = c["page"], c["H"], c["D"]
        if own:
            st["pages"] = moin.KV8Pages(st["data"], H, D, P)
        if c["kind"] == "attend":
            st["q"] = _normal(g, (st["T"], c["heads"], D))
            if own:   # the step's plan: one for all layers; it deals the pages as the table has them
                st["plan"] = moin.KVPlan(st["ctx"])
                rest = order[held:]
                free = torch.cat([rest[total - held:], rest[:total - held].flip(0)]).cuda()
                st["plan"].build(kv.cuda(), new.cuda(), st["T"], before.cuda(), free, torch.tensor([free.numel()], dtype=I32, device="cuda"),
                                 n_pages=st["n_pages"], page_tokens=P, n_heads=c["heads"], n_kv=H, max_new=st["max_new"])
            return st
        st["kv"] = torch.cat([_keys_like(g, (st["T"], H, D)), _keys_like(g, (st["T"], H, D))], 1)
        table, off = st["table"].cpu(), st["off"].cpu().long()

        def slots_of(s, pos):
            return table[s, pos // P] * P + (pos % P).to(I32)

        t = torch.arange(st["T"])
        s = torch.searchsorted(off[1:], t, right=True)
        pos = kv[s].long() + t - off[s]
        st["slots"] = slots_of(s, pos).to(I32).cuda()
        # the blocks that the step touches, and the places in them that hold tokens afterwards
        first, last = kv.long() // 64, _ceil(kv.long() + new.long(), 64)
        b = torch.arange(int(last.max()))
        bs, bb = ((b >= first[:, None]) & (b < last[:, None]) & (new > 0)[:, None]).nonzero(as_tuple=True)
        place = bb[:, None] * 64 + torch.arange(64)                                       # positions [blocks, 64]
        there = place < (kv + new).long()[bs][:, None]
        st.update(blk_page=table[bs, bb * 64 // P].long().cuda(), blk=(bb % (P // 64)).cuda(), there=there.cuda(),
                  is_new=(there & (place >= kv.long()[bs][:, None])).cuda(),
                  src=(off[bs][:, None] + place - kv.long()[bs][:, None]).clamp(0, st["T"] - 1).cuda())
        at = there.nonzero(as_tuple=True)
        st["held"] = slots_of(bs[at[0]], place[at]).to(I32).cuda()                        # every slot of those blocks in use
        return st
    S, d_in, d_out, r, E = c["S"], c["d_in"], c["d_out"], c["r"], c["E"]
    lens = _some(c, c["len_lo"], c["len_hi"], 3)
    T = int(lens.sum())
    st.update(T=T, off=_offsets(lens).cuda(), lens=lens.cuda(), x=_normal(g, (T, d_in)) * torch.exp(0.7 * _normal(g, (T, 1), dtype=F32)).to(BF16))
    W = _normal(g, (d_out, d_in), d_in ** -0.5) * torch.exp(0.5 * _normal(g, (d_out, 1), dtype=F32)).to(BF16)
    codes, st["ws"] = _to_i8(W)
    st["W"] = torch.zeros((d_out, max(256, _ceil(d_in, 128) * 128)), dtype=torch.int8, device="cuda")
    st["W"][:, :d_in] = codes
    if r:
        p = torch.arange(1, E + 1, dtype=F64) ** -1.1     # few experts serve most requests
        ids = torch.multinomial(p, S, replacement=True, generator=_gen(seed, "cpu"))
        st["ids"] = torch.randperm(E, generator=_gen(seed + 1, "cpu"))[ids].to(I32).cuda()
        st["A"], st["B"] = _normal(g, (E, r, d_in), d_in ** -0.5), _normal(g, (E, d_out, r), r ** -0.5)
    if own:
        st["w8"] = moin.I8Weight(st["W"], st["ws"], d_in)
        if r:   # the batch's grouping: one for all projections of all layers
            st["plan"] = moin.Plan(st["ctx"])
            st["plan"].build(st["off"], st["ids"], T, E)
    return st


# ---- one pass -------------------------------------------------------------------------------------------

def _dtype(c):
    return BF16 if c["y"] == "bf16" else F32


def run(st):
    c = st["case"]
    if own:
        return _run_own(c, st)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend, "linear": _plain_linear}[c["kind"]](c, st)


def _run_own(c, st):
    from paper_2410_09687_amd import moin
    ctx = st["ctx"]
    if c["kind"] == "rotate":
        h, H = c["heads"], c["H"]
        q, k = moin.moin_qk_norm_rope(ctx, st["qkv"][:, :h], st["qkv"][:, h:h + H], positions=st["pos"], freqs=st["freqs"],
                                      q_gain=st["gain_q"] if c["norm"] else None, k_gain=st["gain_k"] if c["norm"] else None,
                                      norm=c["norm"], eps=EPS, neighbours=c["pairs"] == "neighbours")
        return dict(q=q, k=k)
    if c["kind"] == "append":
        H = c["H"]
        moin.moin_kv8_append(ctx, st["pages"], st["kv"][:, :H], st["kv"][:, H:], st["off"], st["slots"])
        k, v = moin.moin_kv8_gather(ctx, st["pages"], st["held"])
        return dict(k=k, v=v)
    if c["kind"] == "attend":
        y, lse = moin.moin_kv8_attention(ctx, st["plan"], st["pages"], st["q"], st["table"], window=c["window"], y_dtype=_dtype(c),
                                         want_lse=True)
        return dict(y=y, lse=lse)
    if c["r"]:
        return moin.moin_lora_linear_i8_planned(ctx, st["plan"], st["x"], st["w8"], st["A"], st["B"], SCALE, y_dtype=_dtype(c))
    return moin.moin_i8_linear(ctx, st["x"], st["w8"], y_dtype=_dtype(c))


def _plain_rotate(c, st):
    h, H, R = c["heads"], c["H"], c["rot"]
    turns = st["pos"].to(F64)[:, None] * (st["freqs"] / (2.0 * math.pi))
    angle = (turns - turns.floor()).to(F32) * (2.0 * math.pi)
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def one(x, gain):
        x = x.to(F32)
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.to(F32)
        out = x.clone()
        at = (slice(0, R // 2), slice(R // 2, R)) if c["pairs"] == "halves" else (slice(0, R, 2), slice(1, R, 2))
        a, b = x[..., at[0]], x[..., at[1]]
        out[..., at[0]], out[..., at[1]] = a * cos - b * sin, b * cos + a * sin
        return out.to(BF16)

    return dict(q=one(st["qkv"][:, :h], st["gain_q"]), k=one(st["qkv"][:, h:h + H], st["gain_k"]))


def _plain_append(c, st):
    H, D = c["H"], c["D"]
    rec, E = _records_of(st["data"], c)
    old = _unlayout(rec[st["blk_page"], :, st["blk"]], D)
    E_old = E[st["blk_page"], :, st["blk"]].to(I32)                                         # [blocks, H, 2]
    is_new, there = st["is_new"][:, :, None, None], st["there"][:, :, None, None]
    begun = (st["there"] & ~st["is_new"]).any(1)[:, None]
    out = []
    for i in range(2):
        x = st["kv"][:, i * H:(i + 1) * H][st["src"]].to(F32)                               # [blocks, 64, H, D]
        e_new = _scale_byte(torch.where(is_new, x.abs(), 0.0).amax((1, 3)))
        e_old = torch.where(begun, E_old[..., i], 0)
        e = torch.maximum(e_new, e_old)
        shrink = _unit((127 + e_old - e).clamp(min=1))[:, None, :, None]
        was = old[i].view(E4M3).to(F32) * shrink
        z = torch.where(is_new, x * _unit(254 - e)[:, None, :, None], torch.where(there, was, 0.0))
        held = (_to_e4m3(z).to(F32) * _unit(e)[:, None, :, None]).to(BF16)
        out.append(held[st["there"]])
    return dict(k=out[0], v=out[1])


def _plain_attend(c, st):
    S, H, D, n, T, B = c["S"], c["H"], c["D"], st["max_new"], st["T"], c["page"] // 64
    G = c["heads"] // H
    nb = _ceil(st["max_len"], 64)
    blk = torch.arange(nb, device="cuda")
    page = st["table"][:, blk // B].long().clamp(min=0)
    rec, E = _records_of(st["data"], c)
    codes = _unlayout(rec[page, :, blk % B].flatten(0, 1), D)                               # [S nb, 64, H, D]
    unit = _unit(E[page, :, blk % B].to(I32).clamp(1, 254)).flatten(0, 1)                   # [S nb, H, 2]
    k, v = ((codes[i].view(E4M3).to(F32) * unit[:, None, :, None, i]).reshape(S, nb * 64, H, D).permute(0, 2, 1, 3) for i in range(2))
    L = nb * 64
    off, lens = st["off"].long(), st["len"].long()
    new = off[1:] - off[:-1]
    row = torch.arange(n, device="cuda")
    tok = (off[:-1, None] + row).clamp(max=T - 1)                                           # [S, n]
    q = st["q"][tok].to(F32).view(S, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(S, H, n * G, D)
    key = torch.arange(L, device="cuda")
    held = key < lens[:, None]
    k, v = (torch.where(held[:, None, :, None], x, 0.0) for x in (k, v))                    # no key is read beyond a request's end
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * D ** -0.5
    pos = (lens - new)[:, None] + row                                                       # [S, n]
    seen = (key <= pos[..., None]) & (pos[..., None] >= 0)
    if c["window"]:
        seen = seen & (key > pos[..., None] - c["window"])
    s = s.view(S, H, n, G, L).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = (s - torch.where(m == -math.inf, 0.0, m)).exp_()
    sums = p.sum(-1, keepdim=True)
    y = torch.matmul(p.view(S, H, n * G, L), v).view(S, H, n, G, D) / torch.where(sums == 0, 1.0, sums)
    lse = (m + sums.log()).squeeze(-1)
    real = row < new[:, None]                                                               # [S, n], in the order of the tokens
    return dict(y=y.permute(0, 2, 1, 3, 4).reshape(S, n, H * G, D)[real].to(_dtype(c)),
                lse=lse.permute(0, 2, 1, 3).reshape(S, n, H * G)[real])


def _to_i8(x):
    """Codes and scales of the rows of x, the quotients in 64 bits."""
    s = (x.to(F32).abs().amax(1).to(F64) / 127.0).to(F32).clamp(min=2.0 ** -126)
    return torch.round(x.to(F64) / s.to(F64)[:, None]).to(torch.int8), s


def _plain_linear(c, st):
    T, d_in = st["T"], c["d_in"]
    xq, s = _to_i8(st["x"])
    y = (xq.to(F32) @ st["W"][:, :d_in].to(F32).t()) * s[:, None] * st["ws"]
    if c["r"]:
        A, B, x = st["A"], st["B"], st["x"].to(F32)
        ids = st["ids"].long().repeat_interleave(st["lens"].long(), output_size=T)
        used, at = torch.unique(ids, return_inverse=True)
        # the tokens of each adapter side by side, padded to the most that one has
        order = at.argsort(stable=True)
        count = torch.bincount(at, minlength=used.numel())
        place = torch.arange(T, device="cuda") - (count.cumsum(0) - count)[at[order]]
        xs = torch.zeros((used.numel(), int(count.max()), d_in), dtype=F32, device="cuda")
        xs[at[order], place] = x[order]
        u = torch.bmm(xs, A[used].to(F32).transpose(1, 2).contiguous())
        z = torch.bmm(u, B[used].to(F32).transpose(1, 2).contiguous())
        y[order] += SCALE * z[at[order], place]
    return y.to(_dtype(c))


# ---- from the definitions, in 64 bits -------------------------------------------------------------------

def _power(e):
    """2^e, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def _e4m3_value(code):
    """What E4M3 bytes stand for."""
    code = code.to(I32)
    e, m = (code >> 3) & 15, (code & 7).to(F64)
    mag = torch.where(e == 0, m * 2.0 ** -9, (8.0 + m) * _power(e - 10))
    mag = torch.where((code & 127) == 127, math.nan, mag)
    return torch.where(code > 127, -mag, mag)


def _on_grid(x):
    """x to the nearest value of E4M3, ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))).clamp(min=-6)
    step = _power(e - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def exact(case, seed):
    c = case
    st = _plain_state(case, seed)
    if c["kind"] == "rotate":
        h, H, R, D = c["heads"], c["H"], c["rot"], c["D"]
        at = st["pos"].to(F64)[:, None] * torch.exp(torch.arange(R // 2, dtype=F64, device="cuda") * (-2.0 * math.log(THETA) / R))
        turn = torch.polar(torch.ones_like(at), at)[:, None]

        def one(x, gain):
            x = x.to(F64)
            if c["norm"]:
                x = x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * gain.to(F64)
            z = x[..., :R]
            z = z.unflatten(-1, (2, R // 2)).transpose(-1, -2) if c["pairs"] == "halves" else z.unflatten(-1, (R // 2, 2))
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            z = z.transpose(-1, -2).flatten(-2) if c["pairs"] == "halves" else z.flatten(-2)
            return torch.cat([z, x[..., R:]], -1)

        return dict(q=one(st["qkv"][:, :h], st["gain_q"]), k=one(st["qkv"][:, h:h + H], st["gain_k"]))
    if c["kind"] == "append":
        H, D = c["H"], c["D"]
        rec, E = _records_of(st["data"], c)
        t = torch.arange(64, device="cuda")
        ch = torch.arange(D, device="cuda")
        at_k = (t // 16)[:, None] * 16 * D + (ch // 64) * 1024 + (t % 16)[:, None] * 64 + ch % 64
        at_v = 64 * D + ch * 64 + ((t // 4 % 4) * 16 + (t // 32) * 8 + (t // 16 % 2) * 4 + t % 4)[:, None]
        n = st["blk_page"].numel()
        out = [[], []]
        for lo in range(0, n, 256):     # (a few blocks at a time)
            sl = slice(lo, min(n, lo + 256))
            r, e0 = rec[st["blk_page"][sl], :, st["blk"][sl]], E[st["blk_page"][sl], :, st["blk"][sl]].to(F64)
            new, there = st["is_new"][sl], st["there"][sl]
            began = (there & ~new).any(1)
            for i, at in enumerate((at_k, at_v)):
                was = _e4m3_value(r[:, :, at]).permute(0, 2, 1, 3)                          # [blocks, 64, H, D]
                x = st["kv"][:, i * H:(i + 1) * H][st["src"][sl]].to(F64)
                top = torch.where(new[:, :, None, None], x.abs(), 0.0).amax((1, 3))
                # the smallest power of two in whose units the largest value is below 464
                e = torch.floor(torch.log2(top.clamp(min=2.0 ** -300))) - 8
                e = torch.where(top / _power(e) >= 464, e + 1, e).clamp(-117, 119)
                e = torch.where(began[:, None], torch.maximum(e, e0[..., i] - 127), e)
                unit = _power(e)[:, None, :, None]
                old = torch.where(there[:, :, None, None] & ~new[:, :, None, None], was * _power(e0[..., i] - 127)[:, None, :, None], 0.0)
                held = _on_grid(torch.where(new[:, :, None, None], x, old) / unit) * unit
                out[i].append(held[there])
        return dict(k=torch.cat(out[0]), v=torch.cat(out[1]))
    if c["kind"] == "linear":
        d_in = c["d_in"]
        x = st["x"].to(F64)
        s = (x.abs().amax(1) / 127.0).to(F32).to(F64).clamp(min=2.0 ** -126)
        y = ((x / s[:, None]).round() @ st["W"][:, :d_in].to(F64).t()) * s[:, None] * st["ws"].to(F64)
        if c["r"]:
            off, ids = st["off"].tolist(), st["ids"].tolist()
            for e in set(ids):
                rows = torch.cat([torch.arange(off[i], off[i + 1], device="cuda") for i in range(c["S"]) if ids[i] == e])
                y[rows] += SCALE * (x[rows] @ st["A"][e].to(F64).t() @ st["B"][e].to(F64).t())
        return y
    H, D, P, G = c["H"], c["D"], c["page"], c["heads"] // c["H"]
    y = torch.zeros((st["T"], c["heads"], D), dtype=F64, device="cuda")
    lse = torch.full((st["T"], c["heads"]), -math.inf, dtype=F64, device="cuda")
    rec, E = _records_of(st["data"], c)
    off, lens, table = st["off"].tolist(), st["len"].tolist(), st["table"].tolist()
    t = torch.arange(64, device="cuda")
    ch = torch.arange(D, device="cuda")
    at_k = (t // 16)[:, None] * 16 * D + (ch // 64) * 1024 + (t % 16)[:, None] * 64 + ch % 64
    at_v = 64 * D + ch * 64 + ((t // 4 % 4) * 16 + (t // 32) * 8 + (t // 16 % 2) * 4 + t % 4)[:, None]
    for s in range(c["S"]):
        n, L = off[s + 1] - off[s], lens[s]
        if not n or not L:
            continue
        pages = torch.tensor(table[s][:_ceil(L, P)], device="cuda")
        r = rec[pages].transpose(1, 2).reshape(-1, H, 128 * D)                              # [records][H][bytes]
        e = E[pages].transpose(1, 2).reshape(-1, H, 2).to(F64)
        pos = L - n + torch.arange(n, device="cuda")
        lo, hi = (pos - c["window"] + 1 if c["window"] else pos * 0).clamp(min=0), pos + 1
        key = torch.arange(L, device="cuda")
        out = (key < lo[:, None]) | (key >= hi[:, None])                                    # [n, L]
        for h in range(H):
            k = (_e4m3_value(r[:, h][:, at_k]) * _power(e[:, h, 0] - 127)[:, None, None]).view(-1, D)[:L]
            v = (_e4m3_value(r[:, h][:, at_v]) * _power(e[:, h, 1] - 127)[:, None, None]).view(-1, D)[:L]
            q = st["q"][off[s]:off[s + 1], h * G:(h + 1) * G].to(F64)                       # [n, G, D]
            z = (q.reshape(n * G, D) @ k.t().contiguous()).view(n, G, L) / math.sqrt(D)
            z.masked_fill_(out[:, None], -math.inf)
            a = torch.logsumexp(z, -1)
            w = torch.where(a[..., None] == -math.inf, 0.0, (z - a[..., None]).exp())
            lse[off[s]:off[s + 1], h * G:(h + 1) * G] = a
            y[off[s]:off[s + 1], h * G:(h + 1) * G] = (w.view(n * G, L) @ v).view(n, G, D)
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
    if c["kind"] == "rotate":
        n = float(c["T"] * (c["heads"] + c["H"]) * c["D"])
        return dict(bytes=n * ((2 if c["x"] == "bf16" else 4) + 2) + 4.0 * c["T"], flops=n * (7 if c["norm"] else 3))
    if c["kind"] == "append":
        kv, new = _lens(c)
        T, held = float(new.sum()), float((new + kv % 64)[new > 0].sum())
        row = 2.0 * c["H"] * c["D"]
        return dict(bytes=row * (T * 3 + held * 3) + 4 * (T + held), flops=0.0)
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
        return dict(bytes=keys * c["H"] * (2.0 * c["D"] + 2 / 64) + T * c["heads"] * (c["D"] * (2 + (2 if c["y"] == "bf16" else 4)) + 4),
                    flops=4.0 * pairs * c["heads"] * c["D"])
    T, d_in, d_out, r = int(_some(c, c["len_lo"], c["len_hi"], 3).sum()), c["d_in"], c["d_out"], c["r"]
    b = float(d_in * d_out + 4 * d_out + T * (2 * d_in + (2 if c["y"] == "bf16" else 4) * d_out))
    f = 2.0 * T * d_in * d_out
    if r:
        p = torch.arange(1, c["E"] + 1, dtype=F64) ** -1.1
        distinct = float((1 - (1 - p / p.sum()) ** c["S"]).sum())
        b += 2 * distinct * r * (d_in + d_out)
        f += 2.0 * T * r * (d_in + d_out)
    return dict(bytes=b, flops=f)
