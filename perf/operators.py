"""The paged 8-bit cache, measured: page tables and slot maps, the store, and the attention that reads the cache.

`run` computes a case in elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.  A
case's kind is one of

  map     hca_paged_map: pages given and taken back, start positions, row offsets and the slot of every new token
  store   hca_paged_store: blocks that became whole are coded in 8 bits, the open block's rows kept in 16 bits
  attend  hca_paged_attend: softmax attention of every sequence's queries over its cache

What the cache holds (P tokens per page, D channels, n pages, s sequences, h KV heads):
  kv     8-bit codes [n, h, 2, P * D]: keys, then values, in tiles of 16 tokens
           keys    [P/16][D/64][4 g][16 t][16 e]        token t of the tile, channel 64 * second + 16 g + e
           values  [P/16][D/64][4 g][16 c][4 u][4 j]    token 4 g + j of the tile, channel 64 * second + 16 u + c
  scale  fp32 [n, h, 2]: what one step of a page's codes stands for, keys and values
  open   16-bit [s, h, 2, P * D]: the rows of each sequence's last block while it is not whole, in the same tiles
A sequence of length L has L // P whole pages; its remaining L % P tokens are in its open rows.
"""
import math

import torch

own = False

QMAX = {"int8": 127.0, "e4m3": 448.0}
FLOOR = 2.0 ** -64            # the least scale: 1 / scale and the sums of weights stay finite
ELEM = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # bookkeeping of one decode step of a small batch: nothing but latency
        dict(name="map-decode-16", kind="map", seqs=16, page=16, max_pages=512, mix="decode", n=8000),
        # a busy step: requests that end, prompts that arrive in chunks, the others one token each, idle slots
        dict(name="map-mixed-256", kind="map", seqs=256, page=16, max_pages=2048, mix="mixed", n=20000, new=1500),
        # one decode step's keys and values of a Llama-3-8B layer, 64 sequences at their own lengths
        dict(name="store-decode-64", kind="store", seqs=64, hkv=8, hq=32, d=128, page=64, elem="bf16", code="e4m3", n=5000, new=1,
             ragged=True, fused=True),
        # prompts of different lengths written at once, out of a fused projection's rows
        dict(name="store-prompts-32k", kind="store", seqs=6, hkv=8, hq=32, d=128, page=64, elem="f16", code="int8", n=0, new=8192,
             ragged=True, fused=True),
        # one request of a few hundred tokens: latency
        dict(name="attend-1x777", kind="attend", seqs=1, hq=32, hkv=8, d=128, page=16, elem="f16", code="int8", n=777, q=1,
             causal=True, ragged=False),
        # a served batch, every sequence at its own length
        dict(name="attend-32x8k", kind="attend", seqs=32, hq=32, hkv=8, d=128, page=64, elem="bf16", code="e4m3", n=8192, q=1,
             causal=True, ragged=True),
        # one long context: a single layer's share of 1 Mi tokens
        dict(name="attend-1m", kind="attend", seqs=1, hq=32, hkv=8, d=128, page=128, elem="f16", code="int8", n=1048576, q=1,
             causal=True, ragged=False),
        # four long contexts in the smallest pages, one value head for eight query heads
        dict(name="attend-4x128k-p16", kind="attend", seqs=4, hq=32, hkv=4, d=128, page=16, elem="bf16", code="int8", n=131072, q=1,
             causal=True, ragged=True),
        # drafted tokens checked together: five queries per sequence
        dict(name="attend-drafts-8x32k", kind="attend", seqs=8, hq=32, hkv=8, d=128, page=32, elem="f16", code="e4m3", n=32768, q=5,
             causal=True, ragged=True),
        # one chunk of a long prompt against what is cached of it
        dict(name="attend-chunk-2k", kind="attend", seqs=1, hq=32, hkv=8, d=128, page=64, elem="f16", code="e4m3", n=34000, q=2048,
             causal=True, ragged=False),
        # whole prompts against themselves
        dict(name="attend-prompts-5x4k", kind="attend", seqs=5, hq=32, hkv=8, d=128, page=64, elem="bf16", code="int8", n=4096,
             q=4096, causal=True, ragged=True),
        # a decoder's prompts against an encoder's states: no mask, 64 channels per head
        dict(name="attend-encoder-4x1500", kind="attend", seqs=4, hq=8, hkv=8, d=64, page=32, elem="f16", code="e4m3", n=1500,
             q=300, causal=False, ragged=True),
    ]


def _log(rng, lo, hi):
    """A size whose logarithm is uniform between those of lo and hi."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["map", "store", "store", "attend", "attend", "attend", "attend"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "map":
        n = _log(rng, 100, 30000)
        new = _log(rng, 1, 2000)
        return dict(kind=kind, seqs=_log(rng, 1, 256), page=page, max_pages=(n + new) // page + 2 + rng.randint(0, 500),
                    mix=rng.choice(["decode", "mixed"]), n=n, new=new)
    hq, hkv = rng.choice([(32, 8), (32, 8), (16, 8), (8, 8), (4, 1), (1, 1), (14, 7), (32, 4), (24, 4), (16, 1)])
    c = dict(kind=kind, hq=hq, hkv=hkv, d=rng.choice([128, 128, 64]), page=page, elem=rng.choice(["f16", "bf16"]),
             code=rng.choice(["int8", "e4m3"]), ragged=rng.random() < 0.7)
    if kind == "store":
        if rng.random() < 0.5:
            return dict(c, seqs=_log(rng, 1, 256), n=_log(rng, 1, 8000), new=1, fused=rng.random() < 0.5)
        seqs = _log(rng, 1, 32)
        return dict(c, seqs=seqs, n=rng.choice([0, 0, _log(rng, 1, 8000)]), new=_log(rng, 2, min(16384, max(2, 49152 // seqs))),
                    fused=rng.random() < 0.5)
    form = rng.choice(["decode", "decode", "drafts", "prompt", "encoder"])
    if form in ("decode", "drafts"):
        seqs = _log(rng, 1, 64)
        return dict(c, seqs=seqs, n=_log(rng, 1, min(1048576, 4194304 // (seqs * hkv))),
                    q=1 if form == "decode" else rng.randint(2, 12), causal=True)
    seqs = _log(rng, 1, 8)
    q = _log(rng, 13, 4096 if seqs < 3 else 2048)
    n = _log(rng, 20, 4000) if form == "encoder" else max(q, _log(rng, 20, 16384 // seqs))
    return dict(c, seqs=seqs, n=n, q=q, causal=form == "prompt")


# ---- sizes that follow from a case ----------------------------------------------------------------

def _spread(most, count, ragged, step):
    """`count` whole numbers up to `most`, the first the largest; ragged: down to about a third of it, in no round steps."""
    if not ragged:
        return [most] * count
    return [max(1, most - i * (2 * most // 3) // max(1, count) - (step * i) % max(1, most // 5 + 1)) if i else most for i in range(count)]


def _lens(c):
    """(tokens held before the call, new tokens or queries) per sequence."""
    s, P = c["seqs"], c["page"]
    if c["kind"] == "map":
        n = _spread(c["n"], s, True, 13)
        if c["mix"] == "decode":
            return n, [1] * s
        new = _spread(c["new"], s, True, 7)
        return n, [(-1 if i % 16 == 3 else new[i] if i % 16 == 5 else 0 if i % 16 == 9 else 1) for i in range(s)]
    if c["kind"] == "store":
        n = _spread(c["n"], s, c["ragged"], 13) if c["n"] else [0] * s
        new = [1] * s if c["new"] == 1 else _spread(c["new"], s, c["ragged"], 11)
        if c["new"] > 1:      # chunks of a prompt end at whole blocks, all but the last
            n = [x // P * P for x in n]
        return n, new
    n = _spread(c["n"], s, c["ragged"], 13)
    q = [c["q"]] * s if c["q"] < 13 else _spread(c["q"], s, c["ragged"], 5)
    return (n, [min(a, b) for a, b in zip(n, q)]) if c["causal"] else (n, q)


def _ceil(a, b):
    return -(-a // b)


def work(case):
    c = case
    n, new = _lens(c)
    P = c["page"]
    if c["kind"] == "map":
        T = [max(t, 0) for t in new]
        pages = sum(_ceil(a + t, P) - _ceil(a, P) for a, t in zip(n, T)) + sum(_ceil(a, P) for a, t in zip(n, new) if t < 0)
        return {"bytes": 8 * c["seqs"] + 12 * c["seqs"] + 8 * pages + 12 * sum(T), "flops": 2 * c["seqs"] + 3 * sum(T)}
    H, D = c["hkv"], c["d"]
    if c["kind"] == "store":
        whole = sum((a + t) // P - a // P for a, t in zip(n, new))
        held = sum(a % P for a, t in zip(n, new) if (a + t) // P > a // P)
        left = sum((a + t) % P if (a + t) // P > a // P else t for a, t in zip(n, new))
        return {"bytes": 2 * H * D * (2 * sum(new) + 2 * held + whole * P + 2 * left) + 8 * H * whole + 12 * c["seqs"] + 4 * whole,
                "flops": 4 * 2 * H * D * whole * P}
    m = new
    read = sum(2 * H * (a // P * P * D + a % P * D * 2) + 8 * H * (a // P) + 4 * (a // P) for a in n)
    rows = sum(m)
    pairs = sum(t * a - (t * (t - 1) // 2 if c["causal"] else 0) for a, t in zip(n, m))
    return {"bytes": read + rows * c["hq"] * (4 * D + 4) + 8 * c["seqs"], "flops": 4 * D * c["hq"] * pairs}


# ---- inputs ---------------------------------------------------------------------------------------

def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + tag)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _rows(shape, g, outlier, elem):
    """Rows of keys or values; `outlier` channels per head stand out eightfold, as they do in keys."""
    x = torch.randn(shape, generator=g, device="cuda")
    if outlier:
        x[..., 5 :: shape[-1] // outlier] *= 8.0
    return x.to(ELEM[elem])


def _code(x, code):
    """(codes of x [..., P, D] with one scale per block, the scales)."""
    amax = x.abs().amax((-1, -2))
    scale = (amax.double() / QMAX[code]).float().clamp_min(FLOOR)
    y = (x * (1.0 / scale.double()).float()[..., None, None]).clamp(-QMAX[code], QMAX[code])
    return (y.round().to(torch.int8) if code == "int8" else y.to(torch.float8_e4m3fn)), scale


def _tiled(k, v):
    """[..., P, D] keys and values -> the cache's order [..., 2, P * D]."""
    *b, P, D = k.shape
    z = len(b)
    at = list(range(z))
    k = k.reshape(*b, P // 16, 16, D // 64, 4, 16).permute(*at, z, z + 2, z + 3, z + 1, z + 4).reshape(*b, P * D)
    v = v.reshape(*b, P // 16, 4, 4, D // 64, 4, 16).permute(*at, z, z + 3, z + 1, z + 5, z + 4, z + 2).reshape(*b, P * D)
    return torch.stack((k, v), len(b))


def _plain_order(kv, P, D):
    """Views of [..., 2, P * D]: keys [..., P/16, 16, D/64, 4, 16], values [..., P/16, 4, 4, D/64, 4, 16]; tokens, then channels."""
    k, v = kv.select(-2, 0), kv.select(-2, 1)
    z = k.dim() - 1
    at = list(range(z))
    k = k.unflatten(-1, (P // 16, D // 64, 4, 16, 16)).permute(*at, z, z + 3, z + 1, z + 2, z + 4)
    v = v.unflatten(-1, (P // 16, D // 64, 4, 16, 4, 4)).permute(*at, z, z + 2, z + 5, z + 1, z + 4, z + 3)
    return k, v


def prepare(case, seed):
    c = case
    n, new = _lens(c)
    s, P = c["seqs"], c["page"]
    T = [max(t, 0) for t in new]
    after = [a + t for a, t in zip(n, T)] if c["kind"] != "attend" else n
    cu = [0]
    for t in T:
        cu.append(cu[-1] + t)
    pages = [_ceil(a, P) for a in (n if c["kind"] == "map" else after)]
    max_pages = c.get("max_pages") or max(pages) + 3
    spare = sum(_ceil(a, P) for a in after) + 7 if c["kind"] == "map" else 5
    n_pages = sum(pages) + spare
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device="cuda").int()
    tables = torch.full((s, max_pages), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(s):
        tables[b, : pages[b]] = order[at : at + pages[b]]
        at += pages[b]
    st = dict(case=c, P=P, s=s, n_pages=n_pages, max_pages=max_pages, tables=tables, total=cu[-1], max_new=max(T), nmax=max(after),
              cu=_i32(cu))
    if c["kind"] == "map":
        free = torch.full((n_pages + 1,), -1, dtype=torch.int32, device="cuda")       # one place more: the plain form's bin
        free[: n_pages - at] = order[at:]
        st.update(add=_i32(new), lens=_i32(n), free=free, count=_i32([n_pages - at]), lens_out=_i32([0] * s), count_out=_i32([0]),
                  start=_i32([0] * s), cu=_i32([0] * (s + 1)), tok=torch.full((3, cu[-1]), -5, dtype=torch.int32, device="cuda"))
        return st
    H, D, elem = c["hkv"], c["d"], c["elem"]
    st.update(H=H, D=D, hq=c["hq"])
    open_ = torch.empty(s + 1, H, 2, P * D, dtype=ELEM[elem], device="cuda")
    open_[:] = _tiled(_rows((s + 1, H, P, D), _gen(seed, 2), 4, elem), _rows((s + 1, H, P, D), _gen(seed, 3), 0, elem))
    kv = torch.zeros(n_pages + 1, H, 2, P * D, dtype=torch.uint8, device="cuda")      # one page more: the plain form's bin
    scale = torch.ones(n_pages + 1, H, 2, device="cuda")
    st.update(open=open_, kv=kv, scale=scale)
    if c["kind"] == "store":
        st["start"] = _i32(n)
        if c["fused"]:        # keys and values are slices of a fused projection's output
            x = _rows((cu[-1], c["hq"] + 2 * H, D), _gen(seed, 4), 0, elem)
            x[:, c["hq"] : c["hq"] + H, 5 :: D // 4] *= 8.0
            st.update(k=x[:, c["hq"] : c["hq"] + H], v=x[:, c["hq"] + H :])
        else:
            st.update(k=_rows((cu[-1], H, D), _gen(seed, 4), 4, elem), v=_rows((cu[-1], H, D), _gen(seed, 5), 0, elem))
        return st
    gk, gv = _gen(seed, 4), _gen(seed, 5)
    for p in range(0, n_pages, 4096):                     # a few pages' worth at a time: 32-bit rows are large
        m = min(4096, n_pages - p)
        k, ks = _code(_rows((m, H, P, D), gk, 4, elem).float(), c["code"])
        v, vs = _code(_rows((m, H, P, D), gv, 0, elem).float() * (0.5 + torch.rand((m, H, 1, 1), generator=gv, device="cuda")), c["code"])
        kv[p : p + m] = _tiled(k.view(torch.uint8), v.view(torch.uint8))
        scale[p : p + m] = torch.stack((ks, vs), -1)
    # queries: logits with a spread of about two and a half
    st["q"] = (torch.randn((cu[-1], c["hq"], D), generator=_gen(seed, 6), device="cuda") * 1.4).to(ELEM[elem])
    st.update(lens=_i32(n), sm=1.0 / math.sqrt(D), y=torch.zeros_like(st["q"]), lse=torch.zeros(cu[-1], c["hq"], device="cuda"))
    return st


# ---- the passes -----------------------------------------------------------------------------------

def _map_plain(s):
    P, mp = s["P"], s["max_pages"]
    dev = s["lens"].device
    n, add = s["lens"].long(), s["add"].long()
    gone = add < 0
    T = add.clamp_min(0)
    held = (n + P - 1) // P
    back = torch.where(gone, held, 0)
    j = torch.arange(mp, device=dev)
    bin_ = s["n_pages"]
    to = torch.where(gone[:, None] & (j < held[:, None]), s["count"].long() + (back.cumsum(0) - back)[:, None] + j, bin_)
    s["free"].scatter_(0, to.reshape(-1), s["tables"].reshape(-1))
    avail = s["count"].long() + back.sum()
    n0 = torch.where(gone, 0, n)
    first = (n0 + P - 1) // P
    c = T.cumsum(0)
    fits = (n0 + T <= mp * P) & (c <= s["total"])
    need = torch.where(fits, (n0 + T + P - 1) // P - first, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= avail))
    rank = (upto - need)[:, None] + j - first[:, None]
    mine = ok[:, None] & (j >= first[:, None]) & (j < (first + need)[:, None])
    got = s["free"][(avail - 1 - rank).clamp(0, bin_)]
    s["tables"].copy_(torch.where(mine, got, s["tables"]))
    start = torch.where(ok, n0, -1)
    s["start"].copy_(start)
    s["lens_out"].copy_(n0 + torch.where(ok, T, 0))
    s["count_out"].copy_(avail - torch.where(ok, need, 0).sum())
    s["cu"][1:].copy_(c.clamp_max(s["total"]))
    t = torch.arange(s["total"], device=dev)
    seq = torch.searchsorted(c, t, right=True).clamp_max(s["s"] - 1)
    pos = torch.where(ok[seq], start[seq] + t - (c - T)[seq], -1)
    slot = torch.where(pos >= 0, s["tables"][seq, pos.clamp_min(0) // P].long() * P + pos % P, -1)
    s["tok"].copy_(torch.where(t < c[-1], torch.stack((seq, pos, slot)), s["tok"]))


def _store_plain(s):
    P, H, D, c = s["P"], s["H"], s["D"], s["case"]
    dev = s["kv"].device
    start, cu = s["start"].long(), s["cu"].long()
    T = cu[1:] - cu[:-1]
    blk = start[:, None] // P + torch.arange(s["max_new"] // P + 2, device=dev)                       # [s, blocks]
    p = blk[:, :, None] * P + torch.arange(P, device=dev)
    i = p - start[:, None, None]
    new = (i >= 0) & (i < T[:, None, None])
    whole = ((blk + 1) * P <= (start + T)[:, None]) & (T > 0)[:, None]
    src = (cu[:-1, None, None] + i).clamp(0, max(s["total"] - 1, 0))
    x = torch.stack((s["k"][src], s["v"][src]), 2)                                                     # [s, blocks, 2, P, H, D]
    ok, ov = _plain_order(s["open"][: s["s"]], P, D)
    old = torch.stack((ok.reshape(s["s"], H, P, D), ov.reshape(s["s"], H, P, D)), 1).transpose(2, 3)[:, None]
    x = torch.where(new[:, :, None, :, None, None], x, old).transpose(3, 4)                             # [s, blocks, 2, H, P, D]
    y, scale = _code(x.float(), c["code"])
    to = torch.where(whole, s["tables"].long()[torch.arange(s["s"], device=dev)[:, None], blk.clamp_max(s["max_pages"] - 1)], s["n_pages"])
    s["kv"][to] = _tiled(y[:, :, 0].view(torch.uint8), y[:, :, 1].view(torch.uint8))
    s["scale"][to] = scale.transpose(2, 3)
    # rows of the block that stays open
    tk, tv = _plain_order(s["open"], P, D)
    row = torch.where(new & ~whole[:, :, None], torch.arange(s["s"], device=dev)[:, None, None], s["s"]).reshape(-1)
    o = (p % P).reshape(-1)
    x = x.permute(2, 0, 1, 4, 3, 5).reshape(2, -1, H, D)                                                # rows [s * blocks * P]
    tk.permute(0, 2, 3, 1, 4, 5, 6)[row, o // 16, o % 16] = x[0].unflatten(-1, (D // 64, 4, 16))
    tv.permute(0, 2, 3, 4, 1, 5, 6, 7)[row, o // 16, o % 16 // 4, o % 4] = x[1].unflatten(-1, (D // 64, 4, 16))


def _attend_plain(s):
    P, H, D, c, B = s["P"], s["H"], s["D"], s["case"], s["s"]
    dev = s["kv"].device
    G = s["hq"] // H
    n, cu = s["lens"].long(), s["cu"].long()
    m = cu[1:] - cu[:-1]
    blocks = s["nmax"] // P + 1
    ids = torch.nn.functional.pad(s["tables"], (0, 1))[:, :blocks].clamp_min(0).long()
    kv = s["kv"].view(torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn)
    k, v = _plain_order(kv.view(torch.uint8)[ids].view(kv.dtype), P, D)
    scale = s["scale"][ids][..., None, None, None]                                                      # [B, blocks, H, 2, 1, 1, 1]
    k = (k.float() * scale[:, :, :, 0, ..., None, None]).reshape(B, blocks, H, P, D)
    v = (v.float() * scale[:, :, :, 1, ..., None, None, None]).reshape(B, blocks, H, P, D)
    ok, ov = _plain_order(s["open"][:B], P, D)
    b = torch.arange(B, device=dev)
    k[b, n // P] = ok.reshape(B, H, P, D).float()
    v[b, n // P] = ov.reshape(B, H, P, D).float()
    k = k.transpose(1, 2).reshape(B, H, blocks * P, D)
    v = v.transpose(1, 2).reshape(B, H, blocks * P, D)
    i = torch.arange(s["max_new"], device=dev)
    src = (cu[:-1, None] + i).clamp(0, s["total"] - 1)
    q = s["q"][src].float().reshape(B, -1, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, -1, D)         # rows: head, then query
    z = torch.matmul(q, k.transpose(2, 3)) * s["sm"]
    sees = (n - m)[:, None] + i + 1 if c["causal"] else n[:, None].expand(B, s["max_new"])
    hidden = torch.arange(blocks * P, device=dev) >= torch.minimum(sees, n[:, None])[..., None]          # [B, queries, tokens]
    z = z.reshape(B, H, G, s["max_new"], -1).masked_fill_(hidden[:, None, None], -math.inf)
    top = z.amax(-1, keepdim=True).clamp_min(-1e30)
    z = z.sub_(top).exp_()
    l = z.sum(-1, keepdim=True)
    y = torch.matmul(z.reshape(B, H, -1, z.shape[-1]), v).reshape(B, H, G, s["max_new"], D) / torch.where(l > 0, l, 1.0)
    lse = (top + l.log())[..., 0]
    t = torch.arange(s["total"], device=dev)
    seq = torch.searchsorted(cu[1:], t, right=True)
    at = t - cu[seq]
    s["y"].copy_(y.permute(0, 3, 1, 2, 4)[seq, at].reshape(s["total"], H * G, D))
    s["lse"].copy_(lse.permute(0, 3, 1, 2)[seq, at].reshape(s["total"], H * G))


def _run_own(s):
    from paper_2507_19823_amd import binding as B
    c = s["case"]
    if "shape" not in s:      # the handle that a program keeps: plain sizes
        s["shape"] = B.make_paged_shape(s["s"], c.get("hq", 1), c.get("hkv", 1), s["P"], s["n_pages"], s["max_pages"],
                                        head_dim=c.get("d", 128), elem=c.get("elem", "f16"), code=c.get("code", "int8"))
        if c["kind"] == "attend":
            s["ws"] = torch.empty(B.hca_paged_workspace_bytes(s["shape"], s["total"], s["max_new"]), dtype=torch.uint8, device="cuda")
    if c["kind"] == "map":
        B.hca_paged_map(s["shape"], s["add"], s["lens"], s["lens_out"], s["tables"], s["free"], s["count"], s["count_out"], s["total"],
                        s["start"], s["cu"], s["tok"][0], s["tok"][1], s["tok"][2])
    elif c["kind"] == "store":
        B.hca_paged_store(s["shape"], s["k"], s["k"].stride(0), s["v"], s["v"].stride(0), s["total"], s["start"], s["cu"], s["tables"],
                          s["kv"], s["scale"], s["open"])
    else:
        B.hca_paged_attend(s["shape"], s["q"], s["q"].stride(0), s["cu"], s["total"], s["max_new"], s["lens"], s["nmax"], s["tables"],
                           s["kv"], s["scale"], s["open"], s["sm"], c["causal"], s["y"], s["lse"], s["ws"])


def run(state):
    s = state
    kind = s["case"]["kind"]
    if own:
        _run_own(s)
    else:
        {"map": _map_plain, "store": _store_plain, "attend": _attend_plain}[kind](s)
    if kind == "map":
        return dict(tables=s["tables"], free=s["free"][: s["n_pages"]], lens=s["lens_out"], count=s["count_out"], start=s["start"],
                    cu=s["cu"], tok=s["tok"])
    if kind == "store":
        codes = s["kv"][: s["n_pages"]].view(torch.int8 if s["case"]["code"] == "int8" else torch.float8_e4m3fn)
        return dict(kv=_plain_order(codes, s["P"], s["D"]), scale=s["scale"][: s["n_pages"]],
                    open=_plain_order(s["open"][: s["s"]], s["P"], s["D"]))
    return dict(y=s["y"], lse=s["lse"])


# ---- the definitions, in 64 bits ------------------------------------------------------------------

def _at_key(t, ch, D):
    """Place of (token t, channel ch) in a page's keys."""
    return t // 16 * (16 * D) + ch // 64 * 1024 + ch % 64 // 16 * 256 + t % 16 * 16 + ch % 16


def _at_value(t, ch, D):
    return t // 16 * (16 * D) + ch // 64 * 1024 + t % 16 // 4 * 256 + ch % 16 * 16 + ch % 64 // 16 * 4 + t % 4


def exact(case, seed):
    c = case
    if c["kind"] == "map":
        return None
    s = prepare(case, seed)
    P, H, D = s["P"], s["H"], s["D"]
    n, new = _lens(c)
    tables = s["tables"].tolist()
    ch = torch.arange(D, device="cuda")
    cu = s["cu"].tolist()
    if c["kind"] == "store":
        scale, open_ = s["scale"].double(), s["open"].double()
        for b in range(s["s"]):
            a, t = n[b], new[b]
            for which, (rows, at) in enumerate(((s["k"], _at_key), (s["v"], _at_value))):
                x = rows[cu[b] : cu[b + 1]].double()                                # [t, H, D]
                o = torch.arange(a % P, device="cuda")[:, None]
                x = torch.cat((open_[b, :, which][:, at(o, ch, D)].transpose(0, 1), x))   # from the first token of the open block on
                k = x.shape[0] // P
                if k:
                    amax = x[: k * P].reshape(k, P, H, D).abs().amax((1, 3))
                    ids = torch.tensor(tables[b][a // P : a // P + k], device="cuda")
                    scale[ids, :, which] = (amax / QMAX[c["code"]]).clamp_min(FLOOR)
                left = x.shape[0] - k * P
                o = torch.arange(left, device="cuda")[:, None]
                open_[b, :, which, at(o, ch, D)] = x[k * P :].permute(1, 0, 2)
        return dict(kv=[None, None], scale=scale[: s["n_pages"]], open=_plain_order(open_[: s["s"]], P, D))
    y = torch.zeros(s["total"], s["hq"], D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["total"], s["hq"], dtype=torch.float64, device="cuda")
    G = s["hq"] // H
    kind = torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn
    for b in range(s["s"]):
        a, t = n[b], new[b]
        pos = torch.arange(a, device="cuda")
        page = s["tables"][b].long()[pos // P]
        for h in range(H):
            x = []
            for which, at in enumerate((_at_key, _at_value)):
                place = at((pos % P)[:, None], ch, D)
                w = s["kv"].view(-1)[((page * H + h) * 2 + which)[:, None] * (P * D) + place].view(kind).float().double()
                w *= s["scale"][page, h, which].double()[:, None]
                w[a // P * P :] = s["open"][b, h, which].double()[place[a // P * P :]]
                x.append(w)
            for g in range(G):
                z = s["q"][cu[b] : cu[b + 1], h * G + g].double() @ x[0].T * (1.0 / math.sqrt(D))
                if c["causal"]:
                    z.masked_fill_(pos > (a - t + torch.arange(t, device="cuda"))[:, None], -math.inf)
                lse[cu[b] : cu[b + 1], h * G + g] = torch.logsumexp(z, 1)
                y[cu[b] : cu[b + 1], h * G + g] = torch.softmax(z, 1) @ x[1]
    return dict(y=y, lse=lse)
