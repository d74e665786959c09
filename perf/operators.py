"""The block cache's operators: what is measured of them, and their plain forms.

A decode instance holds the keys and values of its resident blocks in 8 bits
(e4m3, one power-of-two scale for each block and head).  A case is a dict of
plain values; ``kind`` names the operator:

  attend   attention of the sequences' newest tokens over their blocks
           (BlockCache.attend), with the blocks' attention weights on demand;
  store    quantisation of new keys and values into the blocks and the blocks'
           contents read back in 16 bits (BlockCache.store, BlockCache.read);
  evict    every instance keeps its heaviest blocks (Selector.evict);
  reclaim  the sequences' block weights summed over the pages of one instance
           (BlockCache.weigh), and its lightest pages given up.

``own`` is set by whoever measures: false, ``run`` computes the plain forms
with elementary torch operations; true, it calls the library.
"""
import math

import numpy as np
import torch

own = False

UNIT = float(1 << 24)   # page weights: fixed point, 2^-24 of one row's whole attention
F8 = torch.float8_e4m3fn


def _attend(name, seqs, new, ctx, **kw):
    c = dict(kind="attend", seqs=seqs, new=new, ctx=ctx, ragged=True, fresh=False, heads=64, kv_heads=8, dim=128,
             block=512, dtype="bfloat16", shared=0, weights=False)
    c.update(kw)
    return {"name": name, **c} if name else c


def _store(name, seqs, new, ctx, **kw):
    c = dict(kind="store", seqs=seqs, new=new, ctx=ctx, ragged=True, fresh=False, kv_heads=8, dim=128, block=512,
             dtype="bfloat16")
    c.update(kw)
    return {"name": name, **c} if name else c


def _evict(name, segs, entries, **kw):
    c = dict(kind="evict", segs=segs, entries=entries, ragged=True, keep=0.5, newest=0)
    c.update(kw)
    return {"name": name, **c} if name else c


def listed():
    return [
        # the only request of an idle instance, a short chat: pure latency (16-token blocks as in the method's paper)
        _attend("decode-one", 1, 1, 700, block=16),
        # an instance's ordinary batch behind a common system prompt, block weights kept for the eviction
        _attend("decode-batch", 64, 1, 16384, shared=1, weights=True),
        # long documents, one token each: the largest caches
        _attend("decode-long", 8, 1, 131071, dtype="float16", ragged=False),
        # three proposed tokens for each sequence of a small model with an odd head group, odd lengths
        _attend("decode-odd", 37, 3, 5003, heads=15, kv_heads=5, dim=64, block=32, dtype="float16", weights=True),
        # a batch of whole prompts, packed, nothing cached before them
        _attend("prompt-packed", 6, 2777, 2777, fresh=True, block=16),
        # two chunks of long prompts after a long cached prefix, with the blocks' weights
        _attend("prompt-chunk", 2, 1024, 32768, ragged=False, weights=True),
        # one decoded token of every sequence into its open block
        _store("store-token", 64, 1, 16384),
        # the keys and values of arriving prompts
        _store("store-prompt", 16, 16384, 16384, fresh=True, dtype="float16"),
        # a 64-GPU cluster's decode instances halve their resident sets, the newest blocks stay
        _evict("evict-64gpu", 48, 4096, newest=64),
        # a 1,024-GPU cluster's decode instances with 65,536 resident blocks each
        _evict("evict-1024gpu", 768, 65536, ragged=False),
        # one instance under memory pressure: its sequences' weights, then its lightest pages
        dict(name="reclaim", kind="reclaim", seqs=64, blocks=1024, shared=16, keep=0.75),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "prompt", "store", "evict", "reclaim"])
    hq, hk, d = rng.choice([(64, 8, 128), (32, 8, 128), (32, 32, 128), (15, 5, 64), (8, 1, 128), (40, 8, 128),
                            (16, 4, 64), (16, 2, 256), (24, 2, 128)])
    block = rng.choice([16, 32, 64, 128, 512, 512])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16"])
    w = rng.random() < 0.5
    if kind == "decode":
        new = rng.choice([1, 1, 1, 2, 4, 7])
        ctx = _log_int(rng, 16, 131072)
        most = max(1, min(256, (1 << 30) // (ctx * hk * d)))   # at most the largest listed cache
        return _attend(None, _log_int(rng, 1, most), new, max(ctx, new), heads=hq, kv_heads=hk, dim=d, block=block,
                       dtype=dtype, ragged=rng.random() < 0.8, weights=w,
                       shared=rng.choice([0, 0, 1]) if block <= ctx // 16 else 0)
    if kind == "prompt":
        new = _log_int(rng, 9, 4096)
        ctx = new if rng.random() < 0.5 else _log_int(rng, new, 32768)
        most = max(1, min(16, (1 << 22) * 16 // (ctx * new), (1 << 27) // (ctx * hk * d)))
        return _attend(None, _log_int(rng, 1, most), new, ctx, fresh=ctx == new, heads=hq, kv_heads=hk, dim=d,
                       block=block, dtype=dtype, weights=w)
    if kind == "store":
        new = rng.choice([1, 1, _log_int(rng, 2, 16384)])
        most = max(1, min(256, (1 << 27) // (new * hk * d)))
        ctx = _log_int(rng, new, 16384)
        most = max(1, min(most, (1 << 29) // (ctx * hk * d)))
        return _store(None, _log_int(rng, 1, most), new, ctx, fresh=ctx == new, kv_heads=hk, dim=d, block=block,
                      dtype=dtype)
    if kind == "evict":
        n = _log_int(rng, 3, 262144)
        return _evict(None, _log_int(rng, 1, max(1, min(100000, 40000000 // n))), n, ragged=rng.random() < 0.7,
                      keep=rng.choice([0.1, 0.25, 0.5, 0.75, 0.9]), newest=rng.choice([0, 0, 1, 32]))
    blocks = _log_int(rng, 2, 4096)
    return dict(kind="reclaim", seqs=_log_int(rng, 1, 256), blocks=blocks, shared=rng.randint(0, blocks // 2),
                keep=rng.choice([0.25, 0.5, 0.9]))


# ------------------------------------------------------------------ inputs

def _lengths(case):
    """(new tokens, tokens held) of every sequence, the case's own whatever the
    seed; the first has the most of both."""
    r = np.random.RandomState(case["seqs"] * 1000003 + case["new"] * 1009 + case["ctx"])
    n, new, ctx = case["seqs"], case["new"], case["ctx"]
    a, c = np.full(n, new), np.full(n, ctx)
    if case["ragged"]:
        if new > 8:
            a = np.exp(r.uniform(math.log(max(1, new // 16)), math.log(new), n)).astype(np.int64)
        c = np.exp(r.uniform(math.log(max(1, ctx // 32)), math.log(ctx), n)).astype(np.int64)
        a[0], c[0] = new, ctx
        c = np.maximum(c, a)
    return a, a.copy() if case["fresh"] else c


def _pow2(e):
    """2^e in 32 bits by its exponent field (a power function is rounded)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _gen(seed, dev):
    g = torch.Generator(device=dev)
    g.manual_seed(seed * 7919 + 17)
    return g


def _tables(case, held, seed, dev):
    """Block tables [seqs][longest]: pages in random order, the first `shared` blocks common."""
    bt, r = case["block"], np.random.RandomState((seed + 1) % (1 << 32))
    nb = -(-held // bt)
    sh = int(min(case.get("shared", 0), nb.min() - 1))        # every sequence's last block is its own
    width = max(1, int(nb.max()))
    private = int(nb.sum()) - sh * (len(nb) - 1)
    n_pages = private + 3                                     # three that no sequence holds
    order = r.permutation(n_pages)
    table = np.zeros((len(nb), width), np.int64)
    at = sh
    fill = np.zeros(n_pages, np.int64)                        # tokens valid in each page
    for s, k in enumerate(nb):
        table[s, :sh] = order[:sh]
        table[s, sh:k] = order[at:at + k - sh]
        at += int(k) - sh
        fill[table[s, :k]] = bt
        if held[s] % bt:
            fill[table[s, k - 1]] = held[s] % bt
    return (torch.from_numpy(table).to(dev), torch.from_numpy(fill).to(dev), n_pages, width)


def _cache(case, fill, n_pages, g, dev):
    """Blocks as the cache holds them: keys by token, values by dimension in
    tiles of 64 tokens; slots that no token has reached hold NaN."""
    bt, hk, d = case["block"], case["kv_heads"], case["dim"]
    t = min(bt, 64)
    slot = torch.arange(bt, device=dev)
    empty = slot[None, :] >= fill[:, None]
    n = n_pages * hk * bt * d
    k, v = torch.empty(n, dtype=torch.uint8, device=dev), torch.empty(n, dtype=torch.uint8, device=dev)
    for x in (k, v):
        for i in range(0, n, 1 << 28):
            m = min(1 << 28, n - i)
            x[i:i + m] = (torch.randn(m, generator=g, device=dev) * 100).clamp_(-448, 448).to(F8).view(torch.uint8)
    k, v = k.view(n_pages, hk, bt, d), v.view(n_pages, hk, bt // t, d, t)
    k.masked_fill_(empty[:, None, :, None], 0x7F)
    v.masked_fill_(empty.view(n_pages, 1, bt // t, 1, t), 0x7F)
    ks, vs = (_pow2(torch.randint(-9, -5, (n_pages, hk), generator=g, device=dev)) for _ in range(2))
    return k, v, ks, vs


def _off(counts, dev):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)).to(dev)


def _prepare_attend(case, seed):
    dev, dt = torch.device("cuda"), getattr(torch, case["dtype"])
    new, held = _lengths(case)
    g = _gen(seed, dev)
    table, fill, n_pages, width = _tables(case, held, seed, dev)
    k, v, ks, vs = _cache(case, fill, n_pages, g, dev)
    q = torch.randn((int(new.sum()), case["heads"], case["dim"]), generator=g, device=dev).mul_(2).to(dt)
    return dict(case=case, k=k, v=v, ks=ks, vs=vs, q=q, tok_off=_off(new, dev), table=table.to(torch.int32),
                held=torch.from_numpy(held.astype(np.int32)).to(dev), most=int(new.max()), scale=case["dim"] ** -0.5)


def _prepare_store(case, seed):
    dev, dt = torch.device("cuda"), getattr(torch, case["dtype"])
    hk, d, bt = case["kv_heads"], case["dim"], case["block"]
    new, held = _lengths(case)
    g = _gen(seed, dev)
    table, fill, n_pages, width = _tables(case, held, seed, dev)
    k, v, ks, vs = _cache(case, fill, n_pages, g, dev)
    n = int(new.sum())
    # slices of one product's rows [queries | keys | values], as a layer hands them over
    kv = torch.randn((n, 2 * hk, d), generator=g, device=dev)
    kv *= torch.exp(0.5 * torch.randn((n, 2 * hk, 1), generator=g, device=dev))
    kv = kv.to(dt)
    first = (held - new) // bt * bt                           # the blocks that the new tokens touch, whole
    back = held - first
    return dict(case=case, k=k, v=v, ks=ks, vs=vs, new_k=kv[:, :hk], new_v=kv[:, hk:], tok_off=_off(new, dev),
                table=table.to(torch.int32), held=torch.from_numpy(held.astype(np.int32)).to(dev), most=int(new.max()),
                back_off=_off(back, dev), back_n=int(back.sum()), back_most=int(back.max()))


def _entries(case):
    """Resident blocks of every instance."""
    n = np.full(case["segs"], case["entries"])
    if case["ragged"]:
        r = np.random.RandomState(case["segs"] * 1009 + case["entries"])
        n = np.exp(r.uniform(0, math.log(case["entries"] + 1), case["segs"])).astype(np.int64)
        n[0] = case["entries"]
    return n


def _held_by(case):
    """Blocks of every sequence."""
    r = np.random.RandomState(case["seqs"] * 1009 + case["blocks"])
    nb = np.exp(r.uniform(math.log(max(1, case["blocks"] // 8)), math.log(case["blocks"]), case["seqs"])).astype(np.int64)
    nb[0] = case["blocks"]
    return nb


def _prepare_evict(case, seed):
    dev = torch.device("cuda")
    n = _entries(case)
    g = _gen(seed, dev)
    total = int(n.sum())
    # heavy-tailed weights of a few significant digits (many equal ones), a tenth never attended
    w = torch.exp(torch.randn(total, generator=g, device=dev) * 2 + 8).to(torch.int64) << 12
    w[torch.rand(total, generator=g, device=dev) < 0.1] = 0
    h = torch.randint(1, 1 << 62, (total,), generator=g, device=dev)
    keep = np.ceil(n * case["keep"]).astype(np.int64)
    return dict(case=case, off=_off(n, dev), weight=w, hashes=h, keep=torch.from_numpy(keep.astype(np.int32)).to(dev),
                n_keep=int(keep.sum()), newest=case["newest"])


def _prepare_reclaim(case, seed):
    dev = torch.device("cuda")
    nb = _held_by(case)
    held = nb * 16 - np.random.RandomState(seed % (1 << 32)).randint(0, 16, case["seqs"])
    g = _gen(seed, dev)
    table, fill, n_pages, width = _tables(dict(block=16, shared=case["shared"]), held, seed, dev)
    bw = torch.exp(torch.randn((case["seqs"], width), generator=g, device=dev) * 1.5 - 2)   # of one layer and step
    h = torch.randint(1, 1 << 62, (n_pages,), generator=g, device=dev)
    keep = max(1, int(case["keep"] * n_pages))
    return dict(case=case, table=table.to(torch.int32), held=torch.from_numpy(held.astype(np.int32)).to(dev), bw=bw,
                n_pages=n_pages, hashes=h, off=_off([n_pages], dev), n_keep=keep,
                keep=torch.full((1,), keep, dtype=torch.int32, device=dev),
                page_weight=torch.zeros(n_pages, dtype=torch.int64, device=dev),
                tok_off=_off(np.zeros(case["seqs"], np.int64), dev))


def prepare(case, seed):
    return {"attend": _prepare_attend, "store": _prepare_store, "evict": _prepare_evict,
            "reclaim": _prepare_reclaim}[case["kind"]](case, seed)


# ------------------------------------------------------------------ plain forms

def _blocks(x, scale, table, tiles):
    """Keys or values [seqs, kv heads, tokens, dim] of every table's pages, in 32 bits."""
    y = x[table]                                              # [S, nb, Hkv, bt, D] or [S, nb, Hkv, bt / T, D, T]
    y = y.view(F8).float()
    if tiles:
        y = y.transpose(-1, -2).flatten(3, 4)
    y = y * scale[table][..., None, None]
    return y.transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c = s["case"]
    S, hk, g, d, mn = c["seqs"], c["kv_heads"], c["heads"] // c["kv_heads"], c["dim"], s["most"]
    q, off, held, table = s["q"], s["tok_off"], s["held"].long(), s["table"].long()
    n = off[1:] - off[:-1]
    k, v = _blocks(s["k"], s["ks"], table, False), _blocks(s["v"], s["vs"], table, True)
    tok = torch.arange(k.shape[2], device=q.device)
    v = torch.where((tok[None, :] < held[:, None])[:, None, :, None], v, torch.zeros((), device=q.device))
    j = torch.arange(mn, device=q.device)
    rows = (off[:-1, None] + j).clamp(max=q.shape[0] - 1)
    qp = q[rows].float().view(S, mn, hk, g, d).permute(0, 2, 1, 3, 4).reshape(S, hk, mn * g, d)
    sc = torch.matmul(qp, k.transpose(-1, -2).contiguous()) * s["scale"]
    last = held[:, None] - n[:, None] + j                     # the last token that row j of a sequence sees
    last = torch.where(j < n[:, None], last, -1)
    seen = (tok <= last[..., None])[:, None, :, None, :]      # [S, 1, mn, 1, tokens]
    sc = sc.view(S, hk, mn, g, -1).masked_fill_(~seen, -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = sc.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    p /= torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p.view(S, hk, mn * g, -1), v).view(S, hk, mn, g, d).transpose(1, 2).reshape(S, mn, hk * g, d)
    row = torch.arange(q.shape[0], device=q.device)
    seq = torch.searchsorted(off[1:].contiguous(), row, right=True)
    out = [o[seq, row - off[seq]].to(q.dtype)]
    if c["weights"]:
        out.append(p.sum((1, 2, 3), dtype=torch.float64).view(S, table.shape[1], -1).sum(-1).float())
    return out


def _plain_store(s):
    c = s["case"]
    bt = c["block"]
    off, back, held, table = s["tok_off"], s["back_off"], s["held"].long(), s["table"].long()
    row = torch.arange(s["back_n"], device=off.device)
    seq = torch.searchsorted(back[1:].contiguous(), row, right=True)
    pos = held[seq] - (back[seq + 1] - row)                   # the row's token in its sequence
    page, slot = table[seq, pos // bt], pos % bt
    fresh = pos - (held - (off[1:] - off[:-1]))[seq]          # the new token that the row is, or below zero
    new = torch.where(fresh >= 0, off[seq] + fresh, 0)
    is_new = (fresh >= 0)[:, None, None]
    out = []
    for old, scale, x, t in ((s["k"], s["ks"], s["new_k"], 0), (s["v"], s["vs"], s["new_v"], min(bt, 64))):
        x = x[new].float()
        was = old[page, :, slot] if not t else old[page, :, slot // t, :, slot % t]
        sc = scale[page]
        amax = torch.where(is_new, x, 0.0).abs().amax(-1)
        block = torch.zeros_like(scale).index_reduce_(0, page, amax, "amax", include_self=True)
        m, e = torch.frexp(block)                             # block = m 2^e, m in [1/2, 1); 448 = 0.875 * 2^9
        e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-126)
        need = _pow2(e)[page]
        begun = torch.zeros(scale.shape[0], device=off.device).index_reduce_(0, page, (fresh < 0).float(), "amax", include_self=True)[page]
        now = torch.where(begun[:, None] > 0, torch.maximum(sc, need), need)[..., None]
        y = torch.where(is_new, x, was.view(F8).float() * sc[..., None])
        out.append(((y / now).to(F8).float() * now).to(s["new_k"].dtype))
    return out


def _plain_keep(off, weight, hashes, keep, newest, n_keep):
    n = weight.numel()
    row = torch.arange(n, device=off.device)
    seg = torch.searchsorted(off[1:].contiguous(), row, right=True)
    size = off[1:] - off[:-1]
    keep = torch.minimum(keep.long(), size)
    if newest:
        pinned = row >= (off[1:] - torch.clamp(keep, max=newest))[seg]
        weight = torch.where(pinned, torch.full_like(weight, (1 << 63) - 1), weight)
    order = torch.sort(weight, descending=True, stable=True).indices
    order = order[torch.sort(seg[order], stable=True).indices]
    stays = torch.empty(n, dtype=torch.bool, device=off.device)
    stays[order] = row - off[seg] < keep[seg]                 # `order` goes segment by segment, as the rows do
    at = torch.sort(~stays, stable=True).indices[:n_keep]
    out_off = torch.zeros_like(off)
    out_off[1:] = torch.cumsum(keep, 0)
    return [out_off, (at - off[seg[at]]).to(torch.int32), hashes[at]]


def _plain_reclaim(s):
    table, held, bw = s["table"].long(), s["held"].long(), s["bw"]
    block = torch.arange(table.shape[1], device=table.device)
    has = block < ((held + 15) // 16)[:, None]
    add = torch.where(has, torch.round(bw.double() * UNIT).long(), 0)
    pw = torch.zeros(s["n_pages"], dtype=torch.int64, device=table.device)
    pw.index_add_(0, table.flatten(), add.flatten())
    return [pw] + _plain_keep(s["off"], pw, s["hashes"], s["keep"], 0, s["n_keep"])


# ------------------------------------------------------------------ the library's calls

def _selector(s):
    from paper_2606_03910_amd import netkv
    if "sel" not in s:
        s["sel"] = _selector.kept = getattr(_selector, "kept", None) or netkv.Selector(0)
    return s["sel"]


def _own_cache(s, off, n, most):
    """The instance's cache and the batch's sequences, as its program keeps them from layer to layer."""
    from paper_2606_03910_amd import netkv
    cache = netkv.BlockCache(_selector(s), s["k"].view(-1), s["v"].view(-1), s["ks"].view(-1), s["vs"].view(-1),
                             s["case"]["kv_heads"], s["case"]["dim"], s["case"]["block"])
    return cache, _sequences(s, off, n, most)


def _sequences(s, off, n, most):
    from paper_2606_03910_amd import netkv
    return netkv.Sequences(off.view(torch.uint64), s["held"].view(torch.uint32), s["table"].view(torch.uint32), n, most)


def _own_attend(s):
    if "plan" not in s:
        s["plan"] = _own_cache(s, s["tok_off"], s["q"].shape[0], s["most"])
    cache, seqs = s["plan"]
    if s["case"]["weights"]:
        return list(cache.attend(seqs, s["q"], s["scale"], weights=True))
    return [cache.attend(seqs, s["q"], s["scale"])]


def _own_store(s):
    if "plan" not in s:
        s["plan"] = _own_cache(s, s["tok_off"], s["new_k"].shape[0], s["most"])
        s["back"] = _sequences(s, s["back_off"], s["back_n"], s["back_most"])
    cache, seqs = s["plan"]
    cache.store(seqs, s["new_k"], s["new_v"])
    return list(cache.read(s["back"], s["new_k"].dtype))


def _kept(r):
    return [r["hash_off"].view(torch.int64), r["pos"].view(torch.int32), r["hashes"].view(torch.int64)]


def _own_evict(s):
    return _kept(_selector(s).evict(dict(hash_off=s["off"].view(torch.uint64), hashes=s["hashes"].view(torch.uint64)),
                                    s["weight"].view(torch.uint64), s["keep"].view(torch.uint32), s["newest"], s["n_keep"]))


def _own_reclaim(s):
    sel = _selector(s)
    from paper_2606_03910_amd import netkv
    if "plan" not in s:
        s["plan"] = _sequences(s, s["tok_off"], 0, 0)
    s["page_weight"].zero_()
    netkv.netkv_kv_weigh(sel.h, s["plan"], 16, s["bw"], s["page_weight"].view(torch.uint64), sel.device)
    r = sel.evict(dict(hash_off=s["off"].view(torch.uint64), hashes=s["hashes"].view(torch.uint64)),
                  s["page_weight"].view(torch.uint64), s["keep"].view(torch.uint32), 0, s["n_keep"])
    return [s["page_weight"]] + _kept(r)


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"attend": _own_attend, "store": _own_store, "evict": _own_evict, "reclaim": _own_reclaim}[kind](state)
    if kind == "attend":
        return _plain_attend(state)
    if kind == "store":
        return _plain_store(state)
    if kind == "evict":
        return _plain_keep(state["off"], state["weight"], state["hashes"], state["keep"], state["newest"], state["n_keep"])
    return _plain_reclaim(state)


# ------------------------------------------------------------------ work

def work(case):
    """Bytes that have to be read and written once, and operations, of one pass."""
    kind = case["kind"]
    if kind == "evict":
        n = _entries(case)
        kept = int(np.ceil(n * case["keep"]).sum())
        return {"bytes": int(8 * n.sum() + (8 + 12) * kept + 20 * len(n)), "flops": int(n.sum())}
    if kind == "reclaim":
        nb = _held_by(case)
        pages = int(nb.sum()) - (case["seqs"] - 1) * int(min(case["shared"], nb.min() - 1))
        return {"bytes": int(8 * nb.sum() + pages * (8 + case["keep"] * 20)), "flops": int(nb.sum() + pages)}
    new, held = _lengths(case)
    hk, d = case["kv_heads"], case["dim"]
    if kind == "store":
        back = held - (held - new) // case["block"] * case["block"]
        return {"bytes": int(hk * d * 2 * (new.sum() * (2 + 1) + back.sum() * (1 + 2))), "flops": int(4 * hk * d * back.sum())}
    sh = int(min(case["shared"], (-(-held // case["block"])).min() - 1)) * case["block"]
    tokens = int(held.sum()) - sh * (case["seqs"] - 1)
    seen = int((new * held - new * (new - 1) // 2).sum())
    b = 2 * tokens * hk * d + 4 * int(new.sum()) * case["heads"] * d
    if case["weights"]:
        b += 4 * int((-(-held // case["block"])).sum())
    return {"bytes": int(b), "flops": 4 * d * case["heads"] * seen}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The operators' definitions in 64 bits, sequence by sequence."""
    kind = case["kind"]
    if kind == "attend":
        return _exact_attend(prepare(case, seed))
    if kind == "store":
        return _exact_store(prepare(case, seed))
    return None   # whole numbers only: equal, or wrong


def _two_to(e):
    """2^e in 64 bits, exactly."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _values(x):
    """What e4m3 bytes stand for, from the format's definition."""
    x = x.to(torch.int64)
    e, m = (x >> 3) & 15, x & 7
    mag = torch.where(e == 0, m.double() / 8 * 2.0 ** -6, (1 + m.double() / 8) * _two_to(e - 7))
    mag = torch.where((x & 127) == 127, math.nan, mag)
    return torch.where(x >= 128, -mag, mag)


def _held_blocks(s, seq, h, n):
    """Keys and values [n, dim] of a sequence's first n tokens, one head."""
    bt = s["case"]["block"]
    pages = s["table"][seq, :-(-n // bt)].long()
    k = _values(s["k"][pages, h]) * s["ks"][pages, h].double()[:, None, None]
    v = _values(s["v"][pages, h]) * s["vs"][pages, h].double()[:, None, None, None]
    return k.reshape(-1, k.shape[-1])[:n], v.permute(0, 1, 3, 2).reshape(-1, v.shape[2])[:n]


def _exact_attend(s):
    c = s["case"]
    g, bt = c["heads"] // c["kv_heads"], c["block"]
    off, held = s["tok_off"].tolist(), s["held"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    w = torch.zeros(s["table"].shape, dtype=torch.float64, device=s["q"].device)
    for i, n in enumerate(held):
        a = off[i + 1] - off[i]
        for h in range(c["kv_heads"]):
            k, v = _held_blocks(s, i, h, n)
            k = k.T.contiguous()
            total = torch.zeros(n, dtype=torch.float64, device=out.device)
            for r in range(0, a, 512):
                q = s["q"][off[i] + r:off[i] + min(r + 512, a), h * g:(h + 1) * g].double()
                z = torch.matmul(q.reshape(-1, c["dim"]), k) * s["scale"]
                z = z.view(q.shape[0], g, n)
                late = torch.arange(n, device=out.device)[None, :] > n - a + r + torch.arange(q.shape[0], device=out.device)[:, None]
                z = torch.where(late[:, None, :], -math.inf, z)
                p = torch.exp(z - torch.logsumexp(z, -1, keepdim=True))
                out[off[i] + r:off[i] + r + q.shape[0], h * g:(h + 1) * g] = torch.matmul(p, v)
                total += p.sum((0, 1))
            pad = torch.zeros(-(-n // bt) * bt, dtype=torch.float64, device=out.device)
            pad[:n] = total
            w[i, :-(-n // bt)] += pad.view(-1, bt).sum(1)
    return [out, w] if c["weights"] else [out]


def _round_e4m3(x):
    """To the nearest multiple of the format's step at x, ties to the even one."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60))).clamp(min=-6)
    step = _two_to(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_store(s):
    c = s["case"]
    bt, hk, d = c["block"], c["kv_heads"], c["dim"]
    off, back, held = s["tok_off"].tolist(), s["back_off"].tolist(), s["held"].tolist()
    outs = []
    for name, x, sc in (("k", s["new_k"], s["ks"]), ("v", s["new_v"], s["vs"])):
        out = torch.zeros((s["back_n"], hk, d), dtype=torch.float64, device=x.device)
        for i, n in enumerate(held):
            a = off[i + 1] - off[i]
            was = n - a                                       # tokens before the call
            start = was // bt * bt
            m = n - start
            val = torch.zeros((-(-m // bt) * bt, hk, d), dtype=torch.float64, device=x.device)
            val[was - start:m] = x[off[i]:off[i + 1]].double()
            blocks = val.view(-1, bt, hk, d)
            amax = blocks.abs().amax((1, 3))
            need = _two_to(torch.ceil(torch.log2(amax / 448)).clamp(min=-126))
            need = torch.where((need > 2.0 ** -126) & (need * 224 >= amax), need / 2, need)   # log2 is rounded
            need = torch.where(need * 448 < amax, need * 2, need)
            if was > start:
                page = int(s["table"][i, start // bt])
                raw = _values(s[name][page])
                raw = raw if name == "k" else raw.permute(0, 1, 3, 2).reshape(hk, bt, d)
                blocks[0, :was - start] = (raw[:, :was - start] * sc[page].double()[:, None, None]).transpose(0, 1)
                need[0] = torch.maximum(need[0], sc[page].double())
            q = _round_e4m3(blocks / need[:, None, :, None]) * need[:, None, :, None]
            out[back[i]:back[i + 1]] = q.view(-1, hk, d)[:m]
        outs.append(out)
    return outs
