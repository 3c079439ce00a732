"""Operators of a paged KV cache held in 8 bits with a scale for each block of tokens and head, and of its pages.

  attend   tree attention over such a cache, a few layers of one step: plan, then layer by layer
  write    a step's own rows quantised behind the prefixes, layer by layer, then the accepted path kept in all layers
  fork     sequences that end are freed, others are continued twice: whole pages shared, the part-filled one copied
  defrag   the pages in use moved together at the front of the pool, tables renumbered

A cache entry is an E4M3 byte and stands for code * scale; K and V of a layer have scales [page][kv head][128 / block], a
page is 128 slots.  Where rows are written, the scale of a block is the smallest power of two 2^e >= 2^-100 that holds
the largest magnitude (amax <= 448 * 2^e); a block that holds entries of the prefix keeps its scale unless the new rows need
a larger one, and then its entries are encoded again.

Sizes are those of the workloads in paper_2603_08899_b200/inputs.py and of the parity tests (32 query heads on 8 kv heads of 128,
trees of 60 nodes with 4 contemplate rows, 16 soft prompts, prefixes of 512 to 16384) or generic ones in between.
"""
import math

import numpy as np
import torch

own = False

PAGE = 128
DEPTH = 64                  # entries of an accepted path
CASE = dict(attend=dict(B=1, Hq=32, Hkv=8, D=128, T=60, C=4, S=16, block=128, L=4, lo=4096, hi=4096),
            write=dict(B=1, Hkv=8, D=128, T=60, C=4, block=64, L=8, lo=500, hi=500),
            fork=dict(B=4, n=2, Hkv=8, D=128, L=4, block=64, eight=True, lo=300, hi=3000),
            defrag=dict(pages=256, used=160, moved=40, Hkv=8, D=128, L=4, block=64, eight=True))


def _case(kind, name=None, **kw):
    c = dict(CASE[kind], kind=kind, **{})
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, plain decoding of single tokens, eight layers: launches and latency
        _case("attend", "decode_one", T=1, C=0, S=0, L=8, lo=2048, hi=2048),
        # a full server decoding single tokens, long and short prefixes: the cache is read once, nothing else counts
        _case("attend", "decode_batch64", B=64, T=1, C=0, S=0, L=2, lo=100, hi=8192, block=64),
        # a few users with short chains of drafts and groups of eight query heads, odd prefixes
        _case("attend", "chain_g8", B=7, Hq=64, T=5, C=1, L=4, lo=37, hi=5001, block=64),
        # head dim 64, a whole tree
        _case("attend", "tree_d64", B=4, D=64, L=4, lo=1500, hi=2500, block=32),
        # one user, a whole tree, prefix 4096
        _case("attend", "tree_one"),
        # a full server, whole trees, ragged prefixes 512..16384
        _case("attend", "tree_batch32", B=32, L=1, lo=512, hi=16384),
        # one user's step written into eight layers
        _case("write", "write_one", lo=4099, hi=4099, block=32),
        # a full server's step, one contemplate row per node, blocks of a page
        _case("write", "write_batch32", B=32, C=60, L=16, block=128, lo=200, hi=1200),
        # two continuations of one small batch
        _case("fork", "fork_two"),
        # a server that continues half of its sequences twice, bf16 pages of 16 layers
        _case("fork", "fork_batch32", B=48, n=24, L=16, eight=False, lo=200, hi=1500),
        # a small pool
        _case("defrag", "defrag_small"),
        # a large pool, a third of the pages in use on the move
        _case("defrag", "defrag_large", pages=1500, used=900, moved=300, L=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "write", "fork", "defrag"])
    block = rng.choice([32, 64, 128])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 4, 8])
    if kind == "attend":
        T = rng.choice([1, 1, _log(rng, 2, 64), 30, 60])
        C = rng.choice([0, min(T, 4), rng.randint(0, T)])
        G = rng.choice([1, 2, 3, 4, 4, 8, 16])
        B = _log(rng, 1, 32)
        hi = _log(rng, 60, 8000)
        L = rng.randint(1, 4)
        keys = B * hi * L
        if keys * (T + C) * G * Hkv * D > 1.2e11:
            L, hi = 1, max(60, int(hi * 1.2e11 / (B * hi * (T + C) * G * Hkv * D)) if B * hi * (T + C) * G * Hkv * D > 1.2e11 else hi)
        return _case(kind, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, T=T, C=C, S=rng.choice([0, 0, 16, rng.randint(1, 128)]), block=block, L=L,
                     lo=rng.choice([hi, max(1, hi // 30), rng.randint(0, 20)]), hi=hi)
    if kind == "write":
        T = rng.choice([1, _log(rng, 2, 64), 60])
        hi = _log(rng, 20, 1200)
        return _case(kind, B=_log(rng, 1, 32), Hkv=Hkv, D=D, T=T, C=rng.randint(0, T), block=block, L=rng.randint(1, 12), lo=rng.randint(0, hi), hi=hi)
    if kind == "fork":
        n = _log(rng, 1, 24)
        return _case(kind, B=n + rng.randint(1, 24), n=n, Hkv=Hkv, D=D, L=rng.randint(1, 12), block=block, eight=rng.random() < 0.6, lo=rng.randint(1, 200),
                     hi=_log(rng, 200, 2000))
    pages = _log(rng, 20, 1400)
    used = rng.randint(pages // 3, pages - 4)
    return _case(kind, pages=pages, used=used, moved=rng.randint(1, min(used, pages - used)), Hkv=Hkv, D=D, L=rng.randint(1, 10), block=block,
                 eight=rng.random() < 0.6)


def _lengths(c, B):
    return [int(round(c["lo"] + (c["hi"] - c["lo"]) * (i + 0.5) / B)) for i in range(B)]


def work(c):
    D, Hkv, L = c["D"], c["Hkv"], c["L"]
    if c["kind"] == "attend":
        R, B = c["T"] + c["C"], c["B"]
        keys = sum(p + R for p in _lengths(c, B))
        scales = 2 * 4 * Hkv * keys / c["block"]
        return {"bytes": L * (2 * keys * Hkv * D + scales + 2 * B * R * c["Hq"] * D * 2 + 2 * c["S"] * Hkv * D), "flops": L * 4.0 * R * c["Hq"] * D * keys / B * B}
    if c["kind"] == "write":
        return {"bytes": L * 2.0 * c["B"] * (c["T"] + c["C"]) * Hkv * D * 3, "flops": 0}
    e = 1 if c["eight"] else 2
    page = 2.0 * L * PAGE * Hkv * D * e
    return {"bytes": 2 * page * (c["n"] if c["kind"] == "fork" else c["moved"]), "flops": 0}


# --------------------------------------------------------------------------- inputs
def _codes(g, shape):
    """E4M3 codes of normal values, 96 to a standard deviation."""
    x = torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda")
    for i in range(shape[0]):                        # a layer at a time: fp32 in between
        x[i] = (torch.randn(shape[1:], generator=g, device="cuda") * 96).clamp_(-448, 448).to(torch.float8_e4m3fn)
    return x


def _scales(g, shape):
    return torch.exp2(torch.randint(-8, -5, shape, generator=g, device="cuda").float())


def _tree(r, B, T, C):
    parent = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        parent[:, i] = i - 1 - r.randint(0, min(i, 5), B)
    owner = np.sort(np.argsort(r.rand(B, T), axis=1)[:, :C], axis=1).astype(np.int32) if C <= T else r.randint(0, T, (B, C)).astype(np.int32)
    return parent, owner


def _tables(r, need, spare=3):
    """Pages of sequences that need so many, in no order, and a few that nobody has."""
    n = int(sum(need)) + spare
    perm, table, at = r.permutation(n), np.full((len(need), max(need) + 2), -1, np.int32), 0
    for b, k in enumerate(need):
        table[b, :k] = perm[at:at + k]
        at += k
    return n, table


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def prepare(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    L, Hkv, D, nb = c["L"], c["Hkv"], c["D"], PAGE // c["block"]
    s = {"case": dict(c)}
    if c["kind"] in ("attend", "write"):
        B, T, C = c["B"], c["T"], c["C"]
        P = r.permutation(_lengths(c, B)).astype(np.int32)
        n, table = _tables(r, [-(-(int(p) + T + C) // PAGE) for p in P])
        parent, owner = _tree(r, B, T, C)
        s.update(P=_dev(P), n_pages=n, table=_dev(table), parent=_dev(parent), owner=_dev(owner), most=int(P.max()) + T + C,
                 k=_codes(g, (L, n * PAGE, Hkv, D)), v=_codes(g, (L, n * PAGE, Hkv, D)), ks=_scales(g, (L, n, Hkv, nb)), vs=_scales(g, (L, n, Hkv, nb)))
    if c["kind"] == "attend":
        S = c["S"]
        s.update(q=torch.randn((L, B, T + C, c["Hq"], D), generator=g, device="cuda").bfloat16())
        s.update(k_soft=_codes(g, (L, S, Hkv, D)), v_soft=_codes(g, (L, S, Hkv, D)), ks_soft=_scales(g, (L, Hkv, nb)), vs_soft=_scales(g, (L, Hkv, nb)))
    if c["kind"] == "write":
        # rows of the size of the cached ones, some of them larger
        rows = [torch.randn((L, B, T + C, Hkv, D), generator=g, device="cuda") * torch.exp2(torch.randint(-2, 2, (L, B, T + C, 1, 1), generator=g, device="cuda"))
                for _ in range(2)]
        a = r.randint(0, min(T, 8), B).astype(np.int32)
        path = np.full((B, DEPTH), -1, np.int32)
        for b in range(B):
            path[b, 0] = 0
            path[b, 1:a[b] + 1] = np.sort(r.permutation(np.arange(1, T))[:a[b]])
        s.update(k_rows=rows[0].bfloat16(), v_rows=rows[1].bfloat16(), a=_dev(a), path=_dev(path))
    if c["kind"] == "fork":
        # rows 0..B-1: sequences, rows B..B+n-1: their continuations, empty at first
        P = r.permutation(_lengths(c, c["B"])).astype(np.int32)
        n, table = _tables(r, [-(-int(p) // PAGE) for p in P], spare=c["n"] + 5)
        table = np.concatenate([table, np.full((c["n"], table.shape[1]), -1, np.int32)])
        src = r.permutation(c["B"])[:c["n"]].astype(np.int32)
        s.update(src=_dev(src), dst=_dev(np.arange(c["B"], c["B"] + c["n"], dtype=np.int32)), length=_dev(P[src]))
    if c["kind"] == "defrag":
        # `moved` of the pages in use lie behind the first `used`; a few rows of tables name them, a tenth twice
        n, used, moved = c["pages"], c["used"], c["moved"]
        ids = np.concatenate([np.sort(r.permutation(used)[:used - moved]), used + np.sort(r.permutation(n - used)[:moved])])
        ids = np.concatenate([r.permutation(ids), r.permutation(ids)[:used // 10]])
        width = max(2, len(ids) // 12)
        table = np.full((-(-len(ids) // width), width + 1), -1, np.int32)
        for i in range(len(table)):
            part = ids[i * width:(i + 1) * width]
            table[i, :len(part)] = part
    if c["kind"] in ("fork", "defrag"):
        ref = np.bincount(table[table >= 0].reshape(-1), minlength=n).astype(np.int32)
        s.update(n_pages=n, table=_dev(table), ref=_dev(ref))
        if c["eight"]:
            s.update(k=_codes(g, (L, n * PAGE, Hkv, D)), v=_codes(g, (L, n * PAGE, Hkv, D)), ks=_scales(g, (L, n, Hkv, nb)), vs=_scales(g, (L, n, Hkv, nb)))
        else:
            s.update(k=torch.randn((L, n * PAGE, Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16),
                     v=torch.randn((L, n * PAGE, Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16))
        if c["kind"] == "defrag":
            s.update(table0=s["table"].clone(), ref0=s["ref"].clone())
    return s


# --------------------------------------------------------------------------- the plain forms
def _sees(s):
    """[B][R][T] the tree rows that a row sees, contemplate rows' own slots apart."""
    c = s["case"]
    B, T, C = c["B"], c["T"], c["C"]
    up = (s["parent"][:, :, None] == torch.arange(T, device="cuda")).float() + torch.eye(T, device="cuda")
    up = up @ up
    up = up @ up
    up = up @ up
    up = (up > 0).float()
    up = up @ up
    up = up @ up
    up = ((up @ up) > 0).float()
    own_nodes = torch.gather(up, 1, s["owner"].long()[:, :, None].expand(B, C, T))
    return torch.cat([up, own_nodes], 1) > 0


def _attend_layer(s, l, sees, pos, page):
    c = s["case"]
    B, R, Hkv, D, S, bl = c["B"], c["T"] + c["C"], c["Hkv"], c["D"], c["S"], c["block"]
    G, N = c["Hq"] // Hkv, pos.numel()
    slot = page * PAGE + pos % PAGE

    def values(codes, scales, soft, soft_scales):
        x = codes.view(torch.uint8)[slot.reshape(-1)].view(torch.float8_e4m3fn).float().view(B, N, Hkv, D)
        x = x * scales[page, :, (pos % PAGE) // bl].view(B, N, Hkv, 1)
        y = soft.float() * soft_scales[:, torch.arange(S, device="cuda") // bl].t()[:, :, None]
        return torch.cat([x, y.expand(B, S, Hkv, D)], 1).transpose(1, 2)
    k = values(s["k"][l], s["ks"][l], s["k_soft"][l], s["ks_soft"][l])
    q = s["q"][l].float().view(B, R, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * R, D)
    w = torch.matmul(q * D ** -0.5, k.transpose(2, 3)).view(B, Hkv, G, R, N + S)
    del k
    w = w.masked_fill_(~sees[:, None, None], -math.inf)
    w = w.sub_(w.amax(-1, keepdim=True)).exp_()
    total = w.sum(-1)
    v = values(s["v"][l], s["vs"][l], s["v_soft"][l], s["vs_soft"][l]).masked_fill_(~sees.any(1)[:, None, :, None], 0)
    o = torch.matmul(w.view(B, Hkv, G * R, N + S), v).view(B, Hkv, G, R, D) / total[..., None]
    return o.permute(0, 3, 1, 2, 4).reshape(B, R, c["Hq"], D).bfloat16()


def _attend(s):
    c = s["case"]
    B, T, C, R, S = c["B"], c["T"], c["C"], c["T"] + c["C"], c["S"]
    pos = torch.arange(s["most"], device="cuda")
    page = s["table"][:, :(s["most"] + PAGE - 1) // PAGE].clamp(min=0).long()[:, pos // PAGE]
    at = pos[None, :] - s["P"][:, None]                                             # [B][N] tree slot, negative: prefix
    rows = torch.arange(R, device="cuda")
    tree = torch.gather(_sees(s), 2, at.clamp(0, T - 1).long()[:, None, :].expand(B, R, -1)) & ((at >= 0) & (at < T))[:, None, :]
    sees = (at < 0)[:, None, :] | tree | ((at[:, None, :] == rows[None, :, None]) & (rows >= T)[None, :, None])
    sees = torch.cat([sees, (rows >= T)[None, :, None].expand(B, R, S)], 2)
    return {"out": [_attend_layer(s, l, sees, pos, page) for l in range(c["L"])]}


def _needed(x):
    """The smallest power of two, 2^-100 at least, that times 448 holds the largest finite magnitude of the last axis."""
    amax = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875), -100).clamp(min=-100)
    return torch.ldexp(torch.ones_like(amax), e)


def _encode(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _place(s, pos):
    """Slot in the pool, and block of the scales, of positions [B][n]."""
    c = s["case"]
    page = torch.gather(s["table"].long(), 1, (pos // PAGE).long())
    return page * PAGE + pos % PAGE, page * (PAGE // c["block"]) + (pos % PAGE) // c["block"]


def _raise(s, codes, flat, need, blocks, keep_to, fresh):
    """Scales of the blocks raised to what the new entries need, kept entries of the block at P encoded again."""
    c = s["case"]
    bl = c["block"]
    new = flat.clone()
    if fresh is not None:
        new[blocks[fresh]] = 0.0
    new.index_reduce_(0, blocks.reshape(-1), need.reshape(-1, c["Hkv"]), "amax")
    pos = (s["P"] // bl * bl)[:, None] + torch.arange(bl, device="cuda")
    keep = pos <= keep_to[:, None]
    slot, block = _place(s, torch.where(keep, pos, s["P"][:, None]))
    slot, block = slot[keep], block[keep]
    codes[slot] = _encode(codes[slot].view(torch.float8_e4m3fn).float() * flat[block][..., None] / new[block][..., None])
    return new


def _write_layer(s, codes, scales, rows):
    c = s["case"]
    B, R, Hkv, D, bl = c["B"], c["T"] + c["C"], c["Hkv"], c["D"], c["block"]
    codes = codes.view(torch.uint8)
    flat = scales.transpose(1, 2).reshape(-1, Hkv)
    # the rows behind the prefix
    pos = s["P"][:, None] + torch.arange(R, device="cuda")
    slot, block = _place(s, pos)
    x = rows.float()
    flat = _raise(s, codes, flat, _needed(x), block, s["P"] - 1, pos // bl * bl >= s["P"][:, None])
    codes[slot] = _encode(x / flat[block][..., None])
    # the accepted path
    K = torch.arange(1, max(2, c["T"]), device="cuda")[None, :].expand(B, -1)
    live = K <= s["a"][:, None]
    src, src_block = _place(s, s["P"][:, None] + torch.where(live, s["path"][:, 1:1 + K.shape[1]], 0))
    dst, dst_block = _place(s, s["P"][:, None] + torch.where(live, K, 0))
    x = codes[src].view(torch.float8_e4m3fn).float() * flat[src_block][..., None]
    need = torch.where(live[..., None], _needed(x), 0.0)
    flat = _raise(s, codes, flat, need, dst_block, s["P"], None)
    codes[dst[live]] = _encode(x / flat[dst_block][..., None])[live]
    scales.copy_(flat.view(-1, PAGE // bl, Hkv).transpose(1, 2))


def _write(s):
    for l in range(s["case"]["L"]):
        _write_layer(s, s["k"][l], s["ks"][l], s["k_rows"][l])
        _write_layer(s, s["v"][l], s["vs"][l], s["v_rows"][l])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "length": s["P"] + s["a"] + 1}


def _move_pages(s, src, dst):
    c = s["case"]
    for name in ("k", "v"):
        x = s[name].view(torch.uint8).view(c["L"], s["n_pages"], -1)
        x[:, dst] = x[:, src]
    if c["eight"]:
        for name in ("ks", "vs"):
            s[name][:, dst] = s[name][:, src]


def _pools(s):
    return {name: s[name] for name in ("k", "v", "ks", "vs") if name in s}


def _fork(s):
    table, ref, src, dst = s["table"], s["ref"], s["src"].long(), s["dst"].long()
    # the continuations of the step before end
    gone = table[dst]
    ref.index_add_(0, gone.clamp(min=0).reshape(-1).long(), -(gone >= 0).int().reshape(-1))
    table[dst] = -1
    # others begin
    full, rest = s["length"] // PAGE, s["length"] % PAGE != 0
    free = torch.sort((ref != 0).int(), stable=True).indices
    new = free[(torch.cumsum(rest, 0) - 1).clamp(min=0)].int()
    j = torch.arange(table.shape[1], device="cuda")
    row = table[src]
    last = torch.gather(row, 1, full.long()[:, None].clamp(max=table.shape[1] - 1))[:, 0]
    row = torch.where(j < full[:, None], row, torch.where((j == full[:, None]) & rest[:, None], new[:, None], -1))
    table[dst] = row
    ref.index_add_(0, row.clamp(min=0).reshape(-1).long(), (row >= 0).int().reshape(-1))
    _move_pages(s, last[rest].long(), new[rest].long())
    return {"table": table, "ref": ref, **_pools(s)}


def _defrag(s):
    table, ref, n = s["table"], s["ref"], s["n_pages"]
    table.copy_(s["table0"])
    ref.copy_(s["ref0"])
    used, ids = ref > 0, torch.arange(n, device="cuda")
    n_used = used.sum()
    src, dst = torch.nonzero(used & (ids >= n_used))[:, 0], torch.nonzero(~used & (ids < n_used))[:, 0]
    new = torch.where(used, ids, -1)
    new[src] = dst
    ref[dst] = ref[src]
    ref[src] = 0
    table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()], -1))
    _move_pages(s, src, dst)
    return {"table": table, "ref": ref, "map": new.int(), "used": n_used.int().reshape(1), **_pools(s)}


# --------------------------------------------------------------------------- the framework's calls
def _handles(s):
    """What a program over this library sets up once: context, dims, workspace, plan, outputs, addresses of the layers."""
    from paper_2603_08899_b200 import binding as cb
    c = s["case"]
    h = {"ctx": cb.confu_create(0)}
    T, C = c.get("T", 1), c.get("C", 0)
    eight = c.get("eight", True)
    dims = cb.make_dims(c.get("B", 1), c.get("Hq", c["Hkv"]), c["Hkv"], c["D"], T, C, c.get("S", 0), cb.FP8_BLOCK if eight else torch.bfloat16)
    h.update(dims=dims)

    def addresses(x):
        return torch.tensor([x[l].data_ptr() for l in range(c["L"])], dtype=torch.int64, device="cuda")
    h.update(k=addresses(s["k"]), v=addresses(s["v"]))
    if eight:
        h.update(ks=addresses(s["ks"]), vs=addresses(s["vs"]))
        cb.confu_set_kv_block_scale_layers(h["ctx"], h["ks"], h["vs"], c["block"])
    if c["kind"] in ("attend", "write"):
        cb.confu_set_paging(h["ctx"], s["table"], s["table"].shape[1])
        h["status"] = torch.zeros(c["B"], dtype=torch.int32, device="cuda")
    if c["kind"] == "attend":
        h["ws"] = torch.empty(cb.confu_workspace_bytes(h["ctx"], dims), dtype=torch.uint8, device="cuda")
        cb.confu_set_workspace(h["ctx"], h["ws"])
        h["plan"] = torch.empty(cb.confu_plan_bytes(h["ctx"], dims), dtype=torch.uint8, device="cuda")
        h["out"] = torch.empty_like(s["q"])
        h["layers"] = [(s["q"][l], s["k"][l], s["v"][l], s["k_soft"][l] if c["S"] else None, s["v_soft"][l] if c["S"] else None, h["out"][l],
                        (s["ks"][l], s["vs"][l], s["ks_soft"][l] if c["S"] else None, s["vs_soft"][l] if c["S"] else None)) for l in range(c["L"])]
    elif c["kind"] == "write":
        h["layers"] = [(s["k_rows"][l], s["v_rows"][l], s["k"][l], s["v"][l], s["ks"][l], s["vs"][l]) for l in range(c["L"])]
        h["length"] = torch.empty_like(s["P"])
    else:
        h["pages"] = cb.make_pages(s["ref"], s["table"])
        h["ws"] = torch.empty(cb.confu_pages_workspace_bytes(s["n_pages"]), dtype=torch.uint8, device="cuda")
        h["status"] = torch.zeros(c.get("n", 1), dtype=torch.int32, device="cuda")
        h["used"] = torch.empty(1, dtype=torch.int32, device="cuda")
        h["map"] = torch.empty(s["n_pages"], dtype=torch.int32, device="cuda")
    return h


def _own(s):
    from paper_2603_08899_b200 import binding as cb
    c = s["case"]
    h = s.get("handles")
    if h is None:
        h = s["handles"] = _handles(s)
    ctx, dims = h["ctx"], h["dims"]
    if c["kind"] == "attend":
        cb.confu_tree_plan(ctx, dims, None, s["P"], s["parent"], s["owner"] if c["C"] else None, h["plan"], h["status"])
        for q, k, v, k_soft, v_soft, out, scales in h["layers"]:
            cb.confu_set_kv_block_scales(ctx, *scales, c["block"])
            cb.confu_tree_attention(ctx, dims, q, k, v, s["n_pages"] * PAGE, None, s["P"], k_soft, v_soft, None, None, h["plan"], out, None, h["status"])
        return {"out": list(h["out"])}
    if c["kind"] == "write":
        for k_rows, v_rows, k, v, ks, vs in h["layers"]:
            cb.confu_set_kv_block_scales(ctx, ks, vs, None, None, c["block"])
            cb.confu_kv_append(ctx, dims, k_rows, v_rows, k, v, None, s["P"])
        cb.confu_kv_compact(ctx, dims, c["L"], h["k"], h["v"], None, s["P"], s["a"], s["path"], h["length"], h["status"])
        return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"], "length": h["length"]}
    if c["kind"] == "fork":
        cb.confu_pages_free(ctx, h["pages"], s["dst"], h["status"])
        cb.confu_pages_fork(ctx, dims, c["L"], h["k"], h["v"], h["pages"], s["src"], s["dst"], s["length"], h["ws"], h["status"])
        return {"table": s["table"], "ref": s["ref"], **_pools(s)}
    s["table"].copy_(s["table0"])
    s["ref"].copy_(s["ref0"])
    cb.confu_pages_compact(ctx, dims, c["L"], h["k"], h["v"], h["pages"], h["map"], h["used"], h["ws"])
    return {"table": s["table"], "ref": s["ref"], "map": h["map"], "used": h["used"], **_pools(s)}


def run(s):
    if own:
        return _own(s)
    return {"attend": _attend, "write": _write, "fork": _fork, "defrag": _defrag}[s["case"]["kind"]](s)


# --------------------------------------------------------------------------- 64 bits, one sequence or page at a time
def _e4m3():
    """The value of every code: sign, 4 bits of exponent (bias 7), 3 of mantissa; 0x7f and 0xff are not numbers."""
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[code] = math.nan if code & 127 == 127 else -x if code >> 7 else x
    return v


def _nearest(x, values):
    """Codes of the nearest E4M3 values, ties to the even code, 448 at most."""
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(values[:127], a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - values[lo], values[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def _exact_attend(c, s):
    val = torch.from_numpy(_e4m3()).cuda()
    R, T, G, bl, outs = c["T"] + c["C"], c["T"], c["Hq"] // c["Hkv"], c["block"], []
    parent, owner, P, table = (s[n].cpu().numpy() for n in ("parent", "owner", "P", "table"))
    for l in range(c["L"]):
        out = torch.zeros((c["B"], R, c["Hq"], c["D"]), dtype=torch.float64, device="cuda")
        for b in range(c["B"]):
            n = int(P[b]) + R
            page = torch.from_numpy(np.repeat(table[b, :-(-n // PAGE)], PAGE)[:n].astype(np.int64)).cuda()
            off = torch.arange(n, device="cuda") % PAGE
            see = np.zeros((R, n + c["S"]), bool)
            see[:, :P[b]] = True
            for i in range(R):
                node = i if i < T else owner[b, i - T]
                see[i, P[b] + i] = True
                while node >= 0:
                    see[i, P[b] + node] = True
                    node = parent[b, node]
                see[i, n:] = i >= T
            see = torch.from_numpy(see).cuda()

            def read(codes, scales, soft, soft_scales, h):
                x = val[codes.view(torch.uint8)[page * PAGE + off, h].long()] * scales[page, h, off // bl].double()[:, None]
                y = val[soft.view(torch.uint8)[:, h].long()] * soft_scales[h, torch.arange(c["S"], device="cuda") // bl].double()[:, None]
                return torch.cat([x, y])
            for h in range(c["Hkv"]):
                k = read(s["k"][l], s["ks"][l], s["k_soft"][l], s["ks_soft"][l], h)
                v = read(s["v"][l], s["vs"][l], s["v_soft"][l], s["vs_soft"][l], h)
                z = s["q"][l][b, :, h * G:(h + 1) * G].double() @ k.t() / math.sqrt(c["D"])          # [R][G][n]
                p = torch.softmax(torch.where(see[:, None], z, -math.inf), -1)
                out[b, :, h * G:(h + 1) * G] = p @ v
        outs.append(out)
    return {"out": outs}


def _exact_write(c, s):
    val, bl, R, nb = _e4m3(), c["block"], c["T"] + c["C"], PAGE // c["block"]
    P, table, a, path = (s[n].cpu().numpy() for n in ("P", "table", "a", "path"))
    found = {}
    for codes_name, scales_name, rows_name in (("k", "ks", "k_rows"), ("v", "vs", "v_rows")):
        codes, scales = s[codes_name].view(torch.uint8).cpu().numpy(), s[scales_name].double().cpu().numpy()
        rows = s[rows_name].double().cpu().numpy()

        def needed(x):                                   # of every head of entries [...][Hkv][D]
            top = np.abs(x).max(axis=tuple(i for i in range(x.ndim) if i != x.ndim - 2))
            return np.array([2.0 ** max(-100, math.ceil(math.log2(t / 448) - 1e-12)) if t > 0 else 2.0 ** -100 for t in top])

        def put(l, b, slots, x, kept, fresh):
            """Entries x [n][Hkv][D] into slots of sequence b; kept: slots that keep their entries."""
            for j in sorted({p // bl for p in slots}):
                page, sub = table[b, j * bl // PAGE], j * bl % PAGE // bl
                mine = [i for i, p in enumerate(slots) if p // bl == j]
                stay = [page * PAGE + p % PAGE for p in kept if p // bl == j]
                was = scales[l, page, :, sub].copy()
                now = needed(x[mine]) if fresh and not stay else np.maximum(was, needed(x[mine]))
                for p in stay:
                    codes[l, p] = _nearest(val[codes[l, p]] * was[:, None] / now[:, None], val)
                codes[l, [page * PAGE + slots[i] % PAGE for i in mine]] = _nearest(x[mine] / now[:, None], val)
                scales[l, page, :, sub] = now
        for l in range(c["L"]):
            for b in range(c["B"]):
                first = int(P[b]) // bl * bl
                put(l, b, [int(P[b]) + i for i in range(R)], rows[l, b], range(first, int(P[b])), True)
                if a[b] > 0:
                    at = [int(P[b]) + int(path[b, i]) for i in range(1, a[b] + 1)]
                    x = np.stack([val[codes[l, table[b, p // PAGE] * PAGE + p % PAGE]] * scales[l, table[b, p // PAGE], :, p % PAGE // bl][:, None] for p in at])
                    put(l, b, [int(P[b]) + i for i in range(1, a[b] + 1)], x, range(first, int(P[b]) + 1), False)
        found[codes_name], found[scales_name] = torch.from_numpy(val[codes]), torch.from_numpy(scales)
    return {**found, "length": torch.from_numpy((P + a + 1).astype(np.int32))}


def _exact_pages(c, s):
    """Copies are the same numbers: the pools with the pages copied one by one."""
    table, ref = s["table"].cpu().numpy(), s["ref"].cpu().numpy()
    if c["kind"] == "fork":
        src, dst, length = (s[n].cpu().numpy() for n in ("src", "dst", "length"))
        pairs, more = [], {}
        for i in range(c["n"]):
            for j in range(-(-int(length[i]) // PAGE)):
                page = table[src[i], j]
                if (j + 1) * PAGE > length[i]:
                    pairs.append((int(page), int(np.flatnonzero(ref == 0)[0])))
                    page = pairs[-1][1]
                table[dst[i], j] = page
                ref[page] += 1
    else:
        n_used = int((ref > 0).sum())
        new = np.where(ref > 0, np.arange(s["n_pages"]), -1).astype(np.int32)
        holes = [p for p in range(n_used) if ref[p] == 0]
        pairs = [(p, holes.pop(0)) for p in range(n_used, s["n_pages"]) if ref[p] > 0]
        for p, q in pairs:
            new[p], ref[q], ref[p] = q, ref[p], 0
        table = np.where(table >= 0, new[np.maximum(table, 0)], -1).astype(np.int32)
        more = {"map": torch.from_numpy(new), "used": torch.tensor([n_used], dtype=torch.int32)}
    found = {}
    for name, x in _pools(s).items():
        pages = x.view(c["L"], s["n_pages"], -1)
        for p, q in pairs:
            pages[:, q] = pages[:, p]
        found[name] = x
    return {"table": torch.from_numpy(table), "ref": torch.from_numpy(ref), **more, **found}


def exact(c, seed):
    s = prepare(c, seed)
    return {"attend": _exact_attend, "write": _exact_write, "fork": _exact_pages, "defrag": _exact_pages}[c["kind"]](c, s)
