"""What the second set of attention-side operators is measured on: rotary positions with several axes, the
fused norm + rotation + write into a cache held in 4 bits, attention over that cache, and the life of a
cache's pages (forking, freeing, compacting).

A 4-bit cache holds E2M1 codes, two to a byte with the even element in the low four bits, and an E4M3 scale for every 16
elements of a head; both stand for code * scale * k_scale (v_scale).  Widths and head counts are those of the library's workloads
(5120+1024 and 8192+1024 columns, heads of 128) and a few generic ones; token counts go from one decode step to a prompt.
"""
import math

import torch

own = False

BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
EPS = 1e-6
KS, VS = 2.0 ** -8, 2.0 ** -7     # what a unit of K, of V in the 4-bit cache stands for
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # E2M1's magnitudes by code; bit 3 is the sign


# ---- cases ------------------------------------------------------------------------------------------

def _axes(tokens, dq, dk, head_dim=128, rot_dim=128, layout="half", assign="blocks", inverse=False, dtype="bf16"):
    return dict(op="axes", tokens=tokens, dq=dq, dk=dk, head_dim=head_dim, rot_dim=rot_dim, layout=layout, assign=assign,
                inverse=inverse, dtype=dtype)


def _append(tokens, dq, dk, head_dim=128, rot_dim=128, layout="half", norm="layerwise", page=16, axes=False):
    return dict(op="append", tokens=tokens, dq=dq, dk=dk, head_dim=head_dim, rot_dim=rot_dim, layout=layout, norm=norm,
                page=page, axes=axes)


def _attn(seqs, new, ctx, heads_q, heads_kv, head_dim=128, page=16, window=0, ragged=True):
    return dict(op="attn", seqs=seqs, new=new, ctx=ctx, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim, page=page,
                window=window, ragged=ragged)


def _fork(forks, ctx, layers, heads=8, head_dim=128, page=16, parents=1):
    return dict(op="fork", forks=forks, ctx=ctx, layers=layers, heads=heads, head_dim=head_dim, page=page, parents=parents)


def _compact(pages, rows, layers, heads=8, head_dim=128, page=16, live=0.6):
    return dict(op="compact", pages=pages, rows=rows, layers=layers, heads=heads, head_dim=head_dim, page=page, live=live)


def listed():
    return [
        # one decode step of a batch of 64 with time, height and width positions: a small call, latency counts
        dict(_axes(64, 5120, 1024), name="axes_decode"),
        # the backward pass of a training step over text and image patches, the axes dealt to the pairs in turn
        dict(_axes(16384, 5120, 1024, assign="turns", inverse=True), name="axes_backward"),
        # the cache write of one decode step
        dict(_append(64, 5120, 1024), name="append_decode"),
        # the cache write of a prompt, the norm over whole rows
        dict(_append(16384, 5120, 1024), name="append_prefill"),
        # one decode step of a few short sequences, five query heads to a key head
        dict(_attn(8, 1, 1000, 40, 8), name="attn_decode_small"),
        # one decode step of a full serving batch
        dict(_attn(64, 1, 8192, 64, 8), name="attn_decode"),
        # the same with fewer and longer sequences, pages of 64
        dict(_attn(16, 1, 32000, 64, 8, page=64), name="attn_decode_long"),
        # chunks of new tokens of four sequences next to what is in the cache
        dict(_attn(4, 512, 8192, 40, 8), name="attn_chunk"),
        # eight samples of one prompt dropped and drawn again, the cache of one layer
        dict(_fork(8, 1000, 1), name="fork_small"),
        # a beam step of a batch over all layers: every row forked anew from one of 32 parents
        dict(_fork(96, 2045, 32, parents=32), name="fork_large"),
        # a small pool of one layer after some sequences have ended
        dict(_compact(512, 16, 1), name="compact_small"),
        # the FP8 pool of eight layers packed before its tail is handed back
        dict(_compact(4096, 96, 8), name="compact_large"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["axes", "append", "attn", "attn", "attn", "fork", "compact"])
    head_dim = rng.choice([64, 96, 128, 128])
    layout = rng.choice(["half", "interleaved"])
    rot_dim = rng.choice([head_dim, head_dim // 2])
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8])
    if op == "axes":
        return _axes(_log(rng, 1, 12000), hkv * group * head_dim, hkv * head_dim, head_dim, rot_dim, layout,
                     rng.choice(["blocks", "turns"]), rng.random() < 0.5, rng.choice(["bf16", "e4m3"]))
    if op == "append":
        return _append(_log(rng, 1, 12000), hkv * group * head_dim, hkv * head_dim, head_dim, rot_dim, layout,
                       rng.choice(["layerwise", "headwise"]), rng.choice([16, 24, 64]), rng.random() < 0.5)
    if op == "fork":
        forks = _log(rng, 1, 96)
        return _fork(forks, _log(rng, 1, 2048), rng.randint(1, 16), hkv, head_dim, rng.choice([16, 24, 64]), rng.randint(1, forks))
    if op == "compact":
        return _compact(_log(rng, 64, 4096), _log(rng, 1, 64), rng.randint(1, 8), hkv, head_dim, rng.choice([8, 16]), rng.uniform(0.05, 0.95))
    kind = rng.choice(["decode", "decode", "verify", "chunk"])
    seqs = _log(rng, 1, 64) if kind != "chunk" else _log(rng, 1, 8)
    new = 1 if kind == "decode" else rng.randint(2, 17) if kind == "verify" else _log(rng, 33, 1024)
    ctx = new + _log(rng, 1, 8192)
    seqs = max(1, min(seqs, 600_000_000 // (hkv * group * new * ctx)))   # no more pairs than the listed chunks have
    return _attn(seqs, new, ctx, hkv * group, hkv, head_dim, rng.choice([16, 24, 64, 128]), rng.choice([0, 0, 1024]), rng.random() < 0.7)


# ---- inputs -----------------------------------------------------------------------------------------

def _kv_lens(c):
    """Keys per sequence, the new tokens among them; a ragged batch spreads them over the upper three quarters."""
    old = c["ctx"] - c["new"]
    if not c["ragged"]:
        return [c["ctx"]] * c["seqs"]
    return [c["new"] + min(old, 1 + int(old * (0.25 + 0.75 * ((i + 1) * 0.6180339887 % 1.0)))) for i in range(c["seqs"])]


def _new_lens(c):
    """New tokens per sequence; in a ragged batch of chunks every third one is shorter."""
    return [max(1, c["new"] // 3) if c["ragged"] and i % 3 == 2 else c["new"] for i in range(c["seqs"])]


def _normal(g, shape, dtype, sigma=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype is F8 else dtype).mul_(sigma)
    return x.to(dtype)


def _place(tokens, g):
    """Positions [3, tokens] (time, height, width) of text with images of 24 x 32 patches between: text moves all three on
    together, a patch stands at its row and column."""
    t = torch.arange(tokens, device="cuda")
    first = torch.randint(0, 4096, (1,), generator=g, device="cuda")
    image, at = t // 1024, t % 1024                 # 768 patches, then 256 tokens of text
    base = first + image * (32 + 256)
    patch = at < 768
    text = base + 32 + at - 768
    return torch.stack((torch.where(patch, base, text), torch.where(patch, base + at // 32, text),
                        torch.where(patch, base + at % 32, text)))


def _axis_of_pair(c):
    """Which axis turns each pair: time first and then height and width in blocks (2 : 3 : 3), or the three in turn."""
    n = c["rot_dim"] // 2
    i = torch.arange(n)
    a = n // 4
    b = a + (n - a) // 2
    axis = (i >= a).long() + (i >= b).long() if c.get("assign", "blocks") == "blocks" else i % 3
    return axis.to(torch.uint8).cuda()


def _pool(g, blocks):
    """Blocks of 16 normal values as a 4-bit cache holds them, chosen again and again: codes as int64 [blocks], scales as bytes."""
    x = torch.randn((65536, 16), generator=g, device="cuda")
    code, scale = _quantise(x, KS)
    byte = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8)
    pick = torch.randint(0, 65536, (blocks,), generator=g, device="cuda", dtype=torch.int32)
    return byte.view(torch.int64).view(-1)[pick], scale.view(torch.uint8).view(-1)[pick]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    D = c.get("head_dim")
    if c["op"] in ("axes", "append"):
        T, dq, dk = c["tokens"], c["dq"], c["dk"]
        s["inv_freq"] = (10000.0 ** (-2.0 * torch.arange(c["rot_dim"] // 2, dtype=torch.float64) / c["rot_dim"])).cuda()
        if c["op"] == "axes" or c["axes"]:
            s["positions"], s["axis"] = _place(T, g).contiguous(), _axis_of_pair(c)
        else:
            s["positions"], s["axis"] = torch.randint(0, 32768, (1,), generator=g, device="cuda") + torch.arange(T, device="cuda"), None
    if c["op"] == "axes":
        dt = F8 if c["dtype"] == "e4m3" else BF16
        s["q"], s["k"] = _normal(g, (T, dq), dt), _normal(g, (T, dk), dt)
    elif c["op"] == "append":
        qkv = _normal(g, (T, dq + 2 * dk), BF16)       # the fused projection's output
        s["q"], s["k"], s["v"] = qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:]
        s["gamma_q"] = (torch.rand(dq, generator=g, device="cuda") + 0.5).to(BF16)
        s["gamma_k"] = (torch.rand(dk, generator=g, device="cuda") + 0.5).to(BF16)
        page, heads = c["page"], dk // D
        pages = T // page + 2 if T > 256 else T        # a prompt fills pages; a decode step has one sequence per token
        order = torch.randperm(pages, generator=g, device="cuda")
        t = torch.arange(T, device="cuda")
        s["slots"] = (order[t // page] * page + t % page if T > 256
                      else order * page + torch.randint(0, page, (T,), generator=g, device="cuda"))
        # both sides of the pool, a page's heads one after the other; seen as [page, token, head, d]
        codes, scales = _pool(g, 2 * pages * heads * page * D // 16)
        s["codes"] = codes.view(torch.uint8).view(2, pages, heads, page, D // 2).transpose(2, 3)
        s["scales"] = scales.view(F8).view(2, pages, heads, page, D // 16).transpose(2, 3)
        # what the codes' bytes stand for, to hand the cache's values back
        low = torch.arange(256) % 16
        high = torch.arange(256) // 16
        value = torch.tensor(STEPS + tuple(-v for v in STEPS))
        s["table"] = torch.stack((value[low], value[high]), 1).to(F8).view(torch.int16).view(-1).cuda()
    elif c["op"] == "attn":
        page = c["page"]
        kv, new = _kv_lens(c), _new_lens(c)
        need = [-(-n // page) for n in kv]
        pages, cols = sum(need) + 3, -(-c["ctx"] // page)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        row = torch.arange(cols, device="cuda")[None, :]
        at = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1, None] + row
        s["block_table"] = torch.where(row < torch.tensor(need, device="cuda")[:, None], order[at.clamp(max=pages - 1)], 0).to(torch.int32)
        s["kv_lens"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
        s["q_starts"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
        s["q"] = _normal(g, (sum(new), c["heads_q"] * D), BF16)   # normalised and rotated queries
        codes, scales = _pool(g, 2 * pages * c["heads_kv"] * page * D // 16)
        s["codes"] = codes.view(torch.uint8).view(2, pages, c["heads_kv"], page, D // 2).transpose(2, 3)
        s["scales"] = scales.view(F8).view(2, pages, c["heads_kv"], page, D // 16).transpose(2, 3)
    elif c["op"] == "fork":
        # parents' rows hold their sequences, the forks' rows are empty; some pages more than are wanted, in no order
        n, P, page = c["forks"], c["parents"], c["page"]
        lens = [max(1, c["ctx"] - (7 * i) % max(1, c["ctx"] // 4)) for i in range(P)]
        need = [-(-v // page) for v in lens]
        cols, pages = max(need) + 1, sum(need) + n + 5
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        row = torch.arange(cols, device="cuda")[None, :]
        at = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1, None] + row
        there = row < torch.tensor(need, device="cuda")[:, None]
        s["block_table"] = torch.full((P + n, cols), -1, dtype=torch.int32, device="cuda")
        s["block_table"][:P] = torch.where(there, order[at.clamp(max=pages - 1)], -1)
        s["lens"] = torch.tensor(lens + [0] * n, dtype=torch.int32, device="cuda")
        s["refs"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
        s["refs"][order[:sum(need)].long()] = 1
        s["children"] = torch.arange(P, P + n, dtype=torch.int32, device="cuda")
        s["parents"] = torch.randint(0, P, (n,), generator=g, device="cuda", dtype=torch.int32)
        s["pool"] = _normal(g, (c["layers"], 2, pages, page, c["heads"], D), BF16)
    else:
        # rows of very unequal lengths hold the live pages, spread over the pool; one page in sixteen is in two rows
        N, R, page = c["pages"], c["rows"], c["page"]
        live = max(1, min(N - 1, int(N * c["live"])))
        order = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
        share = [0.1 + (i + 1) * 0.6180339887 % 1.0 for i in range(R)]
        edges = [int(live * sum(share[:i]) / sum(share)) for i in range(R)] + [live]
        count = [b - a for a, b in zip(edges, edges[1:])]
        shared = [1 if i % 2 and n > 8 else 0 for i, n in enumerate(count)]
        cols = max(n + 1 for n in count)
        row = torch.arange(cols, device="cuda")[None, :]
        n = torch.tensor(count, device="cuda")[:, None]
        more = torch.tensor(shared, device="cuda")[:, None]
        at = torch.where(row < n, torch.tensor(edges[:-1], device="cuda")[:, None] + row, row % live)
        s["block_table"] = torch.where(row < n + more, order[at.clamp(max=N - 1)], -1).to(torch.int32)
        s["lens"] = ((n + more) * page - (n + more > 0) * 3)[:, 0].to(torch.int32)
        s["refs"] = torch.zeros(N, dtype=torch.int32, device="cuda")
        held = s["block_table"][row < n + more].long()
        s["refs"].index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
        # what a pass changes is brought back first, so that every pass packs the same pool
        s["table_now"], s["refs_now"] = s["block_table"].clone(), s["refs"].clone()
        s["pool"] = _normal(g, (c["layers"], 2, N, page, c["heads"], D), F8)
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def _round(x, dtype):
    return x.clamp(-448.0, 448.0).to(F8) if dtype is F8 else x.to(dtype)


def _rotate(x, s, c, sign):
    """Rotates the first rot_dim columns of every head; x [T, heads, head_dim] in 32 bits."""
    pos = s["positions"].double()
    pos = pos[:, None] if s["axis"] is None else pos[s["axis"].long()].T
    angle = pos * s["inv_freq"]
    cos = torch.cos(angle).float()[:, None, :]
    sin = (torch.sin(angle) * sign).float()[:, None, :]
    r = c["rot_dim"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["layout"] == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((ya, yb), -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat((ya, yb), -1)
    return torch.cat((y, x[..., r:]), -1)


def _quantise(x, scale):
    """Codes (0..15) and E4M3 scales of x [..., 16 n] in 32 bits: a block's largest magnitude stands at 6 times its scale."""
    b = x.unflatten(-1, (-1, 16)) * (1.0 / scale)
    f = (b.abs().amax(-1) / 6.0).clamp(max=448.0).to(F8)
    w = f.float()[..., None]
    a = torch.where(w > 0, b / w, 0.0)
    m = a.abs()
    code = ((m > 0.25).int() + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5.0))   # ties to the even code
    return torch.where(a < 0, code + 8, code).flatten(-2), f


def _plain_axes(s, c):
    out = {}
    for n in ("q", "k"):
        x = s[n].float().view(c["tokens"], -1, c["head_dim"])
        out[n] = _round(_rotate(x, s, c, -1.0 if c["inverse"] else 1.0).reshape(s[n].shape), s[n].dtype)
    return out


def _plain_norm(x, gamma, c):
    x = x.float()
    h = x.view(x.shape[0], -1, c["head_dim"]) if c["norm"] == "headwise" else x[:, None, :]
    y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)
    return y.reshape(x.shape) * gamma.float()


def _values(s):
    """The codes of the pool as the numbers they are, [2, page, token, head, d]."""
    return s["table"][s["codes"].int()].view(F8)


def _plain_append(s, c):
    heads = lambda x: x.reshape(c["tokens"], -1, c["head_dim"])
    q = _rotate(heads(_plain_norm(s["q"], s["gamma_q"], c)), s, c, 1.0)
    k = _rotate(heads(_plain_norm(s["k"], s["gamma_k"], c)), s, c, 1.0)
    page, token = s["slots"] // c["page"], s["slots"] % c["page"]
    for side, x, scale in ((0, k, KS), (1, heads(s["v"].float()), VS)):
        code, f = _quantise(x, scale)
        s["codes"][side][page, token] = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
        s["scales"].view(torch.uint8)[side][page, token] = f.view(torch.uint8)
    return {"q": q.reshape(c["tokens"], -1).to(BF16), "codes": _values(s), "scales": s["scales"]}


def _plain_attn(s, c):
    B, H, D, n, L = c["seqs"], c["heads_kv"], c["head_dim"], c["new"], c["ctx"]
    G = c["heads_q"] // H
    key = torch.arange(L, device="cuda")
    page, token = s["block_table"].long()[:, key // c["page"]], key % c["page"]
    value = torch.tensor(STEPS + tuple(-v for v in STEPS), device="cuda")

    def widen(side, scale):
        code = s["codes"][side][page, token].int()                                                   # [B, L, H, D/2]
        x = torch.stack((value[code % 16], value[code // 16]), -1).flatten(-2).unflatten(-1, (-1, 16))
        return (x * (s["scales"].view(torch.uint8)[side][page, token].view(F8).float()[..., None] * scale)).flatten(-2)

    k = widen(0, KS).permute(0, 2, 3, 1)                                                             # [B, H, D, L]
    v = widen(1, VS).permute(0, 2, 1, 3)                                                             # [B, H, L, D]
    starts, lens = s["q_starts"].long(), s["kv_lens"].long()
    i = torch.arange(n, device="cuda")
    rows = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)                                    # [B, n]
    q = s["q"].float().view(-1, H, G, D)[rows].permute(0, 2, 3, 1, 4)                                # [B, H, G, n, D]
    pos = (lens - (starts[1:] - starts[:-1]))[:, None] + i                                           # [B, n]
    seen = (key <= pos[:, :, None]) & (key < lens[:, None, None])
    if c["window"]:
        seen &= key > pos[:, :, None] - c["window"]
    seen = seen[:, None, None]                                                                       # [B, 1, 1, n, L]
    score = (q.reshape(B, H, G * n, D) @ k).view(B, H, G, n, L).mul_(1.0 / math.sqrt(D))
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True).clamp_(min=-3.0e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, G * n, L) @ v).view(B, H, G, n, D) / total.clamp(min=1e-30)
    lse = (top + torch.log(total)).squeeze(-1)
    t = torch.arange(s["q"].shape[0], device="cuda")
    b = torch.searchsorted(starts[1:], t, right=True)
    at = t - starts[b]
    return {"out": o.permute(0, 3, 1, 2, 4)[b, at].reshape(s["q"].shape).to(BF16), "lse": lse.permute(0, 3, 1, 2)[b, at].reshape(-1, H * G)}


def _plain_fork(s, c):
    table, lens, refs, page = s["block_table"], s["lens"], s["refs"], c["page"]
    parents, children = s["parents"].long(), s["children"].long()
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    # the samples of the last step go: their rows give their pages up
    held = col < (-(-lens[children] // page))[:, None]
    refs.index_add_(0, table[children].clamp(min=0).flatten().long(), -held.flatten().int())
    # whole pages are shared; a page that is not full is copied to the lowest page that nobody holds
    n = lens[parents]
    part = n % page > 0
    free = torch.argsort((refs > 0).int(), stable=True).int()
    fresh = free[torch.cumsum(part, 0) - part.long()]
    full = (n // page)[:, None]
    rows = torch.where(col < full, table[parents], torch.where((col == full) & part[:, None], fresh[:, None], -1))
    src = table[parents, (n // page).long().clamp(max=table.shape[1] - 1)]
    table[children] = rows
    lens[children] = n
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().int())
    src, dst = torch.where(part, src, 0).long(), torch.where(part, fresh, 0).long()                 # nothing to copy: page 0 onto itself
    s["pool"][:, :, dst] = s["pool"][:, :, src]
    return {"block_table": table, "lens": lens, "refs": refs, "pool": s["pool"]}


def _plain_compact(s, c):
    table, refs, page = s["table_now"], s["refs_now"], c["page"]
    table.copy_(s["block_table"])
    refs.copy_(s["refs"])
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.shape[0], device="cuda")
    src, dst = (live & (at >= count)).nonzero()[:, 0], (~live & (at < count)).nonzero()[:, 0]
    to = at.clone()
    to[src] = dst
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    held = col < (-(-s["lens"] // page))[:, None]
    table.copy_(torch.where(held, to[table.clamp(min=0).long()].int(), table))
    refs[dst], refs[src] = refs[src], 0
    s["pool"].view(torch.uint8)[:, :, dst] = s["pool"].view(torch.uint8)[:, :, src]
    return {"block_table": table, "refs": refs, "live": count.int().view(1), "pool": s["pool"]}


def _own_axes(s, c):
    from paper_2608_09160_b200 import attn
    q, k = attn.qknorm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], c["head_dim"], axis=s["axis"],
                            interleaved=c["layout"] == "interleaved", inverse=c["inverse"])
    return {"q": q, "k": k}


def _own_append(s, c):
    from paper_2608_09160_b200 import attn
    codes, scales = s["codes"], s["scales"]
    q = attn.qknorm_fwd_append_e2m1(s["q"], s["k"], s["v"], s["gamma_q"], s["gamma_k"], s["positions"], s["inv_freq"], s["slots"],
                                    codes[0], codes[1], scales[0], scales[1], EPS, axis=s["axis"], headwise=c["norm"] == "headwise",
                                    interleaved=c["layout"] == "interleaved", k_scale=KS, v_scale=VS)
    return {"q": q, "codes": _values(s), "scales": scales}


def _own_attn(s, c):
    from paper_2608_09160_b200 import attn
    codes, scales = s["codes"], s["scales"]
    lse = torch.empty((s["q"].shape[0], c["heads_q"]), dtype=torch.float32, device="cuda")
    out = attn.qknorm_attn_paged_e2m1(s["q"], codes[0], codes[1], scales[0], scales[1], s["block_table"], s["kv_lens"], s["q_starts"],
                                      c["new"], c["ctx"], window=c["window"], k_scale=KS, v_scale=VS, lse=lse)
    return {"out": out, "lse": lse}


def _own_fork(s, c):
    from paper_2608_09160_b200 import pages
    pages.qknorm_pages_free(s["refs"], s["block_table"], s["lens"], s["children"], c["page"])
    pages.qknorm_pages_fork(s["pool"], s["refs"], s["block_table"], s["lens"], s["parents"], s["children"], c["page"], page_dim=2)
    return {"block_table": s["block_table"], "lens": s["lens"], "refs": s["refs"], "pool": s["pool"]}


def _own_compact(s, c):
    from paper_2608_09160_b200 import pages
    s["table_now"].copy_(s["block_table"])
    s["refs_now"].copy_(s["refs"])
    live = pages.qknorm_pages_compact(s["pool"], s["refs_now"], s["table_now"], s["lens"], c["page"], page_dim=2)
    return {"block_table": s["table_now"], "refs": s["refs_now"], "live": live, "pool": s["pool"]}


def run(state):
    c = state["case"]
    if own:
        return {"axes": _own_axes, "append": _own_append, "attn": _own_attn, "fork": _own_fork, "compact": _own_compact}[c["op"]](state, c)
    return {"axes": _plain_axes, "append": _plain_append, "attn": _plain_attn, "fork": _plain_fork, "compact": _plain_compact}[c["op"]](state, c)


# ---- what a pass cannot do without ------------------------------------------------------------------

def _keys(c):
    """(keys that some row of each sequence sees, visible pairs of rows and keys) over the batch."""
    seen = pairs = 0
    for L, n in zip(_kv_lens(c), _new_lens(c)):
        w = c["window"] or L
        seen += min(L, w + n - 1)
        pairs += sum(min(L - n + i + 1, w) for i in range(n))
    return seen, pairs


def work(case):
    c = case
    D = c["head_dim"]
    if c["op"] == "axes":
        e = 1 if c["dtype"] == "e4m3" else 2
        n = c["tokens"] * (c["dq"] + c["dk"])
        return {"bytes": 2 * n * e + c["tokens"] * 24 + c["rot_dim"] * 4, "flops": 3 * n * c["rot_dim"] // D}
    if c["op"] == "append":
        T, dq, dk = c["tokens"], c["dq"], c["dk"]
        return {"bytes": T * (4 * dq + 4 * dk + 2 * dk * 9 // 16 + (32 if c["axes"] else 16)) + 2 * (dq + dk) + c["rot_dim"] * 4,
                "flops": T * (dq + dk) * 10}
    if c["op"] == "attn":
        seen, pairs = _keys(c)
        rows = sum(_new_lens(c))
        return {"bytes": 2 * seen * c["heads_kv"] * D * 9 // 16 + rows * c["heads_q"] * (4 * D + 4)
                         + 4 * sum(-(-n // c["page"]) for n in _kv_lens(c)) + 8 * c["seqs"] + 4,
                "flops": 4 * pairs * c["heads_q"] * D}
    one = 2 * c["layers"] * c["page"] * c["heads"] * D          # elements of a page over all layers
    if c["op"] == "fork":
        cols = -(-c["ctx"] // c["page"])
        return {"bytes": c["forks"] * (4 * one + 12 * cols + 16), "flops": c["forks"] * cols}
    live = c["live"]
    return {"bytes": int(c["pages"] * live * (1 - live)) * 2 * one + 8 * c["pages"] + int(8 * c["pages"] * live), "flops": c["pages"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _exact_turn(x, s, c):
    """Every pair as a complex number, times exp(+-i * angle)."""
    r, pos = c["rot_dim"], s["positions"]
    y = x.clone()
    one = [(2 * i, 2 * i + 1) if c["layout"] == "interleaved" else (i, i + r // 2) for i in range(r // 2)]
    ia, ib = (torch.tensor(v, device=x.device) for v in zip(*one))
    which = [0] * (r // 2) if s["axis"] is None else s["axis"].tolist()
    at = torch.stack([(pos if s["axis"] is None else pos[a]).double() for a in which], 1)            # [T, pairs]
    angle = (at * s["inv_freq"])[:, None, :] * (-1.0 if c.get("inverse") else 1.0)
    z = torch.complex(x[..., ia], x[..., ib]) * torch.polar(torch.ones_like(angle), angle)
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def _exact_codes(x, scale):
    """(values of the codes, scales) of x [..., D]: each value of a block to the nearest of E2M1's sixteen."""
    b = (x / scale).unflatten(-1, (-1, 16))
    f = torch.minimum(b.abs().amax(-1) / 6.0, torch.tensor(448.0, device=x.device, dtype=torch.float64)).to(F8)
    a = b / f.double().clamp(min=2.0 ** -40)[..., None] * (f.double() > 0)[..., None]
    steps = torch.tensor(STEPS, device=x.device, dtype=torch.float64)
    mid = (steps[1:] + steps[:-1]) / 2
    m = a.abs()
    low = torch.bucketize(m, mid)                    # a tie stays below
    tie = (m == mid[low.clamp(max=6)]) & (low < 7) & (low % 2 == 1)
    return (steps[low + tie.long()] * a.sign()).flatten(-2), f


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    D = c.get("head_dim")
    if c["op"] == "axes":
        return {n: _exact_turn(s[n].double().view(c["tokens"], -1, D), s, c).reshape(s[n].shape) for n in ("q", "k")}
    if c["op"] == "append":
        def side(x, gamma):
            x = x.double()
            w = D if c["norm"] == "headwise" else x.shape[1]
            ms = x.reshape(x.shape[0], -1, w).pow(2).mean(2).add(EPS).rsqrt().repeat_interleave(w, 1)
            return _exact_turn((x * ms * gamma.double()).view(c["tokens"], -1, D), s, c)
        byte = s["codes"].long()
        steps = torch.tensor(STEPS, device="cuda", dtype=torch.float64)
        half = lambda n: steps[n & 7] * (1 - 2 * (n >> 3)).double()
        codes = torch.stack((half(byte & 15), half(byte >> 4)), -1).flatten(-2)
        scales = s["scales"].double()
        for i, x, unit in ((0, side(s["k"], s["gamma_k"]), KS), (1, s["v"].double().reshape(c["tokens"], -1, D), VS)):
            v, f = _exact_codes(x, unit)
            at = (s["slots"] // c["page"], s["slots"] % c["page"])
            codes[i][at], scales[i][at] = v, f.double()
        return {"q": side(s["q"], s["gamma_q"]).reshape(c["tokens"], -1), "codes": codes, "scales": scales}
    if c["op"] == "attn":
        H, G = c["heads_kv"], c["heads_q"] // c["heads_kv"]
        out = torch.zeros((s["q"].shape[0], H, G, D), dtype=torch.float64, device="cuda")
        lse = torch.zeros((s["q"].shape[0], H, G), dtype=torch.float64, device="cuda")
        starts, lens, table = s["q_starts"].tolist(), s["kv_lens"].tolist(), s["block_table"].tolist()
        steps = torch.tensor(STEPS, device="cuda", dtype=torch.float64)
        for b in range(c["seqs"]):
            r0, r1, L = starts[b], starts[b + 1], lens[b]
            used = torch.tensor(table[b][:-(-L // c["page"])], device="cuda")
            kv = []
            for i, unit in ((0, KS), (1, VS)):
                byte = s["codes"][i][used].flatten(0, 1)[:L].long()
                half = lambda n: steps[n & 7] * (1 - 2 * (n >> 3)).double()
                x = torch.stack((half(byte & 15), half(byte >> 4)), -1).flatten(-2)
                f = s["scales"].view(torch.uint8)[i][used].view(F8).flatten(0, 1)[:L].double().repeat_interleave(16, -1)
                kv.append(x * f * unit)
            k, v = kv
            pos = torch.arange(L - (r1 - r0), L, device="cuda")[:, None]
            key = torch.arange(L, device="cuda")[None, :]
            hide = (key > pos) | ((key <= pos - c["window"]) if c["window"] else False)
            for h in range(H):
                q = s["q"][r0:r1].double().view(r1 - r0, H, G, D)[:, h].transpose(0, 1)             # [G, n, D]
                x = (torch.matmul(q, k[:, h].T) / math.sqrt(D)).masked_fill_(hide, -math.inf)
                z = torch.logsumexp(x, -1)
                lse[r0:r1, h] = z.T
                out[r0:r1, h] = torch.matmul(x.sub_(z[..., None]).exp_(), v[:, h]).transpose(0, 1)
        return {"out": out.view(s["q"].shape[0], -1), "lse": lse.view(s["q"].shape[0], -1)}
    page, pool = c["page"], s["pool"]
    table, lens, refs = s["block_table"].tolist(), s["lens"].tolist(), s["refs"].tolist()
    moved = []
    if c["op"] == "fork":
        for parent, child in zip(s["parents"].tolist(), s["children"].tolist()):
            full, rest = divmod(lens[parent], page)
            table[child] = table[parent][:full] + [-1] * (len(table[parent]) - full)
            lens[child] = lens[parent]
            for e in table[child][:full]:
                refs[e] += 1
            if rest:
                fresh = refs.index(0)
                refs[fresh] = 1
                moved.append((table[parent][full], fresh))
                table[child][full] = fresh
        extra = {"lens": torch.tensor(lens, dtype=torch.int32)}
    else:
        live = sum(r > 0 for r in refs)
        holes = (p for p in range(live) if refs[p] == 0)
        to = {p: next(holes) for p in range(live, len(refs)) if refs[p] > 0}
        moved = list(to.items())
        for row, n in zip(table, lens):
            for j in range(-(-n // page)):
                row[j] = to.get(row[j], row[j])
        for a, b in moved:
            refs[b], refs[a] = refs[a], 0
        extra = {"live": torch.tensor([live], dtype=torch.int32)}
    got = pool.double()
    for a, b in moved:
        got[:, :, b] = pool[:, :, a].double()
    return {"block_table": torch.tensor(table, dtype=torch.int32), "refs": torch.tensor(refs, dtype=torch.int32), "pool": got, **extra}
