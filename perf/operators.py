"""What the attention-side operators are measured on: rotary positions, the fused norm + rotation +
cache write, and attention over a paged cache.

Widths and head counts are those of the library's five workloads (4096+4096, 5120+5120, 5120+1024 and
8192+1024 columns, heads of 128) and a few generic ones; token counts go from one decode step to a prompt.
"""
import math

import torch

own = False

BF16, F8 = torch.bfloat16, torch.float8_e4m3fn
EPS = 1e-6


# ---- cases ------------------------------------------------------------------------------------------

def _rope(tokens, dq, dk, head_dim=128, rot_dim=128, layout="half", inverse=False, dtype="bf16", factor=1.0, max_pos=32768):
    return dict(op="rope", tokens=tokens, dq=dq, dk=dk, head_dim=head_dim, rot_dim=rot_dim, layout=layout,
                inverse=inverse, dtype=dtype, factor=factor, max_pos=max_pos)


def _append(tokens, dq, dk, head_dim=128, rot_dim=128, layout="half", norm="layerwise", cache="bf16", page=16, max_pos=32768):
    return dict(op="append", tokens=tokens, dq=dq, dk=dk, head_dim=head_dim, rot_dim=rot_dim, layout=layout,
                norm=norm, cache=cache, page=page, max_pos=max_pos)


def _attn(seqs, new, ctx, heads_q, heads_kv, head_dim=128, page=16, cache="bf16", window=0, ragged=True):
    return dict(op="attn", seqs=seqs, new=new, ctx=ctx, heads_q=heads_q, heads_kv=heads_kv, head_dim=head_dim,
                page=page, cache=cache, window=window, ragged=ragged)


def listed():
    return [
        # one decode step of a batch of 64, 32 + 32 heads: the smallest call, latency counts
        dict(_rope(64, 4096, 4096), name="rope_decode"),
        # a long prompt of a grouped-head layer, frequencies stretched eightfold
        dict(_rope(16384, 5120, 1024, factor=8.0, max_pos=262144), name="rope_prefill"),
        # the backward pass of a training step, interleaved pairs in half of every head
        dict(_rope(8191, 5120, 5120, rot_dim=64, layout="interleaved", inverse=True), name="rope_backward"),
        # FP8 activations of the large layer
        dict(_rope(8192, 8192, 1024, dtype="e4m3"), name="rope_e4m3"),
        # the cache write of one decode step
        dict(_append(64, 5120, 1024), name="append_decode"),
        # the cache write of a prompt, the norm over whole rows
        dict(_append(16384, 5120, 1024), name="append_prefill"),
        # an FP8 cache with pages of 64, the norm over every head
        dict(_append(8191, 8192, 1024, norm="headwise", cache="e4m3", page=64), name="append_e4m3"),
        # one decode step of a few short sequences, five query heads to a key head
        dict(_attn(8, 1, 1000, 40, 8), name="attn_decode_small"),
        # one decode step of a full serving batch
        dict(_attn(64, 1, 8192, 64, 8), name="attn_decode"),
        # the same from an FP8 cache, fewer and longer sequences
        dict(_attn(16, 1, 32000, 64, 8, cache="e4m3", page=64), name="attn_decode_e4m3"),
        # chunks of new tokens of four sequences next to what is in the cache, window of 4096 keys
        dict(_attn(4, 512, 8192, 40, 8, window=4096), name="attn_chunk"),
        # a whole prompt
        dict(_attn(1, 8192, 8192, 40, 8, page=64), name="attn_prefill"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attn", "attn"])
    head_dim = rng.choice([64, 96, 128, 128])
    layout = rng.choice(["half", "interleaved"])
    rot_dim = rng.choice([head_dim, head_dim // 2])
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 4, 5, 7, 8])
    if op == "rope":
        return _rope(_log(rng, 1, 12000), hkv * group * head_dim, hkv * head_dim, head_dim, rot_dim, layout,
                     rng.random() < 0.5, rng.choice(["bf16", "e4m3"]), rng.choice([1.0, 8.0]), _log(rng, 1000, 1000000))
    if op == "append":
        return _append(_log(rng, 1, 12000), hkv * group * head_dim, hkv * head_dim, head_dim, rot_dim, layout,
                       rng.choice(["layerwise", "headwise"]), rng.choice(["bf16", "e4m3"]), rng.choice([16, 24, 64]),
                       _log(rng, 1000, 1000000))
    kind = rng.choice(["decode", "verify", "chunk"])
    seqs = _log(rng, 1, 64) if kind != "chunk" else _log(rng, 1, 8)
    new = 1 if kind == "decode" else rng.randint(2, 17) if kind == "verify" else _log(rng, 33, 2048)
    ctx = new + _log(rng, 1, 8192)
    seqs = max(1, min(seqs, 1_300_000_000 // (hkv * group * new * ctx)))   # no more pairs than the whole prompt has
    return _attn(seqs, new, ctx, hkv * group, hkv, head_dim, rng.choice([16, 24, 64, 128]), rng.choice(["bf16", "bf16", "e4m3"]),
                 rng.choice([0, 0, 1024]), rng.random() < 0.7)


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


def _inv_freq(rot_dim, factor):
    """theta^(-2i/rot_dim); stretched: slow dimensions divided by `factor`, fast ones kept, a ramp between."""
    i = torch.arange(rot_dim // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * i / rot_dim)
    if factor != 1.0:
        turns = 32768.0 * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f / factor * (1 - keep) + f * keep
    return f.cuda()


def _normal(g, shape, dtype, sigma=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype is F8 else dtype).mul_(sigma)
    return x.to(dtype)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"case": c}
    if c["op"] in ("rope", "append"):
        T, dq, dk = c["tokens"], c["dq"], c["dk"]
        s["inv_freq"] = _inv_freq(c["rot_dim"], c.get("factor", 1.0))
        s["mscale"] = 0.1 * math.log(c["factor"]) + 1.0 if c.get("factor", 1.0) != 1.0 else 1.0
        # a decode step has sequences of any length; a prompt's positions run on
        first = torch.randint(0, max(1, c["max_pos"] - T), (1,), generator=g, device="cuda")
        s["positions"] = (torch.randint(0, c["max_pos"], (T,), generator=g, device="cuda") if T <= 256
                          else first + torch.arange(T, device="cuda"))
    if c["op"] == "rope":
        dt = F8 if c["dtype"] == "e4m3" else BF16
        s["q"], s["k"] = _normal(g, (T, dq), dt), _normal(g, (T, dk), dt)
    elif c["op"] == "append":
        qkv = _normal(g, (T, dq + 2 * dk), BF16)       # the fused projection's output
        s["q"], s["k"], s["v"] = qkv[:, :dq], qkv[:, dq:dq + dk], qkv[:, dq + dk:]
        s["gamma_q"] = (torch.rand(dq, generator=g, device="cuda") + 0.5).to(BF16)
        s["gamma_k"] = (torch.rand(dk, generator=g, device="cuda") + 0.5).to(BF16)
        page, heads = c["page"], dk // c["head_dim"]
        pages = T // page + 2 if T > 256 else T        # a prompt fills pages; a decode step has one sequence per token
        order = torch.randperm(pages, generator=g, device="cuda")
        t = torch.arange(T, device="cuda")
        s["slots"] = (order[t // page] * page + t % page if T > 256
                      else order * page + torch.randint(0, page, (T,), generator=g, device="cuda"))
        dt = F8 if c["cache"] == "e4m3" else BF16
        for n in ("k_cache", "v_cache"):
            s[n] = _normal(g, (pages, page, heads, c["head_dim"]), dt)
        s["k_scale"], s["v_scale"] = (0.03125, 0.0625) if dt is F8 else (1.0, 1.0)
    else:
        D, page = c["head_dim"], c["page"]
        kv, new = _kv_lens(c), _new_lens(c)
        need = [-(-n // page) for n in kv]
        pages, cols = sum(need) + 3, -(-c["ctx"] // page)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        row = torch.arange(cols, device="cuda")[None, :]
        at = torch.tensor([0] + need, device="cuda").cumsum(0)[:-1, None] + row
        s["block_table"] = torch.where(row < torch.tensor(need, device="cuda")[:, None], order[at.clamp(max=pages - 1)], 0).to(torch.int32)
        s["kv_lens"] = torch.tensor(kv, dtype=torch.int32, device="cuda")
        s["q_starts"] = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
        dt = F8 if c["cache"] == "e4m3" else BF16
        s["q"] = _normal(g, (sum(new), c["heads_q"] * D), BF16)   # normalised and rotated queries
        s["k_scale"], s["v_scale"] = (0.03125, 0.0625) if dt is F8 else (1.0, 1.0)
        s["k_cache"] = _normal(g, (pages, page, c["heads_kv"], D), dt, 1.0 / s["k_scale"])
        s["v_cache"] = _normal(g, (pages, page, c["heads_kv"], D), dt, 1.0 / s["v_scale"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------

def _round(x, dtype):
    return x.clamp(-448.0, 448.0).to(F8) if dtype is F8 else x.to(dtype)


def _rotate(x, s, c, sign):
    """Rotates the first rot_dim columns of every head; x [T, heads, head_dim] in 32 bits."""
    angle = s["positions"].double()[:, None] * s["inv_freq"]
    cos = (torch.cos(angle) * s["mscale"]).float()[:, None, :]
    sin = (torch.sin(angle) * (sign * s["mscale"])).float()[:, None, :]
    r = c["rot_dim"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["layout"] == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((ya, yb), -1).flatten(-2) if c["layout"] == "interleaved" else torch.cat((ya, yb), -1)
    return torch.cat((y, x[..., r:]), -1)


def _plain_rope(s, c):
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


def _plain_append(s, c):
    heads = lambda x: x.reshape(c["tokens"], -1, c["head_dim"])
    q = _rotate(heads(_plain_norm(s["q"], s["gamma_q"], c)), s, c, 1.0)
    k = _rotate(heads(_plain_norm(s["k"], s["gamma_k"], c)), s, c, 1.0)
    for n, x in (("k", k), ("v", heads(s["v"].float()))):
        pool = s[n + "_cache"]
        raw = torch.uint8 if pool.dtype is F8 else torch.int16
        pool.view(raw).view(-1, *pool.shape[2:])[s["slots"]] = _round(x / s[n + "_scale"], pool.dtype).view(raw)
    return {"q": q.reshape(c["tokens"], -1).to(BF16), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attn(s, c):
    B, H, D, n, L = c["seqs"], c["heads_kv"], c["head_dim"], c["new"], c["ctx"]
    G = c["heads_q"] // H
    key = torch.arange(L, device="cuda")
    slot = s["block_table"].long()[:, key // c["page"]] * c["page"] + key % c["page"]
    k = s["k_cache"].view(-1, H, D)[slot].float().mul_(s["k_scale"]).permute(0, 2, 3, 1)            # [B, H, D, L]
    v = s["v_cache"].view(-1, H, D)[slot].float().mul_(s["v_scale"]).permute(0, 2, 1, 3)            # [B, H, L, D]
    starts, lens = s["q_starts"].long(), s["kv_lens"].long()
    i = torch.arange(n, device="cuda")
    rows = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)                                   # [B, n]
    q = s["q"].float().view(-1, H, G, D)[rows].permute(0, 2, 3, 1, 4)                               # [B, H, G, n, D]
    pos = (lens - (starts[1:] - starts[:-1]))[:, None] + i                                          # [B, n]
    seen = (key <= pos[:, :, None]) & (key < lens[:, None, None])
    if c["window"]:
        seen &= key > pos[:, :, None] - c["window"]
    seen = seen[:, None, None]                                                                      # [B, 1, 1, n, L]
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


def _own_rope(s, c):
    from paper_2608_09160_b200 import attn
    q, k = attn.qknorm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], c["head_dim"],
                            interleaved=c["layout"] == "interleaved", inverse=c["inverse"], mscale=s["mscale"])
    return {"q": q, "k": k}


def _own_append(s, c):
    from paper_2608_09160_b200 import attn
    q = attn.qknorm_fwd_append(s["q"], s["k"], s["v"], s["gamma_q"], s["gamma_k"], s["positions"], s["inv_freq"], s["slots"],
                               s["k_cache"], s["v_cache"], EPS, headwise=c["norm"] == "headwise",
                               interleaved=c["layout"] == "interleaved", k_scale=s["k_scale"], v_scale=s["v_scale"])
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _own_attn(s, c):
    from paper_2608_09160_b200 import attn
    lse = torch.empty((s["q"].shape[0], c["heads_q"]), dtype=torch.float32, device="cuda")
    out = attn.qknorm_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["kv_lens"], s["q_starts"],
                                 c["new"], c["ctx"], window=c["window"], k_scale=s["k_scale"], v_scale=s["v_scale"], lse=lse)
    return {"out": out, "lse": lse}


def run(state):
    c = state["case"]
    if own:
        return {"rope": _own_rope, "append": _own_append, "attn": _own_attn}[c["op"]](state, c)
    return {"rope": _plain_rope, "append": _plain_append, "attn": _plain_attn}[c["op"]](state, c)


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
    if c["op"] == "rope":
        e = 1 if c["dtype"] == "e4m3" else 2
        n = c["tokens"] * (c["dq"] + c["dk"])
        return {"bytes": 2 * n * e + c["tokens"] * 8 + c["rot_dim"] * 4, "flops": 3 * n * c["rot_dim"] // c["head_dim"]}
    if c["op"] == "append":
        e = 1 if c["cache"] == "e4m3" else 2
        T, dq, dk = c["tokens"], c["dq"], c["dk"]
        return {"bytes": T * (4 * dq + 2 * dk * (2 + e) + 16) + 2 * (dq + dk) + c["rot_dim"] * 4,
                "flops": T * (dq + dk) * 7}
    e = 1 if c["cache"] == "e4m3" else 2
    seen, pairs = _keys(c)
    rows = sum(_new_lens(c))
    return {"bytes": 2 * seen * c["heads_kv"] * c["head_dim"] * e + rows * c["heads_q"] * (4 * c["head_dim"] + 4)
                     + 4 * sum(-(-n // c["page"]) for n in _kv_lens(c)) + 8 * c["seqs"] + 4,
            "flops": 4 * pairs * c["heads_q"] * c["head_dim"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _exact_turn(x, pos, freq, c, mscale):
    """Every pair as a complex number, times mscale * exp(+-i * angle)."""
    r = c["rot_dim"]
    y = x.clone()
    one = [(2 * i, 2 * i + 1) if c["layout"] == "interleaved" else (i, i + r // 2) for i in range(r // 2)]
    ia, ib = (torch.tensor(v, device=x.device) for v in zip(*one))
    angle = pos.double()[:, None, None] * freq * (-1.0 if c.get("inverse") else 1.0)
    z = torch.complex(x[..., ia], x[..., ib]) * torch.polar(torch.full_like(angle, mscale), angle)
    y[..., ia], y[..., ib] = z.real, z.imag
    return y


def exact(case, seed):
    s, c = prepare(case, seed), dict(case)
    D = c["head_dim"]
    if c["op"] == "rope":
        return {n: _exact_turn(s[n].double().view(c["tokens"], -1, D), s["positions"], s["inv_freq"], c, s["mscale"]).reshape(s[n].shape)
                for n in ("q", "k")}
    if c["op"] == "append":
        def side(x, gamma):
            x = x.double()
            w = D if c["norm"] == "headwise" else x.shape[1]
            ms = x.reshape(x.shape[0], -1, w).pow(2).mean(2).add(EPS).rsqrt().repeat_interleave(w, 1)
            return _exact_turn((x * ms * gamma.double()).view(c["tokens"], -1, D), s["positions"], s["inv_freq"], c, 1.0)
        got = {"q": side(s["q"], s["gamma_q"]).reshape(c["tokens"], -1)}
        for n, x in (("k", side(s["k"], s["gamma_k"])), ("v", s["v"].double().reshape(c["tokens"], -1, D))):
            pool = s[n + "_cache"].double()
            pool.view(-1, *pool.shape[2:])[s["slots"]] = x / s[n + "_scale"]
            got[n + "_cache"] = pool
        return got
    H, G = c["heads_kv"], c["heads_q"] // c["heads_kv"]
    out = torch.zeros((s["q"].shape[0], H, G, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((s["q"].shape[0], H, G), dtype=torch.float64, device="cuda")
    starts, lens, table = s["q_starts"].tolist(), s["kv_lens"].tolist(), s["block_table"].tolist()
    for b in range(c["seqs"]):
        r0, r1, L = starts[b], starts[b + 1], lens[b]
        used = table[b][:-(-L // c["page"])]
        k = s["k_cache"][used].double().flatten(0, 1)[:L] * s["k_scale"]
        v = s["v_cache"][used].double().flatten(0, 1)[:L] * s["v_scale"]
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
