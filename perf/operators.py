"""What the operators of the growing 8-bit cache cost: rotary positions, the write into the cache, attention over it, eviction by
accumulated attention weight.  Each has a plain form of elementary torch operations (the module's `own` is false) beside the
library's call (`own` is true).

  rotary    queries and keys of the tokens of a step or of a prompt, turned by the angles of their positions
  append    their keys and values, held in 8 bits (E4M3) with one scale per block of tokens and head, into the cache of one layer
  attend    one token per sequence over that cache, all rows or listed ones, with the weights that the rows gather where eviction wants them
  evict     which rows of every layer, sequence and head stay
  compact   these rows moved together, with their scales and gathered weights

Cache of L layers: K, V [L][Hkv][T_total][D] bytes; sequence b's rows start at cu_tok[b], and its block t of `block` rows has scale
[L][Hkv][cu_tok[b] / block + b + t], a power of two.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D = 128                                   # head dimension
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn
MOST_ROWS = 1 << 21                       # rows x KV heads (x layers) of a drawn cache
MOST_TURNED = 32768 * 40                  # tokens x heads that a drawn rotation turns


def _case(name, op, **kw):
    c = {"name": name, "op": op, "layers": 1, "q_heads": 32, "kv_heads": 8, "dtype": "bf16", "batch": 1, "block": 64}
    c.update(kw)
    return c


def listed():
    return [
        # the smallest call: the tokens of one decode step of a few sequences, fp32, part of the head turned
        _case("rotary_step", "rotary", dtype="f32", tokens=5, rot=64, interleaved=True, far=131072, mscale=1.2),
        # a prompt on its way into the pool
        _case("rotary_prompt", "rotary", tokens=32768, rot=128, interleaved=False, far=32768, mscale=1.0),
        # the decode step of a batch: one token per sequence into blocks that are partly filled
        _case("append_step", "append", batch=16, new_min=1, new_max=1, held_min=1000, held_max=9000),
        # a prompt behind a short resident prefix
        _case("append_prompt", "append", new_min=32768, new_max=32768, held_min=77, held_max=77),
        # a resident window of recent tokens: latency
        _case("attend_window", "attend", dtype="f32", held_min=257, held_max=257, listed=0, weights=False, block=32),
        # the rows a retrieval has listed, out of a 32K context
        _case("attend_listed", "attend", held_min=32768, held_max=32768, listed=2048, weights=False),
        # one sequence over its whole long context
        _case("attend_long", "attend", held_min=131072, held_max=131072, listed=0, weights=False),
        # a ragged batch of a serving step that gathers the weights, wide groups
        _case("attend_batch", "attend", q_heads=64, batch=16, held_min=8192, held_max=32768, listed=0, weights=True),
        # eviction from one short layer
        _case("evict_small", "evict", held_min=2100, held_max=2100, keep=1024, sink=4, recent=256),
        # eviction from all layers of a long context
        _case("evict_long", "evict", layers=32, held_min=32768, held_max=32768, keep=4096, sink=4, recent=1024),
        # what follows it: the kept rows of one layer, and of all layers
        _case("compact_small", "compact", held_min=2100, held_max=2100, keep=1024),
        _case("compact_long", "compact", layers=16, held_min=16384, held_max=16384, keep=8192),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: 1 to 32K tokens turned, 1 to 32 sequences of up to 128K rows, both types, groups of 1 to 8."""
    op = rng.choice(["rotary", "append", "attend", "attend", "evict", "compact"])
    kv_heads = rng.choice([1, 2, 8, 8, 8, 16])
    c = {"op": op, "layers": 1, "kv_heads": kv_heads, "q_heads": kv_heads * rng.choice([1, 2, 4, 8]),
         "dtype": rng.choice(["bf16", "bf16", "f32"]), "batch": 1, "block": rng.choice([16, 32, 64, 128])}
    if op == "rotary":
        heads = c["kv_heads"] + c["q_heads"]
        c.update(tokens=_log(rng, 1, min(32768, MOST_TURNED // heads // (2 if c["dtype"] == "f32" else 1))),
                 rot=rng.choice([32, 64, 96, 128, 128, 2 * rng.randint(1, 64)]), interleaved=rng.random() < 0.5,
                 far=_log(rng, 1024, 1 << 20), mscale=rng.choice([1.0, round(rng.uniform(0.7, 1.6), 3)]))
        return c
    if op in ("append", "attend"):
        c["batch"] = _log(rng, 1, 32)
    else:
        c["layers"], c["batch"] = _log(rng, 1, 32), _log(rng, 1, 8)
    most = min(131072, max(64, MOST_ROWS // (c["layers"] * c["batch"] * kv_heads)))
    hi = _log(rng, 32, most)
    lo = _log(rng, max(1, hi // 8), hi)
    c.update(held_min=lo, held_max=hi)
    if op == "append":
        hi = _log(rng, 1, max(1, min(32768 // c["batch"], 8 * 32768 // (c["batch"] * kv_heads))))
        c.update(new_min=_log(rng, 1, hi), new_max=hi)
    elif op == "attend":
        c["listed"] = 0 if rng.random() < 0.6 else _log(rng, 1, hi)
        c["weights"] = not c["listed"] and rng.random() < 0.5
    else:
        c["keep"] = _log(rng, max(1, hi // 8), hi)
        if op == "evict":
            c["sink"] = min(rng.choice([0, 1, 4, 16]), c["keep"] // 4)
            c["recent"] = rng.randint(0, c["keep"] // 2)
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Rows of the sequences, new rows, and room behind them: the case's own, so that every seed's outputs have one shape."""
    rng, B = np.random.RandomState(case["held_min"] + 7 * case["held_max"] + 31 * case["batch"]), case["batch"]
    held = rng.randint(case["held_min"], case["held_max"] + 1, B).astype(np.int64)
    new = rng.randint(case["new_min"], case["new_max"] + 1, B).astype(np.int64) if case["op"] == "append" else np.zeros(B, np.int64)
    return held, new, new + rng.randint(0, 2 * case["block"], B)


def _scale_of(a):
    """2^e, e the smallest with a <= 448 * 2^e, at least 2^-100."""
    m, e = torch.frexp(a.double())                              # a = m * 2^e, 0.5 <= m < 1
    e = e - 9 + (m > 0.875).int()                               # 448 = 0.875 * 2^9
    return torch.where(a > 0, torch.ldexp(torch.ones_like(m), e.clamp(min=-100)), torch.ldexp(torch.ones_like(m), torch.full_like(e, -100))).float()


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _cache(case, held, spare, g):
    """A cache of `held` rows per sequence (spare[b] more have room), in 8 bits."""
    L, H, blk, B = case["layers"], case["kv_heads"], case["block"], case["batch"]
    cu = np.concatenate([[0], np.cumsum(held + spare)]).astype(np.int32)
    T = int(cu[-1])
    NS = T // blk + B
    # rows of unlike lengths, as keys and values are: the scales of the blocks differ
    scale = torch.ldexp(torch.ones((), device=DEV), torch.randint(-8, -5, (2, L, H, NS), device=DEV, generator=g, dtype=torch.int32))
    cache = torch.randn(2, L, H, T, D, device=DEV, generator=g, dtype=torch.bfloat16).mul_(60.0).clamp_(-448.0, 448.0).to(F8)
    return {"cu": cu, "T": T, "NS": NS, "K": cache[0].view(torch.uint8), "V": cache[1].view(torch.uint8), "ks": scale[0].contiguous(),
            "vs": scale[1].contiguous(), "cu_tok": torch.from_numpy(cu).to(DEV)}


def _context(case, tokens, batch):
    import paper_2504_00970_amd as skv
    return skv.Context(skv.Desc(n_layers=case["layers"], n_q_heads=case["q_heads"], n_kv_heads=case["kv_heads"],
                                kv_dtype={"f32": skv.SKV_F32, "bf16": skv.SKV_BF16}[case["dtype"]], max_tokens=tokens, max_sentences=1,
                                max_budget=1, max_batch=batch))


def prepare(case, seed):
    g, dt, L, H, B = _gen(seed), TYPE[case["dtype"]], case["layers"], case["kv_heads"], case["batch"]
    s = {"case": case}
    if case["op"] == "rotary":
        n, half = case["tokens"], case["rot"] // 2
        s["q"] = torch.randn(n, case["q_heads"], D, device=DEV, generator=g).to(dt)
        s["k"] = torch.randn(n, H, D, device=DEV, generator=g).to(dt)
        first = np.random.RandomState(seed % (1 << 31)).randint(0, max(1, case["far"] - n))
        s["pos"] = torch.arange(first, first + n, dtype=torch.int32, device=DEV)
        s["inv_freq"] = torch.tensor([500000.0 ** (-i / half) for i in range(half)], dtype=torch.float64, device=DEV)
        s["q_out"], s["k_out"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        if own:
            s["ctx"] = _context(case, n, 1)
        return s
    rng = np.random.RandomState(seed % (1 << 31))
    held, new, spare = _lengths(case)
    s.update(_cache(case, held, spare, g))
    n_tok = torch.from_numpy(np.repeat(held, H).astype(np.int32)).to(DEV).view(B, H)
    s["n_tok"], s["max_n"] = n_tok, int(held.max())
    if case["op"] == "append":
        cu_new = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        n = int(cu_new[-1])
        s["n"], s["max_new"], s["cu_new"] = n, int(new.max()), torch.from_numpy(cu_new).to(DEV)
        length = torch.exp(0.4 * torch.randn(2, n, 1, 1, device=DEV, generator=g))      # some rows are longer than all before them
        kv = torch.randn(2, n, H, D, device=DEV, generator=g) * length
        s["k"], s["v"] = kv[0].to(dt), kv[1].to(dt)
        s["acc"] = torch.rand(L, H, s["T"], device=DEV, generator=g)
    elif case["op"] == "attend":
        s["q"] = torch.randn(B, case["q_heads"], D, device=DEV, generator=g).to(dt)
        s["out"] = torch.zeros(B, case["q_heads"], D, device=DEV)
        s["lse"] = torch.zeros(B, case["q_heads"], device=DEV)
        s["idx"], s["n"] = None, n_tok
        if case["listed"]:                                     # runs of neighbours, ascending
            s["max_n"] = case["listed"]
            n = np.minimum(held, rng.randint((case["listed"] + 1) // 2, case["listed"] + 1, B))
            idx = np.zeros((B, H, case["listed"]), np.int32)
            for b in range(B):
                for h in range(H):
                    runs = rng.permutation(-(-held[b] // 25))[: -(-n[b] // 25) + 1]
                    rows = (np.sort(runs)[:, None] * 25 + np.arange(25)).ravel()
                    rows = rows[rows < held[b]][: n[b]]
                    idx[b, h, : len(rows)] = rows
                    n[b] = min(n[b], len(rows))
            s["idx"], s["n"] = torch.from_numpy(idx).to(DEV), torch.from_numpy(np.repeat(n, H).astype(np.int32)).to(DEV).view(B, H)
        s["acc"] = s["acc_out"] = None
        if case["weights"]:
            s["acc"] = torch.rand(L, H, s["T"], device=DEV, generator=g)
            s["acc_out"] = torch.zeros_like(s["acc"])
    else:
        # gathered weights: most rows little, a few much, some none at all
        acc = torch.exp(2.0 * torch.randn(L, H, s["T"], device=DEV, generator=g) - 4.0)
        s["acc"] = acc * (torch.rand(L, H, s["T"], device=DEV, generator=g) > 0.05)
        s["n_tok"] = n_tok.expand(L, B, H).contiguous()
        s["keep_idx"] = torch.full((L, B, H, case["keep"]), -1, dtype=torch.int32, device=DEV)
        s["n_keep"] = torch.full((L, B, H), -1, dtype=torch.int32, device=DEV)
        if case["op"] == "compact":
            keep = np.minimum(held, case["keep"])
            for b in range(B):
                r = torch.rand(L, H, int(held[b]), device=DEV, generator=g)
                rows = r.topk(int(keep[b]), dim=-1).indices.sort(dim=-1).values
                s["keep_idx"][:, b, :, : int(keep[b])] = rows.int()
            s["n_keep"].copy_(torch.from_numpy(keep.astype(np.int32)).to(DEV)[None, :, None].expand(L, B, H))
            s["out"] = [torch.zeros_like(s[x]) for x in ("K", "V", "ks", "vs", "acc")]
    if own:
        s["ctx"] = _context(case, s["T"], B)
        if case["op"] == "attend":
            s["work"] = torch.empty(s["ctx"].cache_attend_work_bytes(B, s["max_n"], case["weights"]), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        ctx, B, T, blk = s["ctx"], case["batch"], s.get("T"), case["block"]
        if op == "rotary":
            ctx.rotary(case["tokens"], s["q"], s["k"], s["pos"], s["inv_freq"], case["rot"], case["interleaved"], case["mscale"], s["q_out"], s["k_out"])
        elif op == "append":
            ctx.cache_append(0, B, s["k"], s["v"], s["n"], s["cu_new"], s["max_new"], s["cu_tok"], s["n_tok"], s["K"], s["V"], s["ks"], s["vs"],
                             T, blk, s["acc"])
        elif op == "attend":
            ctx.cache_attend(0, B, s["q"], s["K"], s["V"], s["ks"], s["vs"], T, blk, s["cu_tok"], s["n"], s["idx"], s["max_n"], s["out"], s["lse"],
                             s["acc"], s["acc_out"], 0.99, s["work"])
        elif op == "evict":
            ctx.cache_evict(B, s["acc"], T, s["cu_tok"], s["n_tok"], s["max_n"], case["keep"], case["sink"], case["recent"], s["keep_idx"], s["n_keep"])
        else:
            ctx.cache_compact(B, s["K"], s["V"], s["ks"], s["vs"], s["acc"], T, blk, s["cu_tok"], s["keep_idx"], case["keep"], s["n_keep"], *s["out"])
    else:
        {"rotary": _rotary, "append": _append, "attend": _attend, "evict": _evict, "compact": _compact}[op](s)
    return _outputs(s)


def _outputs(s):
    op = s["case"]["op"]
    if op == "rotary":
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "append":
        return {"K": s["K"].view(F8), "V": s["V"].view(F8), "ks": s["ks"], "vs": s["vs"], "acc": s["acc"]}
    if op == "attend":
        return {"out": s["out"], "lse": s["lse"], **({"acc": s["acc_out"]} if s["acc"] is not None else {})}
    if op == "evict":
        return {"keep_idx": s["keep_idx"], "n_keep": s["n_keep"]}
    K, V, ks, vs, acc = s["out"]
    return {"K": K.view(F8), "V": V.view(F8), "ks": ks, "vs": vs, "acc": acc}


def _rotary(s):
    case = s["case"]
    rot, half = case["rot"], case["rot"] // 2
    angle = s["pos"].double()[:, None] * s["inv_freq"]
    c, si = (torch.cos(angle) * case["mscale"]).float()[:, None], (torch.sin(angle) * case["mscale"]).float()[:, None]

    def turn(x, out):
        y = x[..., :rot].float()
        y = y.unflatten(-1, (half, 2)) if case["interleaved"] else y.unflatten(-1, (2, half)).transpose(-1, -2)
        a, b = y[..., 0], y[..., 1]
        z = torch.stack((a * c - b * si, b * c + a * si), dim=-1 if case["interleaved"] else -2).flatten(-2)
        out[..., :rot] = z.to(x.dtype)
        out[..., rot:] = x[..., rot:]

    turn(s["q"], s["q_out"])
    turn(s["k"], s["k_out"])


def _append(s):
    case = s["case"]
    blk, H, B = case["block"], case["kv_heads"], case["batch"]
    cu, cu_new, n_tok = s["cu_tok"].long(), s["cu_new"].long(), s["n_tok"].long()
    i = torch.arange(s["n"], device=DEV)
    b = torch.searchsorted(cu_new, i, right=True) - 1
    row = n_tok[b] + (i - cu_new[b])[:, None]                                        # [n][H], local to the sequence
    h = torch.arange(H, device=DEV)
    slot = cu[b][:, None] // blk + b[:, None] + row // blk
    at = cu[b][:, None] + row
    # the blocks that hold rows already: one per sequence and head
    seq = torch.arange(B, device=DEV)[:, None]
    open_row = n_tok // blk * blk                                                     # [B][H]
    open_slot = (cu[:-1, None] // blk + seq + n_tok // blk).clamp(max=s["NS"] - 1)
    r = open_row[..., None] + torch.arange(blk, device=DEV)                           # [B][H][blk]
    there = r < n_tok[..., None]
    old_at = (cu[:-1, None, None] + r).clamp(max=s["T"] - 1)
    has = n_tok % blk > 0

    def store(x, codes, scale):
        codes, scale, x = codes.view(F8)[0], scale[0], x.float()
        most = torch.zeros(H, s["NS"], device=DEV).view(-1)
        most.scatter_reduce_(0, (h * s["NS"] + slot).flatten(), x.abs().amax(-1).flatten(), "amax")
        before = scale[h, open_slot].clone()
        fresh = _scale_of(most).view(H, s["NS"])
        touched = torch.zeros(H, s["NS"], dtype=torch.bool, device=DEV)
        touched[h.expand_as(slot), slot] = True
        held = torch.zeros_like(fresh)
        held[h, open_slot] = torch.where(has, before, 0.0)
        scale.copy_(torch.where(touched, torch.maximum(fresh, held), scale))
        ratio = torch.where(touched[h, open_slot], before / scale[h, open_slot], 1.0)
        old = codes.view(torch.uint8)[h[:, None], old_at].view(F8).float()
        where = there.nonzero(as_tuple=True)
        codes.view(torch.uint8)[where[1], old_at[where]] = (old * ratio[..., None, None])[where].to(F8).view(torch.uint8)
        codes.view(torch.uint8)[h.expand_as(at), at] = (x / scale[h, slot][..., None]).to(F8).view(torch.uint8)

    store(s["k"], s["K"], s["ks"])
    store(s["v"], s["V"], s["vs"])
    s["acc"][0][h.expand_as(at), at] = 0.0


def _attend(s):
    case = s["case"]
    blk, H, B, G = case["block"], case["kv_heads"], case["batch"], case["q_heads"] // case["kv_heads"]
    cu, h = s["cu_tok"].long(), torch.arange(H, device=DEV)[:, None]
    j = torch.arange(s["max_n"], device=DEV).expand(B, H, s["max_n"])
    there = j < s["n"][..., None]
    row = torch.where(there, j if s["idx"] is None else s["idx"].long(), 0)
    at, slot = cu[:-1, None, None] + row, (cu[:-1] // blk + torch.arange(B, device=DEV))[:, None, None] + row // blk
    K = s["K"][0][h, at].view(F8).float() * s["ks"][0][h, slot][..., None]
    x = torch.matmul(s["q"].float().view(B, H, G, D), K.transpose(-1, -2)) / math.sqrt(D)
    del K
    x = x.masked_fill(~there[:, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    z = e.sum(-1, keepdim=True)
    p = e / torch.where(z > 0, z, 1.0)
    V = s["V"][0][h, at].view(F8).float() * s["vs"][0][h, slot][..., None]
    s["out"].copy_(torch.matmul(p, V).view(B, -1, D))
    s["lse"].copy_((m + torch.log(z)).view(B, -1))
    if s["acc"] is not None:
        hh = h.expand(B, H, s["max_n"])[there]
        s["acc_out"][0][hh, at[there]] = 0.99 * s["acc"][0][hh, at[there]] + p.sum(2)[there]


def _evict(s):
    case = s["case"]
    L, H, B, keep = case["layers"], case["kv_heads"], case["batch"], case["keep"]
    cu, n = s["cu_tok"].long(), s["n_tok"].long()[..., None]                          # [L][B][H][1]
    j = torch.arange(s["max_n"], device=DEV)
    at = (cu[:-1, None] + j).clamp(max=s["T"] - 1)                                    # [B][max_n]
    a = s["acc"][:, :, at].transpose(1, 2)                                            # [L][B][H][max_n]
    a = torch.where((j < case["sink"]) | (j >= n - case["recent"]), math.inf, a)
    a = torch.where(j < n, a, -math.inf)
    first = a.sort(dim=-1, descending=True, stable=True).indices[..., :keep]          # equal weights: the lower row first
    first = torch.where(torch.arange(first.shape[-1], device=DEV) < n, first, 1 << 30).sort(dim=-1).values
    kept = first < (1 << 30)
    s["keep_idx"][..., : first.shape[-1]] = torch.where(kept, first.int(), s["keep_idx"][..., : first.shape[-1]])
    s["n_keep"].copy_(n[..., 0].clamp(max=keep))


def _compact(s):
    case = s["case"]
    blk, L, H, B, keep = case["block"], case["layers"], case["kv_heads"], case["batch"], case["keep"]
    cu = s["cu_tok"].long()
    base = (cu[:-1] // blk + torch.arange(B, device=DEV))[:, None, None]
    j = torch.arange(keep, device=DEV)
    there = (j < s["n_keep"].long()[..., None]).nonzero(as_tuple=True)                # l, b, h, j of every kept row
    l, b, h, j = there
    src = s["keep_idx"].long()[there]
    frm, to = cu[b] + src, cu[b] + j
    base = base[b, 0, 0]
    dst_slot = base + j // blk
    flat = (l * H + h) * s["NS"] + dst_slot
    Ko, Vo, kso, vso, acco = s["out"]

    def move(codes, scale, codes_out, scale_out):
        before = scale[l, h, base + src // blk]
        most = torch.zeros(scale.numel(), device=DEV).scatter_reduce_(0, flat, before, "amax").view_as(scale)
        scale_out.copy_(torch.where(most > 0, most, scale_out))
        ratio = before / scale_out[l, h, dst_slot]
        codes_out[l, h, to] = (codes[l, h, frm].view(F8).float() * ratio[:, None]).to(F8).view(torch.uint8)

    move(s["K"], s["ks"], Ko, kso)
    move(s["V"], s["vs"], Vo, vso)
    acco[l, h, to] = s["acc"][l, h, frm]


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------

def work(case):
    L, H, Hq, B = case["layers"], case["kv_heads"], case["q_heads"], case["batch"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "rotary":
        rows = case["tokens"] * (H + Hq)
        return {"bytes": 2 * rows * D * e, "flops": 3 * rows * case["rot"]}
    held = B * (case["held_min"] + case["held_max"]) / 2
    if case["op"] == "append":
        n = B * (case["new_min"] + case["new_max"]) / 2 * H
        return {"bytes": 2 * n * D * (e + 1) + 4 * n, "flops": 2 * 4 * n * D}
    if case["op"] == "attend":
        rows = (min(held, 0.75 * B * case["listed"]) if case["listed"] else held) * H
        return {"bytes": rows * (2 * D + (8 if case["weights"] else 0)) + B * Hq * D * (e + 4), "flops": 4 * rows * (Hq // H) * D}
    if case["op"] == "evict":
        return {"bytes": 4 * L * H * (held + B * case["keep"]), "flops": 4 * L * H * held}
    rows = L * H * min(held, B * case["keep"])
    return {"bytes": rows * (4 * D + 4 + 8), "flops": 2 * rows * D}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------

def _nearest8(x):
    """The value of the nearest E4M3 number, ties to the even one, of |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _power(a):
    """The smallest power of two p with a <= 448 p, for one number."""
    p = 2.0 ** -100
    if a > 0:
        p = max(p, 2.0 ** (math.ceil(math.log2(a / 448.0)) - 1))
        while a > 448.0 * p:
            p *= 2.0
    return p


def exact(case, seed):
    s = prepare(case, seed)
    L, H, B, blk = case["layers"], case["kv_heads"], case["batch"], case["block"]
    if case["op"] == "rotary":
        turns = torch.outer(s["pos"].double(), s["inv_freq"]) / (2 * math.pi)
        z = torch.polar(torch.full_like(turns, case["mscale"]), 2 * math.pi * (turns - torch.round(turns)))[:, None]
        out = []
        for x in (s["q"], s["k"]):
            x = x.double()
            y = x[..., : case["rot"]]
            if case["interleaved"]:
                w = torch.view_as_real(torch.complex(y[..., 0::2], y[..., 1::2]) * z).flatten(-2)
            else:
                w = torch.complex(*y.chunk(2, dim=-1)) * z
                w = torch.cat((w.real, w.imag), dim=-1)
            out.append(torch.cat((w, x[..., case["rot"]:]), dim=-1))
        return {"q": out[0], "k": out[1]}
    if case["op"] == "evict":
        return None
    cu = s["cu"].tolist()
    if case["op"] == "attend":
        G = case["q_heads"] // H
        out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV), torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
        acc = None if s["acc"] is None else torch.zeros(s["acc"].shape, dtype=torch.float64, device=DEV)
        n = s["n"].tolist()
        for b in range(B):
            for h in range(H):
                row = torch.arange(n[b][h], device=DEV) if s["idx"] is None else s["idx"][b, h, : n[b][h]].long()
                if not len(row):
                    continue
                slot = cu[b] // blk + b + row // blk
                K, V = ((s[x][0, h, cu[b] + row].view(F8).double() * s[y][0, h, slot].double()[:, None]) for x, y in (("K", "ks"), ("V", "vs")))
                x = s["q"][b, h * G:(h + 1) * G].double() @ K.T / math.sqrt(D)
                z = torch.logsumexp(x, dim=-1)
                p = torch.exp(x - z[:, None])
                out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = p @ V, z
                if acc is not None:
                    acc[0, h, cu[b] + row] = 0.99 * s["acc"][0, h, cu[b] + row].double() + p.sum(0)
        return {"out": out, "lse": lse, **({} if acc is None else {"acc": acc})}
    if case["op"] == "append":
        if sum(-(-int(x) // blk) + 1 for x in s["cu_new"].diff().tolist()) * H > 20000:
            return None
        held, cu_new, acc = s["n_tok"][:, 0].tolist(), s["cu_new"].tolist(), s["acc"].double()
        for b in range(B):
            acc[0, :, cu[b] + held[b]: cu[b] + held[b] + cu_new[b + 1] - cu_new[b]] = 0.0
        found = {"acc": acc}
        for x, codes, scale in (("k", "K", "ks"), ("v", "V", "vs")):
            c, p = s[codes].view(F8).float().double(), s[scale].double()
            for b in range(B):
                new = s[x][cu_new[b]: cu_new[b + 1]].double().transpose(0, 1)         # [H][m][D]
                done = 0
                while done < new.shape[1]:
                    at = held[b] + done
                    first = at // blk * blk
                    m = min(first + blk - at, new.shape[1] - done)
                    slot, rows = cu[b] // blk + b + at // blk, new[:, done: done + m]
                    fresh = torch.tensor([_power(a) for a in rows.abs().amax((1, 2)).tolist()], dtype=torch.float64, device=DEV)
                    if at > first:
                        fresh = torch.maximum(fresh, p[0, :, slot])
                        c[0, :, cu[b] + first: cu[b] + at] = _nearest8(c[0, :, cu[b] + first: cu[b] + at] * (p[0, :, slot] / fresh)[:, None, None])
                    p[0, :, slot] = fresh
                    c[0, :, cu[b] + at: cu[b] + at + m] = _nearest8(rows / fresh[:, None, None])
                    done += m
            found[codes], found[scale] = c, p
        return {x: found[x] for x in ("K", "V", "ks", "vs", "acc")}
    if L * B * H * case["keep"] > 1 << 21:
        return None
    found = {"acc": torch.zeros(s["acc"].shape, dtype=torch.float64, device=DEV)}
    kept = s["n_keep"][0, :, 0].tolist()
    for codes, scale in (("K", "ks"), ("V", "vs")):
        c, p = torch.zeros(s[codes].shape, dtype=torch.float64, device=DEV), torch.zeros(s[scale].shape, dtype=torch.float64, device=DEV)
        for b in range(B):
            base = cu[b] // blk + b
            for first in range(0, kept[b], blk):
                rows = s["keep_idx"][:, b, :, first: min(first + blk, kept[b])].long()           # [L][H][m]
                own_scale = s[scale].double().gather(2, base + rows // blk)
                p[:, :, base + first // blk] = own_scale.amax(-1)
                x = s[codes].gather(2, (cu[b] + rows)[..., None].expand(*rows.shape, D)).view(F8).float().double()
                at = cu[b] + first
                c[:, :, at: at + rows.shape[-1]] = _nearest8(x * (own_scale / own_scale.amax(-1, keepdim=True))[..., None])
                if codes == "K":
                    found["acc"][:, :, at: at + rows.shape[-1]] = s["acc"].double().gather(2, cu[b] + rows)
        found[codes], found[scale] = c, p
    return {x: found[x] for x in ("K", "V", "ks", "vs", "acc")}
