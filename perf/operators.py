"""The operators around the 8-bit paged KV cache, as cases that can be timed: their plain form, and the calls of this package.

  append   one layer's norms of the query and key heads, rotary embedding and cache append (arb_stage_norm_rope_append)
  attend   append-attention of one layer over a paged cache, scores optionally capped (arb_stage_attention_kv)
  pack     blocks of a bf16 cache into the 8-bit format (arb_kv8_pack)
  unpack   blocks of an 8-bit cache back into bf16 (arb_kv8_unpack)

The 8-bit cache holds a key or value row of one position and kv head as e4m3 elements and one power-of-two scale: with e the
least integer for which max|x| <= 448 * 2^e (and e >= -100), element = e4m3(x * 2^-e), scale byte = e + 127.  Elements come back
as float8_e4m3fn and scales as float8_e8m0fnu, the types whose values they are.

Head layouts are those of the repository's three shapes (workloads/configs.py) and two generic ones (one kv head per query
head; a single kv head).
"""
import math

import torch

own = False

BLOCK = 16
EPS, BASE = 1e-6, 10000.0
LOG2E = 1.4426950408889634

# query heads, kv heads, head dim
HEADS = {
    "tiny": (4, 2, 64),
    "router": (12, 2, 128),
    "target": (32, 8, 128),
    "single": (16, 16, 64),
    "multi": (8, 1, 128),
}


def _case(name, kind, heads, batch, prefix, step, **more):
    c = {"name": name, "kind": kind, "heads": heads, "batch": batch, "prefix_lo": prefix[0], "prefix_hi": prefix[1],
         "step_lo": step[0], "step_hi": step[1], "cache": "e4m3", "norms": False, "softcap": 0.0, "q_scaled": True,
         "lengths_seed": 1}
    c.update(more)
    return c


def _blocks_case(name, kind, heads, blocks, listed_blocks=True):
    return {"name": name, "kind": kind, "heads": heads, "blocks": blocks, "by_list": listed_blocks}


def listed():
    return [
        # one question, one token: the router's decoding step, bound by latency
        _case("append-router-b1-s1", "append", "router", 1, (1531, 1531), (1, 1), norms=True),
        # small ragged steps of the tiny shape into a bf16 cache
        _case("append-tiny-b7-bf16", "append", "tiny", 7, (3, 700), (1, 45), norms=True, cache="bf16", q_scaled=False),
        # one long prompt enters the target's cache
        _case("append-target-b1-s3001", "append", "target", 1, (0, 0), (3001, 3001), norms=True),
        # one question, one token against a middling context: bound by latency
        _case("attend-router-b1-s1", "attend", "router", 1, (1531, 1531), (1, 1)),
        # a serving batch decodes token by token against long ragged contexts: bound by the cache
        _case("attend-target-b32-s1", "attend", "target", 32, (4096, 32768), (1, 1)),
        # the router scores drafted steps: the headline workload's batch
        _case("attend-router-b16-s64", "attend", "router", 16, (2048, 2048), (64, 64)),
        # a chunk of a long prompt, capped scores: bound by the matrix units
        _case("attend-target-chunk-cap", "attend", "target", 1, (6005, 6005), (2048, 2048), softcap=50.0),
        # few ragged tokens per sequence over a bf16 cache, capped scores, queries as they are
        _case("attend-tiny-b9-bf16-cap", "attend", "tiny", 9, (5, 1700), (1, 9), softcap=30.0, cache="bf16", q_scaled=False),
        # one finished prompt moves into the 8-bit cache
        _blocks_case("pack-router-131", "pack", "router", 131),
        # the cache of a whole batch is converted
        _blocks_case("pack-target-8192", "pack", "target", 8192, False),
        # one sequence is read back
        _blocks_case("unpack-tiny-95", "unpack", "tiny", 95),
        # long contexts are read back for a caller that wants bf16
        _blocks_case("unpack-target-9000", "unpack", "target", 9000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    """An inclusive range of lengths inside [lo, hi]; one draw in three is a single length."""
    a, b = sorted((_log(rng, lo, hi), _log(rng, lo, hi)))
    return (b, b) if rng.random() < 1 / 3 else (a, b)


def _cost(c):
    w = work(c)
    return w["flops"] / 4e14 + w["bytes"] / 4e12


def _plain_bytes(c):
    """Memory of the plain form's widest intermediates: padded fp32 scores, keys and values."""
    if c["kind"] != "attend":
        return 0
    n_q, n_kv, hd = HEADS[c["heads"]]
    ctx = c["prefix_hi"] + c["step_hi"]
    return 4 * c["batch"] * ctx * (n_q * c["step_hi"] + 2 * n_kv * hd)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        heads = rng.choice(sorted(HEADS))
        k = rng.randrange(8)
        if k <= 1:
            c = _case("", "append", heads, _log(rng, 1, 64), _span(rng, 1, 20000), _span(rng, 1, 600), norms=rng.random() < 0.7,
                      cache=rng.choice(("e4m3", "e4m3", "bf16")), q_scaled=rng.random() < 0.5)
        elif k <= 3:
            c = _case("", "attend", heads, _log(rng, 1, 64), _span(rng, 16, 32768), (1, rng.choice((1, 1, 2, 5))))
        elif k == 4:
            c = _case("", "attend", heads, _log(rng, 1, 32), _span(rng, 64, 8192), _span(rng, 4, 128))
        elif k == 5:
            c = _case("", "attend", heads, 1, _span(rng, 1, 8000), _span(rng, 200, 2048))
        else:
            c = _blocks_case("", rng.choice(("pack", "unpack")), heads, _log(rng, 1, 9000), rng.random() < 0.7)
        if c["kind"] == "attend":
            c.update(cache=rng.choice(("e4m3", "e4m3", "e4m3", "bf16")), softcap=rng.choice((0.0, 0.0, 30.0, 50.0)),
                     q_scaled=rng.random() < 0.6)
        if "lengths_seed" in c:
            c["lengths_seed"] = rng.randrange(1, 1 << 30)
        del c["name"]
        if _cost(c) <= most and _plain_bytes(c) < 2e10:
            return c


def _lengths(c):
    """Prefix and step lengths of the batch: part of the case, the same for every seed of the inputs."""
    g = torch.Generator().manual_seed(c["lengths_seed"])
    pick = lambda lo, hi: torch.randint(lo, hi + 1, (c["batch"],), generator=g)  # noqa: E731
    return pick(c["prefix_lo"], c["prefix_hi"]), pick(c["step_lo"], c["step_hi"])


def work(case):
    n_q, n_kv, hd = HEADS[case["heads"]]
    row8, row16 = 2 * hd + 2, 4 * hd                       # bytes of a position and kv head: keys, values and scales
    if case["kind"] in ("pack", "unpack"):
        return {"bytes": case["blocks"] * n_kv * BLOCK * (row8 + row16), "flops": 0}
    prefix, step = _lengths(case)
    tokens = int(step.sum())
    row = row8 if case["cache"] == "e4m3" else row16
    if case["kind"] == "append":
        return {"bytes": tokens * ((n_q + 2 * n_kv) * hd * 2 + n_q * hd * 2 + n_kv * row), "flops": 0}
    seen = int((step * prefix + step * (step + 1) // 2).sum())
    return {"bytes": int((prefix + step).sum()) * n_kv * row + 2 * tokens * n_q * hd * 2, "flops": 4 * n_q * hd * seen}


# ------------------------------------------------------------------------------------------- inputs


def _quantize(x):
    """fp32 [..., hd] -> (float8_e4m3fn [..., hd], uint8 scale bytes [...])."""
    m, k = torch.frexp(x.abs().amax(-1))                   # max|x| = m 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, k - 9, k - 8)
    e = torch.where(m == 0, -100, e).clamp(min=-100)
    return (x * torch.exp2(-e.float())[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(elements, scale_bytes):
    return elements.float() * torch.exp2(scale_bytes.float() - 127)[..., None]


def _rows(g, blocks, n_kv, hd, sigma):
    """Key or value rows of whole blocks: row magnitudes vary, two channels in 32 are loud, as in real caches."""
    x = torch.randn(blocks, n_kv, BLOCK, hd, generator=g, device="cuda") * sigma
    x *= torch.exp(0.5 * torch.randn(blocks, n_kv, BLOCK, 1, generator=g, device="cuda"))
    x[..., 3::16] *= 3.0
    return x


def _pools(g, blocks, n_kv, hd, kind, sigma):
    """(k, v, k_scale, v_scale) of a cache; the scales are None for bf16.  Made in pieces: a long cache's fp32 rows need not fit at once."""
    out = []
    for _ in range(2):
        pool = torch.empty(blocks, n_kv, BLOCK, hd, device="cuda", dtype=torch.bfloat16 if kind == "bf16" else torch.float8_e4m3fn)
        scale = None if kind == "bf16" else torch.empty(blocks, n_kv, BLOCK, device="cuda", dtype=torch.uint8)
        for at in range(0, blocks, 8192):
            x = _rows(g, min(8192, blocks - at), n_kv, hd, sigma)
            if kind == "bf16":
                pool[at:at + 8192] = x.bfloat16()
            else:
                q, s = _quantize(x)
                pool[at:at + 8192].view(torch.uint8).copy_(q.view(torch.uint8))
                scale[at:at + 8192] = s
        out += [pool, scale]
    return out[0], out[2], out[1], out[3]


def _model(A, n_q, n_kv, hd):
    """The smallest model that has these heads: the operators of one layer take their shapes from a model."""
    d = 128
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    one = torch.ones(d, device="cuda")

    class W:
        embed, g_final, w_head, b_head = bf(128, d), one, one, 0.0
        wqkv, wo, wgu, wd = [bf((n_q + 2 * n_kv) * hd, d)], [bf(d, n_q * hd)], [bf(2 * d, d)], [bf(d, d)]
        g_attn, g_mlp = [one], [one]

    return A.Model(n_layers=1, d_model=d, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd, d_ffn=d, vocab=128, weights=W,
                   rms_eps=EPS, rope_base=BASE, has_router_head=False, block_gate_up=False)


def prepare(case, seed):
    n_q, n_kv, hd = HEADS[case["heads"]]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case, "heads": (n_q, n_kv, hd)}
    if case["kind"] in ("pack", "unpack"):
        n = case["blocks"]
        room = n + n // 4 if case["by_list"] else n        # the list picks and places blocks of larger pools
        for side, kind in (("src", "bf16" if case["kind"] == "pack" else "e4m3"), ("dst", "e4m3" if case["kind"] == "pack" else "bf16")):
            if side == "src":
                s["src"] = _pools(g, room, n_kv, hd, kind, 1.0)
            elif kind == "bf16":
                s["dst"] = tuple(torch.zeros(room, n_kv, BLOCK, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)) + (None, None)
            else:
                s["dst"] = tuple(torch.zeros(room, n_kv, BLOCK, hd, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)) + \
                    tuple(torch.full((room, n_kv, BLOCK), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
            s[side + "_blocks"] = torch.randperm(room, generator=g, device="cuda")[:n].int() if case["by_list"] else None
        if own:
            import paper_2512_05033_amd as A
            s["A"], s["src_layer"], s["dst_layer"] = A, A.KVLayer(*s["src"]), A.KVLayer(*s["dst"])
        return s
    prefix, step = _lengths(case)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), step.cumsum(0)])
    tokens, batch = int(cu[-1]), case["batch"]
    per_seq = -(-(prefix + step) // BLOCK)
    width = int(per_seq.max())
    if case["kind"] == "append":
        # the pool holds the blocks that the steps write to; a call reads no others
        first = prefix // BLOCK
        used = (torch.arange(width)[None, :] >= first[:, None]) & (torch.arange(width)[None, :] < per_seq[:, None])
    else:
        used = torch.arange(width)[None, :] < per_seq[:, None]
    blocks = int(used.sum())
    table = torch.zeros(batch, width, dtype=torch.int64)
    table[used] = torch.randperm(blocks, generator=torch.Generator().manual_seed(seed))
    s.update(prefix=prefix.cuda(), cu=cu.cuda(), table=table.cuda(), tokens=tokens)
    s["seq"] = torch.repeat_interleave(torch.arange(batch), step).cuda()
    s["pos"] = s["prefix"][s["seq"]] + torch.arange(tokens, device="cuda") - s["cu"][s["seq"]]
    if case["kind"] == "append":
        s["qkv"] = (torch.randn(tokens, (n_q + 2 * n_kv) * hd, generator=g, device="cuda") * 1.5).bfloat16()
        s["gains"] = tuple(1 + 0.3 * torch.randn(hd, generator=g, device="cuda") for _ in range(2)) if case["norms"] else (None, None)
        if case["cache"] == "bf16":
            s["layer"] = tuple(torch.zeros(blocks, n_kv, BLOCK, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)) + (None, None)
        else:
            s["layer"] = tuple(torch.zeros(blocks, n_kv, BLOCK, hd, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)) + \
                tuple(torch.full((blocks, n_kv, BLOCK), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        s["out"] = torch.empty(tokens, n_q * hd, dtype=torch.bfloat16, device="cuda")
    else:
        q = torch.randn(tokens, n_q * hd, generator=g, device="cuda") * 1.2
        s["q"] = (q * (LOG2E / math.sqrt(hd)) if case["q_scaled"] else q).bfloat16()
        s["layer"] = _pools(g, blocks, n_kv, hd, case["cache"], 0.8)
        s["max_step"] = int(step.max())
    if own:
        import paper_2512_05033_amd as A
        s["A"], s["model"], s["kv"] = A, _model(A, n_q, n_kv, hd), A.KVLayer(*s["layer"])
        s["batch"] = A.DeviceBatch(prefix.numpy(), cu.numpy(), table.numpy())
        s["ws"] = torch.empty(max(256, s["model"].workspace_bytes(batch, tokens, int((prefix + step).max()))), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------- the plain forms


def _as_values(layer):
    """A layer's pools as they are returned: elements and scales in the types whose values they hold."""
    k, v, ks, vs = layer
    if ks is None:
        return {"k": k, "v": v}
    return {"k": k, "v": v, "k_scale": ks.view(torch.float8_e8m0fnu), "v_scale": vs.view(torch.float8_e8m0fnu)}


def _store(pool, scale, blk, row, x):
    """x fp32 [T, n_kv, hd] into the slots (blk, row) of every kv head."""
    if scale is None:
        pool[blk, :, row] = x.to(pool.dtype)
    else:
        e, b = _quantize(x)
        pool.view(torch.uint8)[blk, :, row] = e.view(torch.uint8)
        scale[blk, :, row] = b


def _append(s):
    n_q, n_kv, hd = s["heads"]
    T, half = s["tokens"], hd // 2
    u = s["qkv"].float().view(T, n_q + 2 * n_kv, hd)
    q, k, v = u[:, :n_q], u[:, n_q:n_q + n_kv], u[:, n_q + n_kv:]
    if s["gains"][0] is not None:
        q, k = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * g for x, g in zip((q, k), s["gains"]))
    inv = BASE ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = s["pos"].double()[:, None] * inv               # 64 bits: positions of tens of thousands
    c, n = angle.cos().float()[:, None], angle.sin().float()[:, None]
    turn = lambda x: torch.cat([x[..., :half] * c - x[..., half:] * n, x[..., half:] * c + x[..., :half] * n], -1)  # noqa: E731
    f = LOG2E / math.sqrt(hd) if s["case"]["q_scaled"] else 1.0
    blk, row = s["table"][s["seq"], s["pos"] // BLOCK], s["pos"] % BLOCK
    _store(s["layer"][0], s["layer"][2], blk, row, turn(k))
    _store(s["layer"][1], s["layer"][3], blk, row, v)
    return (turn(q) * f).bfloat16().view(T, n_q * hd)


def _attend(s):
    n_q, n_kv, hd = s["heads"]
    B, S, G, T = s["case"]["batch"], s["max_step"], n_q // n_kv, s["tokens"]
    k, v, ks, vs = s["layer"]
    at = s["table"]                                        # [B, width]
    gather = lambda x, sc: (x[at].float() if sc is None else _values(x.view(torch.uint8)[at].view(torch.float8_e4m3fn), sc[at])) \
        .transpose(1, 2).reshape(B, n_kv, -1, hd)  # noqa: E731
    keys, vals = gather(k, ks), gather(v, vs)
    i = torch.arange(T, device="cuda") - s["cu"][s["seq"]]
    q = torch.zeros(B, S, n_q, hd, device="cuda")
    q[s["seq"], i] = s["q"].float().view(T, n_q, hd)
    q = q.view(B, S, n_kv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, n_kv, G * S, hd)
    logits = torch.matmul(q, keys.transpose(-1, -2))
    logits *= 1 / LOG2E if s["case"]["q_scaled"] else 1 / math.sqrt(hd)
    cap = s["case"]["softcap"]
    if cap > 0:
        logits = torch.tanh(logits / cap) * cap
    pos = s["prefix"][:, None] + torch.arange(S, device="cuda")
    seen = torch.arange(keys.shape[2], device="cuda")[None, None, :] <= pos[:, :, None]          # [B, S, ctx]
    logits = logits.view(B, n_kv, G, S, -1).masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, n_kv, G * S, -1), vals).view(B, n_kv, G, S, hd).permute(0, 3, 1, 2, 4)
    return o[s["seq"], i].bfloat16().reshape(T, n_q * hd)


def _convert(s):
    n = s["case"]["blocks"]
    src = slice(0, n) if s["src_blocks"] is None else s["src_blocks"].long()
    dst = slice(0, n) if s["dst_blocks"] is None else s["dst_blocks"].long()
    k, v, ks, vs = s["src"]
    dk, dv, dks, dvs = s["dst"]
    if s["case"]["kind"] == "pack":
        (ek, bk), (ev, bv) = _quantize(k[src].float()), _quantize(v[src].float())
        dk.view(torch.uint8)[dst], dv.view(torch.uint8)[dst] = ek.view(torch.uint8), ev.view(torch.uint8)
        dks[dst], dvs[dst] = bk, bv
    else:
        dk[dst] = _values(k.view(torch.uint8)[src].view(torch.float8_e4m3fn), ks[src]).bfloat16()
        dv[dst] = _values(v.view(torch.uint8)[src].view(torch.float8_e4m3fn), vs[src]).bfloat16()


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        A = s["A"]
        if kind == "append":
            q = A.arb_stage_norm_rope_append(s["model"], s["qkv"], s["kv"], s["batch"], g_q=s["gains"][0], g_k=s["gains"][1],
                                             q_scaled=s["case"]["q_scaled"], out=s["out"])
            return {"q": q, **_as_values(s["layer"])}
        if kind == "attend":
            return A.arb_stage_attention_kv(s["model"], s["q"], s["kv"], s["batch"], softcap=s["case"]["softcap"],
                                            q_scaled=s["case"]["q_scaled"], ws=s["ws"])
        (A.arb_kv8_pack if kind == "pack" else A.arb_kv8_unpack)(s["src_layer"], s["dst_layer"], s["src_blocks"], s["dst_blocks"],
                                                                 n_blocks=s["case"]["blocks"])
        return _as_values(s["dst"])
    if kind == "append":
        return {"q": _append(s), **_as_values(s["layer"])}
    if kind == "attend":
        return _attend(s)
    _convert(s)
    return _as_values(s["dst"])


# ------------------------------------------------------------------------- the definition, 64 bits


def _e4m3_rows(x):
    """The format from its definition: -> (elements, scales), both as fp64 values."""
    m = x.abs().amax(-1)
    e = torch.ceil(torch.log2(m.clamp(min=2.0 ** -120) / 448))
    e = torch.where(448 * torch.exp2(e - 1) >= m, e - 1, e)                # the logarithm may be off by a hair: the definition decides
    e = torch.where(448 * torch.exp2(e) < m, e + 1, e).clamp(min=-100)
    y = x * torch.exp2(-e)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(max=8) - 3)
    return torch.round(y / step) * step, torch.exp2(e)


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    n_q, n_kv, hd = s["heads"]
    if case["kind"] in ("pack", "unpack"):
        n = case["blocks"]
        src, dst = (torch.arange(n, device="cuda") if b is None else b.long() for b in (s["src_blocks"], s["dst_blocks"]))
        out = {}
        for name, pool, scale, to in (("k", s["src"][0], s["src"][2], s["dst"][0]), ("v", s["src"][1], s["src"][3], s["dst"][1])):
            out[name] = torch.zeros(to.shape, dtype=torch.float64, device="cuda")
            if case["kind"] == "pack":
                out[name + "_scale"] = torch.ones(to.shape[:-1], dtype=torch.float64, device="cuda")
            for at in range(0, n, 1024):
                i, j = src[at:at + 1024], dst[at:at + 1024]
                if case["kind"] == "pack":
                    out[name][j], out[name + "_scale"][j] = _e4m3_rows(pool[i].double())
                else:
                    out[name][j] = pool.view(torch.uint8)[i].view(torch.float8_e4m3fn).double() * (2.0 ** (scale[i].double() - 127))[..., None]
        return out
    prefix, cu, table = s["prefix"].tolist(), s["cu"].tolist(), s["table"]
    if case["kind"] == "append":
        x = s["qkv"].double().view(-1, n_q + 2 * n_kv, hd)
        half = hd // 2
        out = {"q": torch.empty(s["tokens"], n_q, hd, dtype=torch.float64, device="cuda")}
        e4m3 = case["cache"] == "e4m3"
        for name, pool in (("k", s["layer"][0]), ("v", s["layer"][1])):
            out[name] = torch.zeros(pool.shape, dtype=torch.float64, device="cuda")
            if e4m3:
                out[name + "_scale"] = torch.ones(pool.shape[:-1], dtype=torch.float64, device="cuda")
        for b in range(case["batch"]):
            y = x[cu[b]:cu[b + 1]]
            pos = prefix[b] + torch.arange(y.shape[0], device="cuda", dtype=torch.float64)
            heads = {}
            for name, lo, hi, g in (("q", 0, n_q, s["gains"][0]), ("k", n_q, n_q + n_kv, s["gains"][1])):
                h = y[:, lo:hi]
                if g is not None:
                    h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * g.double()
                z = torch.complex(h[..., :half], h[..., half:])
                phase = pos[:, None] * torch.exp(-math.log(BASE) * 2 * torch.arange(half, device="cuda", dtype=torch.float64) / hd)
                z = z * torch.polar(torch.ones_like(phase), phase)[:, None]
                heads[name] = torch.cat([z.real, z.imag], -1)
            out["q"][cu[b]:cu[b + 1]] = heads["q"] * (LOG2E / math.sqrt(hd) if case["q_scaled"] else 1.0)
            p = pos.long()
            where = table[b][p // BLOCK], slice(None), p % BLOCK
            for name, rows in (("k", heads["k"]), ("v", y[:, n_q + n_kv:])):
                if e4m3:
                    out[name][where], out[name + "_scale"][where] = _e4m3_rows(rows)
                else:
                    out[name][where] = rows
        out["q"] = out["q"].view(s["tokens"], n_q * hd)
        return out
    k, v, ks, vs = s["layer"]
    out = torch.empty(s["tokens"], n_q, hd, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(-1, n_q, hd)
    for b in range(case["batch"]):
        n, steps = prefix[b] + cu[b + 1] - cu[b], cu[b + 1] - cu[b]
        blocks = table[b, :-(-n // BLOCK)]
        seen = torch.arange(n, device="cuda")[None] <= prefix[b] + torch.arange(steps, device="cuda")[:, None]
        for h in range(n_kv):
            rows = []
            for pool, scale in ((k, ks), (v, vs)):
                if scale is None:
                    r = pool[blocks, h].double()
                else:
                    r = pool.view(torch.uint8)[blocks, h].view(torch.float8_e4m3fn).double() * (2.0 ** (scale[blocks, h].double() - 127))[..., None]
                rows.append(r.reshape(-1, hd)[:n])
            mine = slice(h * (n_q // n_kv), (h + 1) * (n_q // n_kv))
            x = torch.matmul(q[cu[b]:cu[b + 1], mine].transpose(0, 1), rows[0].T)
            x = x / LOG2E if case["q_scaled"] else x / math.sqrt(hd)
            if case["softcap"] > 0:
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            p = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
            out[cu[b]:cu[b + 1], mine] = torch.matmul(p, rows[1]).transpose(0, 1)
    return out.view(s["tokens"], n_q * hd)
