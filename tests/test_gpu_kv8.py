"""The 8-bit KV cache on the GPU, through the C ABI, against plain fp64 implementations on the same inputs.

Bounds, derived: a rounding to bf16 is off by at most u = 2^-8 of the value, to e4m3 by 2^-4 of it (2^-10 of the scale below the
normal range).  Attention rounds every probability, every split's result and the result: with S = sum p |v| and |out| <= S,
  |error| <= u (sum p |v - out| + S + |out|) (1 + u) <= u (2 + 1 + 1) 1.01 S,
and what fp32 does to a logit of up to 50 (hd products, 2^-24 each) moves a probability by less than u / 8, twice (sum and
quotient): 4.3 u S in all, element by element.  Norms and rotation are a few fp32 operations on hd values: 2^-18 of the row's
largest covers them."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import arb_oracle as O
from oracle import kv8_oracle as K8

pytestmark = pytest.mark.gpu

U = 2.0 ** -8
HEADS = {"tiny": (4, 2, 64), "router": (12, 2, 128), "target": (32, 8, 128), "single": (16, 16, 64), "multi": (8, 1, 128)}


@pytest.fixture(scope="module")
def A():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_05033_amd as A
    A.load_library()
    return A


def H():
    import harness
    return harness


_models = {}


def stage_model(heads):
    if heads not in _models:
        hq, hkv, hd = HEADS[heads]
        m = W.ModelShape("stage", 1, 128, hq, hkv, hd, 128, 128)
        _models[heads] = H().make_model(m, W.make_weights(m, 5, "cuda"), has_router_head=False)
    return _models[heads]


def make_batch(A, prefix, steps, seed, spare=3):
    """A shuffled paged batch -> (DeviceBatch, tables, number of pool blocks, blocks of no sequence)."""
    per = [-(-(p + s) // 16) for p, s in zip(prefix, steps)]
    n = sum(per) + spare
    ids = np.random.default_rng(seed).permutation(n).astype(np.int32)
    tables = np.full((len(per), max(per)), int(ids[-1]), np.int32)
    at = 0
    for b, k in enumerate(per):
        tables[b, :k] = ids[at:at + k]
        at += k
    cu = np.concatenate([[0], np.cumsum(steps)]).astype(np.int32)
    return A.DeviceBatch(np.array(prefix, np.int32), cu, tables), tables, n


def rows(shape, seed, sigma=1.0):
    """bf16 rows whose magnitudes differ by position, with two loud channels in 32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda") * sigma * torch.exp(0.7 * torch.randn(*shape[:-1], 1, generator=g, device="cuda"))
    x[..., 3::16] *= 4
    return x.bfloat16()


def layer8(A, n, hkv, hd, fill=None):
    kv = A.KVCache8.empty(1, n, hkv, hd).layers[0]
    if fill is not None:                                         # what slots that were never written may hold
        for t in (kv.k_pool, kv.v_pool):
            t.view(torch.uint8).fill_(fill)
        kv.k_scale.fill_(255)
        kv.v_scale.fill_(255)
    return kv


def layer16(A, n, hkv, hd):
    return A.KVLayer(*(torch.zeros(n, hkv, 16, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)))


def values(kv):
    """fp64 [n, Hkv, 16, hd] keys and values of a layer."""
    if not kv.kv8:
        return kv.k_pool.double(), kv.v_pool.double()
    f = lambda p, s: p.double() * torch.exp2(s.double() - 127)[..., None]
    return f(kv.k_pool, kv.k_scale), f(kv.v_pool, kv.v_scale)


def filled(A, n, hkv, hd, seed, kv8=True, sigma=0.8):
    """A layer whose every slot is written: rows packed by the oracle on the host."""
    k, v = rows((n, hkv, 16, hd), seed, sigma), rows((n, hkv, 16, hd), seed + 1, sigma)
    if not kv8:
        return A.KVLayer(k, v)
    kv = layer8(A, n, hkv, hd)
    put_rows(kv, slice(None), k.double().cpu().numpy(), v.double().cpu().numpy())
    return kv


def put_rows(kv, where, k, v):
    ke, ve, kx, vx = K8.quantize(k, v)
    to8 = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float().cuda().to(torch.float8_e4m3fn).view(torch.uint8)
    byte = lambda e: torch.from_numpy((np.asarray(e) + 127).astype(np.uint8)).cuda()
    kv.k_pool.view(torch.uint8)[where], kv.v_pool.view(torch.uint8)[where] = to8(ke), to8(ve)
    kv.k_scale[where], kv.v_scale[where] = byte(kx), byte(vx)


def attention_ref(heads, q, kv, tables, prefix, steps, cap, q_scaled):
    """fp64 on the GPU -> (out, sum p |v|), [T, Hq, hd]."""
    hq, hkv, hd = HEADS[heads]
    G, T = hq // hkv, sum(steps)
    out, mag = torch.empty(T, hq, hd, dtype=torch.float64, device="cuda"), torch.empty(T, hq, hd, dtype=torch.float64, device="cuda")
    K, V = values(kv)
    qd, at = q[:T, :hq * hd].double().view(T, hq, hd), 0
    for b, (p, s) in enumerate(zip(prefix, steps)):
        n = p + s
        blocks = torch.from_numpy(tables[b, :-(-n // 16)].astype(np.int64)).cuda()
        seen = torch.arange(n, device="cuda")[None] <= p + torch.arange(s, device="cuda")[:, None]
        for h in range(hkv):
            k, v = (x[blocks, h].reshape(-1, hd)[:n] for x in (K, V))
            x = torch.matmul(qd[at:at + s, h * G:(h + 1) * G].transpose(0, 1), k.T)
            x = x * np.log(2.0) if q_scaled else x / np.sqrt(hd)
            if cap:
                x = cap * torch.tanh(x / cap)
            pr = torch.softmax(x.masked_fill(~seen, -np.inf), -1)
            out[at:at + s, h * G:(h + 1) * G] = torch.matmul(pr, v).transpose(0, 1)
            mag[at:at + s, h * G:(h + 1) * G] = torch.matmul(pr, v.abs()).transpose(0, 1)
        at += s
    return out, mag


def queries(T, heads, seed, q_scaled, sigma=1.2, extra=0, more=0):
    hq, hkv, hd = HEADS[heads]
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randn(T + more, hq * hd + extra, generator=g, device="cuda") * sigma
    return (q * (1.4426950408889634 / np.sqrt(hd)) if q_scaled else q).bfloat16()


def check_attention(A, heads, kv, prefix, steps, seed, db, tables, cap=0.0, q_scaled=False, sigma=1.2, **more):
    q = queries(sum(steps), heads, seed, q_scaled, sigma, extra=more.pop("extra", 0))
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, softcap=cap, q_scaled=q_scaled, **more)
    ref, mag = attention_ref(heads, q, kv, tables, prefix, steps, cap, q_scaled)
    err = (got.double().view(ref.shape) - ref).abs()
    assert bool((err <= 4.3 * U * mag + 1e-30).all()), float((err / (mag + 1e-30)).max() / U)
    return q, got


# --------------------------------------------------------------------------------- conversion

@pytest.mark.parametrize("heads,n", [("tiny", 1), ("router", 7), ("target", 33), ("single", 5), ("multi", 3)])
def test_pack_and_unpack_are_the_format_bit_for_bit(A, heads, n):
    hq, hkv, hd = HEADS[heads]
    src = A.KVLayer(rows((n + 4, hkv, 16, hd), 1), rows((n + 4, hkv, 16, hd), 2))
    src.k_pool[0, 0, 0], src.v_pool[0, 0, 1] = 0, 0                                        # rows of zeros
    src.k_pool[0, 0, 2] *= 2.0 ** -100                                                     # below the least scale
    src.k_pool[0, 0, 3] *= 2.0 ** 60
    src.v_pool[0, 0, 4, 1], src.k_pool[0, 0, 5, 2], src.v_pool[0, 0, 6, 3] = float("nan"), float("-inf"), 2.0 ** 120
    src.k_pool[0, 0, 7] = 448.0                                                            # the largest that scale 1 holds
    src.k_pool[0, 0, 8] = 450.0
    order = np.random.default_rng(n).permutation(n + 4)[:n].astype(np.int32)
    if 0 not in order:
        order[0] = 0
    to = np.random.default_rng(n + 1).permutation(n + 4)[:n].astype(np.int32)
    dst = layer8(A, n + 4, hkv, hd, fill=0x55)
    on = lambda a: torch.from_numpy(a).cuda()
    A.arb_kv8_pack(src, dst, on(order), on(to))
    ke, ve, kx, vx = K8.quantize(src.k_pool[on(order).long()].double().cpu().numpy(), src.v_pool[on(order).long()].double().cpu().numpy())
    for pool, scale, el, x in ((dst.k_pool, dst.k_scale, ke, kx), (dst.v_pool, dst.v_scale, ve, vx)):
        assert np.array_equal(pool.double().cpu().numpy()[to], el, equal_nan=True)
        assert np.array_equal(scale.cpu().numpy()[to], x + 127)
        rest = np.setdiff1d(np.arange(n + 4), to)
        assert (pool.view(torch.uint8).cpu().numpy()[rest] == 0x55).all() and (scale.cpu().numpy()[rest] == 255).all()
    back = layer16(A, n + 4, hkv, hd)
    A.arb_kv8_unpack(dst, back, on(to), on(order))
    for pool, el, x in ((back.k_pool, ke, kx), (back.v_pool, ve, vx)):
        got = pool.double().cpu().numpy()
        assert np.array_equal(got[order], el * np.exp2(x.astype(float))[..., None], equal_nan=True)     # exact in bf16
        assert (np.delete(got, order, 0) == 0).all()


def test_pack_of_whole_pools_and_of_a_block_listed_twice(A):
    hq, hkv, hd = HEADS["router"]
    src = A.KVLayer(rows((6, hkv, 16, hd), 3), rows((6, hkv, 16, hd), 4))
    whole, twice = layer8(A, 6, hkv, hd), layer8(A, 6, hkv, hd)
    A.arb_kv8_pack(src, whole)
    A.arb_kv8_pack(src, twice, torch.tensor([2, 2, 5], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 4], dtype=torch.int32, device="cuda"))
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        a, b = (getattr(x, name).view(torch.uint8) for x in (whole, twice))
        assert torch.equal(b[0], a[2]) and torch.equal(b[1], a[2]) and torch.equal(b[4], a[5])
    A.arb_kv8_pack(src, twice, n_blocks=0)
    some = layer8(A, 6, hkv, hd)
    A.arb_kv8_pack(src, some, n_blocks=2)
    assert torch.equal(some.k_pool.view(torch.uint8)[:2], whole.k_pool.view(torch.uint8)[:2]) and not bool(some.k_pool.view(torch.uint8)[2:].any())


# -------------------------------------------------------------------- norms, rotation and append

def append_ref(heads, qkv, prefix, steps, g_q, g_k, q_scaled):
    hq, hkv, hd = HEADS[heads]
    u = qkv.double().cpu().numpy().reshape(sum(steps), -1, hd)
    pos = np.concatenate([p + np.arange(s) for p, s in zip(prefix, steps)])
    gain = lambda g: None if g is None else g.double().cpu().numpy()
    q = O.rope(K8.head_norm(u[:, :hq], gain(g_q), 1e-6), pos, 10000.0)
    k = O.rope(K8.head_norm(u[:, hq:hq + hkv], gain(g_k), 1e-6), pos, 10000.0)
    return q * (np.log2(np.e) / np.sqrt(hd) if q_scaled else 1.0), k, u[:, hq + hkv:], pos


def check_append(A, heads, prefix, steps, kv8, norms, q_scaled, seed, in_place=False, qkv=None):
    hq, hkv, hd = HEADS[heads]
    T = sum(steps)
    db, tables, n = make_batch(A, prefix, steps, seed)
    qkv = rows((T, (hq + 2 * hkv) * hd), seed) if qkv is None else qkv
    g = [1 + 0.4 * torch.randn(hd, generator=torch.Generator(device="cuda").manual_seed(seed + i), device="cuda") if on else None for i, on in enumerate(norms)]
    kv = layer8(A, n, hkv, hd, fill=0x7f) if kv8 else layer16(A, n, hkv, hd)
    before = [x.clone() for x in (kv.k_pool.view(torch.uint8), kv.v_pool.view(torch.uint8))]
    given = qkv.clone()
    got = A.arb_stage_norm_rope_append(stage_model(heads), given, kv, db, g[0], g[1], q_scaled=q_scaled, in_place=in_place)
    q, k, v, pos = append_ref(heads, qkv, prefix, steps, g[0], g[1], q_scaled)
    gq = got.view(T, -1, hd)[:, :hq].double().cpu().numpy()
    big = lambda x: np.abs(x).max(-1, keepdims=True)
    assert (np.abs(gq - q) <= U * np.abs(q) + 2.0 ** -18 * big(q)).all()
    if in_place:
        assert torch.equal(got.view(T, -1, hd)[:, hq:], qkv.view(T, -1, hd)[:, hq:])
    else:
        assert torch.equal(given, qkv)
    seq = np.repeat(np.arange(len(steps)), steps)
    blk, row = tables[seq, pos // 16], pos % 16
    gk, gv = (x.cpu().numpy()[blk, :, row] for x in values(kv))
    if kv8:
        ke, ve, kx, vx = K8.quantize(k, v)
        e = kv.k_scale.cpu().numpy()[blk, :, row].astype(int) - 127
        m = np.maximum(big(k)[..., 0], 1e-30)
        near = np.abs(m / (448 * np.exp2(np.floor(np.log2(m / 448) + 0.5))) - 1) < 2.0 ** -17
        assert (np.abs(e - kx) <= near).all()                    # the scale may only differ where the largest is at a border
        assert (np.abs(gk - k) <= np.maximum(2.0 ** -4 * np.abs(k), 2.0 ** -10 * np.exp2(e.astype(float))[..., None]) + 2.0 ** -18 * big(k)).all()
        assert np.array_equal(gv, ve * np.exp2(vx.astype(float))[..., None])
    else:
        assert (np.abs(gk - k) <= U * np.abs(k) + 2.0 ** -18 * big(k)).all() and np.array_equal(gv, v)
    written = np.zeros((n, 16), bool)
    written[blk, row] = True
    for was, pool in zip(before, (kv.k_pool, kv.v_pool)):
        keep = torch.from_numpy(~written).cuda()[:, None, :, None]
        assert bool(((pool.view(torch.uint8) == was) | ~keep).all())
    if kv8:
        for scale in (kv.k_scale, kv.v_scale):
            assert bool(((scale == 255) | torch.from_numpy(written).cuda()[:, None]).all())
    return kv


@pytest.mark.parametrize("kv8", [True, False])
@pytest.mark.parametrize("heads,prefix,steps", [
    ("router", [1531], [1]), ("tiny", [0, 15, 16, 31, 700], [1, 1, 33, 17, 5]), ("target", [32767, 0], [3, 16]),
    ("single", [9] * 70, [1] * 70), ("multi", [4, 100], [129, 1]), ("tiny", [i % 40 for i in range(300)], [1 + i % 3 for i in range(300)]),
    ("router", [0, 77], [1100, 3])])
def test_norm_rope_append(A, heads, prefix, steps, kv8):
    check_append(A, heads, prefix, steps, kv8, (True, True), False, 11)


@pytest.mark.parametrize("norms,q_scaled,in_place", [((False, False), True, False), ((True, False), False, True), ((False, True), True, True)])
def test_norm_rope_append_forms(A, norms, q_scaled, in_place):
    for kv8 in (True, False):
        check_append(A, "router", [5, 4090], [7, 30], kv8, norms, q_scaled, 12, in_place)


def test_append_of_many_tokens_is_that_of_few(A):
    """From 768 tokens on a lane takes eight pairs and a workgroup two tokens: the same bits as one token fewer."""
    hq, hkv, hd = HEADS["target"]
    prefix, steps = [3, 0, 800], [500, 1, 266]
    db, tables, n = make_batch(A, prefix, steps, 5)
    qkv = rows((767, (hq + 2 * hkv) * hd), 6)
    more = rows((1, (hq + 2 * hkv) * hd), 7)
    both, one = layer8(A, n + 1, hkv, hd), layer8(A, n + 1, hkv, hd)
    g = 1 + 0.2 * torch.randn(hd, device="cuda")
    q1 = A.arb_stage_norm_rope_append(stage_model("target"), qkv, one, db, g, g)
    t4 = np.concatenate([tables, np.full((1, tables.shape[1]), n, np.int32)])
    db4 = A.DeviceBatch(np.array(prefix + [2], np.int32), np.array([0, 500, 501, 767, 768], np.int32), t4)
    q4 = A.arb_stage_norm_rope_append(stage_model("target"), torch.cat([qkv, more]), both, db4, g, g)
    assert torch.equal(q4[:767], q1)
    for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert torch.equal(getattr(both, name).view(torch.uint8)[:n], getattr(one, name).view(torch.uint8)[:n])


def test_rows_of_zeros_and_rows_at_the_border_of_a_scale(A):
    hq, hkv, hd = HEADS["router"]
    qkv = rows((4, (hq + 2 * hkv) * hd), 8).view(4, -1, hd)
    qkv[0, hq:] = 0                                              # key and value of zeros
    qkv[1, hq + hkv:] = 448.0
    qkv[2, hq + hkv:] = 450.0
    qkv[3, :hq] = 0                                              # norm of a row of zeros: 0 / sqrt(eps)
    kv = check_append(A, "router", [20], [4], True, (True, True), False, 9, qkv=qkv.view(4, -1))
    assert sorted(kv.v_scale.unique().tolist())[0] == 27


@pytest.mark.parametrize("tokens", [5, 800])
def test_norms_of_rows_whose_squares_leave_fp32(A, tokens):
    """Rows of magnitudes from 1e-30 to 1e37 are normed like any other (their squares are 0 or infinite in fp32)."""
    hq, hkv, hd = HEADS["router"]
    x = rows((tokens, hq + 2 * hkv, hd), 18, 1.0).float()
    size = torch.tensor([1e-30, 1e-3, 1e18, 1e20, 1e35], device="cuda")[torch.arange(tokens, device="cuda") % 5]
    x[:, :hq + hkv] *= size[:, None, None]
    check_append(A, "router", [20], [tokens], True, (True, True), False, 19, qkv=x.bfloat16().view(tokens, -1))


# ------------------------------------------------------------------------------------ attention

CASES = [
    ("router", [0], [1]), ("router", [1531], [1]), ("target", [0, 1, 15, 16, 63, 64, 65, 127], [1] * 8),
    ("multi", [4000, 17, 900], [1, 2, 1]), ("single", [300, 40, 1000], [16, 5, 9]), ("tiny", [5, 0, 1700, 64], [1, 9, 3, 8]),
    ("router", [2048, 100, 0], [5, 3, 4]), ("target", [700, 64], [8, 7]),
    ("target", [700, 64, 5], [9, 16, 1]), ("router", [2048, 100, 63], [10, 3, 6]), ("tiny", [300, 5], [32, 17]), ("multi", [900, 0], [8, 5]), ("single", [40, 500], [64, 33]),
    ("router", [300, 77, 1000, 0, 2048], [5, 64, 33, 20, 1]), ("target", [4096, 15], [64, 129]), ("tiny", [512, 3, 130], [32, 64, 200]),
    ("tiny", [0], [4300]), ("multi", [200], [300]), ("single", [100, 3], [150, 1]),
]


@pytest.mark.parametrize("heads,prefix,steps", [("router", [2000, 300], [64, 9]), ("target", [700], [16]), ("tiny", [1500], [60]), ("router", [3000], [2])])
@pytest.mark.parametrize("kv8,size", [(True, 1.0), (True, 1e30), (True, 1e-24), (False, 1.0), (False, 1e36), (False, 1e-33)])
def test_parts_hold_values_of_any_size(A, heads, prefix, steps, kv8, size):
    """Cut contexts whose values are large, small, and of columns that differ by 2^20 (2^12 where e4m3 has to hold both)."""
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 25)
    k, v = rows((n, hkv, 16, hd), 26, 0.8), rows((n, hkv, 16, hd), 27, 0.8).float() * size
    v[..., ::7] *= 2.0 ** -12 if kv8 else 2.0 ** -20
    kv = A.KVLayer(k, v.bfloat16())
    if kv8:
        plain, kv = kv, layer8(A, n, hkv, hd)
        A.arb_kv8_pack(plain, kv)
    q = queries(sum(steps), heads, 28, True)
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, softcap=20.0, q_scaled=True)
    ref, mag = attention_ref(heads, q, kv, tables, prefix, steps, 20.0, True)
    # (bf16 and fp32 below 2^-126 round to a multiple of 2^-133)
    assert bool(((got.double().view(ref.shape) - ref).abs() <= 4.3 * U * mag + 2.0 ** -132).all())


# what the long-step kernel cuts into parts of 64, 128 and 192 keys
FINE = [("target", [360], [41]), ("router", [449, 3], [60, 7]), ("router", [2000], [64]), ("tiny", [50], [1200]), ("multi", [92, 5623], [9, 11]),
        ("single", [11], [570]), ("target", [74, 302, 0], [39, 126, 257]), ("multi", [0], [257])]


@pytest.mark.parametrize("kv8", [True, False])
@pytest.mark.parametrize("cap,q_scaled", [(0.0, True), (0.0, False), (20.0, True), (5.0, False)])
@pytest.mark.parametrize("heads,prefix,steps", CASES + FINE)
def test_attention(A, heads, prefix, steps, cap, q_scaled, kv8):
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 21)
    kv = filled(A, n, hkv, hd, 22, kv8)
    check_attention(A, heads, kv, prefix, steps, 23, db, tables, cap, q_scaled, extra=0 if q_scaled else 64)


@pytest.mark.parametrize("heads,prefix,steps", [("router", [9000, 30000], [1, 1]), ("target", [32767], [2]), ("tiny", [20000, 3], [1, 8]), ("multi", [16383], [16]), ("target", [9000, 20000], [16, 9]),
                                                ("single", [7000], [50])])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_attention_over_long_contexts(A, heads, prefix, steps, cap):
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 31)
    kv = filled(A, n, hkv, hd, 32)
    check_attention(A, heads, kv, prefix, steps, 33, db, tables, cap, True)


@pytest.mark.parametrize("heads,prefix,steps,in_a_row,parts", [
    ("router", [130 * i % 7001 for i in range(70)], [1] * 70, 1, 10),       # workgroups that pass from pair to pair, more sequences than a wave
    ("target", [4000, 20, 9000, 700, 64], [2, 4, 1, 3, 1], 0, 36),
    ("tiny", [37 * i % 900 for i in range(300)], [1 + i % 8 for i in range(300)], 1, 4),
    ("single", [5000, 1], [1, 2], 0, 20), ("target", [2048] * 16, [1] * 16, 0, 4), ("router", [767, 0, 63, 64, 500], [1, 2, 1, 1, 5], 0, 1)])
@pytest.mark.parametrize("cap", [0.0, 12.0])
def test_attention_of_few_rows_however_it_is_split(A, heads, prefix, steps, in_a_row, parts, cap):
    from helpers import few_plan
    hq, hkv, hd = HEADS[heads]
    plan = few_plan(A.load_library(), hkv, hd, prefix, steps, max(steps) * hq // hkv)
    assert (plan.in_a_row, plan.parts) == (in_a_row, parts)
    db, tables, n = make_batch(A, prefix, steps, 35)
    kv = filled(A, n, hkv, hd, 36)
    check_attention(A, heads, kv, prefix, steps, 37, db, tables, cap, True)


@pytest.mark.parametrize("heads,prefix,steps", [("router", [700, 64], [2, 1]), ("target", [1000], [40]), ("tiny", [333], [7]), ("target", [650], [13])])
@pytest.mark.parametrize("cap", [0.0, 15.0])
def test_attention_with_scores_that_jump(A, heads, prefix, steps, cap):
    """Queries eight times as large and planted keys: the running maximum moves late, and one key takes nearly all."""
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 41)
    kv = filled(A, n, hkv, hd, 42)
    q = queries(sum(steps), heads, 43, False, 6.0)
    cu = np.concatenate([[0], np.cumsum(steps)])
    for b, (p, s) in enumerate(zip(prefix, steps)):
        for pos in {0, p // 2, p + s - 1}:
            k = np.repeat(q[cu[b + 1] - 1, :hd].double().cpu().numpy()[None] * 0.5, hkv, 0)
            put_rows(kv, (int(tables[b, pos // 16]), slice(None), pos % 16), k, k[:, ::-1])
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, softcap=cap)
    ref, mag = attention_ref(heads, q, kv, tables, prefix, steps, cap, False)
    # logits reach some hundreds here: 2^-24 times the sum of |q k| / sqrt(hd) (at most 2000) times ten for the order of the sum is 2^-10
    assert bool(((got.double().view(ref.shape) - ref).abs() <= (4.3 * U + 4 * 2.0 ** -10) * mag + 1e-30).all())


@pytest.mark.parametrize("heads,prefix,steps", [("router", [300, 77, 1000], [50, 64, 33]), ("tiny", [100, 4500], [4100, 20]), ("router", [100, 77, 0], [50, 64, 250]), ("target", [700], [16])])
def test_long_steps_are_the_attention_over_the_unpacked_cache_bit_for_bit(A, heads, prefix, steps):
    """What an element and its scale stand for is exact in bf16, so where one form serves both caches the products are the same."""
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 51)
    kv, plain = filled(A, n, hkv, hd, 52), layer16(A, n, hkv, hd)
    A.arb_kv8_unpack(kv, plain)
    q = queries(sum(steps), heads, 53, True)
    run = lambda layer: A.arb_stage_attention_kv(stage_model(heads), q, layer, db, softcap=30.0, q_scaled=True)
    assert torch.equal(run(kv), run(plain))


@pytest.mark.parametrize("heads,prefix,steps", [("router", [300, 77, 1000], [50, 64, 33]), ("tiny", [100, 4500], [4100, 20]), ("target", [700, 5], [16, 1]), ("router", [1531], [1])])
@pytest.mark.parametrize("q_scaled", [True, False])
def test_uncapped_over_bf16_is_the_stage_it_generalises_bit_for_bit(A, heads, prefix, steps, q_scaled):
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 54)
    kv, q = filled(A, n, hkv, hd, 55, kv8=False), queries(sum(steps), heads, 56, q_scaled)
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, q_scaled=q_scaled)
    assert torch.equal(got, A.arb_stage_attention(stage_model(heads), q, kv.k_pool, kv.v_pool, db, q_scaled=q_scaled))


@pytest.mark.parametrize("heads,prefix,steps", [("router", [13, 40, 64], [1, 2, 1]), ("target", [5], [60]), ("tiny", [63, 1], [3, 1]), ("router", [600], [1]), ("target", [70, 1], [11, 2])])
@pytest.mark.parametrize("fill,kv8,cap", [(0x7f, True, 0.0), (0xff, True, 9.0), (0xff, False, 9.0)])
def test_slots_past_the_context_may_hold_anything(A, heads, prefix, steps, fill, kv8, cap):
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 61)
    full, kv = filled(A, n, hkv, hd, 62, kv8), layer8(A, n, hkv, hd, fill=fill) if kv8 else layer16(A, n, hkv, hd)
    if not kv8:
        kv.k_pool.fill_(float("nan")), kv.v_pool.fill_(float("nan"))
    for b, (p, s) in enumerate(zip(prefix, steps)):
        for pos in range(p + s):
            at = int(tables[b, pos // 16]), slice(None), pos % 16
            for name in ("k_pool", "v_pool", "k_scale", "v_scale") if kv8 else ("k_pool", "v_pool"):
                a, b_ = (getattr(x, name) for x in (kv, full))
                a.view(torch.uint8 if kv8 else torch.int16)[at] = b_.view(torch.uint8 if kv8 else torch.int16)[at]
    # the tables' unused entries are no block at all
    far = tables.copy()
    for b, (p, s) in enumerate(zip(prefix, steps)):
        far[b, -(-(p + s) // 16):] = 2 ** 30
    db = A.DeviceBatch(db.prefix_host, db.cu_host, far)
    q = queries(sum(steps), heads, 63, True)
    run = lambda layer: A.arb_stage_attention_kv(stage_model(heads), q, layer, db, softcap=cap, q_scaled=True)
    assert bool(torch.isfinite(run(full)).all()) and torch.equal(run(kv), run(full))


@pytest.mark.parametrize("steps", [4, 9, 40])
@pytest.mark.parametrize("bad", ["nan key", "infinite value"])
def test_a_position_that_is_not_finite_is_seen_by_those_that_see_it(A, steps, bad):
    """Append a step whose token 2 is broken in kv head 1, attend: rows before it as without it, rows from it on NaN, head 0 untouched."""
    hq, hkv, hd = HEADS["router"]
    prefix = [30]
    db, tables, n = make_batch(A, prefix, [steps], 71)
    qkv = rows((steps, (hq + 2 * hkv) * hd), 72)
    outs = []
    for broken in (False, True):
        x = qkv.clone().view(steps, -1, hd)
        if broken and bad == "nan key":
            x[2, hq + 1, 5] = float("nan")
        elif broken:
            x[2, hq + hkv + 1, 5] = float("inf")
        kv = filled(A, n, hkv, hd, 73)
        q = A.arb_stage_norm_rope_append(stage_model("router"), x.view(steps, -1), kv, db, q_scaled=True)
        outs.append(A.arb_stage_attention_kv(stage_model("router"), q, kv, db, q_scaled=True).view(steps, hq, hd))
    good, got = outs
    assert torch.equal(got[:2], good[:2]) and torch.equal(got[:, :6], good[:, :6]) and bool(torch.isfinite(good).all())
    assert bool(torch.isnan(got[2:, 6:]).all())


@pytest.mark.parametrize("heads,prefix,steps", [("target", 12000, 4), ("router", 20000, 1), ("tiny", 9000, 16), ("target", 9000, 40), ("router", 30000, 12)])
@pytest.mark.parametrize("kv8,cap", [(True, 0.0), (True, 12.0), (False, 12.0), (False, 0.0)])
def test_a_long_stretch_of_keys_that_are_not_finite(A, heads, prefix, steps, kv8, cap):
    """The first keys of a split context are NaN, up to every fourth tile: whole parts and whole groups of parts.  Whoever sees any
    of them gets NaN; the other sequence is as it was."""
    hq, hkv, hd = HEADS[heads]
    prefix, steps = [prefix, 100], [steps, 1]
    db, tables, n = make_batch(A, prefix, steps, 81)
    kv = filled(A, n, hkv, hd, 82, kv8)
    q = queries(sum(steps), heads, 83, True)
    run = lambda: A.arb_stage_attention_kv(stage_model(heads), q, kv, db, softcap=cap, q_scaled=True)
    good = run()
    assert bool(torch.isfinite(good).all())
    for first in range(0, prefix[0] // 16 - 16, 16):
        bad = torch.from_numpy(tables[0, first:first + 16].astype(np.int64)).cuda()
        if kv8:
            kv.k_pool.view(torch.uint8)[bad] = 0x7f
        else:
            kv.k_pool[bad] = float("nan")
        got = run()
        assert torch.equal(got[steps[0]:], good[steps[0]:]) and bool(torch.isnan(got[:steps[0]]).all()), first


def test_blocks_beyond_32_bit_offsets(A):
    hq, hkv, hd = HEADS["target"]
    n = 300_000                                                  # 4.9 GB a pool of bytes, 9.8 GB of bf16
    prefix, steps = [40, 100], [1, 60]
    db, tables, used = make_batch(A, prefix, steps, 81, spare=0)
    far = A.DeviceBatch(db.prefix_host, db.cu_host, tables + np.int32(n - used))
    near8, near16 = filled(A, used, hkv, hd, 82), layer16(A, used, hkv, hd)
    A.arb_kv8_unpack(near8, near16)
    pool = lambda t, e: torch.empty(n, *t.shape[1:], dtype=t.dtype, device="cuda") if e else None
    far16 = A.KVLayer(*(torch.empty(n, hkv, 16, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)))
    far8 = A.KVLayer(*(torch.empty(n, hkv, 16, hd, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)),
                     *(torch.empty(n, hkv, 16, dtype=torch.uint8, device="cuda") for _ in range(2)))
    here, there = (torch.arange(a, a + used, dtype=torch.int32, device="cuda") for a in (0, n - used))
    A.arb_kv8_unpack(near8, far16, here, there)
    A.arb_kv8_pack(far16, far8, there, there)
    back = layer16(A, used, hkv, hd)
    A.arb_kv8_unpack(far8, back, there, here)
    assert torch.equal(back.k_pool, near16.k_pool) and torch.equal(back.v_pool, near16.v_pool)
    model = stage_model("target")
    qkv = rows((61, (hq + 2 * hkv) * hd), 83)
    for near, away in ((near8, far8), (near16, far16)):
        q = A.arb_stage_norm_rope_append(model, qkv, near, db, q_scaled=True)
        assert torch.equal(A.arb_stage_norm_rope_append(model, qkv, away, far, q_scaled=True), q)
        for sub in (slice(0, 2), slice(0, 1)):                   # long steps and single tokens
            d = [A.DeviceBatch(db.prefix_host[sub], db.cu_host[:sub.stop + 1], t[sub]) for t in (tables, tables + np.int32(n - used))]
            want, got = (A.arb_stage_attention_kv(model, q, kv, x, softcap=25.0, q_scaled=True) for kv, x in zip((near, away), d))
            assert torch.equal(got, want)
    del far8, far16
    torch.cuda.empty_cache()


# ----------------------------------------------------------------------------------- how it is called

def test_more_sequences_than_a_grid_has_planes(A):
    heads, batch = "tiny", 70_000
    hq, hkv, hd = HEADS[heads]
    prefix = np.arange(batch) % 3
    prefix[-1] = 700
    width = 44
    tables = (np.arange(batch, dtype=np.int32) % 50)[:, None] + np.zeros((1, width), np.int32)
    db = A.DeviceBatch(prefix.astype(np.int32), np.arange(batch + 1, dtype=np.int32), tables)
    kv = filled(A, 50, hkv, hd, 94)
    q = queries(batch, heads, 95, True)
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, q_scaled=True)
    for rows_ in (slice(0, 40), slice(batch - 40, batch)):       # two ends of it, as batches of their own
        ref, mag = attention_ref(heads, q[rows_], kv, tables[rows_], prefix[rows_].tolist(), [1] * 40, 0.0, True)
        assert bool(((got[rows_].double().view(ref.shape) - ref).abs() <= 4.3 * U * mag + 1e-30).all())
    assert bool(torch.isfinite(got).all())


def test_rows_behind_the_last_sequence_stay(A):
    heads, prefix, steps = "router", [70, 9], [2, 1]
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 91)
    kv = filled(A, n, hkv, hd, 92)
    q = queries(3, heads, 93, True, more=5)                      # a padded batch: more rows than tokens
    out = torch.full((8, hq * hd), 7.0, dtype=torch.bfloat16, device="cuda")
    A.arb_stage_attention_kv(stage_model(heads), q, kv, db, q_scaled=True, out=out)
    assert bool((out[3:] == 7).all())
    assert torch.equal(out[:3], A.arb_stage_attention_kv(stage_model(heads), q[:3].contiguous(), kv, db, q_scaled=True))


def test_an_empty_batch_is_nothing(A):
    hq, hkv, hd = HEADS["tiny"]
    kv = layer8(A, 2, hkv, hd)
    db = A.DeviceBatch(np.zeros(0, np.int32), np.zeros(1, np.int32), np.zeros((0, 3), np.int32))
    assert A.arb_stage_attention_kv(stage_model("tiny"), torch.zeros(0, hq * hd, dtype=torch.bfloat16, device="cuda"), kv, db).shape == (0, hq * hd)
    assert A.arb_stage_norm_rope_append(stage_model("tiny"), torch.zeros(0, (hq + 2 * hkv) * hd, dtype=torch.bfloat16, device="cuda"), kv, db).shape == (0, hq * hd)


def test_the_binding_refuses_what_does_not_fit(A):
    hq, hkv, hd = HEADS["router"]
    db, tables, n = make_batch(A, [10], [3], 95)
    kv, other = layer8(A, n, hkv, hd), layer8(A, n, hkv, 64)
    model = stage_model("router")
    qkv = torch.zeros(3, (hq + 2 * hkv) * hd, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(3, hq * hd, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: A.arb_stage_attention_kv(model, q, other, db), lambda: A.arb_stage_attention_kv(model, q[:2], kv, db),
                 lambda: A.arb_stage_attention_kv(model, q, kv, db, out=q[:2]), lambda: A.arb_stage_attention_kv(model, q.float(), kv, db),
                 lambda: A.arb_stage_norm_rope_append(model, qkv, other, db), lambda: A.arb_stage_norm_rope_append(model, q, kv, db),
                 lambda: A.arb_stage_norm_rope_append(model, qkv, kv, db, g_q=torch.ones(64, device="cuda")),
                 lambda: A.arb_stage_norm_rope_append(model, qkv, kv, db, out=q, in_place=True),
                 lambda: A.arb_kv8_pack(layer16(A, n, hkv, hd), other), lambda: A.arb_kv8_pack(layer16(A, n, hkv, hd), kv, n_blocks=n + 1),
                 lambda: A.KVLayer(kv.k_pool, kv.v_pool), lambda: A.KVLayer(kv.k_pool, kv.v_pool, kv.k_scale, kv.v_scale[:1]),
                 lambda: A.arb_score_steps_noalloc(model, A.KVCache8([kv]), db, 0.0)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: A.arb_stage_attention_kv(model, q, kv, db, softcap=-1.0), lambda: A.arb_kv8_pack(kv, kv),
                 lambda: A.arb_kv8_unpack(layer16(A, n, hkv, hd), layer16(A, n, hkv, hd))):
        with pytest.raises(A.ArbError):
            call()


def test_a_cache_of_fewer_layers_or_other_heads_is_refused(A):
    shape = W.TINY
    w = W.Workload("kv8", shape, 2, (20, 40), ("fixed", 2, 2), "shuffled", "prefill", 0.0, ("const", 0.0), 779)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 5, 0.0, False)
    fewer = A.KVCache8(kv.layers[:-1])
    other = A.KVCache8.empty(shape.n_layers, batch.n_blocks, shape.n_kv_heads, 128 if shape.head_dim == 64 else 64)
    heads = A.KVCache8.empty(shape.n_layers, batch.n_blocks, shape.n_kv_heads + 1, shape.head_dim)
    x = torch.zeros(batch.total_tokens, shape.d_model, device="cuda")
    for cache in (fewer, other, heads):
        for call in (lambda: A.arb_prefill(model, cache, db), lambda: A.arb_score_steps(model, cache, db, 0.0),
                     lambda: A.arb_stage_layers(model, cache, db, 0, 1, x)):
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        A.KVCache8.empty(1, 2, 2, 64, device="cpu")


def test_two_calls_at_once_on_two_streams(A):
    heads = "router"
    hq, hkv, hd = HEADS[heads]
    model, want, got, todo = stage_model(heads), [], [], []
    for i, (prefix, steps) in enumerate((([9000, 5], [1, 1]), ([3000, 800], [60, 2]))):
        db, tables, n = make_batch(A, prefix, steps, 101 + i)
        todo.append((queries(sum(steps), heads, 103 + i, True), filled(A, n, hkv, hd, 105 + i), db))
    want = [A.arb_stage_attention_kv(model, q, kv, db, q_scaled=True).clone() for q, kv, db in todo]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in todo]
    for _ in range(5):
        got = [A.arb_stage_attention_kv(model, q, kv, db, q_scaled=True, stream=s) for (q, kv, db), s in zip(todo, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("heads,prefix,steps", [("router", [130 * i % 7001 for i in range(70)], [1] * 70), ("target", [4000, 20, 9000], [2, 8, 1]),
                                                ("router", [3000, 300], [40, 64]), ("target", [360], [41])])
def test_nothing_is_written_outside_of_the_least_workspace(A, heads, prefix, steps):
    import re
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 111)
    kv = filled(A, n, hkv, hd, 112)
    q = queries(sum(steps), heads, 113, True)
    run = lambda **k: A.arb_stage_attention_kv(stage_model(heads), q, kv, db, q_scaled=True, **k)
    with pytest.raises(A.ArbError) as e:                         # a host check: nothing is launched
        run(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    need = int(re.search(r"workspace 16 < (\d+) bytes", str(e.value)).group(1))
    buf = torch.full((need + 8192,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((sum(steps) + 2, hq * hd), 3.0, dtype=torch.bfloat16, device="cuda")
    run(ws=buf[4096:4096 + need], out=out)
    assert bool((buf[:4096] == 255).all()) and bool((buf[4096 + need:] == 255).all()) and bool((out[-2:] == 3).all())
    ref, mag = attention_ref(heads, q, kv, tables, prefix, steps, 0.0, True)
    assert bool(((out[:-2].double().view(ref.shape) - ref).abs() <= 4.3 * U * mag + 1e-30).all())


@pytest.mark.parametrize("host,device", [([1000, 300, 900], [200, 100, 900]), ([600, 100, 0], [1000, 300, 900]), ([90 * i % 3001 for i in range(60)], [70 * i % 3001 for i in range(60)])])
def test_lengths_that_differ_on_host_and_device_stay_within_memory(A, host, device):
    """The contract has them equal.  Where they are not, nothing outside the workspace and the output is written; and with fewer keys on
    the device every piece of work is still there, so the result is theirs."""
    import re
    heads, steps = "target", [2, 1, 3] + [1] * (len(host) - 3)
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, [max(a, b) for a, b in zip(host, device)], steps, 131)
    db = A.DeviceBatch(np.array(device, np.int32), db.cu_host, tables)
    db.prefix_host[:] = host
    kv = filled(A, n, hkv, hd, 132)
    q = queries(sum(steps), heads, 133, True)
    run = lambda d, **k: A.arb_stage_attention_kv(stage_model(heads), q, kv, d, q_scaled=True, **k)
    need = 0                                                     # contexts that are not cut need none
    try:
        run(db, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))
    except A.ArbError as e:
        need = int(re.search(r"workspace 16 < (\d+) bytes", str(e)).group(1))
    buf = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((sum(steps) + 2, hq * hd), 3.0, dtype=torch.bfloat16, device="cuda")
    run(db, ws=buf[:need], out=out)
    torch.cuda.synchronize()
    assert bool((buf[need:] == 255).all()) and bool((out[-2:] == 3).all())
    if all(h >= d for h, d in zip(host, device)):
        ref, mag = attention_ref(heads, q, kv, tables, device, steps, 0.0, True)
        assert bool(((out[:-2].double().view(ref.shape) - ref).abs() <= 4.3 * U * mag + 1e-30).all())


def test_two_captured_graphs_share_a_workspace(A):
    todo = []
    for i, (heads, prefix, steps, cap) in enumerate((("router", [5000, 40], [1, 2], 0.0), ("router", [900, 2000], [50, 64], 20.0), ("target", [2048] * 4, [3] * 4, 0.0))):
        hq, hkv, hd = HEADS[heads]
        db, tables, n = make_batch(A, prefix, steps, 121 + i)
        q, kv = queries(sum(steps), heads, 124 + i, True), filled(A, n, hkv, hd, 127 + i)
        todo.append([heads, q, kv, db, cap, torch.empty_like(q)])
    ws = torch.empty(max(stage_model(h).workspace_bytes(db.batch, db.total_tokens, db.max_ctx) for h, _, _, db, _, _ in todo), dtype=torch.uint8, device="cuda")
    call = lambda h, q, kv, db, cap, out: A.arb_stage_attention_kv(stage_model(h), q, kv, db, softcap=cap, q_scaled=True, ws=ws, out=out)
    want, graphs = [call(*t).clone() for t in todo], []
    for t in todo:
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(*t)
        graphs.append(g)
    for i in (0, 1, 0, 2, 2, 1, 0):
        todo[i][5].fill_(9.0)
        graphs[i].replay()
        eager = call(*todo[(i + 1) % 3]).clone()                 # and eager work between the replays, on the same workspace
        torch.cuda.synchronize()
        assert torch.equal(todo[i][5], want[i]) and torch.equal(eager, want[(i + 1) % 3])


# ------------------------------------------------------------------------------ the whole forward

def _forward_session(A, w, seed, softcap, norms, kv8=True, four_bit=False):
    m, h = w.model, H()
    batch = W.make_batch(w)
    weights = W.make_weights(m, w.seed, "cuda", gain_jitter=0.1, b_head=0.0)
    weights_of_model = A.QuantizedWeights(weights) if four_bit else weights
    g = torch.Generator().manual_seed(seed)
    gains = tuple([(1 + 0.3 * torch.randn(m.head_dim, generator=g)).cuda() for _ in range(m.n_layers)] for _ in range(2)) if norms else None
    model = A.Model(n_layers=m.n_layers, d_model=m.d_model, n_q_heads=m.n_q_heads, n_kv_heads=m.n_kv_heads, head_dim=m.head_dim,
                    d_ffn=m.d_ffn, vocab=m.vocab, weights=weights_of_model, rms_eps=m.rms_eps, rope_base=m.rope_base,
                    has_router_head=m.has_router_head, head_norms=gains, softcap=softcap)
    kv = A.KVCache8.empty(m.n_layers, batch.n_blocks, m.n_kv_heads, m.head_dim) if kv8 else \
        A.KVCache(*([torch.zeros(batch.n_blocks, m.n_kv_heads, 16, m.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(m.n_layers)] for _ in range(2)))
    return batch, weights, gains, model, kv, h.device_batch(batch)


def _oracle_forward(w, weights, gains, softcap, layers, ids, prefix, cu, tables, four_bit=False):
    """The oracle's forward over the keys and values that the cache really holds (an element that the GPU's bf16 activations put on
    the other side of an e4m3 border is no error of the attention).  -> (final-normed hidden states, [(k, v)] it would have stored)."""
    from helpers import oracle_model, oracle_params
    m, p = oracle_model(w.model), oracle_params(weights)
    for name in ("wqkv", "wo", "wgu", "wd") if four_bit else ():
        setattr(p, name, [O.w4_dequantize(*O.w4_quantize(x)) for x in getattr(p, name)])
    hq, hkv, hd = m.n_q_heads, m.n_kv_heads, m.head_dim
    pos, slots, T = O.positions(prefix, cu), O.slot_mapping(prefix, cu, tables, 16), len(ids)
    h, stored = O.embed(p.embed, ids), []
    for l, kv in enumerate(layers):
        qkv = (O.rmsnorm(h, p.g_attn[l], m.rms_eps) @ O.as_float(p.wqkv[l]).T).reshape(T, -1, hd)
        g = [None if gains is None else x[l].double().cpu().numpy() for x in (gains or (None, None))]
        q = O.rope(K8.head_norm(qkv[:, :hq], g[0], m.rms_eps), pos, m.rope_base)
        k = O.rope(K8.head_norm(qkv[:, hq:hq + hkv], g[1], m.rms_eps), pos, m.rope_base)
        stored.append((k, qkv[:, hq + hkv:]))
        kp, vp = (x.cpu().numpy() for x in values(kv))
        o = np.empty((T, hq, hd))
        for b in range(len(prefix)):
            lo, hi, G = cu[b], cu[b + 1], hq // hkv
            s = O.slot_of(tables[b], np.arange(prefix[b] + hi - lo), 16)
            for c in range(hq):
                o[lo:hi, c], _ = K8.append_attention(q[lo:hi, c], kp[s // 16, c // G, s % 16], vp[s // 16, c // G, s % 16], prefix[b] + np.arange(hi - lo), softcap)
        h = h + o.reshape(T, -1) @ O.as_float(p.wo[l]).T
        h = h + O.swiglu_mlp(O.rmsnorm(h, p.g_mlp[l], m.rms_eps), p.wgu[l], p.wd[l])
    return O.rmsnorm(h, p.g_final, m.rms_eps), stored, slots


def _layers(A, kv):
    return kv.layers if isinstance(kv, A.KVCache8) else [A.KVLayer(k, v) for k, v in zip(kv.k_pools, kv.v_pools)]


@pytest.mark.parametrize("name,steps,norms,softcap,kv8", [
    ("tiny", 32, True, 30.0, True), ("tiny 4-bit", 33, True, 0.0, True), ("tiny 4-bit", 2, False, 20.0, True), ("tiny", 1, True, 0.0, True), ("tiny", 3, False, 0.0, True), ("router", 5, True, 20.0, True),
    ("tiny long", 2, True, 0.0, True), ("tiny long", 3, True, 15.0, False),
    ("tiny long", 40, True, 0.0, True), ("tiny long", 33, False, 25.0, False), ("tiny 4-bit long", 20, False, 30.0, True), ("router", 1, False, 30.0, True), ("tiny", 2, True, 10.0, False), ("tiny", 40, False, 25.0, False)])
def test_prompts_enter_the_cache_and_steps_are_scored_against_them(A, name, steps, norms, softcap, kv8):
    """arb_prefill of whole prompts, then arb_score_steps of a drafted step on the same cache: the cache is what the oracle stores
    up to its rounding, and the hidden states and scores are the oracle's over that cache."""
    from helpers import HIDDEN_TOL, SCORE_TOL, rel_err
    from dataclasses import replace
    four_bit = "4-bit" in name
    shape = W.TINY if name.startswith("tiny") else replace(W.ROUTER_1P5B, n_layers=2, vocab=4096)
    w = W.Workload("kv8", shape, 3, (300, 600) if name.endswith("long") else (40, 230), ("fixed", steps, steps), "shuffled", "prefill", 0.0, ("const", 0.0), 777)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 3, softcap, norms, kv8, four_bit)
    prompts = H().prompt_batch(w, batch)
    A.arb_prefill(model, kv, prompts)
    ids = W.prompt_token_ids(w, batch)
    cu = np.concatenate([[0], np.cumsum(batch.prefix_lens)]).astype(np.int32)
    rounding = 2.0 ** -4 if kv8 else U
    def check(ids, prefix, cu):
        y, stored, slots = _oracle_forward(w, weights, gains, softcap, _layers(A, kv), ids, prefix, cu, batch.block_tables, four_bit)
        for layer, pair in zip(_layers(A, kv), stored):
            for got, want in zip(values(layer), pair):
                g = got.cpu().numpy()[slots // 16, :, slots % 16]
                big = np.abs(want).max(-1, keepdims=True)
                # the element's rounding, the hidden-state bar on what goes into it, and 2^-10 of the scale (at most big / 224)
                assert (np.abs(g - want) <= rounding * np.abs(want) + (HIDDEN_TOL + 2.0 ** -17) * np.abs(want).max()).all()
        return y
    check(ids, np.zeros(batch.batch, np.int32), cu)
    scores, esc, hidden = A.arb_score_steps(model, kv, db, batch.tau, want_hidden=True)
    y = check(batch.token_ids, batch.prefix_lens, batch.cu_step_lens)
    assert rel_err(hidden.double().cpu().numpy(), y) < HIDDEN_TOL
    s = O.router_scores(y, batch.cu_step_lens, weights.w_head.double().cpu().numpy(), 0.0)
    assert np.abs(scores.cpu().numpy() - s).max() < SCORE_TOL
    assert np.array_equal(esc.cpu().numpy(), O.route(scores.cpu().numpy(), batch.tau))
    # layer by layer from the same residual stream: the same bits as in one call
    x = torch.randn(batch.total_tokens, shape.d_model, device="cuda")
    whole = A.arb_stage_layers(model, kv, db, 0, shape.n_layers, x)
    for l in range(shape.n_layers):
        x = A.arb_stage_layers(model, kv, db, l, l + 1, x)
    assert rel_err(x.double().cpu().numpy(), whole.double().cpu().numpy()) < 1e-2


@pytest.mark.parametrize("steps", [2, 7, 40])
def test_capped_scores_without_allocation_are_those_with_a_workspace(A, steps):
    w = W.Workload("kv8", W.TINY, 3, (100, 900), ("fixed", steps, steps), "shuffled", "prefill", 0.0, ("const", 0.0), 780)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 6, 20.0, True, kv8=False)
    A.arb_prefill(model, kv, H().prompt_batch(w, batch))
    want, esc, _ = A.arb_score_steps(model, kv, db, 0.0)
    got, also = torch.empty_like(want), torch.empty_like(esc)
    for _ in range(2):
        got.fill_(float("nan"))
        A.arb_score_steps_noalloc(model, kv, db, 0.0, scores=got, escalate=also)
        assert bool(torch.isfinite(want).all()) and torch.equal(got, want) and torch.equal(also, esc)


@pytest.mark.parametrize("least,most", [(1, 4), (20, 40)])
def test_a_captured_pass_on_the_8bit_cache_replays(A, least, most):
    w = W.Workload("kv8", W.TINY, 3, (100, 900), ("uniform", least, most), "shuffled", "prefill", 0.0, ("const", 0.0), 778)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 4, 30.0, True)
    A.arb_prefill(model, kv, H().prompt_batch(w, batch))
    ws = torch.empty(model.workspace_bytes(batch.batch, batch.total_tokens, db.max_ctx), dtype=torch.uint8, device="cuda")
    scores, esc = torch.empty(3, device="cuda"), torch.empty(3, dtype=torch.uint8, device="cuda")
    run = lambda **k: A.arb_score_steps(model, kv, db, 0.0, ws=ws, scores=scores, escalate=esc, **k)
    run()
    want = scores.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other = torch.randint(0, w.model.vocab, (batch.total_tokens,), dtype=torch.int32, device="cuda")
    first = db.tokens.clone()
    for i in range(4):
        scores.fill_(float("nan"))
        db.tokens.copy_(other if i % 2 else first)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = scores.clone()
        run()                                                    # the eager pass between the replays
        torch.cuda.synchronize()
        assert torch.equal(got, scores) and (torch.equal(got, want) == (i % 2 == 0))


def test_debug_mode_checks_the_ids_of_an_8bit_pass(A, monkeypatch):
    monkeypatch.setenv("ARB_DEBUG_IDS", "1")
    w = W.Workload("kv8", W.TINY, 2, (20, 40), ("fixed", 2, 2), "shuffled", "prefill", 0.0, ("const", 0.0), 779)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 5, 0.0, False)
    A.arb_score_steps(model, kv, db, 0.0)
    bad = batch.block_tables.copy()
    bad[1, 0] = batch.n_blocks
    with pytest.raises(A.ArbError) as e:
        A.arb_score_steps(model, kv, A.DeviceBatch(batch.prefix_lens, batch.cu_step_lens, bad, batch.token_ids), 0.0)
    assert e.value.status == A.ARB_EINVAL and "block_tables[1][0]" in str(e.value)


def test_algorithm_1_runs_on_8bit_caches(A):
    """The loop of Algorithm 1 with 8-bit caches in its three roles: repeatable, and every router score is the score of the recorded
    step on a fresh cache that was filled in the same pieces."""
    from paper_2512_05033_amd.arbitrage import Arbitrage, Role
    questions = [[int(t) for t in W.uniform_ints(77, f"q{b}", n, W.TINY.vocab).numpy()] for b, n in enumerate((5, 18, 33))]
    tables = np.random.default_rng(3).permutation(3 * 5).astype(np.int32).reshape(3, 5)
    m = W.TINY
    def role(name, seed, lm):
        weights = W.make_weights(m, seed, "cuda", gain_jitter=0.1, b_head=0.0)
        return Role(name, H().make_model(m, weights, has_router_head=not lm), A.KVCache8.empty(m.n_layers, 15, m.n_kv_heads, m.head_dim),
                    W.normal_bf16(seed, "lm_head", (m.vocab, m.d_model), 0.02, "cuda") if lm else None)
    def run(tau):
        trace = []
        roles = role("draft", 101, True), role("target", 202, True), role("router", 303, False)
        out, log = Arbitrage(*roles, tables, tau=tau, sep=-7, eos=-5, max_step_tokens=5, trace=trace).run(questions, 3)
        return out, log, trace
    _, log, _ = run(1e9)
    tau = float(np.median([s for b in log for s, _ in log[b]]))
    out, log, trace = run(tau)
    again = run(tau)
    assert out == again[0] and log == again[1]
    assert len({e for b in log for _, e in log[b]}) == 2         # drafts are accepted and regenerated
    fresh = role("router", 303, False)
    for ev in trace:
        if ev[0] != "route":
            continue
        _, b, ctx, z, score, esc = ev
        one = lambda p, ids: A.DeviceBatch(np.array([p], np.int32), np.array([0, len(ids)], np.int32), tables[b:b + 1], np.array(ids, np.int32))
        A.arb_prefill(fresh.model, fresh.kv, one(0, ctx))
        s, e, _ = A.arb_score_steps(fresh.model, fresh.kv, one(len(ctx), z), tau)
        # another batch and other pieces round differently and may move keys over e4m3 borders: the bar of the scores
        assert abs(float(s[0]) - score) < 1e-2
