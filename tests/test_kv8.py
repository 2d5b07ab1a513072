"""The 8-bit KV cache without a GPU: the oracle of its format against the definition, and what the library refuses."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import kv8_oracle as K8
from test_abi import _cfg, _create, _weights

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_05033_amd", "libarb.so")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        pytest.skip("libarb.so is not built")
    from paper_2512_05033_amd import binding
    return binding.load_library()


# ------------------------------------------------------------------------------- the oracle's pins

def test_e4m3_values():
    v = K8.e4m3_values()
    assert v[0x7e] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and v[0x38] == 1 and v[0xc0] == -2
    assert np.isnan(v[[0x7f, 0xff]]).all() and np.isfinite(np.delete(v, [0x7f, 0xff])).all()


def test_e4m3_rounding_is_to_the_nearest_and_to_even():
    values = K8.e4m3_values()[:127]                              # 0 .. 448, ascending with the byte
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.uniform(0, 448, 4000), np.exp2(rng.uniform(-12, 8.8, 4000)), values, (values[1:] + values[:-1]) / 2])
    for sign in (1, -1):
        got = K8.e4m3_round(sign * x)
        at = np.searchsorted(values, x, side="right") - 1
        lo, hi = values[at], values[np.minimum(at + 1, 126)]
        nearest = np.where(x - lo < hi - x, lo, np.where(x - lo > hi - x, hi, np.where(at % 2 == 0, lo, hi)))
        assert np.array_equal(got, sign * nearest)


def test_scale_exponent_is_the_least_one_that_holds_the_row():
    rng = np.random.default_rng(2)
    m = np.concatenate([np.exp2(rng.uniform(-80, 100, 2000)), 448 * 2.0 ** np.arange(-90, 100), np.nextafter(448.0, 500) * 2.0 ** np.arange(-90, 100)])
    e = K8.scale_exponent(m).astype(float)
    assert (m <= 448 * np.exp2(e)).all() and (m > 448 * np.exp2(e - 1)).all()
    assert (K8.scale_exponent(np.array([0.0, 1e-40, 2.0 ** -100])) == -100).all()


def test_a_position_that_is_not_finite_is_marked_in_its_key():
    k = np.ones((4, 64)); v = np.full((4, 64), 2.0)
    k[1, 3], v[2, 5], v[3, 0] = np.nan, np.inf, 2.0 ** 120
    ke, ve, kx, vx = K8.quantize(k, v)
    assert np.isfinite(ke[0]).all() and np.isnan(ke[1:]).all() and (ve[1:] == 0).all() and (kx[1:] == 0).all() and (vx[1:] == 0).all()
    assert (ke[0] * 2.0 ** kx[0] == 1).all() and (ve[0] * 2.0 ** vx[0] == 2).all()


def test_what_is_read_back_is_what_is_stored_again():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(500, 128)) * np.exp2(rng.uniform(-30, 30, size=(500, 1)))
    ke, ve, kx, vx = K8.quantize(x, x[::-1])
    back = ke * np.exp2(kx.astype(float))[:, None]
    k2, _, kx2, _ = K8.quantize(back, back)
    assert np.array_equal(k2 * np.exp2(kx2.astype(float))[:, None], back)
    # half a step of the element: 2^-4 of its value, or half of 2^-9 of the scale below the normal range
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), np.exp2(kx - 10.0)[:, None])).all()


# -------------------------------------------------------------------------------------- refusals

P = 0x1000                                                       # never dereferenced: everything here is refused on the host


def _batch(B, prefix=(10, 20), cu=(0, 4, 8), blocks=4):
    p, c = np.asarray(prefix, np.int32), np.asarray(cu, np.int32)
    bt = B._Batch(len(p), int(c[-1]), blocks, P, P, P, P, p.ctypes.data, c.ctypes.data)
    bt.keep = (p, c)
    return bt


def test_model_properties_are_checked(lib):
    from paper_2512_05033_amd import binding as B
    w, _keep = _weights()
    _, h = _create(lib, _cfg(), w)
    good, hole, odd = (C.c_void_p * 2)(P, P), (C.c_void_p * 2)(P, None), (C.c_void_p * 2)(P, P + 4)
    assert lib.arb_model_set_head_norms(None, good, good) == B.ARB_EINVAL
    assert lib.arb_model_set_head_norms(h, good, None) == B.ARB_EINVAL
    assert lib.arb_model_set_head_norms(h, good, hole) == B.ARB_EINVAL and b"layer 1" in lib.arb_last_error()
    assert lib.arb_model_set_head_norms(h, odd, good) == B.ARB_EINVAL and b"aligned" in lib.arb_last_error()
    assert lib.arb_model_set_head_norms(h, good, good) == B.ARB_OK
    assert lib.arb_model_set_head_norms(h, None, None) == B.ARB_OK
    for cap in (-1.0, 1e-3, 1025.0, float("nan"), float("inf")):
        assert lib.arb_model_set_softcap(h, cap) == B.ARB_EUNSUPPORTED
    for cap in (0.0, 0.01, 30.0, 1024.0):
        assert lib.arb_model_set_softcap(h, cap) == B.ARB_OK
    assert lib.arb_model_set_softcap(None, 0.0) == B.ARB_EINVAL
    lib.arb_model_destroy(h)


def test_forward_on_an_8bit_cache_is_checked_on_the_host(lib):
    from paper_2512_05033_amd import binding as B
    w, _keep = _weights()
    _, h = _create(lib, _cfg(), w)
    t, hole, odd = (C.c_void_p * 2)(P, P), (C.c_void_p * 2)(P, None), (C.c_void_p * 2)(P, P + 8)
    bt = _batch(B)

    def score(kv, ws_bytes=1 << 30):
        return lib.arb_score_steps_kv8(h, C.byref(kv) if kv else None, C.byref(bt), 0.0, P, None, None, P, ws_bytes, None)
    assert score(None) == B.ARB_EINVAL
    assert score(B._KV8(t, t, t, None, 8)) == B.ARB_EINVAL
    assert score(B._KV8(t, t, t, hole, 8)) == B.ARB_EINVAL and b"layer 1" in lib.arb_last_error()
    assert score(B._KV8(t, hole, t, t, 8)) == B.ARB_EINVAL
    assert score(B._KV8(t, odd, t, t, 8)) == B.ARB_EINVAL and b"aligned" in lib.arb_last_error()
    assert score(B._KV8(t, t, t, t, 8), 16) == B.ARB_ECAPACITY
    kv = B._KV8(t, t, t, t, 8)
    assert lib.arb_prefill_kv8(None, C.byref(kv), C.byref(bt), None, P, 1 << 30, None) == B.ARB_EINVAL
    assert lib.arb_stage_layers_kv8(h, C.byref(kv), C.byref(bt), 1, 1, P, P, P, 1 << 30, None) == B.ARB_EINVAL
    empty = B._Batch(0, 0, 4, None, None, None, None, None, None)
    assert lib.arb_prefill_kv8(h, C.byref(kv), C.byref(empty), None, None, 0, None) == B.ARB_OK
    lib.arb_model_destroy(h)


def test_single_stages_are_checked_on_the_host(lib):
    from paper_2512_05033_amd import binding as B
    w, _keep = _weights()
    _, h = _create(lib, _cfg(), w)
    bt = _batch(B)
    width = 4 * 64

    def attend(kv, cap=0.0, q=P, stride=width, out=P, batch=bt, ws=P, ws_bytes=1 << 30, model=h):
        return lib.arb_stage_attention_kv(model, q, stride, 0, C.byref(kv) if kv else None, cap, C.byref(batch), out, ws, ws_bytes, None)

    def append(kv, qkv=P, g_q=None, g_k=None, q_out=None, batch=bt, model=h):
        return lib.arb_stage_norm_rope_append(model, qkv, g_q, g_k, 0, C.byref(kv) if kv else None, C.byref(batch), q_out, None)
    full, half, none = B._KVLayer(P, P, P, P), B._KVLayer(P, P, P, None), B._KVLayer(P, None, None, None)
    for call in (attend, append):
        assert call(None) == B.ARB_EINVAL
        assert call(half) == B.ARB_EINVAL and b"neither" in lib.arb_last_error()
        assert call(none) == B.ARB_EINVAL
        assert call(B._KVLayer(P + 2, P, P, P)) == B.ARB_EINVAL and b"aligned" in lib.arb_last_error()
        assert call(B._KVLayer(P, P, P + 1, P)) == B.ARB_EINVAL
        assert call(full, model=None) == B.ARB_EINVAL
        assert call(full, batch=_batch(B, cu=(0, 4, 4))) == B.ARB_EINVAL
        assert call(full, batch=_batch(B, prefix=(10, 61))) == B.ARB_ECAPACITY
    assert attend(full, cap=-3.0) == B.ARB_EUNSUPPORTED and attend(full, cap=2000.0) == B.ARB_EUNSUPPORTED
    assert attend(full, cap=float("nan")) == B.ARB_EUNSUPPORTED
    assert attend(full, q=None) == B.ARB_EINVAL and attend(full, out=None) == B.ARB_EINVAL and attend(full, q=P + 4) == B.ARB_EINVAL
    assert attend(full, stride=width - 8) == B.ARB_EINVAL and attend(full, stride=width + 4) == B.ARB_EINVAL
    long = _batch(B, prefix=(5000, 20), blocks=400)
    assert attend(full, batch=long, ws_bytes=64) == B.ARB_ECAPACITY and attend(full, batch=long, ws=None) == B.ARB_ECAPACITY
    assert attend(full, ws=P + 8) == B.ARB_EINVAL and attend(full, out=P + 2) == B.ARB_EINVAL
    assert append(full, qkv=None) == B.ARB_EINVAL and append(full, q_out=P + 2) == B.ARB_EINVAL
    assert append(full, g_q=P + 8) == B.ARB_EINVAL and append(full, qkv=P + 8) == B.ARB_EINVAL
    lib.arb_model_destroy(h)


def test_conversion_is_checked_on_the_host(lib):
    from paper_2512_05033_amd import binding as B
    k8, bf = B._KVLayer(P, P, P, P), B._KVLayer(P, P, None, None)
    for convert, src, dst in ((lib.arb_kv8_pack, bf, k8), (lib.arb_kv8_unpack, k8, bf)):
        call = lambda s, d, n=4, heads=2, hd=64: convert(C.byref(s) if s else None, None, C.byref(d) if d else None, None, n, heads, hd, None)
        assert call(src, dst, n=-1) == B.ARB_EINVAL
        assert call(src, dst, heads=0) == B.ARB_ESHAPE
        assert call(src, dst, hd=96) == B.ARB_EUNSUPPORTED
        assert call(None, dst) == B.ARB_EINVAL and call(src, None) == B.ARB_EINVAL
        assert call(dst, src) == B.ARB_EINVAL and b"8-bit side" in lib.arb_last_error()
        assert call(src, src) == B.ARB_EINVAL and call(dst, dst) == B.ARB_EINVAL
        assert call(src, B._KVLayer(P, P + 4, dst.k_scale, dst.v_scale)) == B.ARB_EINVAL
        assert call(src, dst, n=2 ** 31 - 1, heads=64, hd=128) == B.ARB_EUNSUPPORTED          # more workgroups than a launch has
        assert call(None, None, n=0) == B.ARB_OK


def test_the_binding_takes_caches_of_one_kind():
    import torch
    from paper_2512_05033_amd import binding as B
    pool = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.KVLayer(pool, pool)                                    # not on a GPU
    with pytest.raises(ValueError):
        B.KVLayer(pool, pool, torch.zeros(2, 2, 16, dtype=torch.uint8))
    with pytest.raises(ValueError):
        B.KVCache8([])


# ------------------------------------------------------------------ the split of attention over few rows

def test_every_tile_of_a_decoding_batch_has_a_place(lib):
    """Random batches: the planner ends, its workgroups cover the keys, no (sequence, kv head) is cut into more parts than it says, and
    that is what arb_workspace_bytes counts on (one more than a part per 256 keys, 65 at most)."""
    from helpers import few_plan
    rng = np.random.default_rng(0)
    seen = set()
    for _ in range(1500):
        batch = int(np.exp(rng.uniform(0, np.log(300))))
        hi = int(np.exp(rng.uniform(0, np.log(200000))))
        prefix = rng.integers(rng.integers(0, hi + 1) if rng.random() < 0.7 else hi, hi + 1, batch)
        steps = rng.integers(1, 5, batch)
        heads = int(rng.choice([1, 2, 8, 16]))
        plan = few_plan(lib, heads, int(rng.choice([64, 128])), prefix, steps, int(rng.choice([4, 32])))
        tiles = -(-(prefix + steps) // 64)
        assert plan.tiles == tiles.sum() * heads and plan.per >= 1
        if plan.in_a_row:
            assert plan.groups == -(-plan.tiles // plan.per)
            ends = np.cumsum(np.repeat(tiles, heads))
            cuts = (ends - 1) // plan.per - (ends - np.repeat(tiles, heads)) // plan.per + 1
            assert cuts.max() <= plan.parts
        else:
            assert -(-tiles.max() // plan.per) == plan.parts and plan.groups == batch * heads * plan.parts
        assert plan.parts <= min(-(-int(tiles.max()) // 4), 64) + 1
        seen.add((plan.in_a_row, plan.parts > 1))
    assert len(seen) == 3                                        # in a row, even, uncut


def test_parts_of_few_workgroups_are_fine_ones(lib):
    """Random batches: finer parts than 256 keys only where those would leave CUs empty, at most 32 of them and 65536 rows of partial
    results; otherwise what arb_workspace_bytes counts on, a part per 256 keys and 64 at most."""
    from helpers import attention_plan, fine_attention_plan
    import workloads as W
    rng = np.random.default_rng(2)
    finer = 0
    for _ in range(600):
        m = [W.TINY, W.ROUTER_1P5B, W.TARGET_8B][rng.integers(3)]
        batch, hi = int(np.exp(rng.uniform(0, np.log(40)))), int(np.exp(rng.uniform(0, np.log(40000))))
        prefix, steps = rng.integers(0, hi + 1, batch), rng.integers(1, int(rng.choice([12, 80, 600])), batch)
        fine, plain = fine_attention_plan(lib, m, prefix, steps), attention_plan(lib, m, prefix, steps)
        longest = int((prefix + steps).max())
        if fine.kv_chunk >= 256:
            assert fine.max_qtiles == plain.max_qtiles and fine.max_splits == -(-longest // fine.kv_chunk) <= min(-(-longest // 256), 64)
            continue
        finer += 1
        assert fine.kv_chunk % 64 == 0 and fine.kv_chunk >= (64 if longest <= 512 else 128) and longest > 256
        assert fine.max_splits == -(-longest // fine.kv_chunk) <= 32
        assert int(steps.sum()) * m.n_q_heads * fine.max_splits <= 65536
        streamed = sum(-(-int(s) * m.group // 128) * m.n_kv_heads * int(p + s) for p, s in zip(prefix, steps))
        assert streamed < 256 * 256
    assert finer > 50


def test_workspace_covers_a_decoding_batch(lib):
    """arb_workspace_bytes is enough for what a call on an 8-bit cache asks for (a refusal names it)."""
    import re
    from paper_2512_05033_amd import binding as B
    w, _keep = _weights()
    _, h = _create(lib, _cfg(), w)
    t = (C.c_void_p * 2)(P, P)
    kv = B._KV8(t, t, t, t, 1 << 20)
    rng = np.random.default_rng(1)
    for _ in range(300):
        batch, hi = int(np.exp(rng.uniform(0, np.log(100)))), int(np.exp(rng.uniform(0, np.log(100000))))
        prefix, steps = rng.integers(0, hi + 1, batch), rng.integers(1, int(rng.choice([2, 17, 80, 500])), batch)
        bt = _batch(B, prefix, np.concatenate([[0], np.cumsum(steps)]), 1 << 14)
        assert lib.arb_score_steps_kv8(h, C.byref(kv), C.byref(bt), 0.0, P, None, None, P, 16, None) == B.ARB_ECAPACITY
        need = int(re.search(rb"workspace 16 < (\d+) bytes", lib.arb_last_error()).group(1))
        assert need <= lib.arb_workspace_bytes(h, batch, int(steps.sum()), int((prefix + steps).max()))
    lib.arb_model_destroy(h)
