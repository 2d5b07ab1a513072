"""Attention calls that a launch or the kernels' counts cannot hold are refused on the host, before anything is enqueued."""
import ctypes as C
import os
from types import SimpleNamespace

import numpy as np
import pytest

from helpers import attention_plan, fine_attention_plan
from test_abi import _cfg, _create, _weights
from test_kv8 import P, _batch

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_05033_amd", "libarb.so")
SHAPE = SimpleNamespace(group=4, n_kv_heads=8, head_dim=64)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(LIB):
        pytest.skip("libarb.so is not built")
    from paper_2512_05033_amd import binding
    return binding.load_library()


@pytest.fixture
def model(lib):
    w, _keep = _weights()
    _, h = _create(lib, _cfg(n_q_heads=32, n_kv_heads=8), w)
    yield h
    lib.arb_model_destroy(h)


def _ws_bytes(lib, splits, items, tokens):
    f = lib._Z18attention_ws_bytesimiii
    f.restype, f.argtypes = C.c_size_t, [C.c_int, C.c_size_t, C.c_int, C.c_int, C.c_int]
    return f(splits, items, tokens, 32, 64)


# One long step among short ones, without room for the list of the places that hold work: the places are the product of sequences,
# parts, heads and query tiles, 2^24 and more of them, or so many that 32 bits hold none of it.
@pytest.mark.parametrize("batch,longest", [(4096, 16384), (65536, 131072)])
@pytest.mark.parametrize("kv8", [True, False])
def test_more_places_than_a_launch_has(lib, model, batch, longest, kv8):
    from paper_2512_05033_amd import binding as B
    steps = np.ones(batch, np.int64)
    steps[batch // 3] = longest
    prefix = np.zeros(batch, np.int64)
    bt = _batch(B, prefix, np.concatenate([[0], np.cumsum(steps)]), longest // 16)
    plan = (fine_attention_plan if kv8 else attention_plan)(lib, SHAPE, prefix, steps)
    assert batch * plan.max_splits * 8 * plan.max_qtiles >= 1 << 24
    kv = B._KVLayer(P, P, P, P) if kv8 else B._KVLayer(P, P, None, None)
    enough = _ws_bytes(lib, plan.max_splits, 0, int(steps.sum()))
    assert lib.arb_stage_attention_kv(model, P, 32 * 64, 0, C.byref(kv), 0.0, C.byref(bt), P, P, enough, None) == B.ARB_EUNSUPPORTED
    assert b"workgroups in one call" in lib.arb_last_error()
    if not kv8:
        assert lib.arb_stage_attention(model, P, 32 * 64, 0, P, P, C.byref(bt), P, P, enough, None) == B.ARB_EUNSUPPORTED


def test_query_rows_are_counted_in_32_bits(lib, model):
    from paper_2512_05033_amd import binding as B
    T = 1 << 26                                                  # of 32 query heads
    bt = _batch(B, [0], [0, T], T // 16)
    t = (C.c_void_p * 2)(P, P)
    kv, kv8 = B._KV(t, t, 8), B._KV8(t, t, t, t, 8)
    room = 1 << 62
    for st in (lib.arb_stage_attention_kv(model, P, 32 * 64, 0, C.byref(B._KVLayer(P, P, P, P)), 0.0, C.byref(bt), P, P, room, None),
               lib.arb_stage_attention(model, P, 32 * 64, 0, P, P, C.byref(bt), P, P, room, None),
               lib.arb_prefill(model, C.byref(kv), C.byref(bt), None, P, room, None),
               lib.arb_prefill_kv8(model, C.byref(kv8), C.byref(bt), None, P, room, None)):
        assert st == B.ARB_EUNSUPPORTED and b"query heads in one call" in lib.arb_last_error()


def test_the_border_of_a_launch(lib):
    """A launch of 256 threads a workgroup holds 2^24 - 1 of them, places rounded up to whole runs on all XCDs."""
    from helpers import AttentionPlan
    from paper_2512_05033_amd import binding as B
    f = lib._Z22check_attention_launchRK8AttnPlaniiiii
    f.restype, f.argtypes = C.c_int, [C.POINTER(AttentionPlan)] + [C.c_int] * 5

    def check(batch=1, tokens=1, **plan):
        pl = AttentionPlan(**{"kv_chunk": 256, "max_splits": 1, "max_qtiles": 1, "n_items": 0, **plan})
        return f(C.byref(pl), batch, tokens, 32, 8, 64)
    assert check(n_items=(1 << 24) - 8) == B.ARB_OK and check(n_items=(1 << 24) - 7) == B.ARB_EUNSUPPORTED
    assert check(n_items=(1 << 24) - 24, max_qtiles=3) == B.ARB_OK and check(n_items=(1 << 24) - 15, max_qtiles=3) == B.ARB_EUNSUPPORTED
    assert check(n_items=0x7fffffff) == B.ARB_EUNSUPPORTED
    assert check(batch=(1 << 21) - 1) == B.ARB_OK and check(batch=1 << 21) == B.ARB_EUNSUPPORTED
    assert check(batch=1 << 16, max_qtiles=1 << 13) == B.ARB_EUNSUPPORTED        # 2^32
    from helpers import FewPlan
    g = lib._Z19check_attention_fewRK7FewPlanii
    g.restype, g.argtypes = C.c_int, [C.POINTER(FewPlan), C.c_int, C.c_int]
    few = lambda batch, **plan: g(C.byref(FewPlan(**{"per": 8, "in_a_row": 1, "parts": 2, "groups": 512, "tiles": 1 << 20, **plan})), batch, 8)
    assert few((1 << 21) - 1) == B.ARB_OK and few(1 << 21) == B.ARB_EUNSUPPORTED and few(1 << 21, parts=1) == B.ARB_OK    # a merge a pair
    assert few(1, groups=1 << 24) == B.ARB_EUNSUPPORTED and few(1, tiles=0x7fffffff) == B.ARB_EUNSUPPORTED
    assert check(tokens=1 << 24) == B.ARB_OK and check(tokens=1 << 24, max_splits=2) == B.ARB_EUNSUPPORTED   # the merge: 32 rows a workgroup


# The two batches that the static array of arb_score_steps_noalloc is said to hold, with capped scores too, however many sequences they are.
@pytest.mark.parametrize("softcap", [0.0, 30.0])
@pytest.mark.parametrize("shape,tokens,ctx", [
    (dict(d_model=1536, n_q_heads=12, n_kv_heads=2, head_dim=128, d_ffn=8960), 128, 32768),
    (dict(d_model=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, d_ffn=14336), 64, 8192)])
def test_the_static_array_holds_the_batches_that_are_promised(lib, shape, tokens, ctx, softcap):
    from paper_2512_05033_amd import binding as B
    w, _keep = _weights()
    _, h = _create(lib, _cfg(**shape), w)
    assert lib.arb_model_set_softcap(h, softcap) == B.ARB_OK
    for batch in range(1, tokens + 1):
        assert lib.arb_workspace_bytes(h, batch, tokens, ctx) <= B.NOALLOC_SCRATCH_BYTES
    lib.arb_model_destroy(h)
