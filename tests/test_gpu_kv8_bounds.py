"""The 8-bit KV cache and capped scores on the GPU: where the parts' format ends, and passes in pieces."""
import numpy as np
import pytest
import torch

import workloads as W
from test_gpu_kv8 import HEADS, U, A, H, _forward_session, attention_ref, layer8, make_batch, queries, rows, stage_model, values  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,prefix,steps", [("router", [2000, 300], [64, 9]), ("target", [700], [16]), ("tiny", [1500], [60]), ("router", [3000], [2]),
                                                ("router", [5000, 900], [40, 64])])
@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("kv8", [True, False])
def test_parts_of_columns_that_differ_by_more_than_fp16_holds(A, heads, prefix, steps, cap, kv8):
    """Columns down to 2^-45 of the largest.  The results of a cut context's parts are fp16 relative to a power of two that puts their
    row's largest at 2^14 to 2^15 (8-bit cache or capped scores, more than 32 rows): a multiple of 2^-24 at the finest, so a rounding
    is off by half of 2^-24 / 2^14 of the row's largest at most, 2^-39 of it, and the largest of a part is at most that of the values.
    Elsewhere parts keep the precision of every column."""
    hq, hkv, hd = HEADS[heads]
    db, tables, n = make_batch(A, prefix, steps, 35)
    k, v = rows((n, hkv, 16, hd), 36, 0.8), rows((n, hkv, 16, hd), 37, 0.8).float()
    for i, e in enumerate((20, 29, 33, 37, 41, 45)):
        v[..., 1 + i::8] *= 2.0 ** -e
    kv = A.KVLayer(k, v.bfloat16())
    if kv8:                                                      # what e4m3 does not hold beside a row's largest becomes 0 in the cache itself
        plain, kv = kv, layer8(A, n, hkv, hd)
        A.arb_kv8_pack(plain, kv)
    q = queries(sum(steps), heads, 38, True)
    got = A.arb_stage_attention_kv(stage_model(heads), q, kv, db, softcap=cap, q_scaled=True)
    ref, mag = attention_ref(heads, q, kv, tables, prefix, steps, cap, True)
    few = max(steps) * hq // hkv <= (32 if kv8 or hd == 64 else 16)
    finest = 0.0 if few or (not kv8 and cap == 0.0) else 2.0 ** -39 * float(values(kv)[1].abs().max())
    assert bool(((got.double().view(ref.shape) - ref).abs() <= 4.3 * U * mag + finest * (1 + U)).all())


@pytest.mark.parametrize("steps", [1, 5, 40])
@pytest.mark.parametrize("norms,softcap,kv8", [(True, 0.0, True), (False, 30.0, True), (True, 20.0, False), (False, 0.0, False)])
@pytest.mark.parametrize("name", ["tiny", "router"])
def test_layer_by_layer_is_the_whole_pass_bit_for_bit(A, name, norms, softcap, kv8, steps):
    """The same batch, so the same plans: what a layer is given and what it makes of it are the same numbers."""
    from dataclasses import replace
    shape = replace(W.TINY, n_layers=3) if name == "tiny" else replace(W.ROUTER_1P5B, n_layers=3, vocab=4096)
    w = W.Workload("kv8", shape, 3, (40, 900), ("fixed", steps, steps), "shuffled", "prefill", 0.0, ("const", 0.0), 781)
    batch, weights, gains, model, kv, db = _forward_session(A, w, 7, softcap, norms, kv8)
    A.arb_prefill(model, kv, H().prompt_batch(w, batch))
    x = torch.randn(batch.total_tokens, shape.d_model, device="cuda")
    whole = A.arb_stage_layers(model, kv, db, 0, 3, x)
    for l in range(3):
        x = A.arb_stage_layers(model, kv, db, l, l + 1, x)
    assert bool(torch.isfinite(whole).all()) and torch.equal(x, whole)
