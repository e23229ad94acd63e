"""Passes whose logits are no numbers - a weight, a key or a value that is NaN - have no largest logit, hence no next token; what
stands for none must not become the root of the next pass, where it would be looked up in the embedding."""
import numpy as np
import pytest
import torch

import workloads as wl
from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

pytestmark = pytest.mark.gpu


def with_bad_weight(cfg, value):
    w = wl.gen_weights(cfg, 3)
    wd = wl.bf16_bits_to_f32(w["layers"][0]["wd"]).copy() if cfg.dtype else w["layers"][0]["wd"].copy()
    wd[5, 7] = value
    return dict(w, layers=[dict(w["layers"][0], wd=wl.f32_to_bf16_bits(wd) if cfg.dtype else wd)] + w["layers"][1:])


def not_committed(kv, result, vocab):
    """The result has no token, the commit says so every time, and the cache stays as it is."""
    assert not 0 <= result[3] < vocab
    n = B.ts_kv_len(kv)
    for _ in range(2):
        with pytest.raises(B.TsError) as e:
            B.ts_kv_commit(kv)
        assert e.value.status == B.TS_ERR_TOKEN_RANGE and "no next token" in str(e.value)
        assert B.ts_kv_len(kv) == n


@pytest.mark.parametrize("cfg_name,dtype", [("small_fp32", B.TS_DTYPE_F32), ("small_bf16", B.TS_DTYPE_BF16), ("small_bf16", B.TS_DTYPE_MX4)])
def test_weights_that_are_no_numbers(cfg_name, dtype):
    cfg = wl.get_config(cfg_name)
    model = B.ts_model_load(cfg.with_(dtype=dtype), with_bad_weight(cfg, np.nan))
    kvs = [B.ts_kv_alloc(model, 64) for _ in range(2)]
    try:
        for kv in kvs:
            B.ts_prefill(model, kv, [1, 2, 3])
        for _ in range(2):
            not_committed(kvs[0], B.ts_verify(model, kvs[0], [4, 5], [-1, 0]), cfg.vocab)
            not_committed(kvs[0], B.ts_verify(model, kvs[0], [], []), cfg.vocab)
            not_committed(kvs[0], B.ts_verify_sample(model, kvs[0], [4, 5], [-1, 0], 0.7, [0.5, 0.5], 1), cfg.vocab)
            for kv, r in zip(kvs, B.ts_verify_batch(model, kvs, [([4], [-1]), ([], [])])):
                not_committed(kv, r, cfg.vocab)
    finally:
        for kv in kvs:
            B.ts_kv_free(kv)
        B.ts_model_free(model)


@pytest.mark.parametrize("cfg_name", ["small_fp32", "small_bf16"])
def test_appended_keys_that_are_no_numbers_reach_their_own_sequence_only(cfg_name):
    cfg = wl.get_config(cfg_name)
    model = B.ts_model_load(cfg, wl.gen_weights(cfg, 3))
    kvs = [B.ts_kv_alloc(model, 64) for _ in range(2)]
    dt = torch.bfloat16 if cfg.dtype else torch.float32
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    tree = ([4, 5], [-1, 0])
    try:
        for kv in kvs:
            B.ts_prefill(model, kv, [1, 2, 3])
        want = B.ts_verify(model, kvs[1], *tree)
        rows = torch.full((1, cfg.n_kv_heads * cfg.head_dim), float("nan"), dtype=dt, device="cuda")
        table = torch.from_numpy(ops.ts_kv_page_table(kvs[0], 64)).cuda()[None]
        for layer in range(cfg.n_layers):
            ops.ts_kv_append(ops.ts_kv_layer_pages(kvs[0], layer), None, table, ints([2]), ints([0, 1]), None, rows, rows, cfg.rope_theta)
        ops.ts_kv_extend(kvs[0], 1)
        not_committed(kvs[0], B.ts_verify(model, kvs[0], *tree), cfg.vocab)
        both = B.ts_verify_batch(model, kvs, [tree, tree])
        not_committed(kvs[0], both[0], cfg.vocab)
        assert both[1][0] == want[0] and both[1][3] == want[3]
        assert B.ts_verify(model, kvs[1], *tree) == want
        B.ts_kv_commit(kvs[1])
        # Without that position the cache is as it was.  bf16 passes read whole blocks: what the passes before left behind the
        # length makes theirs NaN too, until it is written over.
        B.ts_kv_truncate(kvs[0], 2)
        if cfg.dtype:
            not_committed(kvs[0], B.ts_verify(model, kvs[0], *tree), cfg.vocab)
            K, V = wl.gen_context_kv(cfg, 60, seed=1)
            B.ts_kv_import(kvs[0], K, V)
            B.ts_kv_truncate(kvs[0], 0)
            B.ts_set_pending(kvs[0], 1)
            B.ts_prefill(model, kvs[0], [2, 3])
        assert B.ts_verify(model, kvs[0], *tree) == want
    finally:
        for kv in kvs:
            B.ts_kv_free(kv)
        B.ts_model_free(model)
