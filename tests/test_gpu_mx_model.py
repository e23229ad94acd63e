"""Models whose layers' matrices are 4-bit (TS_DTYPE_MX4): the oracle and the bf16 path with the rounded values as their weights.

A 4-bit model computes what the bf16 model of the rounded values computes: the weights are the same halves, the rows are
the same hi + lo halves, and only the order of the fp32 sums differs, so the tolerances of the bf16 path against the oracle
hold, with the oracle given the rounded weights.  Rounding to four bits is done here by the definition, on the CPU."""
import numpy as np
import pytest
import torch

import gpu_utils as U
import workloads as wl
from oracle import toolspec_oracle as O
from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops
from test_gpu_mx import definition

pytestmark = pytest.mark.gpu
MATRICES = ("wq", "wk", "wv", "wo", "wg", "wu", "wd")


def rounded(w):
    """The weights (bf16 bit patterns) with every layer matrix rounded to 4-bit values, which bf16 holds exactly."""
    out = dict(w, layers=[])
    for layer in w["layers"]:
        q = dict(layer)
        for k in MATRICES:
            x = torch.from_numpy(wl.bf16_bits_to_f32(layer[k]))
            v = definition(x)[0]
            bits = v.to(torch.bfloat16)
            assert bool((bits.double() == v).all())
            q[k] = bits.view(torch.int16).numpy().view(np.uint16)
        out["layers"].append(q)
    return out


@pytest.fixture(scope="module", params=["small_bf16", "small_bf16_hd64"])
def models(request):
    """(config, handle of the 4-bit model, handle of the bf16 model of the rounded weights, its oracle)"""
    cfg = wl.get_config(request.param)
    w = wl.gen_weights(cfg, 77)
    r = rounded(w)
    mx = B.ts_model_load(cfg.with_(dtype=B.TS_DTYPE_MX4), w)
    bf = B.ts_model_load(cfg, r)
    for m in (mx, bf):
        B.ts_model_keep_logits(m, True)
    yield cfg, mx, bf, O.OracleModel(cfg, r, cache=True), r
    B.ts_model_free(mx)
    B.ts_model_free(bf)


@pytest.mark.parametrize("P,n", [(0, 0), (1, 1), (40, 7), (150, 15), (100, 16), (333, 40), (150, 63), (64, 64)])
def test_verify_against_the_oracle(models, P, n):
    cfg, mx, _, omodel, _ = models
    rng = np.random.default_rng(P * 100 + n)
    K, V = wl.gen_context_kv(cfg, P, seed=P + 3)
    kv, okv = U.make_pair(cfg, mx, K, V, int(rng.integers(cfg.vocab)))
    tok = rng.integers(0, cfg.vocab, n).astype(np.int32)
    par = np.array([rng.integers(-1, i) for i in range(n)], np.int32)
    res, oR = U.check_verify(cfg, mx, omodel, kv, okv, tok, par, label="mx %s P %d n %d" % (cfg.name, P, n))
    U.commit_both(cfg, kv, okv, res, oR)
    assert B.ts_model_saturations(mx) == 0
    B.ts_kv_free(kv)


def test_batches_and_ingestion_like_the_bf16_model(models):
    """Passes of every size class of the projections, the same context and trees on both models."""
    cfg, mx, bf, _, _ = models
    rng = np.random.default_rng(9)
    for n_seqs, nodes in ((2, 20), (3, 60), (9, 64), (33, 3), (70, 0)):
        logits, tokens, caches = [], [], []
        contexts = [rng.integers(0, cfg.vocab, int(rng.integers(1, 90))) for _ in range(n_seqs)]
        trees = [(rng.integers(0, cfg.vocab, nodes).astype(np.int32), np.array([rng.integers(-1, i) for i in range(nodes)], np.int32)) for _ in range(n_seqs)]
        for m in (mx, bf):
            kvs = [B.ts_kv_alloc(m, 200) for _ in range(n_seqs)]
            for kv, c in zip(kvs, contexts):
                B.ts_prefill(m, kv, c)
            B.ts_verify_batch(m, kvs, trees)
            rows = n_seqs * (nodes + 1)
            logits.append(B.ts_get_logits(m, 0, rows, cfg.vocab))
            tokens.append(B.ts_get_row_tokens(m, 0, rows))
            caches.append([B.ts_kv_export(kv, 0, len(c), cfg) for kv, c in zip(kvs, contexts)])
            for kv in kvs:
                B.ts_kv_free(kv)
        worst = max(U.rel_l2(a, b) for a, b in zip(*logits))
        print("%s %d x %d: logits %.3g apart, %d of %d tokens differ" % (cfg.name, n_seqs, nodes + 1, worst, int((tokens[0] != tokens[1]).sum()), len(tokens[0])), flush=True)
        assert worst <= U.TOL_BF16_R
        for r in np.nonzero(tokens[0] != tokens[1])[0]:
            top = np.sort(logits[1][r])[-2:]
            assert top[1] - top[0] < U.MARGIN
        for (ka, va), (kb, vb) in zip(*caches):
            for a, b in ((ka, kb), (va, vb)):
                assert U.rel_l2(wl.bf16_bits_to_f32(a), wl.bf16_bits_to_f32(b)) <= 3e-3


def test_rounded_weights_are_kept(models):
    """A model handed over as the values of its codes is the same model, bit for bit."""
    cfg, mx, _, _, r = models
    again = B.ts_model_load(cfg.with_(dtype=B.TS_DTYPE_MX4), r)
    try:
        B.ts_model_keep_logits(again, True)
        got = []
        for m in (mx, again):
            kv = B.ts_kv_alloc(m, 100)
            B.ts_prefill(m, kv, np.arange(50) % cfg.vocab)
            B.ts_verify(m, kv, [1, 2, 3], [-1, 0, 1])
            got.append(B.ts_get_logits(m, 0, 4, cfg.vocab))
            B.ts_kv_free(kv)
        assert np.array_equal(got[0], got[1])
    finally:
        B.ts_model_free(again)


def test_weights_beyond_half_are_refused_and_small_ones_kept():
    cfg = wl.get_config("small_bf16_hd64").with_(n_layers=1)
    w = wl.gen_weights(cfg, 5)

    def with_wo(value):
        x = wl.bf16_bits_to_f32(w["layers"][0]["wo"]).copy()
        x[3, 5] = value
        return dict(w, layers=[dict(w["layers"][0], wo=wl.f32_to_bf16_bits(x))])

    for value in (70000.0, -1e30, 65536.0):
        with pytest.raises(B.TsError) as e:
            B.ts_model_load(cfg.with_(dtype=B.TS_DTYPE_MX4), with_wo(value))
        assert e.value.status == B.TS_ERR_INVALID_ARG and "half range" in str(e.value)
    for value in (49152.0, 65280.0, 2.0 ** -30):
        B.ts_model_free(B.ts_model_load(cfg.with_(dtype=B.TS_DTYPE_MX4), with_wo(value)))
    with pytest.raises(B.TsError):
        B.ts_model_load(cfg.with_(dtype=3), w)
    # tiny weights throughout one matrix: half's subnormal grid, off by less than 3e-8 each
    tiny = wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(w["layers"][0]["wd"]) * np.float32(2.0 ** -9))
    w2 = dict(w, layers=[dict(w["layers"][0], wd=tiny)])
    r2 = rounded(w2)
    m = B.ts_model_load(cfg.with_(dtype=B.TS_DTYPE_MX4), w2)
    B.ts_model_keep_logits(m, True)
    K, V = wl.gen_context_kv(cfg, 30, seed=1)
    kv, okv = U.make_pair(cfg, m, K, V, 3)
    U.check_verify(cfg, m, O.OracleModel(cfg, r2, cache=True), kv, okv, np.array([4, 5], np.int32), np.array([-1, 0], np.int32), label="tiny weights")
    B.ts_kv_free(kv)
    B.ts_model_free(m)


def test_plain_read_reads_what_there_is(models):
    cfg, mx, bf, _, _ = models
    B.ts_profile_enable(mx, True)
    assert B.ts_profile_plain_read(mx, 2) == ops.ts_mx_packed_bytes(2 * cfg.d_ffn, cfg.d_model)
    B.ts_profile_enable(mx, False)


def test_generation_follows_greedy_decoding(models):
    """Steps with drafts emit the tokens that steps without drafts emit (rows of one pass and of another: the same model)."""
    cfg, mx, _, _, _ = models
    kv = B.ts_kv_alloc(mx, 300)
    B.ts_prefill(mx, kv, (np.arange(40) * 7) % cfg.vocab)
    n0 = B.ts_kv_len(kv)
    plain = []
    margins = []
    for _ in range(24):
        _, _, _, bonus = B.ts_verify(mx, kv, [], [])
        lg = np.sort(B.ts_get_logits(mx, 0, 1, cfg.vocab)[0])[-2:]
        margins.append(float(lg[1] - lg[0]))
        B.ts_kv_commit(kv)
        plain.append(bonus)
    B.ts_kv_free(kv)
    kv = B.ts_kv_alloc(mx, 300)
    B.ts_prefill(mx, kv, (np.arange(40) * 7) % cfg.vocab)
    assert B.ts_kv_len(kv) == n0
    out = []
    while len(out) < 24:
        draft = plain[len(out):len(out) + 6]
        l, acc, _, bonus = B.ts_verify(mx, kv, draft, list(range(-1, len(draft) - 1)))
        B.ts_kv_commit(kv)
        out += acc + [bonus]
    B.ts_kv_free(kv)
    first = next((i for i in range(24) if out[i] != plain[i]), None)       # where they part, the two best logits are as good as equal
    print("%s: smallest margin %.3g at step %d, first difference at %s" % (cfg.name, min(margins), int(np.argmin(margins)), first))
    assert first is None or margins[first] < U.MARGIN
