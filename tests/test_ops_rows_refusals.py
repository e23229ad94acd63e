"""Calls over paged caches of any type that must be refused before anything is enqueued (no GPU needed: made-up addresses never reach a
kernel), and the sizes the host computes."""
import ctypes as C
import os

import pytest
import torch

from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

P = 0x10000                                     # 16-byte aligned, not device memory


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2604_13519_amd.build import build_library
        build_library(verbose=False)
    return ops._load()


def refused(status, word):
    assert status == B.TS_ERR_INVALID_ARG
    assert word in B.load_library().ts_last_error().decode(), B.load_library().ts_last_error()


def change(a, kw):
    for k, v in kw.items():
        if k.startswith("pages_"):
            setattr(a.cache.pages, k[6:], v)
        elif k in ("k_scales", "v_scales"):
            setattr(a.cache, k, v)
        else:
            setattr(a, k, v)
    return a


def cache(dtype=1):
    return ops.ts_kv_pages_any(pages=ops.ts_kv_pages(P, P, 10, 2, 64, dtype))


def append_args(**kw):
    return change(ops.ts_kv_append_norm_rope_args(cache=cache(), table=P, table_stride=4, table_width=4, lengths=P, row_offsets=P, n_seqs=2, n_rows=3, n_q_heads=4, dtype=1,
                                                  q=P, q_stride=256, k=P, k_stride=128, v=P, v_stride=128, q_out=P, q_out_stride=256, q_norm=P, k_norm=P, norm_dtype=1,
                                                  norm_eps=1e-6, rope_theta=1e4, rope_magnitude=1.0, rope_dim=64), kw)


def read_args(**kw):
    return change(ops.ts_kv_read_args(cache=cache(), table=P, table_stride=4, table_width=4, starts=P, row_offsets=P, n_seqs=2, n_rows=3, dtype=1, k_out=P, k_stride=128,
                                      v_out=P, v_stride=128), kw)


def rows_args(**kw):
    return change(ops.ts_kv_attend_rows_args(cache=cache(), table=P, table_stride=4, table_width=4, lengths=P, row_offsets=P, n_seqs=2, n_rows=3, max_len=64, n_q_heads=4, dtype=1,
                                             q=P, q_stride=256, out=P, out_stride=256, lse=P, scale=0.1), kw)


PAGES = [(dict(pages_k=None), "null"), (dict(pages_v=None), "null"), (dict(table=None), "null"), (dict(dtype=2), "dtype"), (dict(dtype=3), "dtype"),
         (dict(pages_dtype=2), "dtype of the pages"), (dict(pages_dtype=5), "dtype of the pages"), (dict(pages_n_pages=0), "pages"), (dict(pages_n_kv_heads=0), "KV heads"),
         (dict(pages_head_dim=96), "head_dim"), (dict(pages_head_dim=32), "head_dim"), (dict(pages_head_dim=256, pages_dtype=0), "head_dim"), (dict(pages_head_dim=4, pages_dtype=0), "head_dim"),
         (dict(pages_dtype=3, pages_head_dim=32, k_scales=P, v_scales=P), "head_dim"), (dict(pages_dtype=3), "scales"), (dict(pages_dtype=3, k_scales=P), "scales"),
         (dict(pages_dtype=3, v_scales=P), "scales"), (dict(k_scales=P), "scales"), (dict(v_scales=P), "scales"), (dict(pages_dtype=3, k_scales=P + 8, v_scales=P), "16-byte"),
         (dict(pages_dtype=3, k_scales=P, v_scales=P + 1), "16-byte"), (dict(pages_k=P + 8), "16-byte"), (dict(pages_v=P + 2), "16-byte"), (dict(n_seqs=0), "n_seqs"),
         (dict(n_seqs=(1 << 20) + 1), "n_seqs"), (dict(table_width=0), "table"), (dict(table_stride=3), "table"), (dict(table=P + 2), "misaligned"), (dict(n_rows=-1), "rows"),
         (dict(n_rows=(1 << 23) + 1), "rows"), (dict(row_offsets=P + 2), "misaligned"), (dict(), "not device memory"), (dict(pages_dtype=3, k_scales=P, v_scales=P), "not device memory")]


@pytest.mark.parametrize("kw,word", PAGES + [
    (dict(lengths=None), "null"), (dict(lengths=P + 1), "misaligned"), (dict(row_offsets=None), "row_offsets"), (dict(positions=P + 2), "positions"), (dict(rope_theta=-1.0), "rope_theta"),
    (dict(rope_theta=float("inf")), "rope_theta"), (dict(rope_theta=float("nan")), "rope_theta"), (dict(rope_dim=-2), "rope_dim"), (dict(rope_dim=63), "rope_dim"), (dict(rope_dim=66), "rope_dim"),
    (dict(rope_freqs=P + 2), "rope_freqs"), (dict(rope_magnitude=float("nan")), "rope_magnitude"), (dict(rope_magnitude=float("inf")), "rope_magnitude"), (dict(norm_dtype=2), "norm_dtype"),
    (dict(norm_eps=-1e-9), "norm_eps"), (dict(norm_eps=float("nan")), "norm_eps"), (dict(norm_eps=float("inf")), "norm_eps"), (dict(q_norm=P + 1), "gains"), (dict(k_norm=P + 1), "gains"),
    (dict(q_norm=P + 2, norm_dtype=0), "gains"), (dict(q=None), "belong together"), (dict(q_out=None), "belong together"), (dict(n_q_heads=0), "query heads"), (dict(k=None), "null"),
    (dict(v=None), "null"), (dict(k_stride=127), "stride"), (dict(v_stride=1), "stride"), (dict(q_stride=255), "stride"), (dict(q_out_stride=0), "stride"), (dict(q=P + 1), "aligned"),
    (dict(k=P + 1), "aligned"), (dict(v=P + 1), "aligned")])
def test_append_refusals(lib, kw, word):
    refused(lib.ts_kv_append_norm_rope(C.byref(append_args(**kw)), None), word)


@pytest.mark.parametrize("kw,word", PAGES + [(dict(row_offsets=None), "null"), (dict(starts=P + 2), "starts"), (dict(k_stride=127), "stride"), (dict(v_stride=127), "stride"),
                                             (dict(k_out=P + 1), "aligned"), (dict(v_out=P + 1), "aligned")])
def test_read_refusals(lib, kw, word):
    refused(lib.ts_kv_read(C.byref(read_args(**kw)), None), word)


@pytest.mark.parametrize("kw,word", PAGES + [
    (dict(lengths=None), "null"), (dict(lengths=P + 1), "misaligned"), (dict(n_q_heads=3), "query heads"), (dict(n_q_heads=0), "query heads"), (dict(max_len=-1), "max_len"),
    (dict(max_len=(1 << 30) + 1), "max_len"), (dict(window=-1), "window"), (dict(window=5, ancestors=P), "window and ancestors"), (dict(ancestors=P + 4), "ancestors"),
    (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(q=None), "null"), (dict(out=None), "null"), (dict(q_stride=255), "stride"), (dict(out_stride=100), "stride"),
    (dict(q=P + 1), "aligned"), (dict(out=P + 1), "aligned"), (dict(lse=P + 2), "aligned"), (dict(row_offsets=None, n_rows=1), "rows for 2 sequences"), (dict(max_len=100000), "workspace"),
    (dict(max_len=100000, workspace=P, workspace_bytes=1024), "workspace"), (dict(max_len=100000, workspace=P + 4, workspace_bytes=1 << 30), "workspace"),
    (dict(n_seqs=1 << 20, n_rows=1 << 20, n_q_heads=65536), "too many"), (dict(n_rows=1 << 23), "too many")])
def test_attend_rows_refusals(lib, kw, word):
    refused(lib.ts_kv_attend_rows(C.byref(rows_args(**kw)), None), word)


def test_nothing_to_do_and_null(lib):
    refused(lib.ts_kv_append_norm_rope(None, None), "null")
    refused(lib.ts_kv_read(None, None), "null")
    refused(lib.ts_kv_attend_rows(None, None), "null")
    refused(lib.ts_kv_attend_rows_workspace(1, 1, 4, 2, 64, 100, 0, None), "null")
    refused(lib.ts_kv_attend_rows_workspace(1, 1, 5, 2, 64, 100, 0, C.byref(C.c_uint64())), "query heads")
    refused(lib.ts_kv_attend_rows_workspace(1, 1, 4, 2, 256, 100, 0, C.byref(C.c_uint64())), "head_dim")
    assert lib.ts_kv_append_norm_rope(C.byref(append_args(n_rows=0)), None) == B.TS_OK
    assert lib.ts_kv_read(C.byref(read_args(n_rows=0)), None) == B.TS_OK
    assert lib.ts_kv_read(C.byref(read_args(k_out=None, v_out=None)), None) == B.TS_OK
    assert lib.ts_kv_attend_rows(C.byref(rows_args(n_rows=0)), None) == B.TS_OK


def test_8_bit_pages_are_for_the_calls_that_say_so(lib):
    a = ops.ts_kv_append_args(pages=ops.ts_kv_pages(P, P, 10, 2, 64, 3), table=P, table_stride=4, table_width=4, lengths=P, row_offsets=P, n_seqs=2, n_rows=3, dtype=1, k=P, k_stride=128,
                              v=P, v_stride=128)
    refused(lib.ts_kv_append(C.byref(a), None), "dtype")


def test_workspace_never_shrinks_with_the_length(lib):
    for n, rows, hq, hkv, window in ((1, 1, 32, 8, 0), (8, 8, 64, 8, 0), (3, 50, 6, 2, 500), (1, 65, 32, 8, 0), (64, 64, 16, 1, 0), (16, 528, 32, 8, 300), (5000, 5000, 8, 8, 0)):
        last = 0
        for top in list(range(0, 3000, 37)) + [4096, 32768, 131072, 1 << 30]:
            b = C.c_uint64()
            assert lib.ts_kv_attend_rows_workspace(n, rows, hq, hkv, 128, top, window, C.byref(b)) == B.TS_OK
            assert b.value >= last
            last = b.value


def test_tensors_are_looked_at(lib):
    t = lambda *shape, dtype=torch.float32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    k, v = t(3, 2, 16, 64), t(3, 2, 64, 16)
    k8, v8 = k.to(torch.float8_e4m3fn), v.to(torch.float8_e4m3fn)
    for call in (lambda *p, **kw: ops.ts_kv_append_norm_rope(*p, i(1, 3), i(1), i(2), t(4, 128), t(4, 128), t(4, 128), **kw),
                 lambda *p, **kw: ops.ts_kv_read(*p, i(1, 3), i(1), i(2), 4, **kw), lambda *p, **kw: ops.ts_kv_attend_rows(*p, i(1, 3), i(1), i(2), t(4, 128), 40, **kw)):
        with pytest.raises(ValueError, match="k_pages"):
            call(k, v)
        with pytest.raises(ValueError, match="k_pages"):
            call(k8, v8, scales=(t(3, 2, 16, dtype=torch.uint8),) * 2)
        with pytest.raises(ValueError, match="scales belong"):
            call(k, v, scales=(t(3, 2, 16, dtype=torch.uint8),) * 2)
        with pytest.raises(TypeError, match="v_pages is missing"):
            call(k, None)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        ops.ts_kv_read(k, v, i(1, 3), i(1), i(2), 4, dtype=torch.float16)
    with pytest.raises(ValueError, match="q_norm requires a gradient"):
        class OnGpu(torch.Tensor):
            is_cuda = True
        ops._gain(torch.zeros(64, requires_grad=True).as_subclass(OnGpu), "q_norm", 64, None)
    with pytest.raises(ValueError, match="q_norm: 64 contiguous"):
        ops._gain(t(32), "q_norm", 64, None)
    with pytest.raises(TypeError, match="k_norm"):
        ops._gain(t(64), "k_norm", 64, torch.bfloat16)


class OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU: what is looked at before a call."""
    is_cuda = True


def on_gpu(*shape, dtype=torch.float32, grad=False):
    t = torch.zeros(shape).to(dtype)
    return (t.requires_grad_() if grad else t).as_subclass(OnGpu)


@pytest.mark.parametrize("which", [0, 1])
def test_gradients_of_8_bit_pages_are_refused(lib, which):
    e4m3, byte, i32 = torch.float8_e4m3fn, torch.uint8, torch.int32
    k, v = on_gpu(3, 2, 16, 64, dtype=e4m3, grad=which == 0), on_gpu(3, 2, 64, 16, dtype=e4m3, grad=which == 1)
    scales = (on_gpu(3, 2, 16, dtype=byte), on_gpu(3, 2, 16, dtype=byte))
    table, one, off, rows = on_gpu(1, 3, dtype=i32), on_gpu(1, dtype=i32), on_gpu(2, dtype=i32), on_gpu(4, 128)
    for call in (lambda: ops.ts_kv_append_norm_rope(k, v, table, one, off, rows, rows, rows, scales=scales), lambda: ops.ts_kv_read(k, v, table, one, off, 4, scales=scales),
                 lambda: ops.ts_kv_attend_rows(k, v, table, one, off, rows, 40, scales=scales)):
        with pytest.raises(ValueError, match="pages requires a gradient"):
            call()
    with torch.no_grad():
        ops._any_pages(k, v, scales)


def test_a_gradient_of_lse_is_refused(lib):
    k, v, table, one, off = on_gpu(3, 2, 16, 64), on_gpu(3, 2, 64, 16), on_gpu(4, 3, dtype=torch.int32), on_gpu(4, dtype=torch.int32), on_gpu(2, dtype=torch.int32)
    q, out, lse = on_gpu(4, 128), on_gpu(4, 128), on_gpu(4, 2, grad=True)
    with pytest.raises(ValueError, match="lse requires a gradient"):
        ops.ts_kv_attend_rows(k, v, table, one, off, q, 40, out=out, lse=lse)
    with pytest.raises(ValueError, match="lse requires a gradient"):
        ops.ts_kv_attend(k, v, table, one, q, 40, out=out, lse=lse)


def test_numbers_beyond_32_bits_are_refused(lib):
    for at in range(7):
        sizes = [1, 1, 8, 8, 128, 100, 0]
        sizes[at] += 1 << 32
        with pytest.raises(ValueError, match="32 bits"):
            ops.ts_kv_attend_rows_workspace(*sizes)


@pytest.mark.parametrize("cls,pack", [(ops.ts_kv_append_norm_rope_args, ops._pack_append_norm_rope), (ops.ts_kv_read_args, ops._pack_read), (ops.ts_kv_attend_rows_args, ops._pack_rows)])
def test_packed_arguments_are_the_structure(cls, pack):
    values = []

    def fill(part):
        for name, kind in part._fields_:
            if issubclass(kind, C.Structure):
                fill(getattr(part, name))
            else:
                values.append(0.5 + len(values) if kind is C.c_float else 3 + 1000 * len(values))
                setattr(part, name, values[-1])
        return part
    assert bytes(fill(cls())) == pack(*values)
