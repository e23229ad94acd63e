"""Calls of the device-tensor operators that must be refused before anything is enqueued (no GPU needed: made-up addresses
never reach a kernel), the exports, and the sizes the host computes."""
import ctypes as C
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_2604_13519_amd import binding as B
from paper_2604_13519_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
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


def test_every_declared_operator_is_exported(lib):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "toolspec_ops.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(ts_[a-z_]+)\s*\(", src))
    assert names == set(ops.EXPORTS)
    for n in names:
        assert hasattr(lib, n) and callable(getattr(ops, n))


def test_quantize_refusals(lib):
    q = lib.ts_mx_quantize
    refused(q(P, 2, 4, 64, 64, P, P, None), "dtype")
    refused(q(P, 0, -1, 64, 64, P, P, None), "rows")
    refused(q(P, 0, 4, 64, 63, P, P, None), "row stride")
    refused(q(None, 0, 4, 64, 64, P, P, None), "null")
    refused(q(P, 0, 4, 64, 64, None, P, None), "null")
    refused(q(P, 0, 4, 64, 64, P, None, None), "null")
    refused(q(P, 0, 4, 64, 64, P + 8, P, None), "16-byte")
    refused(q(P + 2, 0, 4, 64, 64, P, P, None), "aligned")
    refused(q(P, 0, 4, 64, 64, P, P, None), "not device memory")
    refused(lib.ts_mx_dequantize(P, P, 4, 64, P, 7, 64, None), "dtype")
    refused(lib.ts_mx_dequantize(P, P, 4, 64, P, 1, 64, None), "not device memory")
    assert q(None, 0, 0, 64, 64, None, None, None) == B.TS_OK and q(None, 0, 4, 0, 0, None, None, None) == B.TS_OK


def test_pack_and_project_refusals(lib):
    n = C.c_uint64()
    refused(lib.ts_mx_packed_bytes(0, 5, C.byref(n)), "matrix")
    refused(lib.ts_mx_packed_bytes(5, (1 << 22) + 1, C.byref(n)), "matrix")
    refused(lib.ts_mx_packed_bytes(5, 5, None), "null")
    refused(lib.ts_mx_pack(P, P, 0, 32, P, None), "matrix")
    refused(lib.ts_mx_pack(P, P, 16, 32, None, None), "null")
    refused(lib.ts_mx_pack(P, P, 16, 32, P + 4, None), "16-byte")
    refused(lib.ts_mx_pack(P, P, 16, 32, P, None), "not device memory")
    p = lib.ts_mx_project
    refused(p(P, 16, 32, P, 3, 1, 32, P, 16, None), "dtype")
    refused(p(P, 16, 32, P, 1, -1, 32, P, 16, None), "rows")
    refused(p(P, 16, 32, P, 1, (1 << 19) + 1, 32, P, 16, None), "rows")
    refused(p(P, 16, 32, P, 1, 1, 31, P, 16, None), "strides")
    refused(p(P, 16, 32, P, 1, 1, 32, P, 15, None), "strides")
    refused(p(P, 16, 32, P, 1, 2, (1 << 22) + 1, P, 16, None), "apart")
    refused(p(P + 1, 16, 32, P, 1, 1, 32, P, 16, None), "aligned")
    refused(p(P, 16, 32, P + 1, 1, 1, 32, P, 16, None), "aligned")
    refused(p(P, 16, 32, None, 1, 1, 32, P, 16, None), "null")
    refused(p(P, 16, 32, P, 1, 1, 32, P, 16, None), "not device memory")
    assert p(None, 16, 32, None, 1, 0, 32, None, 16, None) == B.TS_OK


def test_packed_bytes_cover_the_matrix(lib):
    for n_out, n_in in ((1, 1), (16, 128), (17, 129), (14336, 4096), (1 << 24, 1 << 22)):
        assert ops.ts_mx_packed_bytes(n_out, n_in) == -(-n_out // 16) * -(-n_in // 128) * (16 * 4 * 17)


def append_args(**kw):
    a = ops.ts_kv_append_args(pages=ops.ts_kv_pages(P, P, 10, 2, 64, 1), table=P, table_stride=4, table_width=4, lengths=P, row_offsets=P, n_seqs=2, n_rows=3, n_q_heads=4,
                              dtype=1, q=P, q_stride=256, k=P, k_stride=128, v=P, v_stride=128, q_out=P, q_out_stride=256, rope_theta=1e4)
    return change(a, kw)


def attend_args(**kw):
    a = ops.ts_kv_attend_args(pages=ops.ts_kv_pages(P, P, 10, 2, 64, 1), table=P, table_stride=4, table_width=4, lengths=P, n_seqs=2, max_len=64, window=0, n_q_heads=4,
                              dtype=1, q=P, q_stride=256, out=P, out_stride=256, lse=P, scale=0.1, workspace=None, workspace_bytes=0)
    return change(a, kw)


def change(a, kw):
    for k, v in kw.items():
        if k.startswith("pages_"):
            setattr(a.pages, k[6:], v)
        else:
            setattr(a, k, v)
    return a


SHARED = [(dict(pages_k=None), "null"), (dict(pages_v=None), "null"), (dict(table=None), "null"), (dict(lengths=None), "null"), (dict(dtype=2), "dtype"),
          (dict(pages_dtype=5), "dtype"), (dict(pages_n_pages=0), "pages"), (dict(pages_n_kv_heads=0), "KV heads"), (dict(pages_head_dim=96), "head_dim"),
          (dict(pages_head_dim=32), "head_dim"), (dict(pages_head_dim=256, pages_dtype=0), "head_dim"), (dict(pages_head_dim=4, pages_dtype=0), "head_dim"),
          (dict(pages_k=P + 8), "16-byte"), (dict(pages_v=P + 2), "16-byte"), (dict(n_seqs=0), "n_seqs"), (dict(n_seqs=(1 << 20) + 1), "n_seqs"),
          (dict(table_width=0), "table"), (dict(table_stride=3), "table"), (dict(table=P + 2), "misaligned"), (dict(lengths=P + 1), "misaligned"),
          (dict(q_stride=255), "stride"), (dict(q=P + 1), "aligned"), (dict(), "not device memory")]


@pytest.mark.parametrize("kw,word", SHARED + [
    (dict(n_rows=-1), "rows"), (dict(n_rows=(1 << 23) + 1), "rows"), (dict(row_offsets=None), "row_offsets"), (dict(row_offsets=P + 2), "row_offsets"),
    (dict(rope_theta=-1.0), "rope_theta"), (dict(rope_theta=float("inf")), "rope_theta"), (dict(rope_theta=float("nan")), "rope_theta"),
    (dict(q=None), "belong together"), (dict(q_out=None), "belong together"), (dict(n_q_heads=0), "query heads"), (dict(k=None), "null"), (dict(v=None), "null"),
    (dict(k_stride=127), "stride"), (dict(v_stride=1), "stride"), (dict(q_out_stride=0), "stride"), (dict(k=P + 1), "aligned"), (dict(v=P + 1), "aligned")])
def test_append_refusals(lib, kw, word):
    refused(lib.ts_kv_append(C.byref(append_args(**kw)), None), word)


@pytest.mark.parametrize("kw,word", SHARED + [
    (dict(n_q_heads=3), "query heads"), (dict(n_q_heads=0), "query heads"), (dict(max_len=-1), "max_len"), (dict(max_len=(1 << 30) + 1), "max_len"),
    (dict(window=-1), "window"), (dict(scale=float("inf")), "scale"), (dict(scale=float("nan")), "scale"), (dict(q=None), "null"), (dict(out=None), "null"),
    (dict(out_stride=100), "stride"), (dict(lse=P + 2), "aligned"), (dict(max_len=100000), "workspace"), (dict(max_len=100000, workspace=P, workspace_bytes=1024), "workspace"),
    (dict(max_len=100000, workspace=P + 4, workspace_bytes=1 << 30), "workspace"), (dict(n_seqs=1 << 20, n_q_heads=65536), "too many"), (dict(n_seqs=1 << 20, n_q_heads=32), "too many")])
def test_attend_refusals(lib, kw, word):
    refused(lib.ts_kv_attend(C.byref(attend_args(**kw)), None), word)


def test_null_structs_and_handles(lib):
    refused(lib.ts_kv_append(None, None), "null")
    refused(lib.ts_kv_attend(None, None), "null")
    refused(lib.ts_kv_layer_pages(None, 0, C.byref(ops.ts_kv_pages())), "null")
    refused(lib.ts_kv_page_table(None, (C.c_int32 * 1)(), 1), "null")
    refused(lib.ts_kv_extend(None, 1, None), "null")
    refused(lib.ts_kv_attend_workspace(1, 4, 2, 64, 100, 0, None), "null")
    refused(lib.ts_kv_attend_workspace(1, 5, 2, 64, 100, 0, C.byref(C.c_uint64())), "query heads")
    assert lib.ts_kv_append(C.byref(append_args(n_rows=0)), None) == B.TS_OK


def test_workspace_never_shrinks_with_the_length(lib):
    for n, hq, hkv, window in ((1, 32, 8, 0), (8, 64, 8, 0), (3, 6, 2, 500), (64, 16, 1, 0), (5000, 8, 8, 0)):
        last = 0
        for top in list(range(0, 3000, 37)) + [4096, 32768, 131072, 1 << 30]:
            b = C.c_uint64()
            assert lib.ts_kv_attend_workspace(n, hq, hkv, 128, top, window, C.byref(b)) == B.TS_OK
            assert b.value >= last
            last = b.value


def test_tensors_are_looked_at(lib):
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError, match="not on a GPU"):
        ops.ts_mx_quantize(x)
    with pytest.raises(ValueError, match="contiguous rows"):
        ops.ts_mx_quantize(x.t())
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        ops.ts_mx_quantize(x.half())
    with pytest.raises(ValueError, match="on a GPU"):
        ops.ts_mx_dequantize(torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8), 64)
    with pytest.raises(ValueError, match="k_pages"):
        ops.ts_kv_attend(torch.zeros((3, 2, 16, 64)), torch.zeros((3, 2, 64, 16)), torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 128)), 40)


def test_types_of_values_are_refused_by_name(lib):
    codes, scales = torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8)
    for dtype in (torch.float16, torch.float64, torch.int32, None):
        with pytest.raises(TypeError, match="float32 or bfloat16"):
            ops.ts_mx_dequantize(codes, scales, 64, dtype)


def test_numbers_beyond_32_bits_are_refused(lib):
    """ctypes hands on the low 32 bits of a larger number: sizes of another matrix, a length of zero."""
    big = (1 << 32) + 16
    for call in (lambda: ops.ts_mx_packed_bytes(big, 128), lambda: ops.ts_mx_packed_bytes(16, big), lambda: ops.ts_mx_packed_bytes(-big, 128),
                 lambda: ops.ts_kv_attend_workspace(1, 8, 8, 128, 1 << 32), lambda: ops.ts_kv_attend_workspace(1, 8, 8, 128, 100, 1 << 32),
                 lambda: ops.ts_kv_attend_workspace((1 << 32) + 1, 8, 8, 128, 100), lambda: ops.ts_kv_extend(None, 1 << 32, stream=_NoStream),
                 lambda: ops.ts_kv_layer_pages(None, 1 << 32)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


class _NoStream:
    cuda_stream = 0


def test_tensors_that_require_gradients_are_refused(lib):
    """No call has a backward pass: a result without one in a graph that records them would lose the gradient silently."""
    x = torch.zeros((4, 64), requires_grad=True)
    plain = torch.zeros((4, 64))
    packed = torch.zeros(16 * 4 * 17, dtype=torch.uint8)
    with pytest.raises(ValueError, match="x requires a gradient"):
        ops.ts_mx_quantize(x)
    with pytest.raises(ValueError, match="out requires a gradient"):
        ops._rows(x, "out", 64)
    with pytest.raises(ValueError, match="x requires a gradient"):
        ops.ts_mx_project(packed, 16, x)
    for call in (lambda: ops.ts_mx_quantize(x.detach()), lambda: ops.ts_mx_project(packed, 16, plain)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    with torch.no_grad(), pytest.raises(ValueError, match="not on a GPU"):
        ops.ts_mx_quantize(x)


def test_a_library_on_another_hip_runtime_than_torch_is_refused(lib):
    code = "from paper_2604_13519_amd import binding as B\nB.load_library()\nfrom paper_2604_13519_amd import ops\ntry: ops.ts_mx_packed_bytes(16, 128)\nexcept RuntimeError as e: print(e)"
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    with open("/proc/self/maps") as maps:                  # here torch came first: one runtime
        assert len({line.split()[-1] for line in maps if "libamdhip64" in line}) == 1
    assert r.returncode == 0 and "before torch" in r.stdout, (r.stdout, r.stderr)


@pytest.mark.parametrize("cls,pack", [(ops.ts_kv_append_args, ops._pack_append), (ops.ts_kv_attend_args, ops._pack_attend)])
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
