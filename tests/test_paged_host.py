"""The paged calls on the host: where a row lies, and every call that is refused before anything is launched."""
import ctypes as C
import os
import subprocess
import types

import pytest
import torch

import paper_2510_25600_b200
from paper_2510_25600_b200 import binding as P

CSRC = os.path.join(os.path.dirname(paper_2510_25600_b200.__file__), "csrc")
MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include "paged.cuh"
using namespace purekv;
int main(int n, char** v) {
  if (!strcmp(v[1], "div")) {  // every divisor up to a limit, quotients around its multiples and at the ends of the range
    for (int64_t d = 1; d <= 70000; d = d < 300 ? d + 1 : d + d / 37 + 1) {
      const FastDiv f = FastDiv::of((int32_t)d);
      auto check = [&](int64_t x) { if (x >= 0 && x <= INT32_MAX && f.quotient((uint32_t)x) != (uint32_t)(x / d)) { printf("%lld / %lld\n", (long long)x, (long long)d); exit(1); } };
      for (int64_t m = 0; m < 2000; ++m) for (int e = -1; e <= 1; ++e) { check(m * d + e); check(INT32_MAX / d * d - m * d + e); }
      for (uint32_t x = 1, i = 0; i < 2000; ++i) { x = x * 1664525u + 1013904223u; check(x >> 1); }
      check(INT32_MAX);
    }
    for (int64_t d = 1; d <= INT32_MAX; d = 2 * d + (d & 1)) { const FastDiv f = FastDiv::of((int32_t)d); if (f.quotient(INT32_MAX) != INT32_MAX / d || f.quotient((uint32_t)d - 1) != 0 || f.quotient((uint32_t)d) != 1) { printf("%lld\n", (long long)d); exit(1); } }
    puts("ok");
  } else if (!strcmp(v[1], "row")) {  // row, page size, pages of the pool, pages of the list, the list
    PagedView p = {};
    p.page_stride = 1000003; p.token_stride = 101;
    p.page_size = FastDiv::of(atoi(v[3])); p.n_pages = atoi(v[4]); p.max_pages = atoi(v[5]);
    int32_t list[16];
    for (int i = 6; i < n; ++i) list[i - 6] = atoi(v[i]);
    printf("%lld", (long long)p.row_offset(list, atoi(v[2])));
  } else {  // request: t, then the offsets
    int32_t cu[16];
    for (int i = 3; i < n; ++i) cu[i - 3] = atoi(v[i]);
    printf("%d", request_of(cu, n - 4, atoi(v[2])));
  }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    (d / "main.cpp").write_text(MAIN)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=address,undefined", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "main")], check=True)
    return lambda *a: subprocess.check_output([str(d / "main"), *map(str, a)]).decode().strip()


def test_division(program):
    assert program("div") == "ok"


@pytest.mark.parametrize("row,page,n_pages,table,want", [
    (0, 16, 9, [4, 2], 4 * 1000003), (15, 16, 9, [4, 2], 4 * 1000003 + 15 * 101), (16, 16, 9, [4, 2], 2 * 1000003), (31, 16, 9, [4, 2], 2 * 1000003 + 15 * 101),
    (32, 16, 9, [4, 2], -1), (-1, 16, 9, [4, 2], -1), (2 ** 31 - 1, 16, 9, [4, 2], -1),          # outside the list
    (0, 16, 9, [9], -1), (0, 16, 9, [-1], -1), (0, 16, 9, [2 ** 31 - 1], -1), (0, 16, 0, [0], -1), (0, 16, 9, [], -1),  # no such page
    (13, 7, 9, [0, 8], 8 * 1000003 + 6 * 101), (5, 1, 9, [0, 1, 2, 3, 4, 7], 7 * 1000003),
    (2 ** 31 - 2, 2 ** 31 - 1, 3, [2], 2 * 1000003 + (2 ** 31 - 2) * 101),
    (2 ** 31 - 1, 2 ** 31 - 1, 3, [2, 1], -1),            # a list that could hold more rows than 32 bits count
    (5, 1, 10000, [0, 1, 2, 3, 4, 9000], 9000 * 1000003),  # an offset past 32 bits
])
def test_where_a_row_lies(program, row, page, n_pages, table, want):
    assert int(program("row", row, page, n_pages, len(table), *table)) == want


@pytest.mark.parametrize("t,cu,want", [(0, [0, 3], 0), (2, [0, 3, 3, 7], 0), (3, [0, 3, 3, 7], 2), (6, [0, 3, 3, 7], 2), (9, [0, 3, 3, 7], 2), (0, [0, 0, 0, 1], 2)])
def test_whose_token(program, t, cu, want):
    assert int(program("request", t, *cu)) == want


# ---- refusals of the C calls: addresses are made up, nothing may be launched -----------------------------------------------
class Pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("layer_stride", C.c_int64), ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p), ("n_req", C.c_int32), ("max_pages", C.c_int32), ("table_stride", C.c_int64), ("block_table", C.c_void_p), ("seq_lens", C.c_void_p)]


class Rope(C.Structure):
    _fields_ = [("positions", C.c_void_p), ("axis_stride", C.c_int64), ("inv_freq", C.c_void_p), ("rotary_dim", C.c_int32), ("n_axes", C.c_int32),
                ("sections", C.c_int32 * 4), ("interleaved", C.c_int32)]


X = 1 << 20  # a 16-byte aligned address that nobody reads
_p, _i, _l = C.c_void_p, C.c_int32, C.c_int64
APPEND = [_p, _l, _l] * 3 + [_p, _p, C.POINTER(Pages), C.POINTER(Rope), _p, _i, _i, _i, _i, C.c_int, _p, _p]
COMPACT = [_p, _p, _l, _i, _p, _p, _l, _p, _i, C.c_int, C.POINTER(Pages), _p, _p]
DECODE = [_p, _l, _l, _p, _p, C.POINTER(Pages), _i, _i, C.c_int, C.c_float, _p, C.c_size_t, _p, _p]


def native(name, types, args):
    f = getattr(C.CDLL(P.LIB_PATH), name)
    f.argtypes = types
    return f(*args)


def append(**over):
    a = {**dict(q=X, q_tok=512, q_head=128, k=X, k_tok=256, k_head=128, v=X, v_tok=256, v_head=128, q_out=X, k_out=None, pages=pages(), rope=None, cu=X, tokens=5, h=4,
                hkv=2, d=128, dtype=P.BF16, status=X, stream=None), **over}
    return "purekv_append_paged", APPEND, list(a.values())


def compact(**over):
    a = {**dict(k=X, v=X, stride=5 * 256, layers=1, idx=X, cu=X, tokens=5, ck=X, k_tot=5, dtype=P.BF16, pages=pages(), status=X, stream=None), **over}
    return "purekv_compact_paged", COMPACT, list(a.values())


def decode(**over):
    a = {**dict(q=X, tok=512, head=128, o=X, lse=None, pages=pages(), max_len=0, h=4, dtype=P.BF16, scale=0.0, ws=None, ws_bytes=0, status=X, stream=None), **over}
    return "purekv_decode_paged", DECODE, list(a.values())


def pages(**over):
    a = {**dict(k=X, v=X, layer_stride=0, page_stride=16 * 2 * 128, token_stride=2 * 128, head_stride=128, n_pages=8, page_size=16, n_kv_heads=2, head_dim=128, dtype=P.BF16,
                k_scale=None, v_scale=None, n_req=3, max_pages=4, table_stride=4, block_table=X, seq_lens=X), **over}
    return Pages(*a.values())


def rope(sections=(64,), **over):
    a = {**dict(positions=X, axis_stride=5, inv_freq=X, rotary_dim=128, n_axes=len(sections)), **over}
    return Rope(*a.values(), (C.c_int32 * 4)(*sections[:4]), 0)


def refused(status, call):
    assert native(*call) == status
    buf = C.create_string_buffer(512)
    P._lib.purekv_last_error(buf, 512)
    assert buf.value.startswith(call[0].encode())


BAD_PAGES = [
    (P.ERR_INVALID_ARG, dict(n_req=-1)), (P.ERR_INVALID_ARG, dict(max_pages=-1)), (P.ERR_INVALID_ARG, dict(n_pages=-1)), (P.ERR_INVALID_ARG, dict(page_size=0)),
    (P.ERR_INVALID_ARG, dict(dtype=3)), (P.ERR_UNSUPPORTED, dict(dtype=P.FP32)), (P.ERR_INVALID_ARG, dict(k_scale=X)), (P.ERR_INVALID_ARG, dict(v_scale=X)),
    (P.ERR_INVALID_ARG, dict(block_table=None)), (P.ERR_INVALID_ARG, dict(seq_lens=None)), (P.ERR_INVALID_ARG, dict(table_stride=3)),
    (P.ERR_INVALID_ARG, dict(k=None)), (P.ERR_INVALID_ARG, dict(v=X + 8)), (P.ERR_INVALID_ARG, dict(page_stride=4)), (P.ERR_INVALID_ARG, dict(token_stride=-256)),
    (P.ERR_INVALID_ARG, dict(head_stride=132)), (P.ERR_INVALID_ARG, dict(head_stride=0)),
]


@pytest.mark.parametrize("status,over", BAD_PAGES)
@pytest.mark.parametrize("call", [append, compact, decode])
def test_descriptions_of_a_cache_that_are_refused(call, status, over):
    refused(status, call(pages=pages(**over)))


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_INVALID_ARG, dict(dtype=7)), (P.ERR_INVALID_ARG, dict(tokens=-1)), (P.ERR_UNSUPPORTED, dict(dtype=P.FP32)),
    (P.ERR_UNSUPPORTED, dict(d=120, pages=pages(head_dim=120))), (P.ERR_UNSUPPORTED, dict(d=528, pages=pages(head_dim=528, head_stride=528, token_stride=1056, page_stride=16896))),
    (P.ERR_INVALID_ARG, dict(hkv=4)), (P.ERR_INVALID_ARG, dict(d=64)), (P.ERR_INVALID_ARG, dict(cu=None)),  # 5 tokens of 3 requests
    (P.ERR_INVALID_ARG, dict(q_out=None)), (P.ERR_INVALID_ARG, dict(q=None)), (P.ERR_INVALID_ARG, dict(k=None)), (P.ERR_INVALID_ARG, dict(v=None)),
    (P.ERR_INVALID_ARG, dict(pages=None)), (P.ERR_INVALID_ARG, dict(h=0)), (P.ERR_INVALID_ARG, dict(q=X + 4)), (P.ERR_INVALID_ARG, dict(k_tok=260)),
    (P.ERR_INVALID_ARG, dict(v_head=132)), (P.ERR_INVALID_ARG, dict(k_tok=-256)), (P.ERR_INVALID_ARG, dict(pages=None, v=None, k_out=X + 2)),
    (P.ERR_INVALID_ARG, dict(rope=rope(inv_freq=None))), (P.ERR_INVALID_ARG, dict(rope=rope(inv_freq=X + 4))), (P.ERR_UNSUPPORTED, dict(rope=rope((12,), rotary_dim=24))),
    (P.ERR_UNSUPPORTED, dict(rope=rope((128,), rotary_dim=256))), (P.ERR_UNSUPPORTED, dict(rope=rope((0,), rotary_dim=0))), (P.ERR_INVALID_ARG, dict(rope=rope(n_axes=0))),
    (P.ERR_INVALID_ARG, dict(rope=rope((16, 16, 16, 16), n_axes=5))), (P.ERR_INVALID_ARG, dict(rope=rope((63,)))), (P.ERR_INVALID_ARG, dict(rope=rope((65, -1)))),
    (P.ERR_INVALID_ARG, dict(rope=rope((32, 32), axis_stride=4))),
])
def test_appends_that_are_refused(status, over):
    refused(status, append(**over))


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(k=None)), (P.ERR_INVALID_ARG, dict(idx=None)), (P.ERR_INVALID_ARG, dict(cu=None)), (P.ERR_INVALID_ARG, dict(ck=None)),
    (P.ERR_INVALID_ARG, dict(layers=-1)), (P.ERR_INVALID_ARG, dict(k_tot=-1)), (P.ERR_INVALID_ARG, dict(tokens=-1)), (P.ERR_INVALID_ARG, dict(tokens=2 ** 31)),
    (P.ERR_INVALID_ARG, dict(layers=2, stride=5 * 256 - 8)), (P.ERR_INVALID_ARG, dict(layers=2, stride=5 * 256 + 4)), (P.ERR_INVALID_ARG, dict(v=X + 8)),
    (P.ERR_INVALID_ARG, dict(layers=2)), (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_UNSUPPORTED, dict(k_tot=2 ** 31 - 1)), (P.ERR_INVALID_ARG, dict(pages=None)),
])
def test_compactions_that_are_refused(status, over):
    refused(status, compact(**over))


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(q=None)), (P.ERR_INVALID_ARG, dict(o=None)), (P.ERR_INVALID_ARG, dict(h=5)), (P.ERR_INVALID_ARG, dict(h=0)), (P.ERR_INVALID_ARG, dict(max_len=-1)),
    (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_INVALID_ARG, dict(q=X + 8)), (P.ERR_INVALID_ARG, dict(tok=516)), (P.ERR_INVALID_ARG, dict(head=-128)),
    (P.ERR_UNSUPPORTED, dict(pages=pages(head_dim=32, head_stride=32, token_stride=64, page_stride=1024))), (P.ERR_UNSUPPORTED, dict(pages=pages(n_req=70000))),
    (P.ERR_INVALID_ARG, dict(pages=None)), (P.ERR_WORKSPACE, dict(max_len=1 << 20)), (P.ERR_WORKSPACE, dict(max_len=1 << 20, ws=X, ws_bytes=1000)),
])
def test_decodes_that_are_refused(status, over):
    refused(status, decode(**over))


def test_nothing_to_do_is_fine():
    assert native(*append(tokens=0)) == P.OK
    assert native(*append(q=None, q_out=None, k=None, v=None, pages=None)) == P.OK
    assert native(*compact(k=None, v=None, idx=None, cu=None, ck=None, k_tot=0)) == P.OK
    assert native(*decode(q=None, o=None, pages=pages(n_req=0, block_table=None, seq_lens=None, k=None, v=None))) == P.OK


# ---- refusals of the binding ------------------------------------------------------------------------------------------------
ON_GPU = "take tensors on a GPU"  # what a call on the CPU is refused for when nothing else is wrong with it
bf16 = dict(dtype=torch.bfloat16)


def decode_args(**over):
    pool = torch.zeros((4, 16, 2, 128), **bf16)
    return {**dict(q=torch.zeros((2, 4, 128), **bf16), k_pages=pool, v_pages=pool, block_table=torch.zeros((2, 2), dtype=torch.int32),
                   seq_lens=torch.ones(2, dtype=torch.int32)), **over}


def append_args(**over):
    pool, new = torch.zeros((4, 16, 2, 128), **bf16), torch.zeros((5, 2, 128), **bf16)
    return {**dict(k=new, v=new, k_pages=pool, v_pages=pool, block_table=torch.zeros((2, 2), dtype=torch.int32), seq_lens=torch.ones(2, dtype=torch.int32),
                   cu_new=torch.zeros(3, dtype=torch.int32)), **over}


def compact_args(**over):
    pool, k = torch.zeros((3, 4, 16, 2, 128), **bf16), torch.zeros((3, 9, 2, 128), **bf16)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)
    a = {**dict(k=k, v=k, idx=i32(3, 2, 4), cu=i32(3), ck=i32(3), k_pages=pool, v_pages=pool, block_table=i32(2, 2), seq_lens=i32(2)), **over}
    return {**{n: x for n, x in a.items() if n not in ("cu", "ck")}, "batch": types.SimpleNamespace(cu_seqlens=a["cu"]), "budget": types.SimpleNamespace(cu_kept=a["ck"])}


@pytest.mark.parametrize("call,args", [(P.purekv_decode_paged, decode_args), (P.purekv_append_paged, append_args), (P.purekv_compact_paged, compact_args)])
def test_the_binding_wants_tensors_on_a_gpu(call, args):
    with pytest.raises(ValueError, match=ON_GPU):
        call(**args())


def refused_by_the_binding(call, args):
    with pytest.raises(ValueError) as e:
        call(**args)
    assert ON_GPU not in str(e.value)


@pytest.mark.parametrize("over", [
    dict(v_pages=torch.zeros((4, 16, 2, 128))), dict(v_pages=torch.zeros((4, 2, 16, 128), **bf16).transpose(1, 2)), dict(seq_lens=torch.ones(2)),
    dict(seq_lens=torch.ones(3, dtype=torch.int32)), dict(block_table=torch.zeros((2, 2), dtype=torch.int64)), dict(block_table=torch.zeros((3, 2), dtype=torch.int32)),
    dict(block_table=torch.zeros((2, 4), dtype=torch.int32)[:, ::2]), dict(block_table=torch.zeros(2, dtype=torch.int32)), dict(q=torch.zeros((2, 4, 64), **bf16)),
    dict(q=torch.zeros((3, 4, 128), **bf16)), dict(q=torch.zeros((2, 4, 128), dtype=torch.float16)), dict(q=torch.zeros((2, 4, 256), **bf16)[:, :, ::2]),
    dict(out=torch.zeros((2, 4, 128))), dict(out=torch.zeros((2, 8, 128), **bf16)[:, ::2]), dict(lse=torch.zeros((2, 4), dtype=torch.float64)), dict(lse=torch.zeros((4, 2))),
    dict(k_pages=torch.zeros((4, 16, 256), **bf16)), dict(k_scale=torch.ones(4)), dict(v_scale=torch.ones(2).double()), dict(status=torch.zeros(2, dtype=torch.int32)),
    dict(ws=torch.zeros(64)[::2]), dict(k_pages=None), dict(seq_lens=None), dict(max_len=2 ** 31),
])
def test_decodes_that_the_binding_refuses(over):
    args = decode_args(**over)
    if over.get("k_pages", 0) is None:
        args["ws"] = torch.zeros(64)
    refused_by_the_binding(P.purekv_decode_paged, args)


@pytest.mark.parametrize("over", [
    dict(v=None), dict(v=torch.zeros((5, 2, 64), **bf16)), dict(v=torch.zeros((5, 2, 128))), dict(cu_new=torch.zeros(4, dtype=torch.int32)),
    dict(cu_new=torch.zeros(3, dtype=torch.int64)), dict(k=None), dict(block_table=None), dict(v_pages=None),
    dict(positions=torch.zeros(5, dtype=torch.int32)),
    dict(positions=torch.zeros(4, dtype=torch.int32), inv_freq=torch.ones(64).double()), dict(positions=torch.zeros(5), inv_freq=torch.ones(64).double()),
    dict(positions=torch.zeros(5, dtype=torch.int32), inv_freq=torch.ones(64)), dict(positions=torch.zeros((2, 5), dtype=torch.int32), inv_freq=torch.ones(64).double()),
    dict(positions=torch.zeros((2, 5), dtype=torch.int32), inv_freq=torch.ones(64).double(), sections=(32, 16, 16)),
    dict(positions=torch.zeros((5, 5), dtype=torch.int32), inv_freq=torch.ones(64).double(), sections=(16, 16, 16, 8, 8)),
    dict(positions=torch.zeros((2, 5), dtype=torch.int32), inv_freq=torch.ones(64).double(), sections=(65, -1)),
    dict(positions=torch.zeros((5, 2), dtype=torch.int32).T, inv_freq=torch.ones(64).double(), sections=(32, 32)),
    dict(q=torch.zeros((4, 4, 128), **bf16)), dict(q=torch.zeros((5, 4, 128))), dict(q=torch.zeros((5, 4, 128), **bf16), q_out=torch.zeros((5, 8, 128), **bf16)[:, ::2]),
    dict(q_out=torch.zeros((5, 4, 128), **bf16)), dict(k_out=torch.zeros((5, 2, 128))), dict(k_out=torch.zeros((5, 2, 64), **bf16)),
])
def test_appends_that_the_binding_refuses(over):
    refused_by_the_binding(P.purekv_append_paged, append_args(**over))


def test_an_append_of_nothing_is_refused():
    refused_by_the_binding(P.purekv_append_paged, {n: None for n in append_args()})


@pytest.mark.parametrize("over", [
    dict(k=torch.zeros((9, 2, 128), **bf16)), dict(v=torch.zeros((3, 9, 2, 64), **bf16)), dict(v=torch.zeros((3, 9, 2, 128))), dict(k=torch.zeros((3, 2, 9, 128), **bf16).transpose(1, 2)),
    dict(idx=torch.zeros((3, 1, 4), dtype=torch.int32)), dict(idx=torch.zeros((3, 2, 4), dtype=torch.int64)), dict(idx=torch.zeros((2, 4), dtype=torch.int32)),
    dict(idx=torch.zeros((3, 2, 8), dtype=torch.int32)[:, :, ::2]), dict(cu=torch.zeros(2, dtype=torch.int32)), dict(ck=torch.zeros(4, dtype=torch.int32)),
    dict(k_pages=torch.zeros((4, 16, 2, 128), **bf16)), dict(k_pages=torch.zeros((2, 4, 16, 2, 128), **bf16)), dict(k_scale=torch.ones(2)),
])
def test_compactions_that_the_binding_refuses(over):
    refused_by_the_binding(P.purekv_compact_paged, compact_args(**over))


def test_heads_of_another_size_are_refused():
    pool = torch.zeros((3, 4, 16, 2, 64), **bf16)
    refused_by_the_binding(P.purekv_compact_paged, compact_args(k_pages=pool, v_pages=pool))


def test_what_is_no_tensor_is_refused():
    with pytest.raises(TypeError):
        P.purekv_decode_paged(**decode_args(lse=3))
