"""The paged calls on the host: where a row lies, and every call that is refused before anything is launched."""
import ctypes as C
import os
import subprocess

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
X = 1 << 20  # a 16-byte aligned address that nobody reads
PAGES = dict(has=1, k=X, v=X, layer=0, page_stride=16 * 2 * 128, token=2 * 128, head=128, n_pages=8, page=16, hkv=2, d=128, dtype=P.BF16, ks=None, vs=None,
             n_req=3, max_pages=4, table_stride=4, table=X, lens=X)


def pages(**over):
    return tuple({**PAGES, **over}.values())


def refused(status, native, *args):
    assert native(*args) == status
    buf = C.create_string_buffer(512)
    P._lib.purekv_last_error(buf, 512)
    assert buf.value.startswith(b"purekv_")


def append(rope=P._NO_ROPE, cu=X, tokens=5, h=4, hkv=2, d=128, dtype=P.BF16, q=(X, 512, 128), k=(X, 256, 128), v=(X, 256, 128), q_out=X, k_out=None, pg=None):
    return (*q, *k, *v, q_out, k_out, *(pages() if pg is None else pg), *rope, cu, tokens, h, hkv, d, dtype, X, None)


ROPE = dict(pos=X, stride=5, freq=X, rot=128, axes=1, s0=64, s1=0, s2=0, s3=0, inter=0)


def rope(**over):
    return tuple({**ROPE, **over}.values())


BAD_PAGES = [
    (P.ERR_INVALID_ARG, dict(n_req=-1)), (P.ERR_INVALID_ARG, dict(max_pages=-1)), (P.ERR_INVALID_ARG, dict(n_pages=-1)), (P.ERR_INVALID_ARG, dict(page=0)),
    (P.ERR_INVALID_ARG, dict(dtype=3)), (P.ERR_UNSUPPORTED, dict(dtype=P.FP32)), (P.ERR_INVALID_ARG, dict(ks=X)), (P.ERR_INVALID_ARG, dict(vs=X)),
    (P.ERR_INVALID_ARG, dict(table=None)), (P.ERR_INVALID_ARG, dict(lens=None)), (P.ERR_INVALID_ARG, dict(table_stride=3)),
    (P.ERR_INVALID_ARG, dict(k=None)), (P.ERR_INVALID_ARG, dict(v=X + 8)), (P.ERR_INVALID_ARG, dict(page_stride=4)), (P.ERR_INVALID_ARG, dict(token=-256)),
    (P.ERR_INVALID_ARG, dict(head=132)), (P.ERR_INVALID_ARG, dict(head=0)),
]


@pytest.mark.parametrize("status,over", BAD_PAGES)
def test_descriptions_of_a_cache_that_are_refused(status, over):
    refused(status, P._marshal.purekv_append_paged, *append(pg=pages(**over)))
    refused(status, P._marshal.purekv_compact_paged, X, X, 5 * 256, 1, X, X, 5, X, 5, P.BF16, *pages(**over), X, None)
    refused(status, P._marshal.purekv_decode_paged, X, 512, 128, X, None, *pages(**over), 0, 4, P.BF16, 0.0, None, 0, X, None)


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_INVALID_ARG, dict(dtype=7)), (P.ERR_INVALID_ARG, dict(tokens=-1)), (P.ERR_UNSUPPORTED, dict(dtype=P.FP32)),
    (P.ERR_UNSUPPORTED, dict(d=120, pg=pages(d=120))), (P.ERR_UNSUPPORTED, dict(d=528, pg=pages(d=528, head=528, token=1056, page_stride=16896))),
    (P.ERR_INVALID_ARG, dict(hkv=4)), (P.ERR_INVALID_ARG, dict(d=64)), (P.ERR_INVALID_ARG, dict(cu=None)),  # 5 tokens of 3 requests
    (P.ERR_INVALID_ARG, dict(q_out=None)), (P.ERR_INVALID_ARG, dict(q=(None, 0, 0))), (P.ERR_INVALID_ARG, dict(k=(None, 0, 0))), (P.ERR_INVALID_ARG, dict(v=(None, 0, 0))),
    (P.ERR_INVALID_ARG, dict(pg=P._NO_PAGES)), (P.ERR_INVALID_ARG, dict(h=0)), (P.ERR_INVALID_ARG, dict(q=(X + 4, 512, 128))), (P.ERR_INVALID_ARG, dict(k=(X, 260, 128))),
    (P.ERR_INVALID_ARG, dict(v=(X, 256, 132))), (P.ERR_INVALID_ARG, dict(k=(X, -256, 128))), (P.ERR_INVALID_ARG, dict(k_out=X + 2)),
    (P.ERR_INVALID_ARG, dict(rope=rope(freq=None))), (P.ERR_INVALID_ARG, dict(rope=rope(freq=X + 4))), (P.ERR_UNSUPPORTED, dict(rope=rope(rot=24, s0=12))),
    (P.ERR_UNSUPPORTED, dict(rope=rope(rot=256, s0=128))), (P.ERR_UNSUPPORTED, dict(rope=rope(rot=0, s0=0))), (P.ERR_INVALID_ARG, dict(rope=rope(axes=0))),
    (P.ERR_INVALID_ARG, dict(rope=rope(axes=5))), (P.ERR_INVALID_ARG, dict(rope=rope(s0=63))), (P.ERR_INVALID_ARG, dict(rope=rope(axes=2, s0=65, s1=-1))),
    (P.ERR_INVALID_ARG, dict(rope=rope(axes=2, s0=32, s1=32, stride=4))),
])
def test_appends_that_are_refused(status, over):
    refused(status, P._marshal.purekv_append_paged, *append(**over))


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(k=None)), (P.ERR_INVALID_ARG, dict(idx=None)), (P.ERR_INVALID_ARG, dict(cu=None)), (P.ERR_INVALID_ARG, dict(ck=None)),
    (P.ERR_INVALID_ARG, dict(layers=-1)), (P.ERR_INVALID_ARG, dict(k_tot=-1)), (P.ERR_INVALID_ARG, dict(tokens=-1)), (P.ERR_INVALID_ARG, dict(tokens=2 ** 31)),
    (P.ERR_INVALID_ARG, dict(layers=2, stride=5 * 256 - 8)), (P.ERR_INVALID_ARG, dict(layers=2, stride=5 * 256 + 4)), (P.ERR_INVALID_ARG, dict(v=X + 8)),
    (P.ERR_INVALID_ARG, dict(layers=2)), (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_UNSUPPORTED, dict(k_tot=2 ** 31 - 1)),
])
def test_compactions_that_are_refused(status, over):
    a = {**dict(k=X, v=X, stride=5 * 256, layers=1, idx=X, cu=X, tokens=5, ck=X, k_tot=5, dtype=P.BF16), **over}
    refused(status, P._marshal.purekv_compact_paged, *a.values(), *pages(), X, None)


@pytest.mark.parametrize("status,over", [
    (P.ERR_INVALID_ARG, dict(q=None)), (P.ERR_INVALID_ARG, dict(o=None)), (P.ERR_INVALID_ARG, dict(h=5)), (P.ERR_INVALID_ARG, dict(h=0)), (P.ERR_INVALID_ARG, dict(max_len=-1)),
    (P.ERR_INVALID_ARG, dict(dtype=P.E4M3)), (P.ERR_INVALID_ARG, dict(q=X + 8)), (P.ERR_INVALID_ARG, dict(tok=516)), (P.ERR_INVALID_ARG, dict(head=-128)),
    (P.ERR_UNSUPPORTED, dict(pg=pages(d=32, head=32, token=64, page_stride=1024))), (P.ERR_UNSUPPORTED, dict(pg=pages(n_req=70000))),
])
def test_decodes_that_are_refused(status, over):
    a = {**dict(q=X, tok=512, head=128, o=X, lse=None, pg=pages(), max_len=0, h=4, dtype=P.BF16), **over}
    refused(status, P._marshal.purekv_decode_paged, a["q"], a["tok"], a["head"], a["o"], a["lse"], *a["pg"], a["max_len"], a["h"], a["dtype"], 0.0, None, 0, X, None)


def test_nothing_to_do_is_fine():
    ok = lambda native, *args: native(*args) == P.OK
    assert ok(P._marshal.purekv_append_paged, *append(tokens=0))
    assert ok(P._marshal.purekv_append_paged, *append(q=(None, 0, 0), q_out=None, k=(None, 0, 0), v=(None, 0, 0), pg=P._NO_PAGES))
    assert ok(P._marshal.purekv_compact_paged, None, None, 0, 0, None, None, 0, None, 0, P.BF16, *pages(), X, None)
    assert ok(P._marshal.purekv_decode_paged, None, 0, 0, None, None, *pages(n_req=0, table=None, lens=None, k=None, v=None), 0, 4, P.BF16, 0.0, None, 0, X, None)


def test_the_binding_wants_tensors_on_one_gpu():
    k = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    pool = torch.zeros((4, 16, 2, 128), dtype=torch.bfloat16)
    table, lens = torch.zeros((2, 2), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for call in (lambda: P.purekv_append_paged(k, k, pool, pool, table, lens), lambda: P.purekv_decode_paged(k, pool, pool, table, lens),
                 lambda: P.purekv_compact_paged(k[None], k[None], torch.zeros((1, 2, 2), dtype=torch.int32), type("B", (), dict(cu_seqlens=lens)),
                                                type("B", (), dict(cu_kept=lens)), pool[None], pool[None], table, lens)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.purekv_append_paged(None, None, None, None, None, None)


class OnGpu:
    """Stands in for the device check, so that the checks of shapes behind it can be seen without a GPU."""

    def __enter__(self):
        self.kept, P._same_device = P._same_device, lambda *t: 0

    def __exit__(self, *_):
        P._same_device = self.kept


@pytest.mark.parametrize("over", [
    dict(v_pages=torch.zeros((4, 16, 2, 128))), dict(v_pages=torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16).transpose(1, 2)), dict(seq_lens=torch.ones(2)),
    dict(seq_lens=torch.ones(3, dtype=torch.int32)), dict(block_table=torch.zeros((2, 2), dtype=torch.int64)), dict(block_table=torch.zeros((3, 2), dtype=torch.int32)),
    dict(block_table=torch.zeros((2, 4), dtype=torch.int32)[:, ::2]), dict(q=torch.zeros((2, 4, 128))), dict(q=torch.zeros((2, 4, 64), dtype=torch.bfloat16)),
    dict(q=torch.zeros((2, 4, 256), dtype=torch.bfloat16)[:, :, ::2]), dict(out=torch.zeros((2, 4, 128))), dict(lse=torch.zeros((2, 4), dtype=torch.float64)),
    dict(lse=torch.zeros((4, 2))), dict(k_pages=torch.zeros((4, 16, 256), dtype=torch.bfloat16)), dict(k_scale=torch.ones(4)), dict(k_scale=torch.ones(2).double()),
])
def test_shapes_that_the_binding_refuses(over):
    pool = torch.zeros((4, 16, 2, 128), dtype=torch.bfloat16)
    a = {**dict(q=torch.zeros((2, 4, 128), dtype=torch.bfloat16), k_pages=pool, v_pages=pool, block_table=torch.zeros((2, 2), dtype=torch.int32),
                seq_lens=torch.ones(2, dtype=torch.int32)), **over}
    if "q" in over and over["q"].dtype is torch.float32:
        a["out"] = torch.zeros((2, 4, 128), dtype=torch.bfloat16)
    with OnGpu(), pytest.raises(ValueError):
        P.purekv_decode_paged(**a)


@pytest.mark.parametrize("over", [
    dict(v=None), dict(v=torch.zeros((5, 2, 64), dtype=torch.bfloat16)), dict(cu_new=torch.zeros(4, dtype=torch.int32)), dict(cu_new=torch.zeros(3, dtype=torch.int64)),
    dict(positions=torch.zeros(4, dtype=torch.int32), inv_freq=torch.ones(64).double()), dict(positions=torch.zeros(5), inv_freq=torch.ones(64).double()),
    dict(positions=torch.zeros(5, dtype=torch.int32), inv_freq=torch.ones(64)), dict(positions=torch.zeros((2, 5), dtype=torch.int32), inv_freq=torch.ones(64).double()),
    dict(positions=torch.zeros((2, 5), dtype=torch.int32), inv_freq=torch.ones(64).double(), sections=(32, 16, 16)), dict(q=torch.zeros((4, 4, 128), dtype=torch.bfloat16)),
    dict(q=torch.zeros((5, 4, 128), dtype=torch.bfloat16), q_out=torch.zeros((5, 8, 128), dtype=torch.bfloat16)[:, ::2]), dict(k_out=torch.zeros((5, 2, 128))),
])
def test_appends_that_the_binding_refuses(over):
    pool, new = torch.zeros((4, 16, 2, 128), dtype=torch.bfloat16), torch.zeros((5, 2, 128), dtype=torch.bfloat16)
    a = {**dict(k=new, v=new, k_pages=pool, v_pages=pool, block_table=torch.zeros((2, 2), dtype=torch.int32), seq_lens=torch.ones(2, dtype=torch.int32),
                cu_new=torch.zeros(3, dtype=torch.int32)), **over}
    with OnGpu(), pytest.raises(ValueError):
        P.purekv_append_paged(**a)
