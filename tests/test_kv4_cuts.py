"""How attention over 4-bit cached keys and values is cut into workgroups: the
host's choice (no GPU) for the sizes that the GPU tests below run."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_32420_amd as P
from paper_2609_32420_amd import build as B
from test_gpu_kv4 import DEV, _bf16, _check_attn, _filled, _tables

CSRC = os.path.join(os.path.dirname(P.__file__), "csrc")
INCLUDE = os.path.join(B.ROOT, "include")

PROBE = r"""
#include "kv4_cut.h"
#include <stdio.h>
using namespace carnator;
int main() {
  long long d, kv_heads, heads, rows, batch, width, block, max_q, causal;
  while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld", &d, &kv_heads, &heads, &rows, &batch, &width, &block,
               &max_q, &causal) == 9) {
    Kv4Attn a{};
    a.c = Kv4{nullptr, 1 << 20, (int)kv_heads, (int)d, block == 64 ? 6 : 7};
    a.heads = (int)heads, a.group = (int)(heads / kv_heads), a.n_rows = (int)rows, a.batch = (int)batch;
    a.width = (int)width, a.max_q = (int)(max_q < rows ? max_q : rows), a.causal = (int)causal;
    const auto [few, many] = cuts(a);
    printf("tile_rows %d few_chunks %d few_columns %d many_tiles %d many_chunks %d turns %d items %d few_bytes %zu many_bytes %zu "
           "groups %lld threads %lld\n", many.tile_rows, few.chunks, few.columns, many.tiles, many.chunks, many.turns, many.items,
           parts_bytes(a, few), parts_bytes(a, many), (long long)(few_groups(a, few) + tile_groups(a, many)),
           (long long)most_threads(a, cuts(a)));
  }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    """cut(d, kv_heads, group, m, width, block, causal, rows, max_q): the choice as a dict."""
    at = tmp_path_factory.mktemp("cut")
    src, exe = str(at / "cut.hip"), str(at / "cut")
    with open(src, "w") as f:
        f.write(PROBE)
    subprocess.run([B.HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", CSRC, "-I", INCLUDE, src, "-o", exe],
                   check=True, capture_output=True)

    def run(d, kv_heads, group, m, width, block=64, causal=True, rows=None, max_q=None):
        sizes = (d, kv_heads, kv_heads * group, rows or sum(m), len(m), width, block, max_q or max(m), int(causal))
        words = subprocess.run([exe], input=" ".join(map(str, sizes)), capture_output=True, text=True, check=True).stdout.split()
        return dict(zip(words[::2], map(int, words[1::2])))

    return run


# d = 128 with tiles of 256 rows and requests of few rows in their grid: queries,
# cached tokens, cached heads, heads to each, table's width, causal; tiles found
# by number, the few rows' axis in parts, the tiles' axis in parts
MIXED = [
    ([700, 2, 700, 31], [4000, 3900, 2000, 4096], 2, 3, 64, False, True, True, True),
    ([900, 5, 900], [2900, 2941, 901], 2, 3, 46, True, True, True, True),
    ([600, 600, 3, 600], [2900, 600, 3001, 0], 2, 3, 52, True, False, True, True),
    ([1000, 600, 3, 1000], [2000, 700, 1999, 1000], 30, 2, 32, True, True, False, False),
    ([600, 3, 1, 600, 0, 600, 9, 600, 600, 600, 600, 600], [900, 1000, 1, 600] + [601, 1024, 77] + [620] * 5, 30, 2, 16, False,
     False, False, False),
]


@pytest.mark.parametrize("case", range(len(MIXED)))
def test_large_tiles_with_few_rows_beside_them_are_chosen(cut, case):
    m, kv, kv_heads, group, width, causal, numbered, few_parts, many_parts = MIXED[case]
    c = cut(128, kv_heads, group, m, width, causal=causal, rows=sum(m) + 1)
    assert min(x * group for x in m if x) <= 32 and max(kv) <= 64 * width
    assert c["tile_rows"] == 256 and (c["items"] > 0) == numbered
    assert (c["few_chunks"] > 1) == few_parts and (c["many_chunks"] > 1) == many_parts


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(MIXED)))
def test_large_tiles_with_few_rows_beside_them(case):
    m, kv, kv_heads, group, width, causal = MIXED[case][:6]
    pages = sum(-(-n // 64) for n in kv) + 1
    pool = _filled(pages, kv_heads, 128, 64, case)
    start = [0] + np.cumsum(m).tolist()
    q = _bf16(start[-1] + 1, kv_heads * group, 128, seed=case + 3)
    _check_attn(q, pool, _tables(kv, 64, pages, case, width=width), start, kv, 64, causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch", [900, 1024, 1025, 2048, 4096, 16384])
def test_workgroups_of_a_ragged_batch_follow_its_tiles(cut, d, batch):
    # a prompt of 8192 beside single tokens, 32 / 8 heads, a table for 16,384
    m = [8192] + [1] * (batch - 1)
    c = cut(d, 8, 4, m, 256)
    # tiles of the rows that there are, a started one a request, the requests of few rows
    assert c["groups"] <= 8 * c["many_chunks"] * (4 * sum(m) // c["tile_rows"] + batch) + max(8 * batch, 8192)
    assert c["groups"] < 1 << 23


def _many_requests(batch):
    """Queries and cached tokens: the tiles lie in every 1024 requests, the longest prompt is the last."""
    rng = np.random.default_rng(batch)
    m = np.where(rng.random(batch) < 0.1, rng.integers(33, 180, batch), rng.integers(0, 3, batch))
    m[-1] = 700
    kv = np.where(rng.random(batch) < 0.2, 0, m + rng.integers(0, 60, batch))
    kv[-1] = 900
    return m.tolist(), kv.tolist()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("batch", [1100, 2048, 4100])
def test_tiles_of_many_requests_are_found_by_number(cut, d, causal, batch):
    m, kv = _many_requests(batch)
    assert cut(d, 3, 1, m, max(-(-n // 64) for n in kv), causal=causal, rows=sum(m) + 1)["items"] > 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,causal", [(1100, True), (1100, False), (2048, True), (4100, True)])
def test_attention_of_many_requests(d, batch, causal):
    m, kv = _many_requests(batch)
    pages = sum(-(-n // 64) for n in kv)
    pool = _filled(pages, 3, d, 64, 6)
    start = [0] + np.cumsum(m).tolist()
    _check_attn(_bf16(start[-1] + 1, 3, d, seed=d), pool, _tables(kv, 64, pages, 5), start, kv, 64, causal)


@pytest.mark.parametrize("d", [64, 128])
def test_parts_of_few_rows_follow_their_workgroups(cut, d):
    # at most 8192 workgroups write parts, each of 64 (d = 64) or 32 rows of d outputs
    # and 16 bytes beside them, whatever the table's width; one alone writes none
    most = 8192 * (64 * (64 * 4 + 16) if d == 64 else 32 * (128 * 4 + 16)) + 512
    for m, kv_heads, group, width in [
            ([1] * 1024, 8, 4, 2048), ([4] * 256, 8, 8, 2048), ([8192] + [1] * 1023, 8, 4, 256), ([8000] + [1] * 1499, 8, 4, 512),
            ([100000] + [1] * 60, 8, 4, 2048), ([100000] + [1] * 1023, 8, 4, 2048), ([1], 8, 4, 1 << 20), ([8] * 900, 1, 8, 1 << 20),
            ([32] * 100, 12, 1, 4096), ([64, 63] * 32, 8, 1, 4096), ([1] * 16384, 12, 2, 2048), ([1, 2, 1] * 341, 4, 8, 300)]:
        c = cut(d, kv_heads, group, m, width)
        assert c["few_bytes"] <= most, (m[:3], c)
        if len(m) * kv_heads > 4096:
            assert c["few_chunks"] == 1 and c["few_bytes"] == 0


IN_TURN = [(1, 1), (3, 1), (20, 1), (1, 9), (3, 9), (1, 30), (2, 7), (40, 1)]  # queries at most, heads to a cached one


def _in_turn(most):
    """Queries of 40 requests (four have any) and their cached tokens."""
    m, kv = [0] * 40, [1 + 3 * b for b in range(40)]
    m[0], m[3], m[20], m[33] = 1, most, min(most, 2), 1
    kv[0], kv[3], kv[9], kv[20] = 9000, 8100, 8192, 4700
    return m, kv


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most,group", IN_TURN)
def test_workgroups_take_parts_in_turn(cut, d, most, group):
    m, kv = _in_turn(most)
    c = cut(d, 60, group, m, 1024)
    assert 1 < c["few_columns"] < -(-max(kv) // 1536) and c["few_chunks"] == -(-65536 // 1536)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("most,group", IN_TURN)
def test_parts_that_a_workgroup_takes_in_turn(d, most, group):
    # tables far wider than the cache, so that a workgroup takes parts far apart under
    # one running sum; pages left out, also at a part's begin; scores that climb and fall
    # from part to part
    kv_heads = 60
    m, kv = _in_turn(most)
    pages = sum(-(-n // 64) for n in kv)
    pool = P.kv4_pool(pages, kv_heads, d, 64)
    n = pages * 64
    k = _bf16(n, kv_heads, d, seed=group).float() + 3 * torch.sin(torch.arange(n, device=DEV) / 700)[:, None, None]
    P.kv4_store(pool, k.to(torch.bfloat16), _bf16(n, kv_heads, d, seed=2), torch.arange(n, dtype=torch.int32, device=DEV), 64)
    table = _tables(kv, 64, pages, 5, width=1024)
    table[3, 0:3] = table[0, 24] = table[0, 90:] = -1
    start = [0] + np.cumsum(m).tolist()
    q = (_bf16(start[-1], kv_heads * group, d, seed=d).float() + 1).to(torch.bfloat16)
    _check_attn(q, pool, table, start, kv, 64, most == 3)


def _workspace(d, kv_heads, group, m, width, block=64):
    c = P.Kv4(0x100000, 1 << 20, kv_heads, d, block)
    return P.lib().carnator_kv4_attn_workspace_size(ctypes.byref(c), kv_heads * group, sum(m), len(m), width, max(m))


def test_workspaces_are_bounded():
    # 3 * 2^28 bytes for the parts of many rows, 143 MB for those of few: below 2^30 together
    for d in (64, 128):
        for m, kv_heads, group, width in [
                ([4096] * 8, 8, 4, 2048), ([8192] + [1] * 1023, 8, 4, 256), ([100000] + [1] * 60, 8, 4, 2048),
                ([8000] + [1] * 1499, 8, 4, 512), ([32760], 12, 1, 512), ([119056], 24, 1, 1 << 20), ([500] * 1000, 8, 8, 1 << 14)]:
            assert _workspace(d, kv_heads, group, m, width) < 1 << 30
    rng = np.random.default_rng(1)
    for _ in range(1000):
        batch = int(2 ** rng.uniform(0, 14))
        most = int(2 ** rng.uniform(0, 17))
        m = [most] + rng.integers(0, max(1, int(most * rng.random()) ** int(rng.integers(0, 2))) + 1, batch - 1).tolist()
        kv_heads, group = int(2 ** rng.uniform(0, 6)), int(2 ** rng.uniform(0, 5))
        if sum(m) * kv_heads * group >= 1 << 31:
            continue
        width = int(2 ** rng.uniform(0, 23))
        assert _workspace(64 << int(rng.integers(0, 2)), kv_heads, group, m, width, 64 << int(rng.integers(0, 2))) < 1 << 30


@pytest.mark.parametrize("d", [64, 128])
def test_a_single_request_of_many_rows_pays_for_no_few(cut, d):
    # 21 frames: the axis whole, no workspace; 256 queries: what the tiles' parts take
    c = cut(d, 12, 1, [4680], 512, causal=False)
    assert c["few_bytes"] == 0 and c["groups"] == 12 * c["many_tiles"] * c["many_chunks"]
    c = cut(d, 12, 1, [256], 32)
    assert c["many_chunks"] > 1 and c["few_bytes"] == 0 and c["groups"] == 12 * c["many_tiles"] * c["many_chunks"]
    assert _workspace(d, 12, 1, [256], 32) == c["many_bytes"] == 256 * 12 * c["many_chunks"] * (4 * d + 16)


def test_a_launch_of_2_32_threads_is_refused(cut):
    # tiles of 256 rows have 512 threads
    def call(rows, batch, most):
        c, q = P.Kv4(0x100000, 4, 1, 128, 64), P.Rows(0x200000, 128, 128)
        return P.lib().carnator_kv4_attn(ctypes.byref(q), rows, 1, ctypes.byref(c), 0x10000, batch, 512, 0x10000, 0x10000,
                                         most, 0, 0.0, 0x60000, 128, 128, None, None, 0, None)

    rows = (1 << 31) - 1
    c = cut(128, 1, 1, [rows], 512)
    assert c["tile_rows"] == 256 and c["groups"] < 1 << 24 and c["threads"] >= 1 << 32
    assert call(rows, 1, rows) == -3 and b"threads" in P.lib().carnator_last_error()
    assert call(1, 1 << 24, 1) == -3


@pytest.mark.parametrize("m,group,width", [([1, 1], 2, 2000), ([300], 2, 200), ([700, 2, 700, 31], 3, 64)])
def test_workspaces_that_do_not_do_are_refused(m, group, width):
    # few rows in parts, tiles in parts, both; nothing is launched
    rows, heads, L = sum(m), 2 * group, P.lib()
    c, q = P.Kv4(0x100000, 4, 2, 128, 64), P.Rows(0x200000, 128 * heads, 128)
    need = _workspace(128, 2, group, m, width)
    assert need > 0

    def call(ws, size):
        return L.carnator_kv4_attn(ctypes.byref(q), rows, heads, ctypes.byref(c), 0x10000, len(m), width, 0x10000, 0x10000,
                                   max(m), 1, 0.0, 0x60000, 128 * heads, 128, None, ws, size, None)

    assert call(0x70000, need - 1) == -5 and call(None, need) == -5 and call(None, 0) == -5
    assert call(0x70010, need) == -4
