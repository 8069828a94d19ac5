"""The operators on a paged cache without a GPU: what the calls refuse, the division of work among CTAs, and their oracle
against second statements of the same definitions."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import operators as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1811_03115_b200", "csrc")
INVALID, SHAPE, NOMEM, UNSUPPORTED = -1, -2, -4, -8


@pytest.fixture(scope="module")
def b():
    from paper_1811_03115_b200.build import build_library
    build_library()
    from paper_1811_03115_b200 import binding
    return binding


P = 0x10000        # an aligned address that no refused call may look at


def _cache(b, **over):
    c = b.bpd_cache(P, P, P, 2, 10, 50, 2, 2, 64, 1)
    for name, value in over.items():
        setattr(c, name, value)
    return C.byref(c)


def _attention(b, cache=None, **over):
    a = dict(q=P, k_new=P, v_new=P, nodes=4, heads=4, q_stride=256, kv_stride=128, lens=P, parents=P, n_nodes=None, scale=1.0, scratch=P,
             scratch_bytes=1 << 40, out=P, lse=None, stream=None)
    a.update(over)
    return b.lib.bpd_op_tree_attention(cache if cache is not None else _cache(b), *a.values())


def _paged(b, cache=None, **over):
    a = dict(means=P, q=P, k_new=P, v_new=P, nodes=4, heads=4, q_stride=256, kv_stride=128, lens=P, parents=P, n_nodes=None, select=2, scale=1.0,
             scratch=P, scratch_bytes=1 << 40, out=P, lse=None, pages=None, stream=None)
    a.update(over)
    return b.lib.bpd_op_page_attention(cache if cache is not None else _cache(b), *a.values())


def _commit(b, cache=None, **over):
    a = dict(k_new=P, v_new=P, nodes=4, kv_stride=128, lens=P, parents=P, tokens=P, top1=P, last_top1=P, n_nodes=None, eos=-1, out_lens=2 * P,
             accepted=P, path=P, following=P, stream=None)
    a.update(over)
    return b.lib.bpd_op_tree_commit(cache if cache is not None else _cache(b), *a.values())


def _weights(b, cache=None, **over):
    a = dict(q=P, nodes=4, heads=4, q_stride=256, lse=P, path=P, accepted=P, lens=P, seen=P, scale=1.0, weights=P, positions=P, stream=None)
    a.update(over)
    return b.lib.bpd_op_cache_weights(cache if cache is not None else _cache(b), *a.values())


def _evict(b, cache=None, **over):
    a = dict(lens=P, seen=P, budget=5, recent=1, weights=P, positions=P, scratch=P, scratch_bytes=1 << 40, out_lens=2 * P, stream=None)
    a.update(over)
    return b.lib.bpd_op_cache_evict(cache if cache is not None else _cache(b), *a.values())


def _means(b, cache=None, **over):
    a = dict(lens_from=P, lens=P, means=P, stream=None)
    a.update(over)
    return b.lib.bpd_op_page_means(cache if cache is not None else _cache(b), *a.values())


@pytest.mark.parametrize("call", [_attention, _paged, _commit, _weights, _evict, _means])
def test_caches_that_every_call_refuses(b, call):
    assert call(b, cache=C.cast(None, C.c_void_p)) == INVALID
    for over, status in (({"k_pool": None}, INVALID), ({"page_table": None}, INVALID), ({"k_pool": P + 8}, INVALID), ({"dtype": 2}, INVALID),
                         ({"dtype": -1}, INVALID), ({"head_dim": 80}, UNSUPPORTED), ({"head_dim": 0}, UNSUPPORTED), ({"head_dim": 256}, UNSUPPORTED),
                         ({"kv_heads": 0}, SHAPE), ({"batch": 0}, SHAPE), ({"batch": 65536}, SHAPE), ({"layers": 0}, SHAPE), ({"n_pages": 0}, SHAPE),
                         ({"n_pages": (1 << 24) + 1}, SHAPE), ({"pages_per_row": 0}, SHAPE), ({"pages_per_row": (1 << 20) + 1}, SHAPE)):
        assert call(b, cache=_cache(b, **over)) == status, over
        assert b.lib.bpd_last_error()


def test_calls_that_write_values_want_them(b):
    for call in (_attention, _paged, _commit, _evict):
        assert call(b, cache=_cache(b, v_pool=None)) == INVALID


@pytest.mark.parametrize("call", [_attention, _paged])
def test_attention_refuses(b, call):
    for name in ("q", "k_new", "v_new", "lens", "parents", "out", "scratch"):
        assert call(b, **{name: None}) == INVALID, name
    for name in ("q", "k_new", "v_new", "out", "scratch"):
        assert call(b, **{name: P + 8}) == INVALID, name
    for over, status in (({"nodes": 0}, SHAPE), ({"nodes": 257}, SHAPE), ({"heads": 0}, SHAPE), ({"heads": 3}, SHAPE), ({"heads": 8192}, SHAPE),
                         ({"q_stride": 248}, SHAPE), ({"q_stride": 260}, INVALID), ({"kv_stride": 64}, SHAPE), ({"kv_stride": 130}, INVALID),
                         ({"q_stride": -256}, SHAPE), ({"scale": 0.0}, INVALID), ({"scale": -1.0}, INVALID), ({"scale": float("nan")}, INVALID),
                         ({"scale": float("inf")}, INVALID), ({"scratch_bytes": 255}, NOMEM), ({"scratch": P + 16}, INVALID)):
        assert call(b, **over) == status, over


def test_page_attention_refuses_selections(b):
    assert _paged(b, select=0) == SHAPE and _paged(b, select=51) == SHAPE and _paged(b, means=None) == INVALID and _paged(b, means=P + 4) == INVALID
    assert b.lib.bpd_op_page_attention_scratch_bytes(_cache(b), 4, 4, 51) == 0


def test_commit_weights_and_eviction_refuse(b):
    for name in ("k_new", "v_new", "lens", "parents", "tokens", "top1", "last_top1", "out_lens", "accepted", "path", "following"):
        assert _commit(b, **{name: None}) == INVALID, name
    assert _commit(b, nodes=300) == SHAPE and _commit(b, kv_stride=120) == SHAPE and _commit(b, kv_stride=132) == INVALID
    assert _commit(b, out_lens=P) == INVALID                 # the lengths themselves
    for name in ("q", "lse", "path", "accepted", "lens", "seen", "weights", "positions"):
        assert _weights(b, **{name: None}) == INVALID, name
    assert _weights(b, heads=5) == SHAPE and _weights(b, nodes=0) == SHAPE and _weights(b, scale=float("nan")) == INVALID
    for name in ("lens", "seen", "weights", "positions", "scratch", "out_lens"):
        assert _evict(b, **{name: None}) == INVALID, name
    assert _evict(b, budget=0) == SHAPE and _evict(b, recent=-1) == SHAPE and _evict(b, recent=6) == SHAPE
    assert _evict(b, scratch_bytes=16) == NOMEM and _evict(b, out_lens=P) == INVALID
    for name in ("lens_from", "lens", "means"):
        assert _means(b, **{name: None}) == INVALID, name
    assert _means(b, means=P + 4) == INVALID


# every CTA of a sequence walks its tree by these arrays, whenever it starts: an output in their place would change the walk
def test_commit_and_eviction_refuse_outputs_in_the_place_of_inputs(b):
    spread = {name: (i + 2) * P for i, name in enumerate(("lens", "parents", "tokens", "top1", "last_top1", "n_nodes"))}
    apart = {name: (i + 20) * P for i, name in enumerate(("out_lens", "accepted", "path", "following"))}
    for out in apart:
        for name, at in spread.items():
            assert _commit(b, **{**spread, **apart, out: at}) == INVALID, (out, name)
            assert b"overlap" in b.lib.bpd_last_error()
        assert _commit(b, **{**spread, **apart, out: P}) == INVALID            # the page table
    # parts of them: 2 sequences of 4 nodes
    assert _commit(b, **{**spread, **apart, "path": spread["last_top1"] - 28}) == INVALID and _commit(b, **{**spread, **apart, "following": spread["top1"] + 28}) == INVALID
    for name in ("lens", "seen"):
        assert _evict(b, **{"lens": 5 * P, "seen": 6 * P, "out_lens": {"lens": 5 * P, "seen": 6 * P}[name] + 4}) == INVALID
        assert b"overlap" in b.lib.bpd_last_error()
    assert _evict(b, lens=5 * P, seen=6 * P, out_lens=P + 396) == INVALID      # the page table's last entry


def test_scratch_grows_with_what_needs_it(b):
    n = b.lib.bpd_op_tree_attention_scratch_bytes(_cache(b), 4, 4)
    assert 0 < n < b.lib.bpd_op_tree_attention_scratch_bytes(_cache(b, batch=640), 64, 4)
    assert b.lib.bpd_op_tree_attention_scratch_bytes(_cache(b, pages_per_row=2), 4, 4) == 0          # whole tiles, nothing to join
    assert b.lib.bpd_op_tree_attention_scratch_bytes(_cache(b, head_dim=7), 4, 4) == 0
    assert b.lib.bpd_op_cache_evict_scratch_bytes(_cache(b), 10 ** 9) == b.lib.bpd_op_cache_evict_scratch_bytes(_cache(b), 3200)


def test_scratch_of_refused_calls_is_none(b):
    many = dict(layers=65535, batch=65535, kv_heads=1024)
    assert _evict(b, cache=_cache(b, **many)) == SHAPE and b.lib.bpd_op_cache_evict_scratch_bytes(_cache(b, **many), 5) == 0
    for over in ({"v_pool": None}, {"v_pool": P + 8}, {"batch": 0}):
        assert b.lib.bpd_op_tree_attention_scratch_bytes(_cache(b, **over), 4, 4) == 0 and b.lib.bpd_op_cache_evict_scratch_bytes(_cache(b, **over), 5) == 0
        assert b.lib.bpd_op_page_attention_scratch_bytes(_cache(b, **over), 4, 4, 2) == 0


def test_expiring_wait_refuses_limits(b):
    assert b.lib.bpd_debug_op_wait_timeout(0, None) == INVALID and b.lib.bpd_debug_op_wait_timeout(2000001, None) == INVALID


def test_binding_refuses_tensors(b):
    import torch
    k = torch.zeros(10, 64, 2, 64)
    with pytest.raises(ValueError, match="CUDA"):
        b._cache(k, k, torch.zeros(2, 5, dtype=torch.int32), False)
    for pool, layered in ((k[None], False), (k, True), (k[:, :32], False), (k.half(), False)):
        with pytest.raises(ValueError, match="pools"):
            b._cache(pool, pool, torch.zeros(2, 5, dtype=torch.int32), layered)
    with pytest.raises(ValueError, match="page_table"):
        b._cache(k, k, torch.zeros(5, dtype=torch.int32), False)


def test_binding_takes_rows_one_stride_apart(b):
    import torch
    cpu, f32 = -1, torch.float32
    fused = torch.zeros(3, 5, 400)
    part = fused[..., 128:256].unflatten(2, (2, 64))
    assert b._expect_rows(part, "x", (3, 5, 2, 64), f32, cpu) == (part.data_ptr(), 400)
    assert b._expect_rows(part.contiguous(), "x", (3, 5, 2, 64), f32, cpu)[1] == 128
    one = fused[:, :1, :128].unflatten(2, (2, 64))           # one node per row: the batch gives the stride
    assert b._expect_rows(one, "x", (3, 1, 2, 64), f32, cpu)[1] == 2000
    assert b._expect_rows(fused[:1, :1, :128].unflatten(2, (2, 64)), "x", (1, 1, 2, 64), f32, cpu)[1] == 128
    layers = torch.zeros(2, 3, 5, 400)[..., :128].unflatten(3, (2, 64))
    assert b._expect_rows(layers, "x", (2, 3, 5, 2, 64), f32, cpu)[1] == 400
    for bad in (fused[:, ::2, :128].unflatten(2, (2, 64))[:, :3], fused.transpose(0, 1)[..., :128].unflatten(2, (2, 64)), fused[..., :256:2].unflatten(2, (2, 64)),
                torch.zeros(3, 5, 64, 2).transpose(2, 3), torch.zeros(1, 1, 2, 64).expand(3, 5, 2, 64)):
        with pytest.raises(ValueError, match="stride"):
            b._expect_rows(bad, "x", tuple(bad.shape), f32, cpu)
    with pytest.raises(ValueError, match="expected"):
        b._expect(torch.zeros(4)[::2], "x", (2,), f32, cpu)


# every unit of every tile falls to exactly one CTA, and the CTAs from a tile's first to its last are those that have units of it
WORK = r"""
#include <cstdio>
#include <initializer_list>

#include "cache_index.hpp"
using namespace bpd::tree;
int main() {
  const long long sizes[] = {1, 2, 3, 40, 147, 148, 149, 443, 444, 445, 1000, 99991, 2147483647LL, 2147483648LL, 5000000000LL};
  for (long long units : sizes)
    for (int grid : {1, 2, 60, 148, 444}) {
      const Runs r = runs_of(units, grid);
      if (r.ctas != (units < grid ? units : grid) || first_unit(r, 0) != 0 || first_unit(r, r.ctas) != units) return 1;
      for (int i = 0; i < r.ctas; ++i) {
        const long long a = first_unit(r, i), z = first_unit(r, i + 1);
        if (a >= z || z - a > units / r.ctas + 1 || cta_of_unit(r, a) != i || cta_of_unit(r, z - 1) != i) return 2;
      }
    }
  if (runs_of(0, 5).ctas != 0) return 9;
  for (int len : {0, 1, 63, 64, 65, 1000})
    for (int nodes : {0, 1, 63, 64, 65, 256})
      for (int group : {1, 3, 16, 17})
        for (int rows : {16, 32, 64}) {
          SeqWork d = dense_work(len, nodes, 4, group, rows), p = paged_work(len, nodes, 3, 4, group, rows);
          if ((long long)d.tiles * rows < 4LL * nodes * group || d.chunks * 64 < len + nodes) return 3;
          if ((long long)p.tiles * rows < 4LL * nodes * group) return 4;
          const int full = len / 64 < 3 ? len / 64 : 3;
          if (p.chunks != full + (len % 64 != 0) + (nodes + 63) / 64) return 5;
        }
  if (pool_row(-1, 10, 5) != -1 || pool_row(10, 10, 5) != -1 || pool_row(2147483647, 10, 5) != -1 || pool_row(9, 10, 70) != 9 * 64 + 6) return 6;
  if (pool_row(16777215, 16777216, 63) != 16777215LL * 64 + 63) return 7;
  if (parent_of(3, 3) != -1 || parent_of(9, 3) != -1 || parent_of(-7, 3) != -1 || parent_of(2, 3) != 2 || parent_of(0, 0) != -1) return 8;
  std::puts("ok");
}
"""


def test_division_of_work(tmp_path):
    (tmp_path / "work.cpp").write_text(WORK)
    subprocess.run([shutil.which("g++"), "-std=c++17", "-O1", "-I", CSRC, "-o", str(tmp_path / "work"),
                    str(tmp_path / "work.cpp")], check=True)
    assert subprocess.run([str(tmp_path / "work")], capture_output=True, text=True).stdout == "ok\n"


# The doubling of find_lines, lane by lane in the orders that a warp's lanes may take between two synchronisations: a lane that
# stores its next round's state while another is between its two reads makes that one skip a part of its line.
def test_lines_by_doubling_need_a_synchronisation_behind_their_reads():
    rng = np.random.default_rng(3)

    def doubled(parents, synchronised):
        n = len(parents)
        mine, mine_up = [1 << t for t in range(n)], [p if 0 <= p < t else -1 for t, p in enumerate(parents)]
        bits, up = list(mine), list(mine_up)
        while any(u >= 0 for u in mine_up):
            bits, up = list(mine), list(mine_up)
            order = rng.permutation(n)
            for i, t in enumerate(order):
                if mine_up[t] < 0:
                    continue
                seen = bits[mine_up[t]]
                if not synchronised:
                    for ahead in order[:i]:                  # these have done their reads
                        bits[ahead], up[ahead] = mine[ahead], mine_up[ahead]
                mine[t], mine_up[t] = mine[t] | seen, up[mine_up[t]]
        return mine
    parents = [max(-1, t - 1 - int(rng.integers(0, 3))) for t in range(60)]
    want = [sum(1 << u for u in plain.line_of(parents, t)) for t in range(60)]
    assert doubled(parents, True) == want and doubled(parents, False) != want
    source = open(os.path.join(CSRC, "tree_attention.cuh")).read()
    rounds = source[source.index("for (int reach = 1"):source.index("void find_lines")]
    assert rounds.count("__syncwarp()") == 3                 # behind a round's stores, behind its reads, behind the last round


# ---------------------------------------------------------------------- the oracle
def test_oracle_attention_is_masked_attention():
    rng = np.random.default_rng(1)
    lens, t, d = [70, 0], 4, 8
    table = np.array([[2, 0], [1, 3]], np.int32)
    k, v = rng.standard_normal((4, 64, 1, d)), rng.standard_normal((4, 64, 1, d))
    q, kn, vn = rng.standard_normal((2, t, 2, d)), rng.standard_normal((2, t, 1, d)), rng.standard_normal((2, t, 1, d))
    parents = np.array([[-1, 0, 0, 2], [-1, -1, 1, 2]], np.int32)
    out, lse = plain.attention(q, kn, vn, k, v, table, lens, parents, [4, 3], 0.5)
    sees = {0: [[0], [0, 1], [0, 2], [0, 2, 3]], 1: [[0], [1], [1, 2]]}
    for b in range(2):
        flat_k, flat_v = k[table[b]].reshape(-1, d)[:lens[b]], v[table[b]].reshape(-1, d)[:lens[b]]
        for node, line in enumerate(sees[b]):
            keys, values = np.vstack([flat_k, kn[b, line, 0]]), np.vstack([flat_v, vn[b, line, 0]])
            e = np.exp(q[b, node] @ keys.T * 0.5)
            np.testing.assert_allclose(out[b, node], e @ values / e.sum(1, keepdims=True), rtol=1e-12)
            np.testing.assert_allclose(lse[b, node], np.log(e.sum(1)), rtol=1e-12)
    assert (out[1, 3] == 0).all() and np.isneginf(lse[1, 3]).all()


def test_oracle_walks_and_evicts_by_hand():
    parents, tokens, top1 = [-1, -1, 0, 1, 1, 4], [7, 8, 1, 2, 3, 9], [1, 3, 0, 0, 9, 5]
    assert plain.accept_path(parents, tokens, top1, 8, 6, 10) == ([1, 4, 5], 5)
    assert plain.accept_path(parents, tokens, top1, 8, 6, 2) == ([1, 4], 9) and plain.accept_path(parents, tokens, top1, 8, 6, 10, eos_id=3) == ([1, 4], 9)
    assert plain.accept_path(parents, tokens, top1, 8, 4, 10) == ([1], 3) and plain.accept_path(parents, tokens, top1, 6, 6, 10) == ([], 6)
    k = np.arange(64.).reshape(1, 1, 64, 1, 1)
    w = np.array([5, 1, np.nan, 4, 4, 0, 9, 2] + [0] * 56, np.float32).reshape(1, 1, 1, 64)
    pos = np.arange(64, dtype=np.int32).reshape(1, 1, 1, 64)
    # the last two tokens (slots 6, 7) stay, then slots 0 and 3: holes 1 and 2 take slots 6 and 7
    lens, w2, p2, k2, _ = plain.evict(w, pos, k, k, np.zeros((1, 1), np.int32), np.array([8]), [8], 4, 2)
    assert lens.tolist() == [4] and p2[0, 0, 0, :4].tolist() == [0, 6, 7, 3] and k2[0, 0, :4, 0, 0].tolist() == [0, 6, 7, 3]
    assert w2[0, 0, 0, :4].tolist() == [5, 9, 2, 4]


def test_oracle_selects_by_score():
    means = np.zeros((1, 6, 1, 4), np.float32)
    means[0, :, 0, 0] = [3, np.nan, 5, 3, 1, 99]
    q = np.zeros((1, 2, 2, 4), np.float32)
    q[0, :, :, 0] = 0.5
    assert plain.select_pages(q, means, [5 * 64 + 9], [1], 2)[0, :, 0].tolist() == [[0, 2], [-1, -1]]
    assert plain.select_pages(q, means, [5 * 64 + 9], [2], 8)[0, 1, 0].tolist() == [0, 1, 2, 3, 4, -1, -1, -1]
