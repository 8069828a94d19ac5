// Tree attention over bf16 caches.
#include <algorithm>
#include <type_traits>

#include "tree_attention_tc.cuh"
#include "tc_host.hpp"
#include "tree_host.hpp"

namespace bpd {
namespace tree {

// Calls whose work is cut into runs, heads of 64 and 128: with more than 64 rows to a key head, and with more than 32 where a
// sequence may have 64 pages or more, tiles are 128 rows and go to the 5th-generation tensor cores.  With fewer, a tile's
// products are short and its softmax is one warp's or two's; with short sequences, the tile's start and end weigh more than its
// chunks.  us of the kernel whose four warps share the keys / of the 128-row one, 8 key heads (16 in the last line):
//   rows                                        16         32         48         64        128
//   8 sequences of 8000, heads of 128        54 / 68    63 / 68    93 / 70    92 / 68   174 / 79
//   8 sequences of 8000, heads of 64         35 / 43    40 / 45    56 / 46    57 / 46   103 / 57
//   1 sequence of 8000, heads of 128         17 / 24    20 / 23    25 / 26    26 / 25    37 / 30
//   32 sequences of 500, heads of 128        25 / 44    33 / 44    46 / 52    50 / 50    91 / 61
//   32 sequences of 500, heads of 64         27 / 53    36 / 56    51 / 60    56 / 62   100 / 78
inline bool many_rows(int rows, long long chunks) { return rows > 64 || (rows > 32 && chunks >= 64); }

template <int D, bool PAGED>
int plan_tc(const AttnArgs& a, AttnPlan* p) {
  const long long per_head = PAGED ? ceil_div(a.G, kTcRows) : ceil_div(a.T * a.G, kTcRows);
  const long long tiles = (long long)a.B * a.Hkv * per_head * (PAGED ? a.T : 1);
  p->tc = 1;
  p->tile_rows = kTcRows;
  p->tiles = (int)tiles;
  p->ctas = (int)std::min<long long>(tiles * max_chunks<PAGED>(a), (long long)kSMs * TcShape<D>::CTAS_PER_SM);
  p->combine_rows = std::min(kTcRows, PAGED ? a.G : a.T * a.G);
  p->end_units = end_units_of(tiles * max_chunks<PAGED>(a), (long long)kSMs * TcShape<D>::CTAS_PER_SM, 8);
  scratch_of(D, p);
  return BPD_OK;
}

// A bf16 matrix [rows, cols], boxes of 64 x 64, 128-byte swizzle.
static int map_of(const void* ptr, long long rows, long long cols, long long ld, CUtensorMap* out) {
  return tc::make_map_3d(ptr, 2, 1, 0, (uint64_t)rows, (uint64_t)cols, (uint64_t)ld, 64, kChunk, true, out);
}

template <int D>
int maps_of(const AttnArgs& a, TcMaps* maps) {
  const long long width = (long long)a.Hkv * D, positions = (long long)a.n_pages * kPagePos, nodes = (long long)a.B * a.T;
  int rc;
  if ((rc = map_of(a.k_pool, positions, width, width, &maps->kp)) || (rc = map_of(a.v_pool, positions, width, width, &maps->vp)) ||
      (rc = map_of(a.k_new, nodes, width, a.kv_stride, &maps->kn)) || (rc = map_of(a.v_new, nodes, width, a.kv_stride, &maps->vn)))
    return rc;
  return BPD_OK;
}

template <int D, bool PAGED>
int launch_tc(const AttnArgs& a, const AttnPlan& p, cudaStream_t st) {
  using S = TcShape<D>;
  TcMaps maps;
  int rc = maps_of<D>(a, &maps);
  if (rc) return rc;
  rc = ensure_smem_limit(reinterpret_cast<const void*>(tree_attention_tc_kernel<D, PAGED>), S::SMEM);
  if (rc) return rc;
  BPD_CUDA(launch_k(tree_attention_tc_kernel<D, PAGED>, dim3(p.ctas), dim3(kTcThreads), S::SMEM, st, PAGED, a, maps));
  ++g_launches;
  return launch_combine<bf16, D, PAGED>(a, p, st);
}

template <> int plan_attention<bf16>(const AttnArgs& a, bool paged, int D, AttnPlan* plan) {
  BPD_TREE_BY_DIM({
    int rc = by_rows<bf16, DD>(a, paged, [&](auto wr, auto pg) { return plan_one<bf16, DD, decltype(wr)::value, decltype(pg)::value>(a, plan); });
    if constexpr (DD >= 64) {
      if (!rc && plan->split && many_rows(paged ? a.G : a.T * a.G, paged ? max_chunks<true>(a) : max_chunks<false>(a))) rc = paged ? plan_tc<DD, true>(a, plan) : plan_tc<DD, false>(a, plan);
    }
    return rc;
  })
}
template <> int launch_attention<bf16>(const AttnArgs& a, bool paged, int D, const AttnPlan& plan, cudaStream_t st) {
  BPD_TREE_BY_DIM({
    if constexpr (DD >= 64) {
      if (plan.tc) return paged ? launch_tc<DD, true>(a, plan, st) : launch_tc<DD, false>(a, plan, st);
    }
    return by_rows<bf16, DD>(a, paged, [&](auto wr, auto pg) { return launch_one<bf16, DD, decltype(wr)::value, decltype(pg)::value>(a, plan, st); });
  })
}

int let_wait_expire(int limit_us, cudaStream_t st) {
  int khz = 0, dev = 0;
  BPD_CUDA(cudaGetDevice(&dev));
  BPD_CUDA(cudaDeviceGetAttribute(&khz, cudaDevAttrClockRate, dev));
  BPD_CUDA(launch_k(op_wait_probe_kernel, dim3(1), dim3(32), 0, st, false, (unsigned long long)limit_us * (unsigned long long)khz / 1000ull));
  ++g_launches;
  return BPD_OK;
}

int take_wait_expired(int* expired, cudaStream_t st) {
  const int zero = 0;
  BPD_CUDA(cudaMemcpyFromSymbolAsync(expired, g_wait_expired, sizeof(int), 0, cudaMemcpyDeviceToHost, st));
  BPD_CUDA(cudaStreamSynchronize(st));
  if (*expired) {
    BPD_CUDA(cudaMemcpyToSymbolAsync(g_wait_expired, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, st));
    BPD_CUDA(cudaStreamSynchronize(st));
  }
  return BPD_OK;
}

}  // namespace tree
}  // namespace bpd
