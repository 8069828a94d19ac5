// Launches of the tree attention kernels, per element type (one translation unit each).
#pragma once
#include "host.hpp"
#include "tree_attention.cuh"

namespace bpd {
namespace tree {

constexpr int kSMs = 148;

// What a call of these sizes needs, and its launches.
struct AttnPlan {
  int ctas, tile_rows, tiles, combine_rows, split, tc, end_units;   // tiles: that could be
  size_t part_bytes, info_bytes;
};
// Tiles of at most so many chunks get a CTA each and need no join: a second launch and its trips to memory cost as much as
// five chunks (one token over 57 positions 9.0 us with runs, 6.2 with whole tiles; 512 tiles of up to three chunks 19.9 / 14.4;
// 16 tiles of up to 135 chunks 19 / 98).
constexpr int kWholeTileChunks = 6;
// Rows of a tile: as few as hold all rows of a key head, 64 at most.
inline int tile_rows_of(bool paged, int rows) { return paged || rows <= 16 ? 16 : (rows <= 32 ? 32 : 64); }

template <typename CT> int plan_attention(const AttnArgs& a, bool paged, int D, AttnPlan* plan);
template <typename CT> int launch_attention(const AttnArgs& a, bool paged, int D, const AttnPlan& plan, cudaStream_t st);

// The most chunks of a tile.
template <bool PAGED>
long long max_chunks(const AttnArgs& a) { return (PAGED ? std::min(a.select, a.ppr) + 1 : a.ppr) + ceil_div(a.T, kChunk); }

// A tile's end (its result, the next one's queries, the pipeline's new start) takes as long as some chunks, `cost` of them, and
// counts as so many where runs are divided: without it, the CTAs that had a tile's end finished last.  Over 8 sequences of 8000,
// heads of 128, with 0 / 2 / 4 / 8 / 12 chunks: 57.7 / 56.2 / 54.9 / 54.6 / 54.8 us (16 rows), 87.4 / 85.4 / 83.3 / 79.7 / 81.0
// (128 rows); fp32, 4000 positions, 64 rows: 292 / 286 / 296 / 314 / 326.  Where CTAs have hardly a chunk each it is left out
// (fp32, 8 heads over 2000 positions: 10.3 us, with it 11.7).
inline int end_units_of(long long units, long long slots, int cost) { return units >= 2 * slots ? cost : 0; }

inline void scratch_of(int D, AttnPlan* p) {
  const size_t part = (size_t)p->ctas * 2 * part_floats(p->combine_rows, D) * 4;
  p->part_bytes = p->split ? (part + 255) / 256 * 256 : 0;
  p->info_bytes = p->split ? ((size_t)p->tiles * sizeof(int2) + 255) / 256 * 256 : 0;
}

template <typename CT, int D, int WR, bool PAGED>
int plan_one(const AttnArgs& a, AttnPlan* p) {
  using S = Shape<CT, D, WR>;
  p->tile_rows = S::R;
  p->tc = 0;
  const long long per_head = PAGED ? ceil_div(a.G, S::R) : ceil_div(a.T * a.G, S::R);
  const long long tiles = (long long)a.B * a.Hkv * per_head * (PAGED ? a.T : 1);
  if (tiles > 0x7fffffffLL) return fail(BPD_E_SHAPE, "batch * nodes * heads out of range");
  p->tiles = (int)tiles;
  p->split = max_chunks<PAGED>(a) > kWholeTileChunks;
  p->ctas = (int)(p->split ? std::min<long long>(tiles * max_chunks<PAGED>(a), (long long)kSMs * S::CTAS_PER_SM) : tiles);
  p->combine_rows = std::min(S::R, PAGED ? a.G : a.T * a.G);
  p->end_units = end_units_of(tiles * max_chunks<PAGED>(a), (long long)kSMs * S::CTAS_PER_SM, sizeof(CT) == 4 ? 2 : 4);
  scratch_of(D, p);
  return BPD_OK;
}

template <typename CT, int D, bool PAGED>
int launch_combine(const AttnArgs& a, const AttnPlan& p, cudaStream_t st) {
  if ((long long)p.tiles * p.combine_rows <= 16 * kSMs)
    BPD_CUDA(launch_k(combine_kernel<CT, D, PAGED, 4>, dim3(p.tiles, p.combine_rows), dim3(kThreads), 0, st, true, a, p.tile_rows));
  else
    BPD_CUDA(launch_k(combine_kernel<CT, D, PAGED, 1>, dim3(p.tiles, ceil_div(p.combine_rows, 4)), dim3(kThreads), 0, st, true, a, p.tile_rows));
  ++g_launches;
  return BPD_OK;
}

template <typename CT, int D, int WR, bool PAGED>
int launch_one(const AttnArgs& a, const AttnPlan& p, cudaStream_t st) {
  using S = Shape<CT, D, WR>;
  const auto kernel = tree_attention_kernel<CT, D, WR, PAGED>;
  int rc = ensure_smem_limit(reinterpret_cast<const void*>(kernel), S::SMEM);
  if (rc) return rc;
  BPD_CUDA(launch_k(kernel, dim3(p.ctas), dim3(kThreads), S::SMEM, st, PAGED, a));
  ++g_launches;
  return p.split ? launch_combine<CT, D, PAGED>(a, p, st) : BPD_OK;
}

template <typename CT, int D, typename F>
int by_rows(const AttnArgs& a, bool paged, F&& f) {
  if (paged) return f(std::integral_constant<int, 1>(), std::true_type());
  switch (tile_rows_of(false, a.T * a.G)) {
    case 16: return f(std::integral_constant<int, 1>(), std::false_type());
    case 32: return f(std::integral_constant<int, 2>(), std::false_type());
    default: return f(std::integral_constant<int, 4>(), std::false_type());
  }
}

#define BPD_TREE_BY_DIM(...)                \
  switch (D) {                                      \
    case 16: { constexpr int DD = 16; __VA_ARGS__ }        \
    case 32: { constexpr int DD = 32; __VA_ARGS__ }        \
    case 64: { constexpr int DD = 64; __VA_ARGS__ }        \
    default: { constexpr int DD = 128; __VA_ARGS__ }       \
  }

// Whether a wait of an operator's kernel has expired on the current device since it was last asked.
int take_wait_expired(int* expired, cudaStream_t st);
// A launch whose wait expires after so long (a self test).
int let_wait_expire(int limit_us, cudaStream_t st);

}  // namespace tree
}  // namespace bpd
