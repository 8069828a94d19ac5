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
// Tiles of at most so many chunks -- by the table's width, which is all the host knows -- get a CTA each and need no join: a
// second launch and its trips to memory cost as much as five chunks.  us with runs / with whole tiles, by chunks of a tile:
//   chunks                              2            3            5            6            7            8            12
//   bf16, heads of 64, 8 tiles      6.9 / 4.9    7.3 / 5.4    7.5 / 6.7    7.5 / 7.4    7.7 / 8.0    7.7 / 8.6    7.7 / 11.0
//   bf16, heads of 64, 512 tiles   15.7 / 11.7  16.9 / 13.7  19.6 / 16.9  20.7 / 18.5  22.1 / 19.8  23.2 / 21.5  28.7 / 29.1
//   bf16, heads of 128, 8 tiles     8.1 / 5.6    8.2 / 6.5    8.7 / 8.2    8.5 / 9.1    8.6 / 10.0   8.6 / 10.8   8.8 / 14.3
//   fp32, heads of 64, 8 tiles      8.4 / 7.2    8.6 / 8.8    8.7 / 11.9   8.7 / 13.5   8.9 / 14.9   8.9 / 16.5   8.8 / 22.8
//   fp32, heads of 64, 512 tiles   22.8 / 18.8  26.8 / 23.3  35.9 / 32.5  42.4 / 37.5  46.7 / 43.2  50.7 / 48.5  66.0 / 66.8
constexpr int kWholeTileChunks = 6;
// Rows of a tile: as few as hold all rows of a key head, 64 at most.  Over selected pages always 16, a node's heads of one key
// head at a time: more heads read their pages again, mostly out of L2.  us with tiles of 16 / 32 / 64 rows, 64 nodes and key
// heads, 32 pages each, bf16 heads of 128: 8 heads to a key head 28 / 32 / 39, 16 31 / 35 / 42, 24 41 / 36 / 44, 32 43 / 38 / 46, 64
// 60 / 49 / 46 (and from 65 the 128-row kernel); fp32: 8 67 / 105 / 175, 24 116 / 112 / 185.
inline int tile_rows_of(bool paged, int rows) { return paged || rows <= 16 ? 16 : (rows <= 32 ? 32 : 64); }

template <typename CT> int plan_attention(const AttnArgs& a, bool paged, int D, AttnPlan* plan);
template <typename CT> int launch_attention(const AttnArgs& a, bool paged, int D, const AttnPlan& plan, cudaStream_t st);

// The most chunks of a tile.
template <bool PAGED>
long long max_chunks(const AttnArgs& a) { return (PAGED ? std::min(a.select, a.ppr) + 1 : a.ppr) + ceil_div(a.T, kChunk); }

// A tile's end (its result, the next one's queries, the pipeline's new start) takes as long as some chunks, `cost` of them, and
// counts as so many where runs are divided: without it, the CTAs that had a tile's end finished last.  us with 0 / 2 / 4 / 8 / 12
// chunks: over 8 sequences of 8000, heads of 128, bf16, 1 row 50.3 / 49.7 / 48.5 / 48.7 / 49.6, 128 rows 89 / 88 / 86 / 82 / 78, heads
// of 64 128 rows 66 / 64 / 62 / 59 / 60; fp32, 4000 positions, heads of 128, 64 rows 300 / 294 / 299 / 313 / 332, heads of 64 16 rows
// 45.7 / 43.5 / 44.0 / 46.8 / 48.4.  Where CTAs have hardly a chunk each it is left out (fp32, 8 heads over 2000 positions: 10.5 us,
// with it 11.4).
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
