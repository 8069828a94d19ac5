// Index arithmetic of the operators on a paged cache, for the host and the device: which units of work a CTA takes, and
// where a position lies.  Nothing here trusts what the caller's device arrays hold: lengths are clamped to the capacity,
// node counts to the tree's width, and a page outside the pool is no page.
#pragma once

#ifdef __CUDACC__
#define BPD_HD __host__ __device__ __forceinline__
#else
#define BPD_HD inline
#endif

namespace bpd {
namespace tree {

constexpr int kPagePos = 64;      // positions of a page
constexpr int kMaxNodes = 256;    // drafted nodes of a sequence

BPD_HD int clamp_int(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }
BPD_HD int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Work is counted in units of one chunk (the up to 64 positions of a page, or 64 nodes) for one tile of query rows.
// A sequence has `tiles` tiles of `chunks` chunks each.
struct SeqWork { int tiles, chunks; };

// Attention over the whole cache: tiles are (key head, rows / R), rows = nodes x group.
BPD_HD SeqWork dense_work(int len, int nodes, int kv_heads, int group, int tile_rows) {
  SeqWork w;
  w.tiles = kv_heads * ceil_div(nodes * group, tile_rows);
  w.chunks = ceil_div(len, kPagePos) + ceil_div(nodes, kPagePos);
  return w;
}
// Attention over selected pages: tiles are (node, key head, rows / R), rows = group; chunks are the selected full pages,
// the open page and the tree.
BPD_HD SeqWork paged_work(int len, int nodes, int select, int kv_heads, int group, int tile_rows) {
  const int full = len / kPagePos;
  SeqWork w;
  w.tiles = nodes * kv_heads * ceil_div(group, tile_rows);
  w.chunks = (select < full ? select : full) + (len % kPagePos ? 1 : 0) + ceil_div(nodes, kPagePos);
  return w;
}

// `units` units over `ctas` <= units CTAs, each a contiguous run of at least one: the first unit of CTA i, and the CTA that
// has unit u.
BPD_HD long long first_unit(long long i, long long units, long long ctas) { return i * units / ctas; }
BPD_HD int cta_of_unit(long long u, long long units, long long ctas) { return (int)(((u + 1) * ctas - 1) / units); }

// Row of the pool ([n_pages, 64] rows) that holds position pos, -1 if the table has no page of the pool for it.
BPD_HD long long pool_row(int page, int n_pages, int pos) {
  return (page < 0 || page >= n_pages) ? -1 : (long long)page * kPagePos + (pos % kPagePos);
}

// A node's parent, if it lies before the node (the order every valid tree has), else -1: walks up always end.
BPD_HD int parent_of(int parent, int node) { return (parent >= 0 && parent < node) ? parent : -1; }

}  // namespace tree
}  // namespace bpd
