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

// `units` units over `ctas` <= units CTAs, each a contiguous run: the first units % ctas of them one unit longer.  (Divisions
// of 64-bit numbers take the device ten times as long as those of 32 bits, and a small call's CTAs wait for them.)
struct Runs {
  long long units;
  int ctas, extra;           // extra: CTAs with size + 1 units
  long long size;
};
BPD_HD Runs runs_of(long long units, int max_ctas) {
  Runs r;
  r.units = units;
  r.ctas = units < max_ctas ? (int)units : max_ctas;
  if (units <= 0) { r.size = 0; r.extra = 0; return r; }
  if (units <= 0x7fffffffLL) {
    const unsigned size = (unsigned)units / (unsigned)r.ctas;
    r.size = size;
    r.extra = (int)((unsigned)units - size * (unsigned)r.ctas);
  } else {
    r.size = units / r.ctas;
    r.extra = (int)(units - r.size * r.ctas);
  }
  return r;
}
// The first unit of CTA i, and the CTA that has unit u.
BPD_HD long long first_unit(const Runs& r, int i) { return i * r.size + (i < r.extra ? i : r.extra); }
BPD_HD int cta_of_unit(const Runs& r, long long u) {
  const long long longer = r.extra * (r.size + 1);
  if (r.units <= 0x7fffffffLL)
    return u < longer ? (int)((unsigned)u / (unsigned)(r.size + 1)) : r.extra + (int)((unsigned)(u - longer) / (unsigned)r.size);
  return u < longer ? (int)(u / (r.size + 1)) : r.extra + (int)((u - longer) / r.size);
}

// Row of the pool ([n_pages, 64] rows) that holds position pos, -1 if the table has no page of the pool for it.
BPD_HD long long pool_row(int page, int n_pages, int pos) {
  return (page < 0 || page >= n_pages) ? -1 : (long long)page * kPagePos + (pos % kPagePos);
}

// A node's parent, if it lies before the node (the order every valid tree has), else -1: walks up always end.
BPD_HD int parent_of(int parent, int node) { return (parent >= 0 && parent < node) ? parent : -1; }

}  // namespace tree
}  // namespace bpd
