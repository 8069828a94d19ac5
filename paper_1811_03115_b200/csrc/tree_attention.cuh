// Attention of drafted nodes over a paged cache and over their own tree.
//
//   out[t] = sum_s softmax_s(scale q_t . k_s) v_s,   s in {cached positions} + {ancestors of t and t itself}
//
// Either every cached position below the sequence's length counts (dense), or the pages that were selected for the node and
// key head, plus the open page (paged).  One kernel for both: a tile of query rows (nodes x heads of a key head's group when
// dense; the heads of the group of one node when paged) walks chunks of 64 keys -- a page is a chunk, so a chunk has one
// table entry -- with the running maximum and sum of the softmax in registers.  Scores and outputs are mma.sync products.
//
// Work is cut by chunks, not by tiles: the chunks of all tiles of all sequences are laid end to end and every CTA takes an
// equal run of them, so ragged batches and single long sequences fill the device alike.  A run that begins or ends inside a
// tile leaves a partial result (maximum, sum, unnormalised output) in the scratch; combine_kernel joins those.
//
// Precision: bf16 caches: scores are exact products summed in fp32; softmax weights go into the second product as two bf16
// planes (w = h + l, 16 bits of mantissa), so the output's error is its own rounding to bf16 (one plane's rounding would add
// as much again); outputs are summed in the tensor core's 32 bits, whose additions truncate: a run of n chunks loses at most
// n 2^-20 of a sum (8 additions a chunk), 2^-12 for a run of 256, where the output is rounded by up to 2^-8.  fp32 caches: every
// operand is three bf16 planes (24 bits), the six largest of the nine products are taken (the rest is below 2^-24), and outputs
// are summed per chunk in the tensor core but across chunks by fp32 FMAs.
#pragma once
#include "attention.cuh"
#include "cache_index.hpp"

namespace bpd {
namespace tree {

using attn::cp_async16;
using attn::ldsm4;
using attn::mma_bf16;
using attn::s_addr;
using attn::split3_pair;

constexpr int kThreads = 128;
constexpr int kPagesAhead = 64;   // pages looked up at a time
constexpr int kChunk = kPagePos;

// 2 units of error, 0 below the smallest normal number.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct AttnArgs {
  const void *q, *k_new, *v_new, *k_pool, *v_pool;
  const int *table, *lens, *parents, *nodes;   // nodes may be null: T each
  const int* pages;                            // paged: [B][T][Hkv][select], ascending, -1 behind the last
  int B, T, H, Hkv, G, ppr, n_pages, select;
  long long q_stride, kv_stride;               // elements between consecutive nodes
  float scale_log2;                            // scale * log2(e)
  void* out;                                   // [B][T][H][D]
  float* lse;                                  // [B][T][H] or null
  float* part;                                 // [ctas][2][R * (D + 2)]
  int end_units;                               // what the end of a tile costs, in chunks
  int split;                                   // 1: equal runs of chunks, joined by combine_kernel; 0: a tile per CTA
  int part_rows;                               // rows of a partial result
  int ctas;                                    // CTAs of the launch
  int2* info;                                  // per tile: 2 * first CTA that has units of it + the slot of its partial result; last CTA
};

// Shared-memory layout of a chunk's rows.  bf16: panels of up to 64 columns, their 16-byte pieces XOR-swizzled so that eight
// consecutive rows' same piece lies in eight different 16-byte columns of the banks; fp32: padded rows (see attention.cuh).
template <typename CT, int D>
struct Rows {
  static constexpr bool F32 = sizeof(CT) == 4;
  static constexpr int PIECES = D * (int)sizeof(CT) / 16;
  static constexpr int PER = 16 / (int)sizeof(CT);
  static constexpr int KP = D + 8, VP = D + 4;             // fp32 pitches (floats)
  static constexpr int K_BYTES = F32 ? kChunk * KP * 4 : kChunk * D * 2;
  static constexpr int V_BYTES = F32 ? kChunk * VP * 4 : kChunk * D * 2;
  static constexpr int STAGE = K_BYTES + V_BYTES;
  __device__ __forceinline__ static uint32_t swz(int row, int piece) {
    constexpr int ACROSS = PIECES >= 8 ? 8 : PIECES, PER_LINE = 8 / ACROSS;      // pieces of a panel's row, rows of 128 bytes
    return (uint32_t)(piece / ACROSS * kChunk * ACROSS + row * ACROSS + ((piece % ACROSS) ^ ((row / PER_LINE) % ACROSS))) * 16u;
  }
  __device__ __forceinline__ static uint32_t k_at(int row, int piece) { return F32 ? (uint32_t)(row * KP + piece * 4) * 4u : swz(row, piece); }
  __device__ __forceinline__ static uint32_t v_at(int row, int piece) { return F32 ? (uint32_t)(row * VP + piece * 4) * 4u : swz(row, piece); }
};

// WR warps side by side over rows (16 each), 4 / WR over the keys of a chunk.
template <typename CT, int D, int WR>
struct Shape {
  static constexpr bool F32 = sizeof(CT) == 4;
  static constexpr int R = 16 * WR, WK = 4 / WR, KW = kChunk / WK;
  static constexpr int QP = D + 8;                          // pitch of a query plane (bf16 elements), fp32 caches only
  static constexpr int Q_BYTES = F32 ? 3 * R * QP * 2 : 0;
  static constexpr int MP = D + 4;                          // pitch of the merge buffer (floats)
  static constexpr int MERGE = WK * R * MP * 4;
  static constexpr int STAGES = F32 ? (D >= 64 ? 2 : 3) : (D >= 128 ? 3 : 4);
  static constexpr int RING = STAGES * Rows<CT, D>::STAGE;
  static constexpr int SMEM = Q_BYTES + (RING > MERGE ? RING : MERGE);
  // as many as shared memory holds (see tree_attention_kernel); the launch divides the work among all of them
  static constexpr int CTAS_PER_SM = F32 ? (D >= 128 ? 1 : (D >= 64 || WR >= 4 ? 2 : 3)) : (D >= 128 ? 2 : 3);
  // Registers of a third CTA are left free where two leave shared memory too: the joining launch's CTAs then wait on the same SMs
  // (32 rows, 2 heads of 64 over 4 x 2000 positions: 13.8 us, with all registers taken 15.6; with 8 heads over 8 x 4000: 65.9 / 65.3).
  static constexpr bool REGISTERS_FOR_JOIN = F32 && D == 64 && WR < 4;
};

// The nodes' lines as bits: bits[word][t] has those of node t's line among nodes 64 * word ..  By doubling: a node takes over
// what its current forefather has seen and that one's forefather, so a chain of 128 takes 7 rounds (walked up row by row it took
// 9 us).  One warp's work: with four, the barriers of the rounds took 7 us.
struct Lines {
  unsigned long long bits[kMaxNodes / 64][kMaxNodes];
  int up[kMaxNodes];
};
template <int PER>
__device__ __forceinline__ void lines_by_warp(Lines& x, const int* parents, int nodes, int lane) {
  constexpr int W = (PER * 32 + 63) / 64;
  unsigned long long mine[PER][W];
  int up[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int t = lane + k * 32;
    up[k] = t < nodes ? parent_of(parents[t], t) : -1;
#pragma unroll
    for (int w = 0; w < W; ++w) mine[k][w] = t / 64 == w ? 1ull << (t % 64) : 0ull;
  }
  for (int reach = 1; reach < nodes; reach *= 2) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int t = lane + k * 32;
      x.up[t] = up[k];
#pragma unroll
      for (int w = 0; w < W; ++w) x.bits[w][t] = mine[k][w];
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (up[k] < 0) continue;
#pragma unroll
      for (int w = 0; w < W; ++w) mine[k][w] |= x.bits[w][up[k]];
      up[k] = x.up[up[k]];
    }
    const bool done = __all_sync(0xffffffffu, [&] { bool d = true;
#pragma unroll
      for (int k = 0; k < PER; ++k) d = d && up[k] < 0;
      return d; }());
    if (done) break;
    __syncwarp();                                           // (a vote orders no memory: these reads come before the next stores)
  }
  __syncwarp();
#pragma unroll
  for (int k = 0; k < PER; ++k)
#pragma unroll
    for (int w = 0; w < W; ++w) x.bits[w][lane + k * 32] = mine[k][w];
}
__device__ __forceinline__ void find_lines(Lines& x, const int* parents, int nodes, int lane) {
  if (nodes <= 32) lines_by_warp<1>(x, parents, nodes, lane);
  else if (nodes <= 64) lines_by_warp<2>(x, parents, nodes, lane);
  else if (nodes <= 128) lines_by_warp<4>(x, parents, nodes, lane);
  else lines_by_warp<kMaxNodes / 32>(x, parents, nodes, lane);
}

// Floats of a partial result: outputs [rows][D], maxima, sums; whole 16 bytes, as the outputs go there four at a time.
__host__ __device__ __forceinline__ long long part_floats(int rows, int D) { return ((long long)rows * (D + 2) + 3) / 4 * 4; }

struct Seq { int len, nodes; SeqWork w; };

template <bool PAGED>
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int b, int tile_rows) {
  Seq s;
  s.len = clamp_int(a.lens[b], 0, a.ppr * kPagePos);
  s.nodes = a.nodes ? clamp_int(a.nodes[b], 0, a.T) : a.T;
  s.w = PAGED ? paged_work(s.len, s.nodes, a.select, a.Hkv, a.G, tile_rows) : dense_work(s.len, s.nodes, a.Hkv, a.G, tile_rows);
  return s;
}

// Tile `local` of a sequence: node (paged only), key head, first row; and its number among all tiles that could be.
struct Tile { int t, h, r0, id; };
template <bool PAGED>
__device__ __forceinline__ Tile tile_of(const AttnArgs& a, int b, int nodes, int local, int tile_rows) {
  Tile x;
  if (PAGED) {
    const int rt = ceil_div(a.G, tile_rows);
    x.t = local / (a.Hkv * rt);
    x.h = local / rt % a.Hkv;
    x.r0 = local % rt * tile_rows;
    x.id = ((b * a.T + x.t) * a.Hkv + x.h) * rt + local % rt;
  } else {
    const int rt = ceil_div(nodes * a.G, tile_rows), rt_all = ceil_div(a.T * a.G, tile_rows);
    x.t = 0;
    x.h = local / rt;
    x.r0 = local % rt * tile_rows;
    x.id = (b * a.Hkv + x.h) * rt_all + local % rt;
  }
  return x;
}

template <typename CT> __device__ __forceinline__ void store4(CT* p, float4 v);
template <> __device__ __forceinline__ void store4<float>(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
template <> __device__ __forceinline__ void store4<bf16>(bf16* p, float4 v) {
  __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&x), *reinterpret_cast<uint32_t*>(&y));
}

// Two floats as two pairs of bf16, high and low.
__device__ __forceinline__ void split2_pair(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  const __nv_bfloat162 l = __floats2bfloat162_rn(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

// A CTA's way through its work, tile by tile.  Every warp keeps one of its own: what it needs of a batch's lengths a warp
// finds out alone, without a barrier.
template <bool PAGED>
struct Walk {
  const AttnArgs& a;
  const int tile_rows;
  Runs runs;
  long long u_begin, u, u_end, seq_first, tile_first;
  int b;
  Seq sq;
  Tile tl;
  int c_begin, c_end;        // chunks of the tile to work on
  int slot, last_cta;        // of the partial result; the CTA that has the tile's last chunk

  __device__ __forceinline__ Walk(const AttnArgs& args, int rows) : a(args), tile_rows(rows) {}
  __device__ __forceinline__ long long units_of(int i) const {
    const SeqWork w = seq_of<PAGED>(a, i, tile_rows).w;
    return (long long)w.tiles * (w.chunks + a.end_units);
  }
  // False if there is nothing for this CTA.
  __device__ __forceinline__ bool begin() {
    if (!a.split) {
      const int rt = PAGED ? ceil_div(a.G, tile_rows) : ceil_div(a.T * a.G, tile_rows);
      int id = blockIdx.x;
      tl.id = id;
      tl.r0 = id % rt * tile_rows;
      id /= rt;
      tl.h = id % a.Hkv;
      id /= a.Hkv;
      tl.t = PAGED ? id % a.T : 0;
      b = PAGED ? id / a.T : id;
      sq = seq_of<PAGED>(a, b, tile_rows);
      c_begin = 0;
      c_end = sq.w.chunks;
      return PAGED ? tl.t < sq.nodes : tl.r0 < sq.nodes * a.G;
    }
    const int lane = threadIdx.x & 31;
    long long sum = 0;
    for (int i = lane; i < a.B; i += 32) sum += units_of(i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    runs = runs_of(sum, (int)gridDim.x);                    // (no CTA that shares a tile may be without a unit)
    if ((int)blockIdx.x >= runs.ctas) return false;
    u = u_begin = first_unit(runs, blockIdx.x);
    u_end = first_unit(runs, blockIdx.x + 1);
    long long before = 0;
    for (int b0 = 0;; b0 += 32) {
      const long long n = b0 + lane < a.B ? units_of(b0 + lane) : 0;
      long long upto = n;                                   // inclusive scan
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const long long x = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += x; }
      const unsigned hit = __ballot_sync(0xffffffffu, before + upto > u_begin);
      if (hit) {
        const int at = __ffs(hit) - 1;
        b = b0 + at;
        seq_first = before + __shfl_sync(0xffffffffu, upto - n, at);
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    sq = seq_of<PAGED>(a, b, tile_rows);
    find();
    return c_begin < c_end || next();
  }
  // The next tile; false if the CTA's run is done.
  __device__ __forceinline__ bool next() {
    if (!a.split) return false;
    do {
      u = tile_first + sq.w.chunks + a.end_units;
      if (u >= u_end) return false;
      while (u >= seq_first + (long long)sq.w.tiles * (sq.w.chunks + a.end_units)) {
        seq_first += (long long)sq.w.tiles * (sq.w.chunks + a.end_units);
        sq = seq_of<PAGED>(a, ++b, tile_rows);
      }
      find();
    } while (c_begin >= c_end);
    return true;
  }
  // The tile that unit u lies in.  (Its chunks' units come first; a run may have nothing but those of its end.)
  __device__ __forceinline__ void find() {
    const int span = sq.w.chunks + a.end_units;
    const long long into = u - seq_first;
    const int local = into <= 0x7fffffffLL ? (int)((unsigned)into / (unsigned)span) : (int)(into / span);
    tile_first = seq_first + (long long)local * span;
    c_begin = (int)(u - tile_first);
    c_end = (int)min((long long)sq.w.chunks, u_end - tile_first);
    tl = tile_of<PAGED>(a, b, sq.nodes, local, tile_rows);
    slot = u == u_begin ? 0 : 1;                            // a CTA leaves at most two partial results: of its first tile, of its last
    last_cta = c_begin == 0 && c_end < sq.w.chunks ? cta_of_unit(runs, tile_first + sq.w.chunks - 1) : (int)blockIdx.x;
  }
  __device__ __forceinline__ int rows() const { return PAGED ? min(tile_rows, a.G - tl.r0) : min(tile_rows, sq.nodes * a.G - tl.r0); }
  // node and head of row r of the tile, and its row of the output
  __device__ __forceinline__ int node_of(int r) const { return PAGED ? tl.t : (tl.r0 + r) / a.G; }
  __device__ __forceinline__ int head_of(int r) const { return tl.h * a.G + (PAGED ? tl.r0 + r : (tl.r0 + r) % a.G); }
  __device__ __forceinline__ long long out_row(int r) const { return ((long long)b * a.T + node_of(r)) * a.H + head_of(r); }
  __device__ __forceinline__ int cache_chunks() const { return sq.w.chunks - ceil_div(sq.nodes, kChunk); }
  __device__ __forceinline__ bool whole() const { return c_begin == 0 && c_end == sq.w.chunks; }
  // Page of cache chunk c (-1: none, or a chunk of the tree), and the number of keys in a chunk.
  __device__ __forceinline__ int page_of(int c) const {
    const int cached = cache_chunks(), full = sq.len / kPagePos;
    if (c >= cached) return -1;
    int logical = c;
    if (PAGED && c < cached - (sq.len % kPagePos ? 1 : 0)) {
      logical = a.pages[((long long)(b * a.T + tl.t) * a.Hkv + tl.h) * a.select + c];
      if (logical < 0 || logical >= full) return -1;
    } else if (PAGED) {
      logical = full;
    }
    const int page = a.table[(long long)b * a.ppr + logical];
    return pool_row(page, a.n_pages, 0) < 0 ? -1 : page;
  }
  __device__ __forceinline__ int keys_of(int c, int page) const {
    const int cached = cache_chunks();
    if (c >= cached) return min(kChunk, sq.nodes - (c - cached) * kChunk);
    if (page < 0) return 0;
    const bool open = sq.len % kPagePos && c == cached - 1;
    return open ? sq.len % kPagePos : kChunk;
  }
};

// Rows behind a sequence's last node: zeros, and a log-sum of nothing.
template <typename CT>
__device__ __forceinline__ void clear_dead_rows(const AttnArgs& a, int D) {
  if (!a.nodes) return;
  for (int i = blockIdx.x; i < a.B * a.T; i += gridDim.x) {
    if (i % a.T < clamp_int(a.nodes[i / a.T], 0, a.T)) continue;
    CT* o = reinterpret_cast<CT*>(a.out) + (long long)i * a.H * D;
    for (int c = threadIdx.x * 4; c < a.H * D; c += blockDim.x * 4) store4<CT>(o + c, make_float4(0.f, 0.f, 0.f, 0.f));
    if (a.lse) for (int c = threadIdx.x; c < a.H; c += blockDim.x) a.lse[(long long)i * a.H + c] = -INFINITY;
  }
}

// (With the pages of bf16 caches brought by TMA instead of every thread's 16-byte copies, the times were the same to 2 %, and
// the tensor maps cost the host a microsecond a call.)
template <typename CT, int D, int WR, bool PAGED>
__global__ void __launch_bounds__(kThreads, (!PAGED && Shape<CT, D, WR>::REGISTERS_FOR_JOIN ? 3 : Shape<CT, D, WR>::CTAS_PER_SM)) tree_attention_kernel(const __grid_constant__ AttnArgs a) {
  using S = Shape<CT, D, WR>;
  using L = Rows<CT, D>;
  pdl_launch_dependents();
  constexpr bool F32 = S::F32;
  constexpr int R = S::R, WK = S::WK, KW = S::KW, KT = D / 16, NT = KW / 8, DT = D / 8;
  extern __shared__ __align__(128) uint8_t ta_smem[];
  __shared__ int s_keys[S::STAGES], s_pages[kPagesAhead];
  __shared__ Lines s_lines;
  __shared__ float s_m[WK][R], s_l[WK][R];
  static_assert(S::CTAS_PER_SM * (S::SMEM + sizeof(s_keys) + sizeof(s_pages) + sizeof(s_lines) + sizeof(s_m) + sizeof(s_l) + 1024) <= 228 * 1024,
                "the CTAs that share an SM do not fit its shared memory (1 KB of it is the system's, per CTA)");
  bf16* qs = reinterpret_cast<bf16*>(ta_smem);
  uint8_t* ring = ta_smem + S::Q_BYTES;
  const uint32_t ring_s = s_addr(ring);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3;
  const int wr = warp % WR, wk = warp / WR;

  clear_dead_rows<CT>(a, D);
  Walk<PAGED> w(a, R);
  const bool work = w.begin();
  if (PAGED) pdl_wait();                                    // the selection (every CTA: what comes after waits for this launch alone)
  if (!work) return;
  int lines_of = -1;                                        // sequence whose lines are in shared memory
  int n = 0;                                                // chunks so far
  // fp32: planes hold numbers up to 3.39e38 only, larger ones and infinities come out of the products as NaN.  A run of a tile's
  // chunks that ends with such a row is done again `from_numbers`: scores in 64 bits, values by FMAs, 8 to 14 times the time (8 sequences
  // of 4000, 16 rows of 64: 43 us, with an infinite value in each 339).
  bool from_numbers = false;
  for (bool more = true; more;) {
    const int rows = w.rows(), b = w.b, cache_chunks = w.cache_chunks(), c_begin = w.c_begin, c_end = w.c_end;
    auto node_of = [&](int r) { return w.node_of(r); };
    auto head_of = [&](int r) { return w.head_of(r); };
    const Tile& tl = w.tl;
    const Seq& sq = w.sq;
    // Pages of the chunks from c0 on, and a barrier.
    auto look_up = [&](int c0) {
      for (int i = tid; i < kPagesAhead && c0 + i < c_end; i += kThreads) s_pages[i] = w.page_of(c0 + i);
      __syncthreads();
    };
    auto load = [&](int c, int stage) {
      const int page = s_pages[(c - c_begin) % kPagesAhead], n_keys = w.keys_of(c, page);
      const uint32_t ks = ring_s + stage * L::STAGE, vs = ks + L::K_BYTES;
      const bool node = c >= cache_chunks;
      if (tid == 0) s_keys[stage] = n_keys;                 // (read behind the barrier at the chunk's turn)
      const long long at = node ? ((long long)b * a.T + (c - cache_chunks) * kChunk) * a.kv_stride + tl.h * D : ((long long)max(page, 0) * kPagePos * a.Hkv + tl.h) * D;
      const long long step = node ? a.kv_stride : (long long)a.Hkv * D;
      constexpr int PER_PASS = kThreads / L::PIECES;
      const int row = tid / L::PIECES, piece = tid % L::PIECES;
      const CT* k = reinterpret_cast<const CT*>(node ? a.k_new : a.k_pool) + at + row * step + piece * L::PER;
      const CT* v = reinterpret_cast<const CT*>(node ? a.v_new : a.v_pool) + at + row * step + piece * L::PER;
      if (n_keys == kChunk) {
#pragma unroll
        for (int r0 = 0; r0 < kChunk; r0 += PER_PASS) {
          cp_async16(ks + L::k_at(r0 + row, piece), k);
          cp_async16(vs + L::v_at(r0 + row, piece), v);
          k += PER_PASS * step;
          v += PER_PASS * step;
        }
      } else {
        // rows behind the last key are filled with zeros: a weight of 0 times what lies there must be 0
#pragma unroll
        for (int r0 = 0; r0 < kChunk; r0 += PER_PASS) {
          const bool there = r0 + row < n_keys;
          const int bytes = there ? 16 : 0;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ks + L::k_at(r0 + row, piece)), "l"(there ? k + r0 * step : reinterpret_cast<const CT*>(a.k_pool)), "r"(bytes) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(vs + L::v_at(r0 + row, piece)), "l"(there ? v + r0 * step : reinterpret_cast<const CT*>(a.v_pool)), "r"(bytes) : "memory");
        }
      }
    };

    // queries: bf16 fragments in registers, fp32 planes in shared memory
    uint32_t qf[F32 ? 1 : KT][4];
    if constexpr (F32) {
      for (int i = tid; i < R * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) x = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.q) + ((long long)b * a.T + node_of(r)) * a.q_stride + head_of(r) * D + c);
        uint32_t p0[3], p1[3];
        split3_pair(x.x, x.y, p0);
        split3_pair(x.z, x.w, p1);
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(qs + (q * R + r) * S::QP + c) = make_uint2(p0[q], p1[q]);
      }
    } else {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = wr * 16 + g + half * 8;
        const bf16* src = reinterpret_cast<const bf16*>(a.q);
        if (r < rows) src += ((long long)b * a.T + node_of(r)) * a.q_stride + head_of(r) * D;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
          qf[k][half] = r < rows ? *reinterpret_cast<const uint32_t*>(src + k * 16 + t4 * 2) : 0u;
          qf[k][half + 2] = r < rows ? *reinterpret_cast<const uint32_t*>(src + k * 16 + t4 * 2 + 8) : 0u;
        }
      }
    }
    float o[DT][4];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // maxima are of scores times scale_log2

    look_up(c_begin);
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s) {
      if (c_begin + s < c_end) load(c_begin + s, (n + s) % S::STAGES);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // the nodes' lines, where the run reaches the tree (the loop's barrier follows; those of the sequence before have been used)
    if (c_end > cache_chunks && lines_of != b) {
      if (warp == 0) find_lines(s_lines, a.parents + (long long)b * a.T, sq.nodes, lane);
      lines_of = b;
    }
    for (int c = c_begin; c < c_end; ++c, ++n) {
      const int stage = n % S::STAGES;
      asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory");
      __syncthreads();                                      // the chunk is there, and the stage before it has been used
      {
        const int cn = c + S::STAGES - 1;
        if (cn < c_end) {
          if ((cn - c_begin) % kPagesAhead == 0) look_up(cn);
          load(cn, (n + S::STAGES - 1) % S::STAGES);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      const uint8_t* kb = ring + stage * L::STAGE;
      const uint8_t* vb = kb + L::K_BYTES;
      const uint32_t ks = ring_s + stage * L::STAGE, vs = ks + L::K_BYTES;
      const int n_keys = s_keys[stage], key0 = wk * KW;

      // scores of the warp's 16 rows and KW keys
      float s[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
      if (F32 && from_numbers) {
        const int ra = min(wr * 16 + g, rows - 1), rb = min(wr * 16 + g + 8, rows - 1);
        const float* qa = reinterpret_cast<const float*>(a.q) + ((long long)b * a.T + node_of(ra)) * a.q_stride + head_of(ra) * D;
        const float* qb = reinterpret_cast<const float*>(a.q) + ((long long)b * a.T + node_of(rb)) * a.q_stride + head_of(rb) * D;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float* kr = reinterpret_cast<const float*>(kb) + (key0 + i * 8 + t4 * 2 + e) * L::KP;
            double sa = 0., sb = 0.;
#pragma unroll 1
            for (int d = 0; d < D; ++d) { sa += (double)qa[d] * (double)kr[d]; sb += (double)qb[d] * (double)kr[d]; }
            s[i][e] = (float)(sa * (double)a.scale_log2);
            s[i][2 + e] = (float)(sb * (double)a.scale_log2);
          }
      } else if constexpr (F32) {
        // Products one behind the other go to different accumulators (J tiles of keys side by side): a chain on one of them
        // would wait for every product's latency (J = 1 over 8 sequences of 4000, 64 rows: 115 us instead of 109, heads of 128 329 instead of 294).
        constexpr int J = NT < 4 ? NT : 4;
        float lo[NT][4];                                    // the smaller products
#pragma unroll
        for (int i = 0; i < NT; ++i) lo[i][0] = lo[i][1] = lo[i][2] = lo[i][3] = 0.f;
#pragma unroll 2
        for (int k = 0; k < KT; ++k) {
          uint32_t aq[3][4];
#pragma unroll
          for (int q = 0; q < 3; ++q) ldsm4(s_addr(qs + (q * R + wr * 16 + (lane & 15)) * S::QP + k * 16 + (lane >> 4) * 8), aq[q]);
#pragma unroll
          for (int i0 = 0; i0 < NT; i0 += J) {
            uint32_t b0[J][3], b1[J][3];
#pragma unroll
            for (int i = 0; i < J; ++i) {
              const float* kr = reinterpret_cast<const float*>(kb) + (key0 + (i0 + i) * 8 + g) * L::KP + k * 16 + t4 * 2;
              const float2 x = *reinterpret_cast<const float2*>(kr), y = *reinterpret_cast<const float2*>(kr + 8);
              split3_pair(x.x, x.y, b0[i]);
              split3_pair(y.x, y.y, b1[i]);
            }
#pragma unroll
            for (int q = 0; q < 3; ++q)
#pragma unroll
              for (int p = 0; p < 3 - q; ++p)
#pragma unroll
                for (int i = 0; i < J; ++i) mma_bf16(p + q == 0 ? s[i0 + i] : lo[i0 + i], aq[q], b0[i][p], b1[i][p]);
          }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] += lo[i][j];
      } else {
#pragma unroll
        for (int k = 0; k < KT; ++k) {
#pragma unroll
          for (int i = 0; i < NT; i += 2) {
            uint32_t bk[4];
            ldsm4(ks + L::swz(key0 + i * 8 + (lane & 7) + (lane >> 4) * 8, k * 2 + ((lane >> 3) & 1)), bk);
            mma_bf16(s[i], qf[k], bk[0], bk[1]);
            mma_bf16(s[i + 1], qf[k], bk[2], bk[3]);
          }
        }
      }
      if (!F32 || !from_numbers) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[i][j] *= a.scale_log2;
      }

      // what the rows do not see
      if (c >= cache_chunks) {
        const int r0 = wr * 16 + g;
        const unsigned long long line0 = r0 < rows ? s_lines.bits[c - cache_chunks][node_of(r0)] : 0ull;
        const unsigned long long line1 = r0 + 8 < rows ? s_lines.bits[c - cache_chunks][node_of(r0 + 8)] : 0ull;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int key = key0 + i * 8 + t4 * 2 + (j & 1);
            if (!(((j < 2 ? line0 : line1) >> key) & 1)) s[i][j] = -INFINITY;
          }
      } else if (n_keys < kChunk) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) if (key0 + i * 8 + t4 * 2 + (j & 1) >= n_keys) s[i][j] = -INFINITY;
      }

      // running maximum and sum; weights
      float n0 = m0, n1 = m1;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        n0 = fmaxf(n0, fmaxf(s[i][0], s[i][1]));
        n1 = fmaxf(n1, fmaxf(s[i][2], s[i][3]));
      }
#pragma unroll
      for (int off = 1; off < 4; off <<= 1) {
        n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, off));
        n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, off));
      }
      // (a row that has seen nothing keeps a maximum of -inf; its weights are taken against 0 and are 0)
      const float base0 = n0 == -INFINITY ? 0.f : n0, base1 = n1 == -INFINITY ? 0.f : n1;
      const float f0 = exp2f(m0 - base0), f1 = exp2f(m1 - base1);
      m0 = n0; m1 = n1;
      l0 *= f0; l1 *= f1;
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        s[i][0] = exp2f(s[i][0] - base0); s[i][1] = exp2f(s[i][1] - base0);
        s[i][2] = exp2f(s[i][2] - base1); s[i][3] = exp2f(s[i][3] - base1);
        l0 += s[i][0] + s[i][1];
        l1 += s[i][2] + s[i][3];
      }

      // A masked node's values may be infinite or not numbers, and 0 times those is not 0 (in 32 bits, numbers too that the
      // first plane rounds to infinity): where the tree's chunk holds such values, its products are taken one by one, without the
      // keys that the row does not see.
      bool odd = false;
      if (c >= cache_chunks) {
        int bad = 0;
        for (int i = tid; i < n_keys * L::PIECES; i += kThreads) {
          const uint4 v = *reinterpret_cast<const uint4*>(vb + L::v_at(i / L::PIECES, i % L::PIECES));
          const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            bad |= F32 ? (x[e] & 0x7fffffffu) >= 0x7f7f8000u : (x[e] & 0x7f800000u) == 0x7f800000u || (x[e] & 0x7f80u) == 0x7f80u;
        }
        odd = __syncthreads_or(bad) != 0;
      }
      if (odd || (F32 && from_numbers)) {
#pragma unroll
        for (int n = 0; n < DT; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= f1; o[n][3] *= f1; }
        // (a weight may be 0 for a key that the row does see: 0 times what is no number is none)
        const int ra = wr * 16 + g, rb = ra + 8;
        const unsigned long long see0 = c < cache_chunks ? ~0ull : (ra < rows ? s_lines.bits[c - cache_chunks][node_of(ra)] : 0ull);
        const unsigned long long see1 = c < cache_chunks ? ~0ull : (rb < rows ? s_lines.bits[c - cache_chunks][node_of(rb)] : 0ull);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) {
            const float w0 = __shfl_sync(0xffffffffu, s[i][kk & 1], (lane & ~3) | (kk >> 1));
            const float w1 = __shfl_sync(0xffffffffu, s[i][2 + (kk & 1)], (lane & ~3) | (kk >> 1));
            const int r = key0 + i * 8 + kk;
#pragma unroll
            for (int n = 0; n < DT; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int d = n * 8 + t4 * 2 + e;
                float x;
                if (F32) x = *reinterpret_cast<const float*>(vb + (r * L::VP + d) * 4);
                else x = __bfloat162float(*reinterpret_cast<const bf16*>(vb + L::swz(r, d / 8) + (d % 8) * 2));
                if ((see0 >> r) & 1) o[n][e] = fmaf(w0, x, o[n][e]);
                if ((see1 >> r) & 1) o[n][2 + e] = fmaf(w1, x, o[n][2 + e]);
              }
          }
      } else if constexpr (F32) {
        uint32_t wp[NT / 2][4][3];                          // the weights' planes, once for all columns
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) {
          split3_pair(s[2 * k][0], s[2 * k][1], wp[k][0]);
          split3_pair(s[2 * k][2], s[2 * k][3], wp[k][1]);
          split3_pair(s[2 * k + 1][0], s[2 * k + 1][1], wp[k][2]);
          split3_pair(s[2 * k + 1][2], s[2 * k + 1][3], wp[k][3]);
        }
        constexpr int J = DT < 4 ? DT : 4;
#pragma unroll
        for (int n0 = 0; n0 < DT; n0 += J) {
          float acc[J][4], lo[J][4];
#pragma unroll
          for (int n = 0; n < J; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = lo[n][e] = 0.f;
#pragma unroll
          for (int k = 0; k < NT / 2; ++k) {
            uint32_t b0[J][3], b1[J][3];
#pragma unroll
            for (int n = 0; n < J; ++n) {
              const float* vr = reinterpret_cast<const float*>(vb) + (key0 + k * 16 + t4 * 2) * L::VP + (n0 + n) * 8 + g;
              split3_pair(vr[0], vr[L::VP], b0[n]);
              split3_pair(vr[8 * L::VP], vr[9 * L::VP], b1[n]);
            }
#pragma unroll
            for (int q = 0; q < 3; ++q) {
              const uint32_t ap[4] = {wp[k][0][q], wp[k][1][q], wp[k][2][q], wp[k][3][q]};
#pragma unroll
              for (int p = 0; p < 3 - q; ++p)
#pragma unroll
                for (int n = 0; n < J; ++n) mma_bf16(p + q == 0 ? acc[n] : lo[n], ap, b0[n][p], b1[n][p]);
            }
          }
#pragma unroll
          for (int n = 0; n < J; ++n) {
            o[n0 + n][0] = fmaf(o[n0 + n][0], f0, acc[n][0] + lo[n][0]); o[n0 + n][1] = fmaf(o[n0 + n][1], f0, acc[n][1] + lo[n][1]);
            o[n0 + n][2] = fmaf(o[n0 + n][2], f1, acc[n][2] + lo[n][2]); o[n0 + n][3] = fmaf(o[n0 + n][3], f1, acc[n][3] + lo[n][3]);
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < DT; ++n) { o[n][0] *= f0; o[n][1] *= f0; o[n][2] *= f1; o[n][3] *= f1; }
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) {
          uint32_t hi[4], lo[4];
          split2_pair(s[2 * k][0], s[2 * k][1], hi[0], lo[0]);
          split2_pair(s[2 * k][2], s[2 * k][3], hi[1], lo[1]);
          split2_pair(s[2 * k + 1][0], s[2 * k + 1][1], hi[2], lo[2]);
          split2_pair(s[2 * k + 1][2], s[2 * k + 1][3], hi[3], lo[3]);
#pragma unroll
          for (int n = 0; n < DT; n += 2) {
            uint32_t bv[4];
            const uint32_t at = vs + L::swz(key0 + k * 16 + (lane & 15), n + (lane >> 4));
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(bv[0]), "=r"(bv[1]), "=r"(bv[2]), "=r"(bv[3]) : "r"(at) : "memory");
            mma_bf16(o[n], hi, bv[0], bv[1]);
            mma_bf16(o[n + 1], hi, bv[2], bv[3]);
            mma_bf16(o[n], lo, bv[0], bv[1]);
            mma_bf16(o[n + 1], lo, bv[2], bv[3]);
          }
        }
      }
    }

    asm volatile("cp.async.wait_all;" ::: "memory");
    if constexpr (F32) {
      bool bad_a = l0 != l0, bad_b = l1 != l1;
#pragma unroll
      for (int n = 0; n < DT; ++n) {
        bad_a |= o[n][0] != o[n][0] || o[n][1] != o[n][1];
        bad_b |= o[n][2] != o[n][2] || o[n][3] != o[n][3];
      }
      // (a query that is no number has no other result: rows of padding may hold such)
      auto is_number = [&](int r) {
        if (r >= rows) return false;
        const float* q = reinterpret_cast<const float*>(a.q) + ((long long)b * a.T + node_of(r)) * a.q_stride + head_of(r) * D;
        bool is = true;
#pragma unroll 1
        for (int d = 0; d < D; ++d) is = is && q[d] == q[d];
        return is;
      };
      const bool again = !from_numbers && ((bad_a && is_number(wr * 16 + g)) || (bad_b && is_number(wr * 16 + g + 8)));
      from_numbers = __syncthreads_or(again);               // (the ring has been used)
      if (from_numbers) continue;
    } else {
      __syncthreads();
    }

    // join the warps that shared the rows
    l0 += __shfl_xor_sync(0xffffffffu, l0, 1); l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
    l1 += __shfl_xor_sync(0xffffffffu, l1, 1); l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    float* mg = reinterpret_cast<float*>(ring);
    if (t4 == 0) {
      s_m[wk][wr * 16 + g] = m0; s_m[wk][wr * 16 + g + 8] = m1;
      s_l[wk][wr * 16 + g] = l0; s_l[wk][wr * 16 + g + 8] = l1;
    }
#pragma unroll
    for (int n = 0; n < DT; ++n) {
      float* at = mg + (wk * R + wr * 16 + g) * S::MP + n * 8 + t4 * 2;
      *reinterpret_cast<float2*>(at) = make_float2(o[n][0], o[n][1]);
      *reinterpret_cast<float2*>(at + 8 * S::MP) = make_float2(o[n][2], o[n][3]);
    }
    __syncthreads();
    const bool whole = w.whole();
    float* part = a.part + ((long long)blockIdx.x * 2 + (a.split ? w.slot : 0)) * part_floats(a.part_rows, D);
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c4 = i % (D / 4) * 4;
      float m = s_m[0][r];
#pragma unroll
      for (int w = 1; w < WK; ++w) m = fmaxf(m, s_m[w][r]);
      const float base = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < WK; ++w) {
        const float f = exp2f(s_m[w][r] - base);
        const float4 y = *reinterpret_cast<const float4*>(mg + (w * R + r) * S::MP + c4);
        l = fmaf(s_l[w][r], f, l);
        x.x = fmaf(y.x, f, x.x); x.y = fmaf(y.y, f, x.y); x.z = fmaf(y.z, f, x.z); x.w = fmaf(y.w, f, x.w);
      }
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const long long at = w.out_row(r);
        store4<CT>(reinterpret_cast<CT*>(a.out) + at * D + c4, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
        if (a.lse && c4 == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
      } else {
        *reinterpret_cast<float4*>(part + r * D + c4) = x;
        if (c4 == 0) { part[a.part_rows * D + r] = m; part[a.part_rows * (D + 1) + r] = l; }
      }
    }
    if (!a.split) return;
    if (c_begin == 0 && tid == 0) a.info[tl.id] = make_int2(blockIdx.x * 2 + w.slot, w.last_cta);
    __syncthreads();                                        // the ring, the lines and the sums are free again
    more = w.next();
  }
}

// Joins the partial results of the tiles that more than one CTA worked on.  grid: (tiles that could be, rows / (4 / SHARE)):
// SHARE (4 or 1) warps to a row, each of which takes 8 partial results at a time, all loads under way together -- one after the
// other, each would cost a trip to L2.  A row's 33 partial results took a warp alone 4 us; where there are thousands of rows
// they fill the device as it is, and warps that find nothing to do cost more (128 rows of 512 tiles: 75 us more).
template <typename CT, int D, bool PAGED, int SHARE>
__global__ void __launch_bounds__(kThreads) combine_kernel(const __grid_constant__ AttnArgs a, int tile_rows) {
  pdl_wait();                                               // (every CTA: the launch after this one waits for this one alone)
  // a lane has 4 columns (D = 128), 2 (64) or 1
  constexpr int E = D >= 64 ? D / 32 : 1, WARPS = kThreads / 32, PER = 8;
  __shared__ float s_m[WARPS], s_l[WARPS], s_x[SHARE > 1 ? WARPS : 1][32 * E];
  const int R = tile_rows, PR = a.part_rows;
  const int id = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = blockIdx.y * (WARPS / SHARE) + warp / SHARE;
  int b, h, t, r0;
  if (PAGED) {
    const int rt = ceil_div(a.G, R);
    r0 = id % rt * R; h = id / rt % a.Hkv; t = id / rt / a.Hkv % a.T; b = id / rt / a.Hkv / a.T;
  } else {
    const int rt = ceil_div(a.T * a.G, R);
    r0 = id % rt * R; h = id / rt % a.Hkv; b = id / rt / a.Hkv; t = 0;
  }
  const int2 who = a.info[id];
  const int nodes = a.nodes ? clamp_int(a.nodes[b], 0, a.T) : a.T;
  const int rows = PAGED ? (t < nodes ? a.G : 0) : nodes * a.G;
  if (r0 + r >= rows) return;
  const int node = PAGED ? t : (r0 + r) / a.G, head = h * a.G + (PAGED ? r0 + r : (r0 + r) % a.G);
  // (a tile that no CTA began -- a wait that expired -- has any number here)
  if (who.x < 0 || (who.x >> 1) >= who.y || who.y >= a.ctas) return;
  const int col = lane * E, first = who.x >> 1, n = who.y - first + 1;
  // all CTAs but the first begin their run inside the tile
  auto part_of = [&](int i) { return a.part + ((long long)(first + i) * 2 + (i == 0 ? (who.x & 1) : 0)) * part_floats(PR, D); };
  float m = -INFINITY, l = 0.f, x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.f;
  for (int i0 = warp % SHARE * PER; i0 < n; i0 += SHARE * PER) {
    float pm[PER], pl[PER], y[PER][E];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool has = i0 + j < n;
      const float* src = part_of(has ? i0 + j : i0);
      pm[j] = has ? src[PR * D + r] : -INFINITY;
      pl[j] = src[PR * (D + 1) + r];
      src += r * D + (col < D ? col : 0);
      if constexpr (E == 4) *reinterpret_cast<float4*>(y[j]) = *reinterpret_cast<const float4*>(src);
      else if constexpr (E == 2) *reinterpret_cast<float2*>(y[j]) = *reinterpret_cast<const float2*>(src);
      else y[j][0] = *src;
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < PER; ++j) top = fmaxf(top, pm[j]);
    const float base = top == -INFINITY ? 0.f : top, f = exp2f(m - base);
    m = top;
    l *= f;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= f;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const bool has = i0 + j < n;                          // (selected here, not branched on: the loads stay side by side)
      const float w = exp2f(pm[j] - base);
      l = fmaf(has ? pl[j] : 0.f, w, l);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(has ? y[j][e] : 0.f, w, x[e]);
    }
  }
  if constexpr (SHARE > 1) {
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
    for (int e = 0; e < E; ++e) s_x[warp][lane * E + e] = x[e];
    __syncthreads();
    if (warp > 0) return;
    m = s_m[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) m = fmaxf(m, s_m[w]);
    const float base = m == -INFINITY ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = exp2f(s_m[w] - base);
      l = fmaf(s_l[w], f, l);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = fmaf(s_x[w][lane * E + e], f, x[e]);
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const long long at = ((long long)b * a.T + node) * a.H + head;
  if (col < D) {
#pragma unroll
    for (int e = 0; e < E; ++e) reinterpret_cast<CT*>(a.out)[at * D + col + e] = from_f<CT>(x[e] * inv);
  }
  if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
}

}  // namespace tree
}  // namespace bpd
