// Operators on a paged cache beside its attention: commit of an accepted path, accumulated attention weights, eviction,
// page means, selection of pages.
#pragma once
#include "tree_attention.cuh"

namespace bpd {
namespace tree {

__device__ __forceinline__ unsigned long long order_bits64(double v) {
  const unsigned long long b = (unsigned long long)__double_as_longlong(v);
  return (b >> 63) ? ~b : (b | (1ull << 63));
}

// ------------------------------------------------------------------ commit of the accepted path
struct CommitArgs {
  const void *k_new, *v_new;          // [layers][B][T] rows of Hkv * D, kv_stride elements apart
  void *k_pool, *v_pool;              // [layers][n_pages][64][Hkv * D]
  const int *table, *lens, *parents, *tokens, *top1, *last_top1, *nodes;
  int layers, B, T, row_pieces, ppr, n_pages, eos, elem;   // row_pieces: 16-byte pieces of a position's keys
  long long kv_stride;
  int *out_lens, *accepted, *path, *next;
};

// grid (B, splits).  Every CTA walks the tree itself (a few steps over arrays in shared memory), then copies its share of
// the accepted rows; the first CTA of a sequence writes the walk down.  Bound by launch and walk latency: a batch of 24
// over 24 layers moves 19 MB.
constexpr int kCommitThreads = 256;
__global__ void __launch_bounds__(kCommitThreads) tree_commit_kernel(const __grid_constant__ CommitArgs a) {
  __shared__ int s_parent[kMaxNodes], s_token[kMaxNodes], s_top1[kMaxNodes], s_path[kMaxNodes], s_row[kMaxNodes], s_n;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31;
  const int nodes = a.nodes ? clamp_int(a.nodes[b], 0, a.T) : a.T;
  // (a length that cannot be takes nothing: a path would be written over what is there)
  const int cap = a.ppr * kPagePos, given = a.lens[b], len = clamp_int(given, 0, cap), room = given < 0 ? 0 : cap - len;
  for (int i = tid; i < nodes; i += kCommitThreads) {
    s_parent[i] = a.parents[(long long)b * a.T + i];
    s_token[i] = a.tokens[(long long)b * a.T + i];
    s_top1[i] = a.top1[(long long)b * a.T + i];
  }
  __syncthreads();
  if (tid < 32) {
    int at = -1, want = a.last_top1[b], n = 0;
    while (n < room) {
      // the lowest child that carries the wanted token; children lie behind their parent, so the walk ends
      int child = -1;
      for (int i0 = (at + 1) & ~31; i0 < nodes; i0 += 32) {
        const int i = i0 + lane;
        const unsigned hit = __ballot_sync(0xffffffffu, i < nodes && i > at && parent_of(s_parent[i < nodes ? i : 0], i) == at && s_token[i < nodes ? i : 0] == want);
        if (hit) { child = i0 + __ffs(hit) - 1; break; }
      }
      if (child < 0) break;
      if (lane == 0) {
        const int pos = len + n;
        s_path[n] = child;
        s_row[n] = (int)pool_row(a.table[(long long)b * a.ppr + pos / kPagePos], a.n_pages, pos);
      }
      ++n;
      at = child;
      want = s_top1[child];
      if (a.eos >= 0 && s_token[child] == a.eos) break;
    }
    if (lane == 0) {
      s_n = n;
      if (blockIdx.y == 0) {
        a.out_lens[b] = len + n;
        a.accepted[b] = n;
        a.next[b] = want;
      }
    }
  }
  __syncthreads();
  const int n = s_n;
  if (blockIdx.y == 0)
    for (int i = tid; i < a.T; i += kCommitThreads) a.path[(long long)b * a.T + i] = i < n ? s_path[i] : -1;
  const int per_layer = 2 * n * a.row_pieces, total = a.layers * per_layer;
  for (int i = blockIdx.y * kCommitThreads + tid; i < total; i += gridDim.y * kCommitThreads) {
    const int layer = i / per_layer, rest = i % per_layer, which = rest / (n * a.row_pieces), j = rest / a.row_pieces % n, piece = rest % a.row_pieces;
    if (s_row[j] < 0) continue;
    const long long per = 16 / a.elem;
    const long long from = (((long long)layer * a.B + b) * a.T + s_path[j]) * a.kv_stride + piece * per;
    const long long to = ((long long)layer * a.n_pages * kPagePos + s_row[j]) * a.row_pieces + piece;
    const char* src = reinterpret_cast<const char*>(which ? a.v_new : a.k_new) + from * a.elem;
    reinterpret_cast<uint4*>(which ? a.v_pool : a.k_pool)[to] = *reinterpret_cast<const uint4*>(src);
  }
}

// ------------------------------------------------------------------ accumulated attention weights
struct WeightArgs {
  const void *q, *k_pool;
  const float* lse;                    // [B][T][H]
  const int *path, *accepted, *lens, *seen, *table;
  int B, T, H, Hkv, G, ppr, n_pages;
  long long q_stride;
  float scale_log2;                    // scale * log2(e)
  float* weights;                      // [B][Hkv][ppr * 64]
  int* positions;
};

// weights[s] += sum over accepted nodes i and heads of exp(scale q . k_s - lse), s <= len + i.
//
// A product with keys on M and (node, head) rows on N whose result is summed over N: no key depends on another, so a warp
// streams 16 keys straight from global memory into fragments (the order of the products' k is free as long as both operands
// agree: a thread takes 16 contiguous bytes) and no key passes through shared memory.  Queries are staged once per CTA.
// Pages of all (sequence, key head) pairs are laid end to end and every CTA takes an equal run of them (with 8 pages a CTA, the
// queries' way into shared memory took as long as the keys).  Bound by reading the keys.
constexpr int kWThreads = 256;
template <typename CT, int D>
struct WShape {
  static constexpr bool F32 = sizeof(CT) == 4;
  static constexpr int PLANES = F32 ? 3 : 1;
  static constexpr int VEC = D >= 32 ? 8 : 4;                      // elements of k a thread takes at once
  static constexpr int STEPS = D / (VEC * 4);                      // such takes per key
  static constexpr int QP = D >= 64 ? D + 32 : (D == 32 ? 32 : 24);   // bf16 elements: two rows' pieces in different banks
  static constexpr int ROWS = F32 ? 32 : 64;                       // (node, head) rows staged at a time
};
template <typename CT, int D>
__global__ void __launch_bounds__(kWThreads) cache_weights_kernel(const __grid_constant__ WeightArgs a) {
  using W = WShape<CT, D>;
  constexpr int VEC = W::VEC, PL = W::PLANES;
  __shared__ __align__(16) bf16 s_q[PL * W::ROWS * W::QP];
  __shared__ __align__(8) float s_hi[W::ROWS], s_lo[W::ROWS];      // log2(e) lse in two parts: its rounding would weigh on every weight alike
  __shared__ int s_step[W::ROWS];                                  // index on the path: the row sees positions <= len + it
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t4 = lane & 3, cap = a.ppr * kPagePos;
  auto length = [&](int b) { return clamp_int(a.lens[b], 0, cap); };
  auto taken = [&](int b, int len) { return clamp_int(a.accepted[b], 0, min(a.T, cap - len)); };
  auto pages_of = [&](int b) { const int len = length(b), got = taken(b, len); return got ? ceil_div(len + got, kPagePos) : 0; };
  // this CTA's run of pages (every warp finds it out alone)
  long long sum = 0;
  for (int i = lane; i < a.B; i += 32) sum += (long long)pages_of(i) * a.Hkv;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const Runs runs = runs_of(sum, (int)gridDim.x);
  if ((int)blockIdx.x >= runs.ctas) return;
  long long u = first_unit(runs, blockIdx.x), seq_first = 0;
  const long long u_end = first_unit(runs, blockIdx.x + 1);
  int b = 0;
  for (int b0 = 0;; b0 += 32) {
    const long long n = b0 + lane < a.B ? (long long)pages_of(b0 + lane) * a.Hkv : 0;
    long long upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const long long x = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += x; }
    const unsigned hit = __ballot_sync(0xffffffffu, seq_first + upto > u);
    if (hit) {
      const int at = __ffs(hit) - 1;
      b = b0 + at;
      seq_first += __shfl_sync(0xffffffffu, upto - n, at);
      break;
    }
    seq_first += __shfl_sync(0xffffffffu, upto, 31);
  }
  int pages = pages_of(b);
  while (u < u_end) {
    while (u >= seq_first + (long long)pages * a.Hkv) {
      seq_first += (long long)pages * a.Hkv;
      pages = pages_of(++b);
    }
    const int into = (int)(u - seq_first), h = into / pages, p_begin = into % pages, p_end = (int)min((long long)pages, p_begin + (u_end - u));
    u += p_end - p_begin;
    const int len = length(b), got = taken(b, len), total = len + got, rows = got * a.G;
    float* wout = a.weights + ((long long)b * a.Hkv + h) * cap;
    int* pout = a.positions + ((long long)b * a.Hkv + h) * cap;
    for (int r0 = 0; r0 < rows; r0 += W::ROWS) {
      const int n = min(W::ROWS, rows - r0), n8 = (n + 7) & ~7;
      __syncthreads();
      for (int i = tid; i < n8 * (D / 4); i += kWThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (r < n) {
          const int node = clamp_int(a.path[(long long)b * a.T + (r0 + r) / a.G], 0, a.T - 1), head = h * a.G + (r0 + r) % a.G;
          const CT* src = reinterpret_cast<const CT*>(a.q) + ((long long)b * a.T + node) * a.q_stride + head * D + c;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = to_f(src[e]);
          if (c == 0) {
            const float lse = a.lse[((long long)b * a.T + node) * a.H + head], hi = lse * 1.44269504f;
            s_hi[r] = hi;
            s_lo[r] = fabsf(hi) < INFINITY ? fmaf(lse, 1.44269504f, -hi) + lse * 1.92596299e-8f : 0.f;
            s_step[r] = (r0 + r) / a.G;
          }
        } else if (c == 0) {
          s_hi[r] = s_lo[r] = 0.f; s_step[r] = 0;                    // padding: add_up leaves these rows out
        }
        if constexpr (W::F32) {
          uint32_t x[3], y[3];
          attn::split3_pair(v[0], v[1], x);
          attn::split3_pair(v[2], v[3], y);
#pragma unroll
          for (int q = 0; q < 3; ++q) *reinterpret_cast<uint2*>(s_q + (q * W::ROWS + r) * W::QP + c) = make_uint2(x[q], y[q]);
        } else {
          *reinterpret_cast<uint2*>(s_q + r * W::QP + c) = make_uint2(attn::pack2(from_f<bf16>(v[0]), from_f<bf16>(v[1])), attn::pack2(from_f<bf16>(v[2]), from_f<bf16>(v[3])));
        }
      }
      __syncthreads();
      // keys of a tile: [take][row half]; 16 (or 8) bytes a take
      struct Keys { uint32_t v[W::STEPS][2][VEC * (int)sizeof(CT) / 4]; bool ok[2]; };
      const int t_end = min(p_end * 4, (total + 15) / 16);
      auto look_up = [&](int tile) { return tile < t_end ? a.table[(long long)b * a.ppr + tile / 4] : -1; };
      auto fetch = [&](int tile, int page, Keys& k) {
        const int pos0 = tile * 16;
        const long long row = pool_row(page, a.n_pages, pos0);
        const CT* kp = reinterpret_cast<const CT*>(a.k_pool) + ((row < 0 ? 0 : row) * a.Hkv + h) * D;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          k.ok[half] = tile < t_end && row >= 0 && pos0 + g + half * 8 < total;
#pragma unroll
          for (int st = 0; st < W::STEPS; ++st) {
            const CT* src = kp + (long long)(g + half * 8) * a.Hkv * D + (t4 + 4 * st) * VEC;
            constexpr int WORDS = VEC * (int)sizeof(CT) / 4;
            if constexpr (WORDS == 2) {
              *reinterpret_cast<uint2*>(k.v[st][half]) = k.ok[half] ? *reinterpret_cast<const uint2*>(src) : make_uint2(0u, 0u);
            } else {
#pragma unroll
              for (int e = 0; e < WORDS; e += 4)
                *reinterpret_cast<uint4*>(&k.v[st][half][e]) = k.ok[half] ? reinterpret_cast<const uint4*>(src)[e / 4] : make_uint4(0u, 0u, 0u, 0u);
            }
          }
        }
      };
      auto add_up = [&](int tile, const Keys& keys) {
        const int pos0 = tile * 16;
        float sum0 = 0.f, sum1 = 0.f;
        for (int n0 = 0; n0 < n8; n0 += 8) {
          float c[4] = {0.f, 0.f, 0.f, 0.f}, lo[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int st = 0; st < W::STEPS; ++st) {
            uint32_t qf[PL][VEC / 2];
#pragma unroll
            for (int q = 0; q < PL; ++q) {
              const bf16* src = s_q + (q * W::ROWS + n0 + g) * W::QP + (t4 + 4 * st) * VEC;
              if constexpr (VEC == 8) {
                const uint4 v = *reinterpret_cast<const uint4*>(src);
                qf[q][0] = v.x; qf[q][1] = v.y; qf[q][2] = v.z; qf[q][3] = v.w;
              } else {
                const uint2 v = *reinterpret_cast<const uint2*>(src);
                qf[q][0] = v.x; qf[q][1] = v.y;
              }
            }
            uint32_t kf[PL][2][VEC / 2];                             // [plane][row half][pairs]
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int e = 0; e < VEC / 2; ++e) {
                if constexpr (W::F32) {
                  uint32_t x[3];
                  attn::split3_pair(__uint_as_float(keys.v[st][half][2 * e]), __uint_as_float(keys.v[st][half][2 * e + 1]), x);
#pragma unroll
                  for (int q = 0; q < PL; ++q) kf[q][half][e] = x[q];
                } else {
                  kf[0][half][e] = keys.v[st][half][e];
                }
              }
#pragma unroll
            for (int k = 0; k < VEC / 4; ++k)
#pragma unroll
              for (int p = 0; p < PL; ++p) {
                const uint32_t aq[4] = {kf[p][0][2 * k], kf[p][1][2 * k], kf[p][0][2 * k + 1], kf[p][1][2 * k + 1]};
#pragma unroll
                for (int q = 0; q < PL - p; ++q) attn::mma_bf16(p + q == 0 ? c : lo, aq, qf[q][2 * k], qf[q][2 * k + 1]);
              }
          }
          const float2 hi = *reinterpret_cast<const float2*>(s_hi + n0 + t4 * 2), low = *reinterpret_cast<const float2*>(s_lo + n0 + t4 * 2);
          float e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = exp2_fast(fmaf(c[j] + lo[j], a.scale_log2, -(j & 1 ? hi.y : hi.x)) - (j & 1 ? low.y : low.x));
          if (pos0 + 16 > len) {                                   // entries of this commit: rows before them do not see them
            const int pos = pos0 + g, step0 = s_step[n0 + t4 * 2], step1 = s_step[n0 + t4 * 2 + 1];
            if (pos > len + step0) e[0] = 0.f;
            if (pos > len + step1) e[1] = 0.f;
            if (pos + 8 > len + step0) e[2] = 0.f;
            if (pos + 8 > len + step1) e[3] = 0.f;
          }
          if (n0 + 8 > n) {                                        // rows of padding: their zeros times an infinite key are no numbers
            if (n0 + t4 * 2 >= n) e[0] = e[2] = 0.f;
            if (n0 + t4 * 2 + 1 >= n) e[1] = e[3] = 0.f;
          }
          sum0 += e[0] + e[1];
          sum1 += e[2] + e[3];
        }
        if constexpr (W::F32) {
          // Planes hold numbers up to 3.39e38 only: larger ones and infinities (0 or not a number in the planes behind the first)
          // make a score that is no number.  Such a tile's scores are taken again in 64 bits, from the numbers themselves.
          if (__any_sync(0xffffffffu, sum0 != sum0 || sum1 != sum1)) {
            sum0 = sum1 = 0.f;
            for (int r = 0; r < n; ++r) {
              const int node = clamp_int(a.path[(long long)b * a.T + (r0 + r) / a.G], 0, a.T - 1);
              const float* src = reinterpret_cast<const float*>(a.q) + ((long long)b * a.T + node) * a.q_stride + (h * a.G + (r0 + r) % a.G) * D;
              double c[2] = {0., 0.};
#pragma unroll
              for (int st = 0; st < W::STEPS; ++st)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                  const double x = src[(t4 + 4 * st) * VEC + e];
#pragma unroll
                  for (int half = 0; half < 2; ++half) c[half] += x * (double)__uint_as_float(keys.v[st][half][e]);
                }
              float w[2];
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                c[half] += __shfl_xor_sync(0xffffffffu, c[half], 1);
                c[half] += __shfl_xor_sync(0xffffffffu, c[half], 2);
                w[half] = pos0 + g + half * 8 > len + s_step[r] ? 0.f : exp2_fast((float)(c[half] * (double)a.scale_log2 - (double)s_hi[r] - (double)s_lo[r]));
              }
              if (t4 == 0) { sum0 += w[0]; sum1 += w[1]; }
            }
          }
        }
        sum0 += __shfl_xor_sync(0xffffffffu, sum0, 1); sum0 += __shfl_xor_sync(0xffffffffu, sum0, 2);
        sum1 += __shfl_xor_sync(0xffffffffu, sum1, 1); sum1 += __shfl_xor_sync(0xffffffffu, sum1, 2);
        if (t4 < 2) {
          const int pos = pos0 + g + t4 * 8;
          const float add = t4 ? (keys.ok[1] ? sum1 : 0.f) : (keys.ok[0] ? sum0 : 0.f);
          if (pos < total) {
            // entries of this commit begin here: nothing of what the slot held before counts
            wout[pos] = pos < len || r0 > 0 ? wout[pos] + add : add;
            if (pos >= len && r0 == 0) pout[pos] = a.seen[b] + pos - len;
          }
        }
      };
      constexpr int STEP = kWThreads / 32;
      int tile = p_begin * 4 + warp, page = look_up(tile);
      if constexpr (W::F32) {
        for (; tile < t_end; tile += STEP) {
          const int next = look_up(tile + STEP);
          Keys k;
          fetch(tile, page, k);
          add_up(tile, k);
          page = next;
        }
      } else {
        // one tile's keys are on their way while the other's are used
        Keys k0, k1;
        fetch(tile, page, k0);
        page = look_up(tile + STEP);
        for (; tile < t_end; tile += 2 * STEP) {
          fetch(tile + STEP, page, k1);
          page = look_up(tile + 2 * STEP);
          add_up(tile, k0);
          fetch(tile + 2 * STEP, page, k0);
          page = look_up(tile + 3 * STEP);
          if (tile + STEP < t_end) add_up(tile + STEP, k1);
        }
      }
    }
  }
}

// ------------------------------------------------------------------ eviction
struct EvictArgs {
  void *k_pool, *v_pool;               // [layers][n_pages][64][Hkv][D]
  const int *table, *lens, *seen;
  int layers, B, Hkv, row_pieces, ppr, n_pages, budget, recent;   // row_pieces: 16-byte pieces of a head's keys, a power of two
  float* weights;                      // [layers][B][Hkv][ppr * 64]
  int* positions;
  int* out_lens;
  int2* moves;                         // scratch: [layers * B * Hkv][moves_cap] rows of the layer's pool (to, from), -1: no page there
  int* counts;                         // scratch: [layers * B * Hkv] of them
  int moves_cap;
  int move_here;                       // 1: the selecting CTA moves the rows itself
};

// The rows of a list's moves, warp `first` of `step`.  Sources lie at or above the budget, targets below it: no row is read
// after it was written, in whatever order they move.  A warp fetches up to 32 moves at once and then has eight 16-byte pieces a lane
// under way (with every piece looking up its move and its pages, 3 trips to memory one behind the other, 256 lists of 850 moves
// took 73 us instead of 38).
__device__ __forceinline__ void move_rows(const EvictArgs& a, int list, int n, int first, int step) {
  const int h = list % a.Hkv, layer = list / a.Hkv / a.B, lane = threadIdx.x & 31;
  const int2* moves = a.moves + (long long)list * a.moves_cap;
  const int pieces = 2 * a.row_pieces, shift = 31 - __clz(pieces);   // of an entry, keys and values
  const long long layer_rows = (long long)layer * a.n_pages * kPagePos;
  constexpr int AT_ONCE = 8;
  const int per = min(32, (n + step - 1) / step);           // entries of a warp
  for (int j0 = first * per; j0 < n; j0 += step * per) {
    const int2 mine = lane < per && j0 + lane < n ? moves[j0 + lane] : make_int2(-1, -1);
    for (int u0 = 0; u0 * 32 < per * pieces; u0 += AT_ONCE) {
      uint4 x[AT_ONCE];
      uint4* to[AT_ONCE];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        const int i = (u0 + k) * 32 + lane, entry = (i >> shift) & 31, rest = i & (pieces - 1);
        const int rt = __shfl_sync(0xffffffffu, mine.x, entry), rf = __shfl_sync(0xffffffffu, mine.y, entry);
        uint4* pool = reinterpret_cast<uint4*>(rest < a.row_pieces ? a.k_pool : a.v_pool) + (rest & (a.row_pieces - 1));
        to[k] = nullptr;
        if (i < per * pieces && rt >= 0 && rf >= 0) {
          to[k] = pool + ((layer_rows + rt) * a.Hkv + h) * a.row_pieces;
          x[k] = pool[((layer_rows + rf) * a.Hkv + h) * a.row_pieces];
        }
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) if (to[k]) *to[k] = x[k];
    }
  }
}

// Selection, a CTA per list (layer, sequence, key head).  An entry's key is its weight as a number whose unsigned order is the
// order of eviction (-0 like 0); NaN is 1, below every number; entries that stay whatever their weight (recent ones, where they
// fit the budget) have all bits set, those that leave whatever theirs (what is not recent, where they do not) have 0.  The
// border is found bit by bit: a candidate stands if at least `budget` keys are not below it, and ends the search where it is
// exactly so many.  A candidate costs one barrier (a radix selection with its histograms and scans took 26 us for 522 entries).
// Ordered scans then list the holes below the budget and the survivors above it.
//
// KEPT keys a thread stay in registers: 16 (lists of up to 8192 slots, two CTAs to an SM) or 32; what is behind them is read
// anew for every candidate.
constexpr int kEvictThreads = 512;
__device__ __forceinline__ unsigned evict_key(float w) { return w != w ? 1u : order_bits(w + 0.f); }
__device__ __forceinline__ unsigned evict_key_of(unsigned key, bool recent, bool recents_stay) {
  return recent == recents_stay ? (recent ? 0xffffffffu : 0u) : key;
}
template <int KEPT>
__global__ void __launch_bounds__(kEvictThreads, KEPT <= 16 ? 2 : 1) cache_evict_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int WARPS = kEvictThreads / 32, SPAN = kEvictThreads * KEPT;
  __shared__ __align__(16) int s_warp[2][WARPS];
  __shared__ int s_at[2][KEPT * WARPS], s_sum[2];
  pdl_launch_dependents();
  const int list = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = list % a.Hkv, b = list / a.Hkv % a.B, layer = list / a.Hkv / a.B;
  const int cap = a.ppr * kPagePos, len = clamp_int(a.lens[b], 0, cap);
  if (layer == 0 && h == 0 && tid == 0) a.out_lens[b] = min(len, a.budget);
  if (len <= a.budget) {
    if (tid == 0) a.counts[list] = 0;
    return;
  }
  float* w = a.weights + (long long)list * cap;
  int* pos = a.positions + (long long)list * cap;
  const long long recent_from = (long long)a.seen[b] - a.recent;
  int turn = 0;
  auto total = [&](int v) {                                // sum over the block
    v = __reduce_add_sync(0xffffffffu, v);
    int* box = s_warp[turn++ & 1];                         // (alternating: one barrier is enough)
    if (lane == 0) box[warp] = v;
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < WARPS; i += 4) { const int4 x = *reinterpret_cast<const int4*>(box + i); sum += (x.x + x.y) + (x.z + x.w); }
    return sum;
  };
  unsigned kept[KEPT], recent = 0;                         // bit k of recent: the entry of turn k is
  const int turns = (min(len, SPAN) + kEvictThreads - 1) / kEvictThreads;
  auto load = [&](int base) {
    recent = 0;
    float wv[4];
    int pv[4];
#pragma unroll
    for (int k0 = 0; k0 < KEPT; k0 += 4) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int i = base + tid + (k0 + k) * kEvictThreads;
        wv[k] = i < len ? w[i] : 0.f;
        pv[k] = i < len ? pos[i] : 0;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        kept[k0 + k] = evict_key(wv[k]);
        if (base + tid + (k0 + k) * kEvictThreads < len && pv[k] >= recent_from) recent |= 1u << (k0 + k);
      }
    }
  };
  load(0);
  int mine = __popc(recent);
  for (int i = SPAN + tid; i < len; i += kEvictThreads) mine += pos[i] >= recent_from;
  const bool recents_stay = total(mine) < a.budget;
  auto settle = [&](int base) {                            // what is not there has key 0
#pragma unroll
    for (int k = 0; k < KEPT; ++k)
      kept[k] = base + tid + k * kEvictThreads < len ? evict_key_of(kept[k], (recent >> k) & 1, recents_stay) : 0u;
  };
  settle(0);
  auto count = [&](unsigned x) {                           // keys that are at least x (x > 0)
    int n = 0;
#pragma unroll
    for (int k = 0; k < KEPT; ++k) n += kept[k] >= x;
    for (int i = SPAN + tid; i < len; i += kEvictThreads) n += evict_key_of(evict_key(w[i]), pos[i] >= recent_from, recents_stay) >= x;
    return total(n);
  };
  unsigned border = 0;
  bool exact = false;
  for (int bit = 31; bit >= 0 && !exact; --bit) {
    const unsigned candidate = border | (1u << bit);
    const int n = count(candidate);
    if (n >= a.budget) border = candidate;
    exact = n == a.budget;
  }
  // of the entries equal to the border the lowest slots stay (there is one that leaves: the border is not all bits)
  const int room = exact ? len : a.budget - count(border + 1);
  int2* moves = a.moves + (long long)list * a.moves_cap;
  int ties = 0, n_holes = 0, n_fill = 0;
  // Entries are numbered in order: the counts of all turns and warps are scanned by one warp, in place.
  auto scan = [&](int which, int n_turns) {
    int run = 0;
    for (int i = lane; i - lane < n_turns * WARPS; i += 32) {
      const int v = i < n_turns * WARPS ? s_at[which][i] : 0;
      int upto = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, upto, o); if (lane >= o) upto += x; }
      if (i < n_turns * WARPS) s_at[which][i] = run + upto - v;
      run += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) s_sum[which] = run;
  };
  const unsigned before = (1u << lane) - 1;
  for (int base = 0; base < len; base += SPAN) {
    if (base > 0) {
      load(base);
      settle(base);
    }
    const int n_turns = base == 0 ? turns : (min(len - base, SPAN) + kEvictThreads - 1) / kEvictThreads;
    unsigned stays = 0;                                    // bit k: the entry of turn k
    if (!exact) {
#pragma unroll
      for (int k = 0; k < KEPT; ++k) {
        if (k >= n_turns) break;
        const unsigned m = __ballot_sync(0xffffffffu, kept[k] == border && base + tid + k * kEvictThreads < len);
        if (lane == 0) s_at[0][k * WARPS + warp] = __popc(m);
      }
      __syncthreads();
      if (warp == 0) scan(0, n_turns);
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
      if (k >= n_turns) break;
      const bool tie = kept[k] == border && base + tid + k * kEvictThreads < len;
      const unsigned m = __ballot_sync(0xffffffffu, tie);
      const bool in = kept[k] > border || (tie && (exact || ties + s_at[0][k * WARPS + warp] + __popc(m & before) < room));
      if (in) stays |= 1u << k;
    }
    if (!exact) ties += s_sum[0];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
      if (k >= n_turns) break;
      const int i = base + tid + k * kEvictThreads;
      const bool in = (stays >> k) & 1;
      const unsigned holes = __ballot_sync(0xffffffffu, i < a.budget && !in), fill = __ballot_sync(0xffffffffu, i >= a.budget && in);
      if (lane == 0) { s_at[0][k * WARPS + warp] = __popc(holes); s_at[1][k * WARPS + warp] = __popc(fill); }
    }
    __syncthreads();
    if (warp < 2) scan(warp, n_turns);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < KEPT; ++k) {
      if (k >= n_turns) break;
      const int i = base + tid + k * kEvictThreads;
      const bool in = (stays >> k) & 1, hole = i < a.budget && !in, filler = i >= a.budget && in;
      const unsigned holes = __ballot_sync(0xffffffffu, hole), fill = __ballot_sync(0xffffffffu, filler);
      if (hole) moves[n_holes + s_at[0][k * WARPS + warp] + __popc(holes & before)].x = i;
      if (filler) moves[n_fill + s_at[1][k * WARPS + warp] + __popc(fill & before)].y = i;
    }
    n_holes += s_sum[0];
    n_fill += s_sum[1];
    __syncthreads();
  }
  // (as many of one as of the other: `budget` entries stay)
  const int n = min(n_holes, n_fill);
  if (tid == 0) a.counts[list] = n;
#pragma unroll 4
  for (int j = tid; j < n; j += kEvictThreads) {
    const int2 m = moves[j];
    w[m.x] = w[m.y];
    pos[m.x] = pos[m.y];
    const int* table = a.table + (long long)b * a.ppr;
    moves[j] = make_int2((int)pool_row(table[m.x / kPagePos], a.n_pages, m.x), (int)pool_row(table[m.y / kPagePos], a.n_pages, m.y));
  }
  if (a.move_here) {
    __syncthreads();
    move_rows(a, list, n, warp, WARPS);
  }
}

// Moves, for lists where they are many: grid (lists, parts).
constexpr int kMoveThreads = 256;
__global__ void __launch_bounds__(kMoveThreads) cache_move_kernel(const __grid_constant__ EvictArgs a) {
  pdl_wait();
  move_rows(a, blockIdx.x, a.counts[blockIdx.x], blockIdx.y * (kMoveThreads / 32) + threadIdx.x / 32, gridDim.y * (kMoveThreads / 32));
}

// ------------------------------------------------------------------ page means
struct MeansArgs {
  const void* k_pool;                  // [layers][n_pages][64][width]
  const int *table, *from, *lens;
  int layers, B, width, ppr, n_pages;  // width = Hkv * D
  float* means;                        // [layers][B][ppr][width]
};

// Means of the keys of the pages that have become full.  Sums are in 64 bits and rounded once: selections go by them, and
// a sum whose rounding depends on its order would make near ties depend on it too.  grid (ppr, B, layers): a CTA per page, a
// thread per 16 bytes of columns and group of positions, eight loads under way at once.  Bound by reading the keys where many
// pages are new (several CTAs share an SM then, and one's sums run under the others' loads; with 512 threads and 16 loads each,
// one CTA to an SM, 8 sequences of up to 60000 took 250 us instead of 110), by a few trips to memory where few are.
constexpr int kMeansThreads = 256, kMeansBatch = 8;
template <typename CT>
__global__ void __launch_bounds__(kMeansThreads, 3) page_means_kernel(const __grid_constant__ MeansArgs a) {
  constexpr int PER = 16 / (int)sizeof(CT);
  __shared__ double s_sum[PER][kMeansThreads];
  const int p = blockIdx.x, b = blockIdx.y, layer = blockIdx.z, cap = a.ppr * kPagePos;
  if (p >= clamp_int(a.lens[b], 0, cap) / kPagePos || p < clamp_int(a.from[b], 0, cap) / kPagePos) return;
  const long long row = pool_row(a.table[(long long)b * a.ppr + p], a.n_pages, 0);
  if (row < 0) return;
  const CT* src = reinterpret_cast<const CT*>(a.k_pool) + ((long long)layer * a.n_pages * kPagePos + row) * a.width;
  float* out = a.means + (((long long)layer * a.B + b) * a.ppr + p) * a.width;
  const int pieces = a.width / PER;
  // groups of positions: as many as there are threads for (a power of two, so that they divide the page), of a batch at least
  int groups = 1;
  while (groups < kPagePos / kMeansBatch && pieces * groups * 2 <= kMeansThreads) groups *= 2;
  const int across = kMeansThreads / groups, g = threadIdx.x / across, rows = kPagePos / groups;
  for (int c0 = 0; c0 < pieces; c0 += across) {
    const int c = c0 + threadIdx.x % across;
    double s[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) s[e] = 0.;
    if (c < pieces) {
      const CT* at = src + (long long)g * rows * a.width + c * PER;
      for (int r0 = 0; r0 < rows; r0 += kMeansBatch) {
        uint4 v[kMeansBatch];
#pragma unroll
        for (int r = 0; r < kMeansBatch; ++r) v[r] = *reinterpret_cast<const uint4*>(at + (long long)(r0 + r) * a.width);
#pragma unroll
        for (int r = 0; r < kMeansBatch; ++r) {
          const uint32_t x[4] = {v[r].x, v[r].y, v[r].z, v[r].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(CT) == 4) {
              s[e] += (double)__uint_as_float(x[e]);
            } else {
              s[2 * e] += (double)__uint_as_float(x[e] << 16);
              s[2 * e + 1] += (double)__uint_as_float(x[e] & 0xffff0000u);
            }
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) s_sum[e][threadIdx.x] = s[e];
    __syncthreads();
    for (int i = threadIdx.x; i < across * PER; i += kMeansThreads) {
      const int col = i % across, e = i / across;
      if (c0 + col >= pieces) continue;
      double sum = 0.;
      for (int k = 0; k < groups; ++k) sum += s_sum[e][k * across + col];
      out[(c0 + col) * PER + e] = (float)(sum / kPagePos);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------ selection of pages
struct SelectArgs {
  const void* q;
  const float* means;                  // [B][ppr][Hkv][D]
  const int *lens, *nodes;
  int B, T, H, Hkv, G, ppr, select, cluster;
  long long q_stride;
  unsigned long long* keys;            // scratch [B][T][Hkv][ppr]
  int* pages;                          // [B][T][Hkv][select]
};

// score(page) = (sum of the group's queries) . mean, in 64 bits: the border of a selection is often close.  The best
// `select` full pages (ties and NaN: the lower page, NaN below everything), listed in ascending order.
//
// For one node a sequence: a cluster per key head.  Its CTAs score a share of the pages each -- a warp takes eight pages at a time and adds up
// their eight sums together -- and the first one finds the border bit by bit, from the top: a candidate stands if at least
// `select` keys are not below it, and ends the search where it is exactly so many.  A candidate costs two barriers
// (the scores of a sequence differ in their first bits, so some 20 candidates do); histograms of digits, with their atomics
// and scans, took five times as long.
constexpr int kSelectThreads = 256, kSelectKept = 8;    // keys a thread keeps in registers
template <typename CT, int D>
__global__ void __launch_bounds__(kSelectThreads) page_select_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int WARPS = kSelectThreads / 32, E = D >= 32 ? D / 32 : 1, BATCH = 8;
  __shared__ double s_q[D];
  __shared__ int s_warp[WARPS];
  pdl_launch_dependents();
  const int id = blockIdx.x / a.cluster, rank = blockIdx.x % a.cluster, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = id % a.Hkv, t = id / a.Hkv % a.T, b = id / a.Hkv / a.T;
  int* out = a.pages + (long long)id * a.select;
  const int full = clamp_int(a.lens[b], 0, a.ppr * kPagePos) / kPagePos;
  const bool alive = !a.nodes || t < a.nodes[b];
  const int n_out = alive ? min(full, a.select) : 0;
  // (these returns are the whole cluster's)
  if (rank == 0) for (int i = n_out + tid; i < a.select; i += kSelectThreads) out[i] = -1;
  if (n_out == 0) return;
  if (full <= a.select) {
    if (rank == 0) for (int i = tid; i < full; i += kSelectThreads) out[i] = i;
    return;
  }
  if (tid < D) {
    double s = 0.;
    const CT* src = reinterpret_cast<const CT*>(a.q) + ((long long)b * a.T + t) * a.q_stride + h * a.G * D + tid;
    for (int g = 0; g < a.G; ++g) s += (double)to_f(src[g * D]);
    s_q[tid] = s;
  }
  __syncthreads();
  unsigned long long* keys = a.keys + (long long)id * a.ppr;
  {
    double q[E];
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = lane * E + e < D ? s_q[lane * E + e] : 0.;
    const float* m = a.means + ((long long)b * a.ppr * a.Hkv + h) * D + (lane * E < D ? lane * E : 0);
    const long long step = (long long)a.Hkv * D;
    for (int p0 = (rank * WARPS + warp) * BATCH; p0 < full; p0 += a.cluster * WARPS * BATCH) {
      float x[BATCH][E];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const float* src = m + min(p0 + k, full - 1) * step;
        if constexpr (E == 4) *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(src);
        else if constexpr (E == 2) *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(src);
        else x[k][0] = *src;
      }
      double s[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        s[k] = 0.;
#pragma unroll
        for (int e = 0; e < E; ++e) if (lane * E < D) s[k] += q[e] * (double)x[k][e];
      }
      // eight sums over 32 lanes: each step halves the sums a lane carries on with
#pragma unroll
      for (int o = 16, k = BATCH / 2; o >= 4; o >>= 1, k >>= 1) {
#pragma unroll
        for (int i = 0; i < k; ++i) {
          const bool up = lane & o;
          const double give = up ? s[i] : s[i + k], keep = up ? s[i + k] : s[i];
          s[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      s[0] += __shfl_xor_sync(0xffffffffu, s[0], 1);
      s[0] += __shfl_xor_sync(0xffffffffu, s[0], 2);
      // the lane's page: bits 4, 3, 2 of its number chose the halves
      const int p = p0 + ((lane >> 4) & 1) * 4 + ((lane >> 3) & 1) * 2 + ((lane >> 2) & 1);
      if ((lane & 3) == 0 && p < full) keys[p] = s[0] != s[0] ? 0ull : order_bits64(s[0] + 0.);
    }
  }
  if (a.cluster > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank > 0) return;
  } else {
    __threadfence_block();
    __syncthreads();
  }
  unsigned long long mine[kSelectKept];
#pragma unroll
  for (int k = 0; k < kSelectKept; ++k) mine[k] = tid + k * kSelectThreads < full ? __ldcg(keys + tid + k * kSelectThreads) : 0ull;
  constexpr int KEPT = kSelectKept * kSelectThreads;
  const int rounds = (full + KEPT - 1) / KEPT;
  // how many keys are at least x (x > 0: what is behind the last page counts as 0)
  auto count = [&](unsigned long long x) {
    int n = 0;
    for (int r = 0; r < rounds; ++r) {
      int hits = 0;
#pragma unroll
      for (int k = 0; k < kSelectKept; ++k) {
        const int p = r * KEPT + tid + k * kSelectThreads;
        const unsigned long long key = r == 0 ? mine[k] : (p < full ? __ldcg(keys + p) : 0ull);
        hits += key >= x;
      }
      n += hits;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    __syncthreads();
    if (lane == 0) s_warp[warp] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) n += s_warp[w];
    return n;
  };
  unsigned long long border = 0;
  bool exact = false;
  for (int bit = 63; bit >= 0 && !exact; --bit) {
    const unsigned long long candidate = border | (1ull << bit);
    const int n = count(candidate);
    if (n >= a.select) border = candidate;
    exact = n == a.select;
  }
  // keys above the border stay, of those equal to it the lowest pages
  int room = exact ? full : a.select - (border == ~0ull ? 0 : count(border + 1));
  int ties = 0, done = 0;
  for (int p0 = 0; p0 < full; p0 += kSelectThreads) {
    const int p = p0 + tid;
    const unsigned long long k = p < full ? __ldcg(keys + p) : 0ull;
    const bool tie = p < full && k == border;
    bool in = p < full && k > border;
    unsigned m = __ballot_sync(0xffffffffu, tie);
    __syncthreads();
    if (lane == 0) s_warp[warp] = __popc(m);
    __syncthreads();
    int before = ties, all = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) { if (i < warp) before += s_warp[i]; all += s_warp[i]; }
    if (tie && before + __popc(m & ((1u << lane) - 1)) < room) in = true;
    ties += all;
    m = __ballot_sync(0xffffffffu, in);
    __syncthreads();
    if (lane == 0) s_warp[warp] = __popc(m);
    __syncthreads();
    int at = done;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) { if (i < warp) at += s_warp[i]; done += s_warp[i]; }
    at += __popc(m & ((1u << lane) - 1));
    if (in && at < a.select) out[at] = p;
  }
}

// The same for several nodes: a cluster per (key head, four nodes).  The means are read once for the four (each node
// for itself, 512 selections among 540 pages of 128 columns took 48 us, so 29), a warp adds up 8 pages x 4 nodes together,
// and a warp then finds each node's border.  From two nodes on: the whole operator over 8 sequences of 30000, 8 key heads of 128, 32
// pages, with a CTA a node / with this: 1 node 35.0 / 31.8 us, 2 51.8 / 48.2, 4 79.4 / 66.4, 8 122 / 109; one sequence, 16 pages: 1
// node 18.3 / 19.8, 2 20.0 / 20.5, 4 22.4 / 21.7.
constexpr int kSelectNodes = 4, kSelectLane = 32;       // keys a lane keeps in registers
template <typename CT, int D>
__global__ void __launch_bounds__(kSelectThreads) page_select_nodes_kernel(const __grid_constant__ SelectArgs a) {
  constexpr int WARPS = kSelectThreads / 32, E = D >= 32 ? D / 32 : 1, BATCH = 8, NB = kSelectNodes;
  __shared__ double s_q[NB][D];
  pdl_launch_dependents();
  const int id = blockIdx.x / a.cluster, rank = blockIdx.x % a.cluster, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int groups = ceil_div(a.T, NB), h = id % a.Hkv, t0 = id / a.Hkv % groups * NB, b = id / a.Hkv / groups;
  const int full = clamp_int(a.lens[b], 0, a.ppr * kPagePos) / kPagePos, nodes = a.nodes ? clamp_int(a.nodes[b], 0, a.T) : a.T;
  auto item = [&](int k) { return ((long long)b * a.T + t0 + k) * a.Hkv + h; };
  // (what decides the next returns is the same for the whole cluster)
  if (rank == 0) {
    for (int i = tid; i < NB * a.select; i += kSelectThreads) {
      const int k = i / a.select, j = i % a.select;
      if (t0 + k >= a.T) break;
      if (t0 + k >= nodes || j >= full) a.pages[item(k) * a.select + j] = -1;
      else if (full <= a.select) a.pages[item(k) * a.select + j] = j;
    }
  }
  if (t0 >= nodes || full <= a.select) return;
  for (int i = tid; i < NB * D; i += kSelectThreads) {
    const int k = i / D, d = i % D;
    double s = 0.;
    if (t0 + k < nodes) {
      const CT* src = reinterpret_cast<const CT*>(a.q) + ((long long)b * a.T + t0 + k) * a.q_stride + h * a.G * D + d;
      for (int g = 0; g < a.G; ++g) s += (double)to_f(src[g * D]);
    }
    s_q[k][d] = s;
  }
  __syncthreads();
  {
    double q[NB][E];
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) q[k][e] = lane * E + e < D ? s_q[k][lane * E + e] : 0.;
    const float* m = a.means + ((long long)b * a.ppr * a.Hkv + h) * D + (lane * E < D ? lane * E : 0);
    const long long step = (long long)a.Hkv * D;
    for (int p0 = (rank * WARPS + warp) * BATCH; p0 < full; p0 += a.cluster * WARPS * BATCH) {
      float x[BATCH][E];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const float* src = m + min(p0 + k, full - 1) * step;
        if constexpr (E == 4) *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(src);
        else if constexpr (E == 2) *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(src);
        else x[k][0] = *src;
      }
      double s[BATCH * NB];                                 // sum of page i / NB, node i % NB
#pragma unroll
      for (int k = 0; k < BATCH; ++k)
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          double v = 0.;
#pragma unroll
          for (int e = 0; e < E; ++e) if (lane * E < D) v += q[n][e] * (double)x[k][e];
          s[k * NB + n] = v;
        }
      // 32 sums over 32 lanes: every step halves the sums a lane carries on with, lane i ends with sum i
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) {
#pragma unroll
        for (int i = 0; i < o; ++i) {
          const bool up = lane & o;
          const double give = up ? s[i] : s[i + o], keep = up ? s[i + o] : s[i];
          s[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
      }
      const int p = p0 + lane / NB, n = lane % NB;
      if (p < full && t0 + n < nodes) a.keys[item(n) * a.ppr + p] = s[0] != s[0] ? 0ull : order_bits64(s[0] + 0.);
    }
  }
  if (a.cluster > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (rank >= NB) return;
  } else {
    __threadfence_block();
    __syncthreads();
  }
  // a warp for a node, in as many CTAs of the cluster as there are
  const int share = min(a.cluster, NB);
  for (int k = rank + warp * share; k < NB && t0 + k < nodes; k += WARPS * share) {
    const unsigned long long* keys = a.keys + item(k) * a.ppr;
    int* out = a.pages + item(k) * a.select;
    unsigned long long mine[kSelectLane];
#pragma unroll
    for (int i = 0; i < kSelectLane; ++i) mine[i] = lane + i * 32 < full ? __ldcg(keys + lane + i * 32) : 0ull;
    auto count = [&](unsigned long long x) {                // keys that are at least x (x > 0)
      int n = 0;
#pragma unroll
      for (int i = 0; i < kSelectLane; ++i) n += mine[i] >= x;
#pragma unroll 8
      for (int p = lane + kSelectLane * 32; p < full; p += 32) n += __ldcg(keys + p) >= x;
      return __reduce_add_sync(0xffffffffu, n);
    };
    unsigned long long border = 0;
    bool exact = false;
    for (int bit = 63; bit >= 0 && !exact; --bit) {
      const unsigned long long candidate = border | (1ull << bit);
      const int n = count(candidate);
      if (n >= a.select) border = candidate;
      exact = n == a.select;
    }
    const int room = exact ? full : a.select - (border == ~0ull ? 0 : count(border + 1));
    const unsigned before = (1u << lane) - 1;
    int ties = 0, done = 0;
    auto list = [&](int p, unsigned long long key) {
      const bool tie = p < full && key == border;
      unsigned m = __ballot_sync(0xffffffffu, tie);
      const bool in = p < full && (key > border || (tie && ties + __popc(m & before) < room));
      ties += __popc(m);
      m = __ballot_sync(0xffffffffu, in);
      const int at = done + __popc(m & before);
      if (in && at < a.select) out[at] = p;
      done += __popc(m);
    };
#pragma unroll
    for (int i = 0; i < kSelectLane; ++i) {
      if (i * 32 >= full) break;
      list(lane + i * 32, mine[i]);
    }
    for (int p0 = kSelectLane * 32; p0 < full; p0 += 32) list(p0 + lane, p0 + lane < full ? __ldcg(keys + p0 + lane) : 0ull);
  }
}

}  // namespace tree
}  // namespace bpd
