// The tree attention of tree_attention.cuh on the 5th-generation tensor cores: bf16 caches with heads of 64 or 128, many rows
// (see many_rows), in calls whose work is cut into runs of chunks.
//
// A tile is 128 query rows of a key head (fewer use fewer of the lanes).  Per chunk of 64 keys: S = Q K^T (tcgen05.mma, both
// operands in shared memory) into tensor memory; a thread per row takes its 64 scores, and puts the weights back where the
// scores were, as two bf16 planes; O += P V (P from tensor memory, V from shared memory as TMA brought it, keys outermost).
// The running maximum a row is scaled by lags behind: O is rescaled only when the maximum has grown by more than 2^8, which
// fp32 sums and bf16 planes carry without loss.
//
// Warps 0-3: softmax (lane = row), epilogue; warp 4: TMA; warp 5: MMA and tensor memory.  Two CTAs share an SM: one's softmax
// runs under the other's products and loads.  Keys and values come page by page as TMA tiles (64 keys x 64 columns, 128-byte
// swizzle); what lies behind a sequence's last key in its open page, or behind its last node in the tree's chunk, comes along
// and is masked, its values zeroed in shared memory (0 times NaN is not 0).
//
// Every wait is bounded; on expiry the CTA notes it (see bpd_op_status).  However it ends, the copies and products it has
// issued are waited for (bounded) before its tensor memory is freed and it returns.
//
// What bounds it: 8 sequences of 8000 and 128 rows, heads of 128, move 268 MB in 70 us of the launch's 79 with the join -- 0.58
// of the copy's rate; the tensor pipe is active 39 % of the time.  A chunk takes a CTA 3000 cycles: about 1000 exponentials and
// the weights' planes, 240 the maximum, up to 1200 waiting for keys or values, the rest tensor-memory traffic and barriers.  Heads of
// 64: 2100 cycles, half of them exponentials.
#pragma once
#include "gemm_tc.cuh"
#include "tree_attention.cuh"

namespace bpd {
namespace tree {

constexpr int kTcThreads = 192, kTcRows = 128;

template <int D>
struct TcShape {
  // Stages of keys and of values, filled independently: a chunk's keys are used up as soon as its scores are there, a chunk
  // ahead of their softmax; its values two softmaxes later.  (In one order of issue, keys waited behind values for whose place a
  // product had to end, and a third of every chunk's 3400 cycles went by waiting.  One stage of keys to three of values: 87 us
  // instead of 84 for 8 sequences of up to 16000, 128 rows, heads of 128.)
  static constexpr int KK = 2, KV = D == 128 ? 2 : 4;
  static constexpr int PANELS = D / 64;                       // of 64 columns
  static constexpr int PANEL = kChunk * 128;                  // bytes of a panel of keys or values
  static constexpr int Q_PANEL = kTcRows * 128;
  static constexpr int Q_BYTES = PANELS * Q_PANEL, KV_BYTES = PANELS * PANEL;
  static constexpr int SMEM = 1024 + Q_BYTES + (KK + KV) * KV_BYTES;
  static constexpr int TMEM_COLS = 256;                       // scores / weights of two chunks (64 columns each), outputs (D)
  static constexpr int CTAS_PER_SM = 2;
};

// A wait of some operator's kernel has expired on this device since it was last asked (see bpd_op_status).
static __device__ int g_wait_expired;

__device__ __forceinline__ bool wait_bar(uint32_t bar, uint32_t parity, volatile int* dead, unsigned long long limit = tc::kSpinCycles) {
  if (tc::mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = clock64();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (tc::mbar_try_wait(bar, parity)) return true;
    if (*dead) return false;
    if ((unsigned long long)(clock64() - t0) > limit) {
      *dead = 1;
      return false;
    }
  }
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// A box of a map's only matrix.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map),
               "r"(bar), "r"(x), "r"(y), "r"(0) : "memory");
}

// kp, vp: the pools as [n_pages * 64][Hkv * D]; kn, vn: the drafted nodes' rows.
struct TcMaps { CUtensorMap kp, vp, kn, vn; };

// The same answer in every lane.
__device__ __forceinline__ bool wait_bar_warp(uint32_t bar, uint32_t parity, volatile int* dead) { return __all_sync(0xffffffffu, wait_bar(bar, parity, dead)); }

#define BPD_TMEM_32(op, X)                                                                                            \
  op(X[0]), op(X[1]), op(X[2]), op(X[3]), op(X[4]), op(X[5]), op(X[6]), op(X[7]), op(X[8]), op(X[9]), op(X[10]),      \
      op(X[11]), op(X[12]), op(X[13]), op(X[14]), op(X[15]), op(X[16]), op(X[17]), op(X[18]), op(X[19]), op(X[20]),   \
      op(X[21]), op(X[22]), op(X[23]), op(X[24]), op(X[25]), op(X[26]), op(X[27]), op(X[28]), op(X[29]), op(X[30]),   \
      op(X[31])
// 32 consecutive columns of this thread's lane; complete after tmem_wait_ld.
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
#define BPD_OUT(x) "=r"(x)
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
      "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : BPD_TMEM_32(BPD_OUT, r) : "r"(at) : "memory");
#undef BPD_OUT
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t (&r)[32]) {
#define BPD_IN(x) "r"(x)
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::BPD_TMEM_32(BPD_IN, r), "r"(at) : "memory");
#undef BPD_IN
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
               "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D += A B with A (128 rows, 16 bf16 of K in 8 columns) in tensor memory.
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// Values as the product's B operand: N (columns) is the contiguous dimension.  Rows of 64 columns (128 bytes, swizzled) are
// keys, eight of them 1024 bytes apart from the next eight; the next 64 columns lie a panel further.
__device__ __forceinline__ uint64_t value_desc(uint32_t saddr, int panel_bytes) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3ffff) >> 4);
  d |= (uint64_t)(panel_bytes >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// One CTA whose wait for a barrier that nothing arrives on expires, and which then ends as the kernel below does.
static __global__ void op_wait_probe_kernel(unsigned long long limit) {
  __shared__ __align__(8) unsigned long long bar;
  __shared__ int dead;
  if (threadIdx.x == 0) {
    dead = 0;
    tc::mbar_init(s_addr(&bar), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    wait_bar(s_addr(&bar), 0, &dead, limit);
    if (dead) g_wait_expired = 1;
  }
}

template <int D, bool PAGED>
__global__ void __launch_bounds__(kTcThreads, 2) tree_attention_tc_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ TcMaps maps) {
  using S = TcShape<D>;
  constexpr int KK = S::KK, KV = S::KV;
  pdl_launch_dependents();
  extern __shared__ uint8_t tt_smem[];
  const uint32_t base = (s_addr(tt_smem) + 1023u) & ~1023u;        // swizzled tiles need 1024-byte alignment
  uint8_t* gen = tt_smem + (base - s_addr(tt_smem));
  const uint32_t q_s = base, k_s = q_s + S::Q_BYTES, v_s = k_s + KK * S::KV_BYTES;
  __shared__ __align__(8) unsigned long long s_bar[2 * (KK + KV) + 9];
  __shared__ uint32_t s_tmem;
  __shared__ int s_dead, s_odd, s_keys[4];
  __shared__ Lines s_lines;
  const uint32_t bars = s_addr(s_bar);
  auto k_full = [&](int n) { return bars + 8 * (n % KK); };         // of chunk n (of the CTA's)
  auto k_empty = [&](int n) { return bars + 8 * (KK + n % KK); };
  auto v_full = [&](int n) { return bars + 8 * (2 * KK + n % KV); };
  auto v_empty = [&](int n) { return bars + 8 * (2 * KK + KV + n % KV); };
  auto s_full = [&](int s) { return bars + 8 * (2 * (KK + KV) + s); };
  auto p_ready = [&](int s) { return bars + 8 * (2 * (KK + KV) + 2 + s); };
  // Two, taken in turn, as for scores and weights: a wait by parity tells a phase from the one before it and the one behind it only,
  // and when the products lag behind (values on their way) a softmax that waits for the last of them may see two end at once.
  auto pv_done = [&](int s) { return bars + 8 * (2 * (KK + KV) + 4 + s); };
  const uint32_t q_ready = bars + 8 * (2 * (KK + KV) + 6), rows_bar = q_ready + 8, end_bar = q_ready + 16;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  clear_dead_rows<bf16>(a, D);
  Walk<PAGED> w(a, kTcRows);
  const bool work = w.begin();                                     // (the same answer in every warp)
  if (PAGED) pdl_wait();                                           // the selection (every CTA: what comes after waits for this launch alone)
  if (!work) return;
  if (tid == 0) {
    for (int s = 0; s < KK; ++s) { tc::mbar_init(k_full(s), 1); tc::mbar_init(k_empty(s), 1); }
    for (int s = 0; s < KV; ++s) { tc::mbar_init(v_full(s), 1); tc::mbar_init(v_empty(s), 1); }
    for (int s = 0; s < 2; ++s) { tc::mbar_init(s_full(s), 1); tc::mbar_init(p_ready(s), 4); tc::mbar_init(pv_done(s), 1); }
    tc::mbar_init(q_ready, 4);
    tc::mbar_init(rows_bar, 4);
    tc::mbar_init(end_bar, 1);
    s_dead = 0;
    s_odd = 0;                                                     // the last tile that had such values
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 5) tc::tmem_alloc(s_addr(&s_tmem), S::TMEM_COLS);
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = s_tmem, o_tmem = tmem + 128;
  volatile int* dead = &s_dead;

  if (warp == 4) {
    // ---- loads: keys and values go their ways independently, each as far ahead as its stages allow
    if (lane == 0) {
      Walk<PAGED> wv = w;
      int nk = 0, nv = 0, ck = w.c_begin, cv = wv.c_begin;
      int page_k = w.page_of(ck), page_v = page_k;                 // (looked up a chunk ahead)
      bool k_left = true, v_left = true;
      auto load = [&](const Walk<PAGED>& at, int c, int page, uint32_t dst, uint32_t bar, const CUtensorMap* pool, const CUtensorMap* drafted) {
        const int cached = at.cache_chunks();
        const bool node = c >= cached;
        // (a page that is not there: some page comes instead, all of it masked)
        const int y = node ? at.b * a.T + (c - cached) * kChunk : max(page, 0) * kPagePos;
        tc::mbar_expect_tx(bar, S::KV_BYTES);
#pragma unroll
        for (int p = 0; p < S::PANELS; ++p) load_box(dst + p * S::PANEL, node ? drafted : pool, bar, at.tl.h * D + p * 64, y);
      };
      unsigned long long t0 = clock64();
      while (k_left || v_left) {
        bool moved = false;
        if (k_left && tc::mbar_test(k_empty(nk), ((nk / KK) & 1) ^ 1)) {
          s_keys[nk % 4] = w.keys_of(ck, page_k);                  // (four chunks on, this one's softmax is done)
          load(w, ck, page_k, k_s + nk % KK * S::KV_BYTES, k_full(nk), &maps.kp, &maps.kn);
          ++nk;
          if (++ck >= w.c_end) { k_left = w.next(); ck = w.c_begin; }
          if (k_left) page_k = w.page_of(ck);
          moved = true;
        }
        if (v_left && tc::mbar_test(v_empty(nv), ((nv / KV) & 1) ^ 1)) {
          load(wv, cv, page_v, v_s + nv % KV * S::KV_BYTES, v_full(nv), &maps.vp, &maps.vn);
          ++nv;
          if (++cv >= wv.c_end) { v_left = wv.next(); cv = wv.c_begin; }
          if (v_left) page_v = wv.page_of(cv);
          moved = true;
        }
        if (moved) {
          t0 = clock64();
        } else if (*dead || (unsigned long long)(clock64() - t0) > tc::kSpinCycles) {
          *dead = 1;
          break;
        }
      }
      // copies in flight land before the shared memory goes, whoever's wait expires (used up, they have landed)
      for (int i = max(0, nk - KK); i < nk; ++i) tc::mbar_wait(k_full(i), (i / KK) & 1);
      for (int i = max(0, nv - KV); i < nv; ++i) tc::mbar_wait(v_full(i), (i / KV) & 1);
    }
  } else if (warp == 5) {
    // ---- products
    if (lane == 0) {
      const uint32_t id_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kChunk >> 3) << 17) | ((uint32_t)(kTcRows >> 4) << 24);
      const uint32_t id_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTcRows >> 4) << 24);
      auto scores = [&](int n) {
        if (!wait_bar(k_full(n), (n / KK) & 1, dead)) return false;
        // The scores take the place of the weights of two chunks before, whose product must have read them: products are in
        // order only where they add to the same sums.
        if (n >= 2 && !wait_bar(pv_done(n & 1), ((n - 2) >> 1) & 1, dead)) return false;
        tc::tc_fence_after();
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          tc::umma_f16(tmem + (n & 1) * 64, tc::smem_desc_sw128(q_s + k / 4 * S::Q_PANEL + (k % 4) * 32),
                       tc::smem_desc_sw128(k_s + n % KK * S::KV_BYTES + k / 4 * S::PANEL + (k % 4) * 32), id_s, k > 0);
        tc::umma_commit(s_full(n & 1));
        tc::umma_commit(k_empty(n));
        return true;
      };
      int n = 0, tile = 0;
      bool ok = true;
      do {
        ok = wait_bar(q_ready, tile & 1, dead);
        tc::tc_fence_after();
        const int count = w.c_end - w.c_begin;
        if (ok) ok = scores(n);
        for (int i = 0; i < count && ok; ++i, ++n) {
          // (the next chunk's scores run ahead, under this one's softmax)
          if (i + 1 < count && !(ok = scores(n + 1))) break;
          if (!(ok = wait_bar(p_ready(n & 1), (n >> 1) & 1, dead)) || !(ok = wait_bar(v_full(n), (n / KV) & 1, dead))) break;
          tc::tc_fence_after();
#pragma unroll
          for (int plane = 0; plane < 2; ++plane)
#pragma unroll
            for (int k = 0; k < kChunk / 16; ++k)
              umma_f16_ts(o_tmem, tmem + (n & 1) * 64 + plane * 32 + k * 8, value_desc(v_s + n % KV * S::KV_BYTES + k * 2048, S::PANEL), id_o,
                          i > 0 || plane > 0 || k > 0);
          tc::umma_commit(v_empty(n));
          tc::umma_commit(pv_done(n & 1));
        }
        ++tile;
      } while (ok && w.next());
      // nothing may read shared memory or write tensor memory once they go: all products end first, whoever's wait has expired
      tc::umma_commit(end_bar);
      tc::mbar_wait(end_bar, 0);
    }
  } else {
    // ---- softmax: a thread per row
    const uint32_t my = (uint32_t)(warp * 32) << 16;
    int n = 0, tile = 0, lines_of = -1, met = 0;
    bool ok = true;
    // the four warps meet (what one of them wrote to shared memory, the others see)
    auto meet = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(rows_bar);
      return wait_bar_warp(rows_bar, met++ & 1, dead);
    };
    do {
      const int rows = w.rows(), r = tid, cached = w.cache_chunks(), count = w.c_end - w.c_begin, b = w.b;
      const bool active = warp * 32 < rows;
      // The warp's queries into swizzled shared memory (its outputs of the tile before have been read), all loads side by side:
      // 16 trips to L2 one after the other would cost as much as five chunks.
      if (active) {
        constexpr int PIECES = D / 8, STEP = 32 / PIECES;          // rows a step
        uint4 x[PIECES];
        const int piece = lane % PIECES;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int row = warp * 32 + i * STEP + lane / PIECES;
          x[i] = make_uint4(0u, 0u, 0u, 0u);
          if (row < rows)
            x[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(a.q) + ((long long)b * a.T + w.node_of(row)) * a.q_stride + w.head_of(row) * D + piece * 8);
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int row = warp * 32 + i * STEP + lane / PIECES;
          *reinterpret_cast<uint4*>(gen + piece / 8 * S::Q_PANEL + row * 128 + ((piece % 8) ^ (row & 7)) * 16) = x[i];
        }
      }
      fence_async_shared();
      tc::tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_ready);
      const bool tree = w.c_end > cached;
      ++tile;
      if (tree && lines_of != b) {
        if (!(ok = meet())) break;                                 // (those of the sequence before have been used)
        if (warp == 0) find_lines(s_lines, a.parents + (long long)b * a.T, w.sq.nodes, lane);
        lines_of = b;
        if (!(ok = meet())) break;
      }
      float m = -INFINITY, l = 0.f;                                // m: what the weights are scaled by, a maximum of the past
      for (int i = 0; i < count; ++i, ++n) {
        const int c = w.c_begin + i, sb = n & 1;
        const bool node = c >= cached;
        if (!(ok = wait_bar_warp(s_full(sb), (n >> 1) & 1, dead))) break;
        tc::tc_fence_after();
        const int n_keys = s_keys[n % 4];
        const bool partial = n_keys < kChunk || node;
        // keys behind the last: their values become 0; in the tree's chunk so do values that are no finite numbers, see below
        if (partial) {
          if (!(ok = wait_bar_warp(v_full(n), (n / KV) & 1, dead))) break;
          uint8_t* vb = gen + (v_s - base) + n % KV * S::KV_BYTES;
          for (int j = tid; j < kChunk * (D / 8); j += 128) {
            const int key = j / (D / 8), piece = j % (D / 8);
            uint4* at = reinterpret_cast<uint4*>(vb + piece / 8 * S::PANEL + key * 128 + ((piece % 8) ^ (key & 7)) * 16);
            if (key >= n_keys) {
              *at = make_uint4(0u, 0u, 0u, 0u);
            } else if (node) {
              uint4 v = *at;
              uint32_t* x = reinterpret_cast<uint32_t*>(&v);
              bool odd = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((x[e] & 0x7f80u) == 0x7f80u) { x[e] &= 0xffff0000u; odd = true; }
                if ((x[e] & 0x7f800000u) == 0x7f800000u) { x[e] &= 0x0000ffffu; odd = true; }
              }
              if (odd) { *at = v; s_odd = tile; }
            }
          }
          fence_async_shared();
        }
        if (active) {
          uint32_t s[64];
          {
            uint32_t (&s0)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[0]);
            uint32_t (&s1)[32] = *reinterpret_cast<uint32_t (*)[32]>(&s[32]);
            tmem_ld32(tmem + my + sb * 64, s0);
            tmem_ld32(tmem + my + sb * 64 + 32, s1);
            tmem_wait_ld();
          }
          if (partial) {
            unsigned long long see = n_keys >= 64 ? ~0ull : (1ull << n_keys) - 1;
            if (node) see &= r < rows ? s_lines.bits[c - cached][w.node_of(r)] : 0ull;
#pragma unroll
            for (int j = 0; j < 64; ++j) if (!((see >> j) & 1)) s[j] = 0xff800000u;
          }
          float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int j = 0; j < 64; ++j) top[j & 3] = fmaxf(top[j & 3], __uint_as_float(s[j]));
          const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale_log2;
          // (a row that has seen nothing keeps a maximum of -inf; its weights are taken against 0 and are 0)
          if (__any_sync(0xffffffffu, now > m + 8.f)) {
            const float higher = fmaxf(m, now), f = higher == -INFINITY ? 1.f : exp2_fast(m - higher);
            m = higher;
            l *= f;
            if (i > 0) {
              if (!(ok = wait_bar_warp(pv_done((n - 1) & 1), ((n - 1) >> 1) & 1, dead))) break;
              tc::tc_fence_after();
#pragma unroll
              for (int d = 0; d < D; d += 32) {
                uint32_t x[32];
                tmem_ld32(o_tmem + my + d, x);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
                tmem_st32(o_tmem + my + d, x);
              }
              tmem_wait_st();
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int at = half * 32 + 2 * j;
              const float p0 = exp2_fast(fmaf(__uint_as_float(s[at]), a.scale_log2, -ref)), p1 = exp2_fast(fmaf(__uint_as_float(s[at + 1]), a.scale_log2, -ref));
              sum[j & 3] += p0 + p1;
              // the high plane is the weight cut off behind 8 bits, the low plane what is left, rounded
              hi[j] = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
              const __nv_bfloat162 rest = __floats2bfloat162_rn(p0 - __uint_as_float(__float_as_uint(p0) & 0xffff0000u),
                                                                p1 - __uint_as_float(__float_as_uint(p1) & 0xffff0000u));
              lo[j] = *reinterpret_cast<const uint32_t*>(&rest);
            }
            tmem_st16(tmem + my + sb * 64 + half * 16, hi);
            tmem_st16(tmem + my + sb * 64 + 32 + half * 16, lo);
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
          tmem_wait_st();
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(sb));
      }
      if (!ok) break;
      // ---- the tile's result
      if (!(ok = wait_bar_warp(pv_done((n - 1) & 1), ((n - 1) >> 1) & 1, dead))) break;
      tc::tc_fence_after();
      if (tree && !(ok = meet())) break;
      const bool whole = w.whole(), odd = tree && s_odd == tile;
      if (active) {
        const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        const long long at = r < rows ? w.out_row(r) : 0;
        float* part = a.part + ((long long)blockIdx.x * 2 + (a.split ? w.slot : 0)) * part_floats(a.part_rows, D);
#pragma unroll
        for (int d = 0; d < D; d += 32) {
          uint32_t x[32];
          tmem_ld32(o_tmem + my + d, x);
          tmem_wait_ld();
          if (r < rows) {
            // Values that were no finite numbers: a row that sees one has no finite output there, whatever its weight.
            if (odd) {
              const int node1 = min(w.sq.nodes, (w.c_end - cached) * kChunk);
              for (int t = max(0, w.c_begin - cached) * kChunk; t < node1; ++t) {
                if (!((s_lines.bits[t / 64][w.node_of(r)] >> (t % 64)) & 1)) continue;
                const bf16* v = reinterpret_cast<const bf16*>(a.v_new) + ((long long)b * a.T + t) * a.kv_stride + w.tl.h * D + d;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const float y = __bfloat162float(v[e]);
                  if (!(fabsf(y) <= 3.402823466e38f)) x[e] = __float_as_uint(__uint_as_float(x[e]) + y);
                }
              }
            }
            if (whole) {
              bf16* o = reinterpret_cast<bf16*>(a.out) + at * D + d;
#pragma unroll
              for (int e = 0; e < 32; e += 8) {
                uint32_t y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const __nv_bfloat162 v2 = __floats2bfloat162_rn(__uint_as_float(x[e + 2 * k]) * inv, __uint_as_float(x[e + 2 * k + 1]) * inv);
                  y[k] = *reinterpret_cast<const uint32_t*>(&v2);
                }
                *reinterpret_cast<uint4*>(o + e) = make_uint4(y[0], y[1], y[2], y[3]);
              }
            }
          }
          if (!whole) {
            // 32 rows x 32 columns through the warp's own rows of the queries' place, so that stores are whole lines
            uint8_t* mine = gen + warp * 4096;
            __syncwarp();                                          // (what was there has been read)
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(mine + lane * 128 + (((e / 4) ^ (lane & 7)) * 16)) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
            __syncwarp();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int row = e * 4 + lane / 8, piece = lane % 8;
              const uint4 y = *reinterpret_cast<const uint4*>(mine + row * 128 + ((piece ^ (row & 7)) * 16));
              if (warp * 32 + row < rows) *reinterpret_cast<uint4*>(part + (long long)(warp * 32 + row) * D + d + piece * 4) = y;
            }
            __syncwarp();                                          // (the next tile's queries go there)
          }
        }
        if (r < rows) {
          if (whole && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.693147180559945f;
          if (!whole) { part[(long long)a.part_rows * D + r] = m; part[(long long)a.part_rows * (D + 1) + r] = l; }
        }
      }
      if (a.split && w.c_begin == 0 && tid == 0) a.info[w.tl.id] = make_int2(blockIdx.x * 2 + w.slot, w.last_cta);
    } while (w.next());
  }
  __syncwarp();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  if (warp == 5) tc::tmem_dealloc(tmem, S::TMEM_COLS);
  if (tid == 0 && s_dead) g_wait_expired = 1;
}

}  // namespace tree
}  // namespace bpd
