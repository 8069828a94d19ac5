// C entry points of the operators on a paged cache.
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "cache_ops.cuh"
#include "tree_host.hpp"

namespace bpd {
namespace tree {

template <> int plan_attention<bf16>(const AttnArgs&, bool, int, AttnPlan*);
template <> int plan_attention<float>(const AttnArgs&, bool, int, AttnPlan*);
template <> int launch_attention<bf16>(const AttnArgs&, bool, int, const AttnPlan&, cudaStream_t);
template <> int launch_attention<float>(const AttnArgs&, bool, int, const AttnPlan&, cudaStream_t);

namespace {

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

int check_cache(const bpd_cache* c, bool need_v) {
  if (!c || !c->k_pool || (need_v && !c->v_pool) || !c->page_table) return fail(BPD_E_INVALID, "null argument");
  if (c->dtype != 0 && c->dtype != 1) return fail(BPD_E_INVALID, "unknown dtype %d", c->dtype);
  if (!aligned(c->k_pool, 16) || !aligned(c->v_pool, 16)) return fail(BPD_E_INVALID, "misaligned pool");
  if (c->head_dim != 16 && c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
    return fail(BPD_E_UNSUPPORTED, "head_dim %d: the operators take 16, 32, 64 and 128", c->head_dim);
  if (c->kv_heads < 1 || c->kv_heads > 1024) return fail(BPD_E_SHAPE, "kv_heads %d out of range (1..1024)", c->kv_heads);
  if (c->batch < 1 || c->batch > 65535) return fail(BPD_E_SHAPE, "batch %d out of range (1..65535)", c->batch);
  if (c->layers < 1 || c->layers > 65535) return fail(BPD_E_SHAPE, "layers %d out of range (1..65535)", c->layers);
  if (c->n_pages < 1 || c->n_pages > (1 << 24)) return fail(BPD_E_SHAPE, "n_pages %d out of range (1..2^24)", c->n_pages);
  if (c->pages_per_row < 1 || c->pages_per_row > (1 << 20)) return fail(BPD_E_SHAPE, "pages_per_row %d out of range (1..2^20)", c->pages_per_row);
  return BPD_OK;
}
int elem_of(const bpd_cache* c) { return c->dtype == 0 ? 4 : 2; }

int check_nodes(int nodes) {
  if (nodes < 1 || nodes > kMaxNodes) return fail(BPD_E_SHAPE, "nodes %d out of range (1..%d)", nodes, kMaxNodes);
  return BPD_OK;
}
int check_heads(const bpd_cache* c, int heads) {
  if (heads < 1 || heads > 4096 || heads % c->kv_heads) return fail(BPD_E_SHAPE, "heads %d: a multiple of kv_heads %d up to 4096", heads, c->kv_heads);
  return BPD_OK;
}
// Rows of `width` elements, `stride` apart, read in 16-byte pieces.
int check_rows(const bpd_cache* c, const void* p, long long stride, long long width, const char* what) {
  if (!p) return fail(BPD_E_INVALID, "null argument");
  if (!aligned(p, 16) || stride * elem_of(c) % 16) return fail(BPD_E_INVALID, "%s: rows must begin on 16-byte boundaries", what);
  if (stride < width) return fail(BPD_E_SHAPE, "%s: stride %lld below the row's %lld elements", what, stride, width);
  return BPD_OK;
}
int check_scale(float scale) {
  if (!(scale > 0.f) || !isfinite(scale)) return fail(BPD_E_INVALID, "scale must be positive and finite");
  return BPD_OK;
}

AttnArgs attn_args(const bpd_cache* c, int nodes, int heads, int select) {
  AttnArgs a;
  memset(&a, 0, sizeof(a));
  a.k_pool = c->k_pool; a.v_pool = c->v_pool; a.table = c->page_table;
  a.B = c->batch; a.T = nodes; a.H = heads; a.Hkv = c->kv_heads; a.G = heads / c->kv_heads;
  a.ppr = c->pages_per_row; a.n_pages = c->n_pages; a.select = select;
  return a;
}
int plan_of(const bpd_cache* c, const AttnArgs& a, bool paged, AttnPlan* plan) {
  return c->dtype == 0 ? plan_attention<float>(a, paged, c->head_dim, plan) : plan_attention<bf16>(a, paged, c->head_dim, plan);
}
struct PagedSizes { size_t keys, pages; };
PagedSizes paged_sizes(const bpd_cache* c, int nodes, int select) {
  const size_t items = (size_t)c->batch * nodes * c->kv_heads;
  return PagedSizes{round256(items * c->pages_per_row * 8), round256(items * select * 4)};
}

int attend(const bpd_cache* c, const void* q, const void* k_new, const void* v_new, int nodes, int heads, long long q_stride,
           long long kv_stride, const int32_t* lens, const int32_t* parents, const int32_t* n_nodes, float scale, bool paged, int select,
           const int* pages, const AttnPlan& plan, char* scratch, void* out, float* lse, cudaStream_t st) {
  AttnArgs a = attn_args(c, nodes, heads, select);
  a.q = q; a.k_new = k_new; a.v_new = v_new; a.lens = lens; a.parents = parents; a.nodes = n_nodes; a.pages = pages;
  a.q_stride = q_stride; a.kv_stride = kv_stride;
  a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  a.out = out; a.lse = lse;
  a.part = reinterpret_cast<float*>(scratch);
  a.info = reinterpret_cast<int2*>(scratch + plan.part_bytes);
  a.split = plan.split;
  a.end_units = plan.end_units;
  a.part_rows = plan.combine_rows;
  a.ctas = plan.ctas;
  return c->dtype == 0 ? launch_attention<float>(a, paged, c->head_dim, plan, st) : launch_attention<bf16>(a, paged, c->head_dim, plan, st);
}

int check_attention(const bpd_cache* c, const void* q, const void* k_new, const void* v_new, int nodes, int heads, long long q_stride,
                    long long kv_stride, const int32_t* lens, const int32_t* parents, float scale, const void* out) {
  int rc = check_cache(c, true);
  if (rc || (rc = check_nodes(nodes)) || (rc = check_heads(c, heads)) || (rc = check_scale(scale))) return rc;
  if (!lens || !parents || !out) return fail(BPD_E_INVALID, "null argument");
  if (!aligned(out, 16)) return fail(BPD_E_INVALID, "misaligned output");
  if ((rc = check_rows(c, q, q_stride, (long long)heads * c->head_dim, "q")) ||
      (rc = check_rows(c, k_new, kv_stride, (long long)c->kv_heads * c->head_dim, "k_new")) ||
      (rc = check_rows(c, v_new, kv_stride, (long long)c->kv_heads * c->head_dim, "v_new"))) return rc;
  return BPD_OK;
}
int check_lists(const bpd_cache* c) {
  if ((long long)c->layers * c->batch * c->kv_heads > 0x7fffffffLL) return fail(BPD_E_SHAPE, "layers * batch * kv_heads out of range");
  return BPD_OK;
}
// The most entries of a list that an eviction moves: from above the budget to below it.
int moves_cap(const bpd_cache* c, int budget) { return std::max(1, std::min(budget, c->pages_per_row * kPagePos - std::min(budget, c->pages_per_row * kPagePos))); }

int check_scratch(const void* scratch, size_t have, size_t need) {
  if (need == 0) return BPD_OK;
  if (!scratch || !aligned(scratch, 256)) return fail(BPD_E_INVALID, "scratch is null or misaligned");
  if (have < need) return fail(BPD_E_NOMEM, "scratch too small: %zu bytes, %zu needed", have, need);
  return BPD_OK;
}

// Outputs that the first CTA of a sequence writes, and arrays that its other CTAs may still have to read, share no memory.
struct Span { const void* at; size_t bytes; const char* name; };
int check_apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span& o : outs)
    for (const Span& i : ins)
      if (o.at && i.at && (uintptr_t)o.at < (uintptr_t)i.at + i.bytes && (uintptr_t)i.at < (uintptr_t)o.at + o.bytes)
        return fail(BPD_E_INVALID, "%s must not overlap %s, which every CTA of a sequence reads", o.name, i.name);
  return BPD_OK;
}

template <typename CT>
int launch_select(SelectArgs& a, int D, cudaStream_t st) {
  const bool several = a.T > 1;
  const long long items = (long long)a.B * (several ? ceil_div(a.T, kSelectNodes) : a.T) * a.Hkv;
  // CTAs for every SM; a share of at least 64 pages each
  a.cluster = 1;
  while (a.cluster < 8 && items * a.cluster * 2 <= 2 * kSMs && a.ppr >= a.cluster * 128) a.cluster *= 2;
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof(cfg));
  cfg.gridDim = dim3((unsigned)(items * a.cluster)); cfg.blockDim = dim3(kSelectThreads); cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)a.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 1 : 0;
  void* ptrs[] = {&a};
  BPD_TREE_BY_DIM(BPD_CUDA(cudaLaunchKernelExC(&cfg, several ? reinterpret_cast<const void*>(page_select_nodes_kernel<CT, DD>) : reinterpret_cast<const void*>(page_select_kernel<CT, DD>), ptrs)); break;)
  ++g_launches;
  return BPD_OK;
}

template <typename CT>
int launch_weights(const WeightArgs& a, int D, cudaStream_t st) {
  const dim3 grid((unsigned)std::min<long long>((long long)a.B * a.Hkv * a.ppr, 2 * kSMs));
  BPD_TREE_BY_DIM(BPD_CUDA(launch_k(cache_weights_kernel<CT, DD>, grid, dim3(kWThreads), 0, st, false, a)); break;)
  ++g_launches;
  return BPD_OK;
}

}  // namespace
}  // namespace tree
}  // namespace bpd

using namespace bpd;
using namespace bpd::tree;

extern "C" {

size_t bpd_op_tree_attention_scratch_bytes(const bpd_cache* cache, int nodes, int heads) {
  if (check_cache(cache, true) || check_nodes(nodes) || check_heads(cache, heads)) return 0;
  AttnPlan plan;
  if (plan_of(cache, attn_args(cache, nodes, heads, 0), false, &plan)) return 0;
  return plan.part_bytes + plan.info_bytes;
}

int bpd_op_tree_attention(const bpd_cache* cache, const void* q, const void* k_new, const void* v_new, int nodes, int heads,
                          int64_t q_stride, int64_t kv_stride, const int32_t* lens, const int32_t* parents, const int32_t* n_nodes,
                          float scale, void* scratch, size_t scratch_bytes, void* out, float* lse, void* cuda_stream) {
  int rc = check_attention(cache, q, k_new, v_new, nodes, heads, q_stride, kv_stride, lens, parents, scale, out);
  if (rc) return rc;
  AttnPlan plan;
  if ((rc = plan_of(cache, attn_args(cache, nodes, heads, 0), false, &plan))) return rc;
  if ((rc = check_scratch(scratch, scratch_bytes, plan.part_bytes + plan.info_bytes))) return rc;
  return attend(cache, q, k_new, v_new, nodes, heads, q_stride, kv_stride, lens, parents, n_nodes, scale, false, 0, nullptr, plan,
                static_cast<char*>(scratch), out, lse, (cudaStream_t)cuda_stream);
}

int bpd_op_page_means(const bpd_cache* cache, const int32_t* lens_from, const int32_t* lens, float* means, void* cuda_stream) {
  int rc = check_cache(cache, false);
  if (rc) return rc;
  if (!lens_from || !lens || !means) return fail(BPD_E_INVALID, "null argument");
  if (!aligned(means, 16)) return fail(BPD_E_INVALID, "misaligned means");
  MeansArgs a;
  a.k_pool = cache->k_pool; a.table = cache->page_table; a.from = lens_from; a.lens = lens; a.layers = cache->layers; a.B = cache->batch;
  a.width = cache->kv_heads * cache->head_dim; a.ppr = cache->pages_per_row; a.n_pages = cache->n_pages; a.means = means;
  const dim3 grid(a.ppr, a.B, a.layers);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (cache->dtype == 0) BPD_CUDA(launch_k(page_means_kernel<float>, grid, dim3(kMeansThreads), 0, st, false, a));
  else BPD_CUDA(launch_k(page_means_kernel<bf16>, grid, dim3(kMeansThreads), 0, st, false, a));
  ++g_launches;
  return BPD_OK;
}

size_t bpd_op_page_attention_scratch_bytes(const bpd_cache* cache, int nodes, int heads, int select) {
  if (check_cache(cache, true) || check_nodes(nodes) || check_heads(cache, heads) || select < 1 || select > cache->pages_per_row) return 0;
  AttnPlan plan;
  if (plan_of(cache, attn_args(cache, nodes, heads, select), true, &plan)) return 0;
  const PagedSizes s = paged_sizes(cache, nodes, select);
  return plan.part_bytes + plan.info_bytes + s.keys + s.pages;
}

int bpd_op_page_attention(const bpd_cache* cache, const float* means, const void* q, const void* k_new, const void* v_new, int nodes,
                          int heads, int64_t q_stride, int64_t kv_stride, const int32_t* lens, const int32_t* parents,
                          const int32_t* n_nodes, int select, float scale, void* scratch, size_t scratch_bytes, void* out, float* lse,
                          int32_t* pages, void* cuda_stream) {
  int rc = check_attention(cache, q, k_new, v_new, nodes, heads, q_stride, kv_stride, lens, parents, scale, out);
  if (rc) return rc;
  if (!means) return fail(BPD_E_INVALID, "null argument");
  if (!aligned(means, 16)) return fail(BPD_E_INVALID, "misaligned means");
  if (select < 1 || select > cache->pages_per_row) return fail(BPD_E_SHAPE, "select %d out of range (1..pages_per_row)", select);
  AttnPlan plan;
  AttnArgs shape = attn_args(cache, nodes, heads, select);
  if ((rc = plan_of(cache, shape, true, &plan))) return rc;
  const PagedSizes s = paged_sizes(cache, nodes, select);
  if ((rc = check_scratch(scratch, scratch_bytes, plan.part_bytes + plan.info_bytes + s.keys + s.pages))) return rc;
  char* base = static_cast<char*>(scratch);
  SelectArgs p;
  p.q = q; p.means = means; p.lens = lens; p.nodes = n_nodes; p.B = shape.B; p.T = nodes; p.H = heads; p.Hkv = shape.Hkv; p.G = shape.G;
  p.ppr = shape.ppr; p.select = select; p.q_stride = q_stride;
  p.keys = reinterpret_cast<unsigned long long*>(base + plan.part_bytes + plan.info_bytes);
  p.pages = pages ? pages : reinterpret_cast<int*>(base + plan.part_bytes + plan.info_bytes + s.keys);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if ((rc = cache->dtype == 0 ? launch_select<float>(p, cache->head_dim, st) : launch_select<bf16>(p, cache->head_dim, st))) return rc;
  return attend(cache, q, k_new, v_new, nodes, heads, q_stride, kv_stride, lens, parents, n_nodes, scale, true, select, p.pages, plan, base,
                out, lse, st);
}

int bpd_op_tree_commit(const bpd_cache* cache, const void* k_new, const void* v_new, int nodes, int64_t kv_stride, const int32_t* lens,
                       const int32_t* parents, const int32_t* tokens, const int32_t* top1, const int32_t* last_top1,
                       const int32_t* n_nodes, int32_t eos_id, int32_t* out_lens, int32_t* out_accepted, int32_t* out_path,
                       int32_t* out_next, void* cuda_stream) {
  int rc = check_cache(cache, true);
  if (rc || (rc = check_nodes(nodes))) return rc;
  if (!lens || !parents || !tokens || !top1 || !last_top1 || !out_lens || !out_accepted || !out_path || !out_next)
    return fail(BPD_E_INVALID, "null argument");
  const long long width = (long long)cache->kv_heads * cache->head_dim;
  if ((rc = check_rows(cache, k_new, kv_stride, width, "k_new")) || (rc = check_rows(cache, v_new, kv_stride, width, "v_new"))) return rc;
  const size_t per_row = (size_t)cache->batch * 4, per_node = per_row * nodes;
  if ((rc = check_apart({{out_lens, per_row, "out_lens"}, {out_accepted, per_row, "out_accepted"}, {out_path, per_node, "out_path"}, {out_next, per_row, "out_next"}},
                        {{lens, per_row, "lens"}, {parents, per_node, "parents"}, {tokens, per_node, "tokens"}, {top1, per_node, "top1"},
                         {last_top1, per_row, "last_top1"}, {n_nodes, per_row, "n_nodes"}, {cache->page_table, per_row * cache->pages_per_row, "the page table"}})))
    return rc;
  CommitArgs a;
  a.k_new = k_new; a.v_new = v_new; a.k_pool = cache->k_pool; a.v_pool = cache->v_pool; a.table = cache->page_table; a.lens = lens;
  a.parents = parents; a.tokens = tokens; a.top1 = top1; a.last_top1 = last_top1; a.nodes = n_nodes;
  a.layers = cache->layers; a.B = cache->batch; a.T = nodes; a.row_pieces = (int)(width * elem_of(cache) / 16); a.ppr = cache->pages_per_row;
  a.n_pages = cache->n_pages; a.eos = eos_id; a.elem = elem_of(cache); a.kv_stride = kv_stride;
  a.out_lens = out_lens; a.accepted = out_accepted; a.path = out_path; a.next = out_next;
  if ((long long)a.layers * 2 * nodes * a.row_pieces > 0x7fffffffLL) return fail(BPD_E_SHAPE, "layers * nodes * kv_heads * head_dim out of range");
  // CTAs for a path of four nodes; longer ones take more turns
  const long long pieces = (long long)a.layers * 2 * std::min(nodes, 4) * a.row_pieces;
  const int splits = (int)std::max<long long>(1, std::min<long long>((pieces + kCommitThreads - 1) / kCommitThreads, std::max(1, 4 * kSMs / a.B)));
  BPD_CUDA(launch_k(tree_commit_kernel, dim3(a.B, splits), dim3(kCommitThreads), 0, (cudaStream_t)cuda_stream, false, a));
  ++g_launches;
  return BPD_OK;
}

int bpd_op_cache_weights(const bpd_cache* cache, const void* q, int nodes, int heads, int64_t q_stride, const float* lse,
                         const int32_t* path, const int32_t* accepted, const int32_t* lens, const int32_t* seen, float scale,
                         float* weights, int32_t* positions, void* cuda_stream) {
  int rc = check_cache(cache, false);
  if (rc || (rc = check_nodes(nodes)) || (rc = check_heads(cache, heads)) || (rc = check_scale(scale))) return rc;
  if (!lse || !path || !accepted || !lens || !seen || !weights || !positions) return fail(BPD_E_INVALID, "null argument");
  if ((rc = check_rows(cache, q, q_stride, (long long)heads * cache->head_dim, "q"))) return rc;
  WeightArgs a;
  a.q = q; a.k_pool = cache->k_pool; a.lse = lse; a.path = path; a.accepted = accepted; a.lens = lens; a.seen = seen;
  a.table = cache->page_table; a.B = cache->batch; a.T = nodes; a.H = heads; a.Hkv = cache->kv_heads; a.G = heads / cache->kv_heads;
  a.ppr = cache->pages_per_row; a.n_pages = cache->n_pages; a.q_stride = q_stride; a.scale_log2 = (float)((double)scale * 1.4426950408889634); a.weights = weights; a.positions = positions;
  if ((long long)a.ppr * a.Hkv > 0x7fffffffLL) return fail(BPD_E_SHAPE, "pages_per_row * kv_heads out of range");
  return cache->dtype == 0 ? launch_weights<float>(a, cache->head_dim, (cudaStream_t)cuda_stream)
                           : launch_weights<bf16>(a, cache->head_dim, (cudaStream_t)cuda_stream);
}

size_t bpd_op_cache_evict_scratch_bytes(const bpd_cache* cache, int budget) {
  if (check_cache(cache, true) || check_lists(cache) || budget < 1) return 0;
  const size_t lists = (size_t)cache->layers * cache->batch * cache->kv_heads;
  return round256(lists * moves_cap(cache, budget) * 8) + round256(lists * 4);
}

int bpd_op_cache_evict(const bpd_cache* cache, const int32_t* lens, const int32_t* seen, int budget, int recent, float* weights,
                       int32_t* positions, void* scratch, size_t scratch_bytes, int32_t* out_lens, void* cuda_stream) {
  int rc = check_cache(cache, true);
  if (rc) return rc;
  if (!lens || !seen || !weights || !positions || !out_lens) return fail(BPD_E_INVALID, "null argument");
  if (budget < 1) return fail(BPD_E_SHAPE, "budget %d must be at least 1", budget);
  if (recent < 0 || recent > budget) return fail(BPD_E_SHAPE, "recent %d out of range (0..budget)", recent);
  if ((rc = check_lists(cache))) return rc;
  if ((rc = check_scratch(scratch, scratch_bytes, bpd_op_cache_evict_scratch_bytes(cache, budget)))) return rc;
  const size_t per_row = (size_t)cache->batch * 4;
  if ((rc = check_apart({{out_lens, per_row, "out_lens"}},
                        {{lens, per_row, "lens"}, {seen, per_row, "seen"}, {cache->page_table, per_row * cache->pages_per_row, "the page table"}}))) return rc;
  EvictArgs a;
  a.k_pool = cache->k_pool; a.v_pool = cache->v_pool; a.table = cache->page_table; a.lens = lens; a.seen = seen; a.layers = cache->layers;
  a.B = cache->batch; a.Hkv = cache->kv_heads; a.row_pieces = cache->head_dim * elem_of(cache) / 16; a.ppr = cache->pages_per_row;
  a.n_pages = cache->n_pages; a.budget = budget; a.recent = recent; a.weights = weights; a.positions = positions; a.out_lens = out_lens;
  const int lists = a.layers * a.B * a.Hkv;
  a.moves = static_cast<int2*>(scratch); a.moves_cap = moves_cap(cache, budget);
  a.counts = reinterpret_cast<int*>(static_cast<char*>(scratch) + round256((size_t)lists * a.moves_cap * 8));
  // Where a list has room for at most 128 moves they are made by the launch that selects them, else all SMs share them in a launch
  // of their own.  us with the moves here / shared, entries in L2: 48 lists, 1152 slots to 1024 12.4 / 14.8, 4096 to 256 13.0 / 14.6,
  // 8000 to 1024 16.7 / 17.6, 8000 to 4000 43 / 31; 256 lists (heads of 128) 17.3 / 18.7, 19.2 / 21.9, 24.0 / 24.2, 89 / 94.
  a.move_here = a.moves_cap <= 128 ? 1 : 0;
  if (a.ppr * kPagePos <= 16 * kEvictThreads) BPD_CUDA(launch_k(cache_evict_kernel<16>, dim3(lists), dim3(kEvictThreads), 0, (cudaStream_t)cuda_stream, false, a));
  else BPD_CUDA(launch_k(cache_evict_kernel<32>, dim3(lists), dim3(kEvictThreads), 0, (cudaStream_t)cuda_stream, false, a));
  ++g_launches;
  if (!a.move_here) {
    // a warp for 32 moves
    const int parts = std::min(ceil_div(a.moves_cap, kMoveThreads), 65535);
    BPD_CUDA(launch_k(cache_move_kernel, dim3(lists, parts), dim3(kMoveThreads), 0, (cudaStream_t)cuda_stream, true, a));
    ++g_launches;
  }
  return BPD_OK;
}

int bpd_debug_op_wait_timeout(int limit_us, void* cuda_stream) {
  if (limit_us < 1 || limit_us > 2000000) return fail(BPD_E_INVALID, "limit_us = %d outside 1..2000000", limit_us);
  return let_wait_expire(limit_us, (cudaStream_t)cuda_stream);
}

int bpd_op_status(void* cuda_stream) {
  int expired = 0;
  const int rc = take_wait_expired(&expired, (cudaStream_t)cuda_stream);
  if (rc) return rc;
  return expired ? fail(BPD_E_TIMEOUT, "a bounded wait of an operator's kernel expired; outputs enqueued since the last call are not valid") : BPD_OK;
}

}  // extern "C"
