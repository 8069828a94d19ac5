// Tree attention over fp32 caches.
#include <algorithm>
#include <type_traits>

#include "tree_host.hpp"

namespace bpd {
namespace tree {

template <> int plan_attention<float>(const AttnArgs& a, bool paged, int D, AttnPlan* plan) {
  BPD_TREE_BY_DIM(return by_rows<float, DD>(a, paged, [&](auto wr, auto pg) { return plan_one<float, DD, decltype(wr)::value, decltype(pg)::value>(a, plan); });)
}
template <> int launch_attention<float>(const AttnArgs& a, bool paged, int D, const AttnPlan& plan, cudaStream_t st) {
  BPD_TREE_BY_DIM(return by_rows<float, DD>(a, paged, [&](auto wr, auto pg) { return launch_one<float, DD, decltype(wr)::value, decltype(pg)::value>(a, plan, st); });)
}

}  // namespace tree
}  // namespace bpd
