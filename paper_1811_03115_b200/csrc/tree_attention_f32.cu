// Tree attention over fp32 caches.
#include <algorithm>
#include <type_traits>

#include "tree_host.hpp"

namespace bpd {
namespace tree {
BPD_TREE_INSTANTIATE(float)
}  // namespace tree
}  // namespace bpd
