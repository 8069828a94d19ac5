// Tree attention over bf16 caches.
#include <algorithm>
#include <type_traits>

#include "tree_host.hpp"

namespace bpd {
namespace tree {
BPD_TREE_INSTANTIATE(bf16)
}  // namespace tree
}  // namespace bpd
