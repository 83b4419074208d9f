// What the host code of mcsd_ops.cu shares with mcsd_api.cu.
#pragma once

#include <stdint.h>

namespace mcsd {

// Depth of a tree, or the MCSD_ERR_* code of a parent array that breaks the layout contract.
__attribute__((visibility("hidden"))) int tree_depth(const int32_t *parent, int n_nodes);
// The value mcsd_last_launch_count reports on this host thread.
__attribute__((visibility("hidden"))) void set_last_launches(int n);

}  // namespace mcsd
