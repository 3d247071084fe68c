// window.hip -- attention with a sliding window and sinks over a bf16 cache
// (plans of msa_plan_window in msa_forward).
//
// The kernels are those of attn.hip with a window's visibility and key axis (see
// attn_device.h): a tile reads the keys that some row of it sees, in whole steps of
// 64, and the planner cuts and deals out those alone.
#include "attn_launch.h"

namespace msa {

int launch_window(const WindowAttnParams& p, int head_dim, int item_rows, int num_wg, void* stream) {
  return launch_tiles(p, head_dim, item_rows, num_wg, stream);
}

}  // namespace msa
