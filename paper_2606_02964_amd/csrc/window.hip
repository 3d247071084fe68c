// window.hip -- attention with a sliding window and sinks over a bf16 cache
// (plans of msa_plan_window in msa_forward).
//
// The kernels are those of attn.hip with a window's visibility and key axis (see
// attn_device.h): a tile reads the sinks and the keys from its first row's window to its last
// row, in whole steps of 64, and the planner cuts and deals out those alone.  Bound as those are: 48 rows over 32K keys
// with a window of 4096 (32 query, 8 KV heads, d = 128) read K/V at 6.2 TB/s (131 us); a prompt of
// 12000 with 1024 keys runs at 870 TFLOP/s of visible pairs (233 us): its tiles have 18 steps, against
// which an item's start and end weigh 5 or 6, and 6% of the keys in them are hidden.  (The next item's
// descriptor and block ids loaded during the one before: the same within 1%.)
#include "attn_launch.h"

namespace msa {

int launch_window(const WindowAttnParams& p, int head_dim, int item_rows, int num_wg, void* stream) {
  return launch_tiles(p, head_dim, item_rows, num_wg, stream);
}

}  // namespace msa
