// The fused attention kernels of attn_fwd.hpp with a sliding window and sink
// tokens: a work item visits the sinks' key blocks and those that the windows
// of its rows reach, in ascending order, and masks inside them.  Alg. 1 takes
// its decisions on the blocks that a row sees, so a block outside its window
// changes nothing (a fully masked block is a no-op), and the first blocks, which
// hold the sinks, are B0 as before.
#include "attn_fwd.hpp"

namespace baps {

namespace {

template <int D, int BLK>
hipError_t launch_window(const AttnParams& p, hipStream_t st)
{
    if ((long long)p.Sq * (p.Hq / p.Hkv) <= kFewFlatRows) return launch_attention_window_few(p, D, BLK, st);
    return p.mode == kModeDefault ? launch_rows<D, BLK, true, kModeDefault | kModeWindow, false, false, false>(p, st)
                                  : launch_rows<D, BLK, true, kModeE2E | kModeWindow, false, false, false>(p, st);
}

}  // namespace

hipError_t launch_attention_window(const AttnParams& p, int D, int block, hipStream_t st)
{
    if (D == 64 && block == 32) return launch_window<64, 32>(p, st);
    if (D == 64 && block == 64) return launch_window<64, 64>(p, st);
    if (D == 64 && block == 128) return launch_window<64, 128>(p, st);
    if (D == 128 && block == 32) return launch_window<128, 32>(p, st);
    if (D == 128 && block == 64) return launch_window<128, 64>(p, st);
    if (D == 128 && block == 128) return launch_window<128, 128>(p, st);
    return hipErrorInvalidValue;
}

}  // namespace baps
