// The fused attention kernels of attn_fwd.hpp with a sliding window and sink
// tokens: a work item visits the sinks' key blocks and those that the windows
// of its rows reach, in ascending order, and masks inside them.  Alg. 1 takes
// its decisions on the blocks that a row sees, so a block outside its window
// changes nothing (a fully masked block is a no-op), and the first blocks, which
// hold the sinks, are B0 as before.  The Default setup takes them for short calls
// only, with 128-key blocks whatever the call's; others go to attn_window_tile.hip.
// Few rows, of either setup, go to attn_decode.hip.
#include "attn_fwd.hpp"

namespace baps {

namespace {

template <int D, int BLK>
hipError_t launch_window(const AttnParams& p, hipStream_t st)
{
    if ((long long)p.Sq * (p.Hq / p.Hkv) <= kFewFlatRows) return launch_attention_window_few(p, D, BLK, st);
    if (p.mode == kModeDefault) {
        int ncu = 0;
        const hipError_t e = cu_count(&ncu);
        if (e != hipSuccess) return e;
        const WindowForm f = window_form(D, (long long)p.Sq * (p.Hq / p.Hkv), p.Hq / p.Hkv, (long long)p.Hkv * p.B, p.Sk, p.window,
                                         p.sinks, ncu);
        if (f.tile) return launch_attention_window_tile(p, D, f.rows, st);
        constexpr int kDefault = kModeDefault | kModeWindow;
        if constexpr (D == 128)
            if (f.rows == 128) return launch_one<D, 128, 8, 2, true, kDefault, false, false, false, false>(p, st);
        return launch_one<D, 128, 4, 2, true, kDefault, false, false, false, false>(p, st);
    }
    return launch_rows<D, BLK, true, kModeE2E | kModeWindow, false, false, false>(p, st);
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
