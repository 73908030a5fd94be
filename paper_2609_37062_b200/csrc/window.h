// Which 16-token tiles of a sequence a windowed plan attends.
//
// The query of a decode step sits at position L - 1 and sees the tokens t with
// t >= L - window or t < sinks.  What it does not see is cut out in whole
// tiles: the plan and the kernels walk the sequence as if the `skip_tiles`
// tiles behind the first `sink_tiles` were not there ("visible" positions),
// and the tiles at the two edges of the gap are masked token by token.  Every
// tile that is walked holds a token that is seen.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define DA_HOST_DEVICE __host__ __device__
#else
#define DA_HOST_DEVICE
#endif

namespace da {

struct WindowCut {
    int32_t sink_tiles;   // tiles in front of the gap (0 when there is no gap)
    int32_t skip_tiles;   // tiles of the gap
    int32_t first;        // first position of the window; what lies in [sinks, first) is not seen
};

DA_HOST_DEVICE inline WindowCut window_cut(int32_t seq_len, int32_t window, int32_t sinks)
{
    WindowCut c = {0, 0, 0};
    if (window <= 0 || seq_len <= window) return c;
    c.first = seq_len - window;
    const int32_t sink_end = sinks < c.first ? sinks : c.first;
    const int32_t sink_tiles = (int32_t)(((int64_t)sink_end + 15) >> 4), window_tile = c.first >> 4;
    if (window_tile > sink_tiles) {
        c.sink_tiles = sink_tiles;
        c.skip_tiles = window_tile - sink_tiles;
    }
    return c;
}

// The tile of the sequence that visible tile `v` is.
DA_HOST_DEVICE inline int32_t window_tile(const WindowCut& c, int32_t v) { return v < c.sink_tiles ? v : v + c.skip_tiles; }

}  // namespace da
