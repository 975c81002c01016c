// The order in which a warp asks for the tiles of its ring, takes them and lets the rest land.  Plain C++, so that a program on the
// host can drive it as the kernel does.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define SHOTKV_BOTH __host__ __device__ __forceinline__
#else
#define SHOTKV_BOTH inline
#endif

namespace shotkv {

// Limit of a wait for what is already on its way into a CTA's memory, about two seconds.  It is not the limit of the other waits,
// which a program may set as short as it likes: a CTA that ended before its copies have landed would leave them to write into the
// memory of the next one.
constexpr long long kLandCycles = 4000000000LL;

// Tiles first, first + step, ... through STAGES stages in turn.  `fetch(tile, stage)` asks for a tile; `landed(stage, parity,
// limit)` waits `limit` cycles at most for the copy that the stage was last asked for, of the phase with that parity.
template <int STAGES>
struct TileRing {
    int first, step, tile, stage = 0;
    uint32_t parity = 0;

    SHOTKV_BOTH TileRing(int first_tile, int tile_step) : first(first_tile), step(tile_step), tile(first_tile) {}

    // The first tiles, of the `all` that there is memory of: how many are wanted may not be known yet.
    template <class Fetch>
    SHOTKV_BOTH void ask(int all, Fetch&& fetch) const {
#pragma unroll
        for (int k = 0; k < STAGES; ++k)
            if (first + k * step < all) fetch(first + k * step, k);
    }
    // Done with a tile: the next one of its stage, if it is below `tiles`.
    template <class Fetch>
    SHOTKV_BOTH void next(int tiles, Fetch&& fetch) {
        if (tile + STAGES * step < tiles) fetch(tile + STAGES * step, stage);
        tile += step;
        turn();
    }
    // What was asked for and not taken, beyond the tiles wanted or after a wait that gave up: it lands before its place is used
    // for something else or the CTA ends.
    template <class Landed>
    SHOTKV_BOTH void land(int all, int tiles, Landed&& landed) {
#pragma unroll 1
        for (int k = 0; k < STAGES; ++k, tile += step)
            if (tile < all && (tile < first + STAGES * step || tile < tiles)) {
                landed(stage, parity, kLandCycles);
                turn();
            }
    }

private:
    SHOTKV_BOTH void turn() {
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (stage == 0) parity ^= 1;
    }
};

}  // namespace shotkv
