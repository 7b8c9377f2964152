// The order in which a group of warps goes through its tiles, apart from what it does with them, so that it can be tried without a device.
//
// In some tiles the warps of a group meet at a barrier that has no limit (`meet`); in every tile each of them waits, with a limit, for the tile's numbers
// (`wait`) and works on them (`work`, which may wait for more).  Limits run out one by one: a warp may give up on a tile that the others
// of its group find there a moment later.  So a warp that gave up works no more, and waits no more, but meets the others in all tiles that are left.
#pragma once

#ifdef __CUDACC__
#define MVLA_WALK __device__ __forceinline__
#else
#define MVLA_WALK inline
#endif

namespace mvla {

// Tiles first, first + step, ... below n: the same ones in every warp of a group.  Whether no wait gave up.
template <class Meet, class Wait, class Work>
MVLA_WALK bool walk_tiles(int first, int n, int step, Meet meet, Wait wait, Work work)
{
    bool ok = true;
    for (int i = first; i < n; i += step) {
        meet(i);
        ok = ok && wait(i) && work(i);
    }
    return ok;
}

}  // namespace mvla
