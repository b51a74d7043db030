// The waits of the layer for a few tokens, and how a call ends on the counters that its blocks wait for one another by.  They are zero before a
// call and have to be zero behind it, so somebody sets them back, and nobody may be reading or adding then.  Plain C++ over an object
// that does it, so that every order in which blocks get there can be played through on the CPU.
//
//   b.join()       all warps of the block are behind their last wait for a counter and their last addition to one
//   b.all_done()   waits until every block's tiles are done; false: given up, and the counters stay as they are
//   b.ticket()     takes the next number, behind join(); who has the last one, and so is behind every block's join(), sets the blocks'
//                  counters back
//   b.clear()      sets a share of the groups' counters back
//   b.sum()        the block's share of the output
//   b.spoil()      marks the counters of a call that was given up, so that none that comes behind it goes by them
//
// The groups' counters are set back by all blocks, and only behind all tiles, not behind the other blocks' warps.  So nobody may be
// reading one who is not needed for a tile (takes_part), and an addition to one has to be behind nobody's back: it is there before
// what tells of all groups together, by which a reader may have gone instead.
#pragma once

#ifdef __CUDACC__
#define CIERA_ON_BOTH __host__ __device__ __forceinline__
#else
#define CIERA_ON_BOTH inline
#endif

namespace ciera {

// A bounded wait.  True once there() is; false when another of the block's waits has run out, or when this one does, which give_up() then
// tells the block and the caller.
template <class There, class GivenUp, class GiveUp>
CIERA_ON_BOTH bool poll(unsigned most, There there, GivenUp given_up, GiveUp give_up) {
    for (unsigned i = 0; i < most; ++i) {
        if (there()) return true;
        if (given_up()) return false;
    }
    give_up();
    return false;
}

// The first counter of a call that was given up: no call gets there by adding.
constexpr unsigned kSpoiled = 1u << 31;

// Whether one of `warps` warps (a power of two), which take stages in turn, has one of a tile's, the first of which is stage `it`.
CIERA_ON_BOTH bool takes_part(unsigned it, unsigned stages, unsigned warp, unsigned warps) { return ((warp - it) & (warps - 1)) < stages; }

// Tells of a block's written tiles: next() waits for one, group() adds it to its group's counter; behind the last whole() adds all of them to
// that of all groups.  (A fence for each tile: 2 us more for five tokens on 256 experts.)
template <class Next, class Group, class Fence, class Whole>
CIERA_ON_BOTH void tell(Next next, Group group, Fence fence, Whole whole) {
    while (next()) group();
    fence();
    whole();
}

template <class Block>
CIERA_ON_BOTH bool end_call(Block& b) {
    b.join();
    if (!b.all_done()) {
        b.spoil();
        return false;
    }
    b.ticket();
    b.clear();
    b.sum();
    return true;
}

}  // namespace ciera
