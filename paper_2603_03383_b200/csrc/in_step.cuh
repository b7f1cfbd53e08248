// The way of warps that meet at named barriers through a worker's pieces.  Such a barrier has no limit: a warp that ended by itself, as a bounded wait of its
// own ran out, would let the others stand at the next one for good.  So it leaves the piece's work, meets the others wherever they may still meet in that piece,
// and all end together at the next one, where they agree on going on.
// Plain control flow, for the kernels and a host compiler alone.
#pragma once

#ifdef __CUDACC__
#define MTV_IN_STEP __device__ __forceinline__
#else
#define MTV_IN_STEP inline
#endif

namespace mtv {

enum class Way { ON, END, LEFT };      // behind a piece: to the next one; there is none (which all see alike); a wait ran out in it

// look(n): whether the n-th piece, or that there is none, could be had.  agree(x): whether all of the warps say x (they meet).  piece(n): works on it.
// follow(): meets the others as they meet in the rest of the piece that was left.  Returns whether the pieces came to their end, the same for all.
template <typename Look, typename Agree, typename Piece, typename Follow>
MTV_IN_STEP bool pieces_in_step(Look &&look, Agree &&agree, Piece &&piece, Follow &&follow) {
#pragma unroll 1
    for (int n = 0; agree(look(n)); ++n) {
        const Way way = piece(n);
        if (way == Way::END) return true;
        if (way == Way::LEFT) {
            follow();
            agree(false);
            return false;
        }
    }
    return false;
}

// Two warps that hold the same rows meet in a key tile: in a piece's first tile, and where one of them asks for it, they exchange their maxima; in its last tile
// they exchange their sums.  The same from tile t on for a warp that left.  asked(): whether the other one asks (they meet).  maxima(last): of the last tile?
template <typename Asked, typename Maxima, typename Sums>
MTV_IN_STEP void follow_tiles(int t, int t0, int t1, Asked &&asked, Maxima &&maxima, Sums &&sums) {
#pragma unroll 1
    for (; t < t1; ++t) {
        if (t == t0 || asked()) maxima(t == t1 - 1);
        if (t == t1 - 1) sums();
    }
}

}  // namespace mtv
