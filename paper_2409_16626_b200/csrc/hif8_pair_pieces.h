// Where an epilogue warp of the pair kernel puts a tile's pieces on their way to C, and what has to have left first.  (Plain C++: the order can be followed on the host.)
#pragma once
#ifdef __CUDACC__
#define HIF8_PIECES_FN __host__ __device__ __forceinline__
#else
#define HIF8_PIECES_FN inline
#endif

namespace hif8 {

// Two places in turn, from the first one on in each tile; the last tile's pieces have one each, and those from the third on have held no piece before.  Within a tile all but the newest
// store have read when a piece is written, which lies in the other place.
struct PiecePlaces {
    int newest = -1;  // place of the store committed last, in the tiles before
    static HIF8_PIECES_FN int place_of(int piece, bool last_tile) { return last_tile ? piece : piece & 1; }
    // Stores that may still read when a tile begins with `place`: the newest, unless the tile before had an odd number of them, so that it lies in this very place.
    HIF8_PIECES_FN int may_still_read(int place) const { return place == newest ? 0 : 1; }
    HIF8_PIECES_FN void stored(int place) { newest = place; }  // by the last store of a tile
};

}  // namespace hif8
