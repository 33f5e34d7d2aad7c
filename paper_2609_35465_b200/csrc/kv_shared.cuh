// What the two kernels of tetra_kv_attend_shared tell each other: k_kv_prefix attends a group's rows to the tokens that its
// sequences share and leaves pieces, k_kv_attend attends each sequence's rows to its own tokens and adds the pieces.
#pragma once
#include "kv_common.cuh"

namespace tetra {
namespace {

constexpr int kPreColumns = 128;                                    // of a piece: rows of a tensor-core product
__host__ __device__ constexpr int pre_slots(int D) { return D == 256 ? 1 : 2; }  // pieces of a part: what fits the SM's 512 columns of tensor memory
__host__ __device__ constexpr int pre_tile(int D) { return kPreColumns * pre_slots(D); }  // columns of an item
// Floats of a piece: sums as [D / 4][column][4], then [column] reference and denominator.
__host__ __device__ constexpr int pre_piece(int D) { return kPreColumns * (D + 2); }

// Where a sequence's share of the pieces is.  An item is (group, kv head, tile of columns), cut into `parts`; a part leaves a piece
// for each 128 columns of its tile, or, where the tile has no more than that, two of the same columns and other tokens.
struct SharedSeq {
    int32_t first;   // blocks that the pieces stand for; 0: none, the sequence reads all of its tokens itself
    int32_t part0;   // of the group's first item
    int32_t parts;   // of an item
    int32_t tiles;   // items of a kv head
    int32_t row0;    // of the group's columns
    int32_t cols;
    int32_t spare[2];
};
static_assert(sizeof(SharedSeq) == 32, "two 16-byte words");

// A column's pieces.
struct PieceRange {
    int32_t first, count, step, column;
};
template <int D>
__device__ __forceinline__ PieceRange pieces_of(const SharedSeq& s, int head, uint32_t column) {
    constexpr uint32_t TILE = pre_tile(D);
    const uint32_t tile = column / TILE, in = column % TILE;
    const bool both = pre_slots(D) == 2 && uint32_t(s.cols) - tile * TILE <= kPreColumns;
    const int32_t part = s.part0 + int32_t(uint32_t(head) * s.tiles + tile) * s.parts;
    PieceRange r;
    r.first = part * pre_slots(D) + (both ? 0 : int32_t(in / kPreColumns));
    r.step = both ? 1 : pre_slots(D);
    r.count = both ? 2 * s.parts : s.parts;
    r.column = int32_t(in % kPreColumns);
    return r;
}

}  // namespace

struct PrefixGroups {
    const int32_t* start;   // [groups + 1]: sequences
    const int32_t* shared;  // [groups]: tokens
    int32_t groups;
};
// Parts that one call may have: as many as the workspace has pieces for.
size_t prefix_parts_most(int head_dim, int64_t rows, int q_heads, int kv_heads, int groups);
size_t prefix_bytes(int head_dim, size_t parts);
// `seqs` [TETRA_KV_MAX_SEQS] and `pieces`: in the workspace.  scale_log2: the scale times log2(e).
cudaError_t launch_prefix(const tetra_kv_cache& cache, int rows, const PrefixGroups& groups, const void* q, int64_t q_stride, float scale_log2, int q_group, int head_dim,
                          void* seqs, float* pieces, size_t parts, cudaStream_t s);

}  // namespace tetra
