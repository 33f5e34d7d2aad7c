// What the kernels of tetra_kv_attend_shared tell each other: k_kv_prefix attends a group's rows to the tokens that its sequences share
// and leaves pieces, k_kv_attend attends each sequence's rows to its own tokens and leaves their sums, k_kv_join adds them.
#pragma once
#include "kv_common.cuh"

namespace tetra {
namespace {

constexpr int kPreColumns = 128;                                    // of a piece: rows of a tensor-core product
__host__ __device__ constexpr int pre_slots(int D) { return D == 256 ? 1 : 2; }  // pieces of a part: what fits the SM's 512 columns of tensor memory
__host__ __device__ constexpr int pre_tile(int D) { return kPreColumns * pre_slots(D); }  // columns of an item
// Floats of a piece: [column][D] sums, then [column] reference and denominator.
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

constexpr int kPreMostCtas = 160, kPreWaves = 2;  // of a launch; parts a CTA where items are few

// Where things are in the workspace of tetra_kv_attend_shared, behind tetra_kv_attend's: the sequences' shares, the sums of their own
// tokens, the pieces; and how many parts may leave pieces.
struct SharedPlaces {
    size_t seqs, own, pieces, end, parts;
    SharedPlaces(int D, int64_t rows, int q_heads, int kv_heads, int groups) {
        const int64_t sharing = groups < rows / 2 ? groups : rows / 2;  // two sequences with a row each, at least
        const int64_t items = (rows * (q_heads / kv_heads) / pre_tile(D) + sharing) * kv_heads, few = kPreWaves * kPreMostCtas;
        parts = size_t(items > few ? items : few);
        seqs = (tetra_kv_workspace_bytes(D) + 255) / 256 * 256;
        own = seqs + size_t(TETRA_KV_MAX_SEQS) * sizeof(SharedSeq);
        pieces = (own + size_t(rows) * q_heads * (D + 2) * sizeof(float) + 255) / 256 * 256;
        end = pieces + parts * pre_slots(D) * pre_piece(D) * sizeof(float);
    }
};

}  // namespace

struct SharedCall {
    KvCache c;
    tetra_kv_groups g;
    const __half* q;
    __half* out;
    int64_t q_stride;
    float scale;        // times log2 e
    int32_t group;      // query heads to a kv head
    SharedSeq* seqs;
    float* own;         // [row][head][D] sums and, from own_ends on, [row][head][2] references and denominators
    int64_t own_ends;
    float* pieces;
    uint32_t most;      // parts
};
cudaError_t launch_prefix(const SharedCall& p, int head_dim, int sms, cudaStream_t s);
cudaError_t launch_join(const SharedCall& p, int head_dim, cudaStream_t s);

}  // namespace tetra
