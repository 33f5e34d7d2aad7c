// What the kernels of tetra_kv_attend_shared tell each other: k_kv_prefix attends a group's rows to the tokens that its sequences share
// and leaves pieces, k_kv_attend attends each sequence's rows to its own tokens and leaves their sums, k_kv_join adds them.
#pragma once
#include "kv_common.cuh"

namespace tetra {
namespace {

constexpr int kPreColumns = 128;                                    // of a piece: rows of a tensor-core product
__host__ __device__ constexpr int pre_slots(int D) { return D == 256 ? 1 : 2; }  // pieces of a part at most: what fits the SM's 512 columns of tensor memory
__host__ __device__ constexpr int pre_tile(int D) { return kPreColumns * pre_slots(D); }  // columns of an item
// Floats of a piece: [column][D] sums, then [column] reference and denominator.
__host__ __device__ constexpr int pre_piece(int D) { return kPreColumns * (D + 2); }
constexpr int kSharedLeast = 8;                                     // blocks: fewer are not worth their pieces

// Blocks that sequence s, with rows [a, b) behind `before` tokens, shares with others of its group and does not read itself.  That goes
// by the sequence and its group alone, so that all kernels know it without each other: where all of its rows see all of the shared blocks,
// none of its own tokens is in them, and the group has other sequences.
struct SharedGroups {
    const int32_t* start;   // [groups + 1]: sequences
    const int32_t* tokens;  // [groups]
    int32_t groups;
};
// The group of sequence s and its sequences [first, last); -1: none, and `lo` is some group.
__device__ __forceinline__ int group_of(const SharedGroups& g, int seqs, int s, int& first, int& last, int& lo) {
    int hi = g.groups;
    lo = 0;  // the last one with start <= s
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(g.start + mid) <= s) lo = mid;
        else hi = mid;
    }
    first = __ldg(g.start + lo);
    last = __ldg(g.start + lo + 1);
    return first >= 0 && last <= seqs && first <= s && s < last ? lo : -1;
}
__device__ __forceinline__ int shared_blocks(const KvCache& c, const SharedGroups& g, int group) {
    const int64_t most = int64_t(c.width) * c.blocks_per_page, blocks = max(__ldg(g.tokens + group), 0) / kKvBlock;
    return int(min(blocks, most));
}
__device__ __forceinline__ bool takes_part(int first, int last, int blocks, int a, int b, int before) {
    return last - first >= 2 && blocks >= kSharedLeast && b > a && int64_t(before) >= int64_t(blocks) * kKvBlock;
}
__device__ __forceinline__ int shared_of(const KvCache& c, const SharedGroups& g, int s, int a, int b, int before) {
    int first, last, which;
    const int group = group_of(g, c.seqs, s, first, last, which);
    const int blocks = shared_blocks(c, g, which);
    return group >= 0 && takes_part(first, last, blocks, a, b, before) ? blocks : 0;
}

// Where a sequence's share of the pieces is.  An item is (group, kv head, tile of columns), cut into `parts`; a part leaves a piece
// for each 128 columns of its tile.
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

// A sequence's own tokens, of items of eight columns: its first run, runs of an item, items of a kv head.
struct OwnSeq {
    int32_t run0, runs, chunks, spare;
};
constexpr int kRunsMost = 8 * 384;  // warps of k_kv_attend's largest grid: runs beside one of each item

constexpr int kPreMostCtas = 160, kPreWaves = 2;  // of a launch; parts a CTA where items are few

// Where things are in the workspace of tetra_kv_attend_shared, behind tetra_kv_attend's: the sequences' shares, the sums of their own
// tokens, the pieces; and how many parts may leave pieces.
struct SharedPlaces {
    size_t seqs, owns, own, pieces, end, parts, runs;
    SharedPlaces(int D, int64_t rows, int q_heads, int kv_heads, int groups) {
        const int64_t sharing = groups < rows ? groups : rows;  // a row each, at least
        const int64_t items = (rows * (q_heads / kv_heads) / pre_tile(D) + sharing) * kv_heads, few = kPreWaves * kPreMostCtas;
        parts = size_t(items > few ? items : few);
        seqs = (tetra_kv_workspace_bytes(D) + 255) / 256 * 256;
        owns = seqs + size_t(TETRA_KV_MAX_SEQS) * sizeof(SharedSeq);
        own = owns + size_t(TETRA_KV_MAX_SEQS) * sizeof(OwnSeq);
        // Items of eight columns are those of calls with no more than eight a sequence on average; no bound gets less with more rows or heads.
        const int64_t most = 8 * TETRA_KV_MAX_SEQS, cols = rows * (q_heads / kv_heads);
        runs = size_t(kv_heads * ((cols < most ? cols : most) / 8 + (rows < TETRA_KV_MAX_SEQS ? rows : TETRA_KV_MAX_SEQS)) + kRunsMost);
        const size_t columns = runs * 8 > size_t(rows) * q_heads ? runs * 8 : size_t(rows) * q_heads;
        pieces = (own + columns * (D + 2) * sizeof(float) + 255) / 256 * 256;
        end = pieces + parts * pre_slots(D) * pre_piece(D) * sizeof(float);
    }
};

// k_kv_attend has nothing of k_kv_prefix's but starts behind what came before that (it is released when k_kv_prefix has waited, so
// the call's operands are complete and it reads them without a wait); its end has to imply that one's.  What it writes, k_kv_join
// reads behind a wait.  (Released at its beginning, k_kv_join waits beside both and takes nothing off: 67.8 and 69.5 us.  With a
// fence at its beginning k_kv_attend takes 1 us longer, and a lookup of its row behind k_kv_join's wait 3, of 56 for 64 answers on
// 16384.)
__device__ __forceinline__ void end_behind_prefix() {
    pdl_release();
    pdl_wait();
}

}  // namespace

struct SharedCall {
    KvCache c;
    SharedGroups g;
    const __half* q;
    __half* out;
    int64_t q_stride;
    float scale;        // times log2 e
    int32_t group;      // query heads to a kv head
    SharedSeq* seqs;
    float* own;         // [row][head][D], or [run][8][D], sums and, from own_ends on, references and denominators of each
    int64_t own_ends;
    OwnSeq* owns;
    bool runs;          // own sums are those of runs, of all sequences; else of items, of sequences that share
    float* pieces;
    uint32_t most;      // parts
    int32_t stages;     // of k_kv_prefix's ring
};
cudaError_t launch_prefix(SharedCall& p, int head_dim, int sms, cudaStream_t s);
cudaError_t launch_join(const SharedCall& p, int head_dim, cudaStream_t s);

}  // namespace tetra
