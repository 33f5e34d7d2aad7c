// New rows into the key/value cache at given positions of several axes (tetra_kv_append_at).
//
// As tetra_kv_append, but a pair is turned by the row's position on the pair's axis, and that has nothing to do with the row's slot.
// A picture comes as one call of some thousand rows, so work is cut by blocks, not rows: a CTA per (block of 16 slots, kv head) makes
// its rows' sines once for the block's keys and all queries of the head group.  Rows of a chat's step are a block each.
//
// What bounds it: a step's rows latency (one row 3.3 us, 64 rows of 40/8 heads 4.4, with tetra_kv_read 5.9 and 8.2); a picture's 2912 rows with
// 32/8 heads of 128 and norms 32 us for 102 MB, twice what the bytes take: 25 million instructions fill 74 % of the schedulers' slots (sines and keys in
// 64 bits, queries).  Four CTAs to an SM (64 registers) instead of three take 3 us off, five (spills) put 3 on.
#include "kv_rows.cuh"

namespace tetra {
namespace {

struct KvAxes {
    const int32_t* positions;  // [row][axes]
    const uint8_t* axis;       // [D / 2]
    int64_t stride;
    int32_t axes;
};

// Cosine and sine of so many turns, in 64 bits: the nearest quarter is taken off, what is left, pi/4 at most, goes into the two
// Taylor series, which cut behind the 13th and 14th power are off by 2e-14 (pi/4)^15 / 15!.  That is 1e-10 of a key's code, where a general
// function to the last bit costs four times as much, a quarter of the kernel.
__device__ __forceinline__ double2 cosine_sine(double turns) {
    const double quarters = rint(4. * turns), y = 6.283185307179586476925 * fma(-0.25, quarters, turns), z = y * y;
    double s = fma(z, 1. / 6227020800., -1. / 39916800.), c = fma(z, -1. / 87178291200., 1. / 479001600.);
    s = fma(s, z, 1. / 362880.), c = fma(c, z, -1. / 3628800.);
    s = fma(s, z, -1. / 5040.), c = fma(c, z, 1. / 40320.);
    s = fma(s, z, 1. / 120.), c = fma(c, z, -1. / 720.);
    s = fma(s, z, -1. / 6.), c = fma(c, z, 1. / 24.);
    s = fma(s * z, y, y), c = fma(fma(c, z, -0.5), z, 1.);
    const int q = int(int64_t(quarters)) & 3;
    const double u = q & 1 ? s : c, v = q & 1 ? c : s;
    return make_double2(q == 1 || q == 2 ? -u : u, q >= 2 ? -v : v);
}

__device__ __forceinline__ double2 turn_of(const KvRows& p, const KvAxes& t, int row, int pair) {
    const int axis = __ldg(t.axis + pair);
    const int at = axis < t.axes ? __ldg(t.positions + row * t.stride + axis) : 0;
    return cosine_sine(double(at) * __ldg(p.inv_freq + pair) * 0.159154943091895335769);  // 1 / 2 pi
}

// The keys and values of n rows of a block, from row r on: a warp takes a row at a time (keys, then values).
template <int D, typename T>
__device__ __forceinline__ void load_block(const KvRows& p, int64_t r, int n, int head, float (&x)[kAppendTasks][D / 32], int lane, int warp) {
#pragma unroll
    for (int k = 0; k < kAppendTasks; ++k) {
        const int task = warp + kAppendWarps * k;
        if (task >= 2 * n) continue;
        if (task < n) load_row<T>(p.k, (r + task) * p.k_stride + head * D, lane, x[k]);
        else load_row<T>(p.v, (r + task - n) * p.v_stride + head * D, lane, x[k]);
    }
}
template <int D>
__device__ __forceinline__ void turn_block(const KvRows& p, int n, const double2* turns, uint32_t* amax, float (&x)[kAppendTasks][D / 32], int lane, int warp) {
    constexpr int E = D / 32;
#pragma unroll
    for (int k = 0; k < kAppendTasks; ++k) {
        const int task = warp + kAppendWarps * k;
        if (task >= 2 * n) continue;
        if (task < n) {
            double z[E];
            turn<E>(x[k], p.k_weight, p.eps, turns + task * (D / 2), lane, z);
#pragma unroll
            for (int i = 0; i < E; ++i) x[k][i] = float(z[i]);
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(x[k][i]) & 0x7FFFFFFFu);  // NaN is above infinity
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (lane == 0) atomicMax(&amax[task < n ? 0 : 1], top);
    }
}

// Few rows a sequence: a CTA for each row, of which the first of a block does the block's work.
template <int D, typename T>
__global__ void __launch_bounds__(kAppendThreads) k_kv_append_at(KvCache c, KvRows p, KvAxes t) {
    constexpr int E = D / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    double2* turns = reinterpret_cast<double2*>(smem);  // [rows of the block][D / 2]
    __shared__ uint32_t amax[2];                        // keys, values
    pdl_wait();
    pdl_release();
    const int r = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    if (threadIdx.x < 2) amax[threadIdx.x] = 0u;
    int a, b;
    const int s = sequence_of(c, r, lane, a, b);
    if (s < 0) return;
    const int64_t slot = int64_t(__ldg(c.lengths + s)) + (r - a);
    const int first = int(slot & (kKvBlock - 1));
    if (r != a && first != 0) return;
    unsigned char* rec = c.record<D>(s, slot >> 4, head);
    const int rows = min(kKvBlock - first, b - r), n = rec ? rows : 0;
    for (int i = threadIdx.x; i < rows * (D / 2); i += kAppendThreads) turns[i] = turn_of(p, t, r + i / (D / 2), i % (D / 2));
    __syncthreads();
    float x[kAppendTasks][E];
    load_block<D, T>(p, r, n, head, x, lane, warp);
    turn_block<D>(p, n, turns, amax, x, lane, warp);
    for (int j = kAppendWarps - 1 - warp; j < rows * p.group; j += kAppendWarps) {  // queries, from the other end of the warps; none without q
        const int row = j / p.group, h = head * p.group + j - row * p.group;
        float xq[E];
        double z[E];
        load_row<T>(p.q, (r + row) * p.q_stride + int64_t(h) * D, lane, xq);
        turn<E>(xq, p.q_weight, p.eps, turns + row * (D / 2), lane, z);
        __half* out = p.q_out + (int64_t(r + row) * c.kv_heads * p.group + h) * D;
#pragma unroll
        for (int i = 0; i < E; ++i) out[lane + 32 * i] = __double2half(z[i]);
    }
    if (!rec) return;
    finish_block<D>(rec, first, n, amax, x, lane, warp);
}

// N values of a row that lie side by side.
template <typename T, int N>
__device__ __forceinline__ void load_side(const T* from, float (&x)[N]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (N == 1) x[0] = from[0];
        if constexpr (N == 2) {
            const float2 v = *reinterpret_cast<const float2*>(from);
            x[0] = v.x, x[1] = v.y;
        }
        if constexpr (N == 4) {
            const float4 v = *reinterpret_cast<const float4*>(from);
            x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
        }
    } else {
        if constexpr (N == 1) x[0] = __half2float(from[0]);
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            const float2 v = __half22float2(reinterpret_cast<const __half2*>(from)[i / 2]);
            x[i] = v.x, x[i + 1] = v.y;
        }
    }
}

// Many rows a sequence: a CTA for each block.  Queries are most of the work; they are rounded to float16 at the end, so from their
// sines on (made in 64 bits, rounded to 32) they are in 32 bits.  That moves a result by 2^-20 of its pair's two sizes together at most (the sum of
// squares 7 2^-24, its root's reciprocal 4, products, sines and rotation 5), where float16 rounds by 2^-11 of the result.  Keys,
// whose codes a last bit may decide, stay in 64, and so does a row whose norm could leave what 32 bits hold: squares of less than 2^-126 are
// nothing beside a mean of 2^-80, and sums up to 2^108 or products up to 2^100 are far from the end.
// SIDE: rows of q are aligned for loads of a lane's D / 64 neighbours at once.
constexpr float kLeastMean = 8.2718061e-25f, kMostMean = 1.2676506e30f, kMostWeight = 1.1529215e18f;  // 2^-80, 2^100, 2^60
template <int D, typename T, bool SIDE>
__global__ void __launch_bounds__(kAppendThreads, D == 256 ? 3 : 4) k_kv_append_blocks(KvCache c, KvRows p, KvAxes t) {
    constexpr int E = D / 32, N = D / 64, PAIRS = D / 2;
    extern __shared__ __align__(16) unsigned char smem[];
    double2* turns = reinterpret_cast<double2*>(smem);                                                             // [16][D / 2]
    float2* turns32 = reinterpret_cast<float2*>(smem + kKvBlock * PAIRS * sizeof(double2));                        // the same
    unsigned char* made = smem + kKvBlock * PAIRS * (sizeof(double2) + sizeof(float2));                            // a record's codes
    __shared__ uint32_t amax[2];
    pdl_wait();
    pdl_release();
    const int head = blockIdx.y, lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, int(threadIdx.x >> 5), 0);
    if (threadIdx.x < 2) amax[threadIdx.x] = 0u;
    int r, a, b;
    int64_t before;
    const int s = block_of(c, blockIdx.x, lane, r, a, b, before);
    if (s < 0) return;
    const int64_t slot = before + (r - a);
    const int first = int(slot & (kKvBlock - 1));
    unsigned char* rec = c.record<D>(s, slot >> 4, head);
    const int rows = min(kKvBlock - first, b - r), n = rec ? rows : 0;
    float x[kAppendTasks][E];
    load_block<D, T>(p, r, n, head, x, lane, warp);
    // Queries, some of a warp's at a time, the next ones on their way: a lane has N neighbours of either half.
    constexpr int AT_ONCE = N == 4 ? 1 : 4;
    const int heads = c.kv_heads * p.group, step_row = p.group ? kAppendWarps / p.group : 0, step_head = p.group ? kAppendWarps % p.group : 0;
    float next[AT_ONCE][2][N];
    int next_row = p.group ? warp / p.group : rows, next_head = p.group ? warp % p.group : 0;
    auto advance = [&](int& row, int& j) {
        row += step_row, j += step_head;
        if (j >= p.group) j -= p.group, ++row;
    };
    auto load = [&](int row, int j) {
#pragma unroll
        for (int o = 0; o < AT_ONCE; ++o) {
            if (row < rows) {
                const T* from = static_cast<const T*>(p.q) + (int64_t(r) + row) * p.q_stride + int64_t(head * p.group + j) * D + lane * N;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (SIDE) load_side<T, N>(from + k * PAIRS, next[o][k]);
                    else
#pragma unroll
                        for (int i = 0; i < N; ++i) next[o][k][i] = float(from[k * PAIRS + i]);
                }
            }
            advance(row, j);
        }
    };
    load(next_row, next_head);
    for (int i = threadIdx.x; i < rows * PAIRS; i += kAppendThreads) {
        const double2 v = turn_of(p, t, r + i / PAIRS, i % PAIRS);
        turns[i] = v;
        turns32[i] = make_float2(float(v.x), float(v.y));
    }
    __syncthreads();
    turn_block<D>(p, n, turns, amax, x, lane, warp);
    __syncthreads();  // amax
    if (n == kKvBlock) {
        // A whole block: its scales are powers of two, of which the reciprocals are exact, and its bytes are put together here.
        float scale[2], by[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float made_for = scale_for(amax[w]);
            scale[w] = amax[w] >= kInfBits ? __uint_as_float(kNanBits) : made_for;
            by[w] = amax[w] >= kInfBits || made_for == 0.f ? 0.f : __uint_as_float((254u << 23) - __float_as_uint(made_for));
        }
#pragma unroll
        for (int k = 0; k < kAppendTasks; ++k) {
            const int task = warp + kAppendWarps * k, token = task & (kKvBlock - 1);
            const bool key = task < kKvBlock;
            const uint32_t at = key ? ((token & 7) * 4 + (lane >> 3)) * 16 + (token >> 3) * 8 + (lane & 7)
                                    : kKvBlock * D + ((lane >> 2) * 4 + (token & 7) / 2) * 16 + (lane & 3) * 4 + (token >> 3) * 2 + (token & 1);
            const float f = by[key ? 0 : 1];
#pragma unroll
            for (int i = 0; i < E; ++i) made[at + 512 * i] = static_cast<unsigned char>((f == 0.f ? 0 : __float2int_rn(x[k][i] * f)) + 128);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += kAppendThreads) reinterpret_cast<uint4*>(rec)[i] = reinterpret_cast<const uint4*>(made)[i];
        if (threadIdx.x == 0) *reinterpret_cast<float2*>(rec + 2 * kKvBlock * D) = make_float2(scale[0], scale[1]);
    } else if (rec) {
        finish_block<D>(rec, first, n, amax, x, lane, warp);
    }

    if (p.group == 0) return;
    float weight[2][N];
    bool plain = true;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            weight[k][i] = p.q_weight ? __ldg(p.q_weight + k * PAIRS + lane * N + i) : 1.f;
            plain = plain && fabsf(weight[k][i]) <= kMostWeight;
        }
    plain = __all_sync(0xFFFFFFFFu, plain);
    bool all_fine = true;
    while (next_row < rows) {
      float batch[AT_ONCE][2][N];
      int row = next_row, j = next_head;
#pragma unroll
      for (int o = 0; o < AT_ONCE; ++o) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < N; ++i) batch[o][k][i] = next[o][k][i];
        advance(next_row, next_head);
      }
      if (next_row < rows) load(next_row, next_head);
#pragma unroll
      for (int o = 0; o < AT_ONCE; ++o, advance(row, j)) {
        if (row >= rows) break;
        float (&now)[2][N] = batch[o];
        bool fine = true;
        if (p.q_weight) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) sum = fmaf(now[k][i], now[k][i], sum);
#pragma unroll
            for (int m = 16; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
            const float mean = fmaf(sum, 1.f / D, float(p.eps));
            fine = plain && mean >= kLeastMean && mean <= kMostMean;
            all_fine = all_fine && fine;
            const float by = rsqrtf(mean);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < N; ++i) now[k][i] *= by * weight[k][i];
        }
        __half* out = p.q_out + ((int64_t(r) + row) * heads + head * p.group + j) * D + lane * N;
        float lo[N], hi[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 u = turns32[row * PAIRS + lane * N + i];
            lo[i] = now[0][i] * u.x - now[1][i] * u.y;
            hi[i] = now[1][i] * u.x + now[0][i] * u.y;
        }
        if (!fine) continue;
        if constexpr (N == 1) {
            out[0] = __float2half_rn(lo[0]);
            out[PAIRS] = __float2half_rn(hi[0]);
        } else {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                if (SIDE) {
                    *reinterpret_cast<__half2*>(out + i) = __floats2half2_rn(lo[i], lo[i + 1]);
                    *reinterpret_cast<__half2*>(out + PAIRS + i) = __floats2half2_rn(hi[i], hi[i + 1]);
                } else {
                    out[i] = __float2half_rn(lo[i]), out[i + 1] = __float2half_rn(lo[i + 1]);
                    out[PAIRS + i] = __float2half_rn(hi[i]), out[PAIRS + i + 1] = __float2half_rn(hi[i + 1]);
                }
            }
        }
      }
    }
    if (all_fine) return;
    // The others as k_kv_append_at makes them; those next to the border are made twice.
#pragma unroll 1
    for (int row = warp / p.group, j = warp % p.group; row < rows; advance(row, j)) {
        float xq[E], sum = 0.f;
        double z[E];
        const int h = head * p.group + j;
        load_row<T>(p.q, (int64_t(r) + row) * p.q_stride + int64_t(h) * D, lane, xq);
#pragma unroll
        for (int i = 0; i < E; ++i) sum = fmaf(xq[i], xq[i], sum);
#pragma unroll
        for (int m = 16; m >= 1; m >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, m);
        const float mean = fmaf(sum, 1.f / D, float(p.eps));
        if (plain && mean >= 2.f * kLeastMean && mean <= 0.5f * kMostMean) continue;
        turn<E>(xq, p.q_weight, p.eps, turns + row * PAIRS, lane, z);
        __half* out = p.q_out + ((int64_t(r) + row) * heads + h) * D;
#pragma unroll
        for (int i = 0; i < E; ++i) out[lane + 32 * i] = __double2half(z[i]);
    }
}

template <int D, typename T, bool SIDE>
int launch_blocks_for(int blocks, const KvCache& c, const KvRows& p, const KvAxes& t, void* stream) {
    constexpr size_t smem = size_t(kKvBlock) * D / 2 * (sizeof(double2) + sizeof(float2)) + 2 * kKvBlock * D;
    static PerDeviceOnce once;  // per instantiation
    if (smem > 48 * 1024 && once.run([] { return cudaFuncSetAttribute(k_kv_append_blocks<D, T, SIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)); }) != cudaSuccess)
        return TETRA_ERR_CUDA;
    return launch_rows(k_kv_append_blocks<D, T, SIDE>, blocks, c.kv_heads, kAppendThreads, smem, stream, c, p, t);
}
template <typename T, bool SIDE>
int launch_blocks(int D, int blocks, const KvCache& c, const KvRows& p, const KvAxes& t, void* stream) {
    return D == 64 ? launch_blocks_for<64, T, SIDE>(blocks, c, p, t, stream) : D == 128 ? launch_blocks_for<128, T, SIDE>(blocks, c, p, t, stream) : launch_blocks_for<256, T, SIDE>(blocks, c, p, t, stream);
}

}  // namespace
}  // namespace tetra

using namespace tetra;

extern "C" int tetra_kv_append_at(const tetra_kv_cache* cache, const tetra_kv_rows* rows, const tetra_kv_axes* axes, void* stream) {
    KvCache c;
    if (!rows || !axes) return TETRA_ERR_NULL;
    int rc = kv_check(cache, rows->rows, c);
    if (rc != TETRA_OK) return rc;
    const int D = cache->head_dim;
    KvRows p;
    rc = kv_check_rows(*rows, c, D, p);
    if (rc != TETRA_OK) return rc;
    if (!rows->inv_freq || !axes->positions || !axes->axis) return TETRA_ERR_NULL;
    if (axes->axes < 1 || axes->axes > TETRA_KV_MAX_AXES || axes->stride < axes->axes) return TETRA_ERR_SHAPE;
    if (!kv_aligned(axes->positions, 4)) return TETRA_ERR_ALIGN;
    if (c.rows == 0) return TETRA_OK;
    const KvAxes t{axes->positions, axes->axis, axes->stride, axes->axes};
    const int64_t blocks = kv_most_blocks(c);
    if (blocks >= c.rows) {
        auto launch = [&](auto kernel) { return launch_rows(kernel, c.rows, c.kv_heads, kAppendThreads, size_t(kKvBlock) * D / 2 * sizeof(double2), stream, c, p, t); };
        if (rows->half_type) return launch(D == 64 ? k_kv_append_at<64, __half> : D == 128 ? k_kv_append_at<128, __half> : k_kv_append_at<256, __half>);
        return launch(D == 64 ? k_kv_append_at<64, float> : D == 128 ? k_kv_append_at<128, float> : k_kv_append_at<256, float>);
    }
    // What a lane loads and stores at once has to be aligned as one.
    const size_t side = size_t(D / 64) * (rows->half_type ? 2 : 4);
    const bool aligned = kv_aligned(p.q, side) && p.q_stride * (rows->half_type ? 2 : 4) % int64_t(side) == 0 && kv_aligned(p.q_out, 2 * size_t(D / 64));
    return aligned ? (rows->half_type ? launch_blocks<__half, true>(D, int(blocks), c, p, t, stream) : launch_blocks<float, true>(D, int(blocks), c, p, t, stream))
                   : (rows->half_type ? launch_blocks<__half, false>(D, int(blocks), c, p, t, stream) : launch_blocks<float, false>(D, int(blocks), c, p, t, stream));
}
