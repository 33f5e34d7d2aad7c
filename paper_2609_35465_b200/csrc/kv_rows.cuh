// Pieces shared by the kernels that bring new rows into the key/value cache (kv_append.cu, kv_append_at.cu): a row's norm and
// rotation, a block's scale, checks of arguments, the launch.
#pragma once
#include "kv_common.cuh"

namespace tetra {
namespace {

constexpr int kAppendThreads = 256, kAppendWarps = kAppendThreads / 32;
constexpr int kAppendTasks = 2 * kKvBlock / kAppendWarps;  // rows of keys or values of a block that are a warp's
constexpr uint32_t kInfBits = 0x7F800000u, kNanBits = 0x7FC00000u;

struct KvRows {
    const void *q, *k, *v;
    __half* q_out;
    const double* inv_freq;
    const float *q_weight, *k_weight;
    int64_t q_stride, k_stride, v_stride;
    double eps;
    int32_t group;  // query heads to a kv head
};

template <typename T, int E>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int lane, float (&x)[E]) {
    const T* src = static_cast<const T*>(base) + at;
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = float(src[lane + 32 * i]);
}

// Head norm and rotation of one head's row; `turns`: cosine and sine for each pair, or nullptr.
template <int E>
__device__ __forceinline__ void turn(const float (&x)[E], const float* weight, double eps, const double2* turns, int lane, double (&z)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) z[i] = double(x[i]);
    if (weight) {
        double sum = 0.;
#pragma unroll
        for (int i = 0; i < E; ++i) sum = fma(z[i], z[i], sum);
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        const double by = 1. / sqrt(sum * (1. / (32 * E)) + eps);
#pragma unroll
        for (int i = 0; i < E; ++i) z[i] *= by * double(__ldg(weight + lane + 32 * i));
    }
    if (turns) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const double2 t = turns[lane + 32 * i];
            const double u = z[i], w = z[i + E / 2];
            z[i] = u * t.x - w * t.y;
            z[i + E / 2] = w * t.x + u * t.y;
        }
    }
}

__device__ __forceinline__ float fdiv(float a, float b) { return __fdiv_rn(a, b); }

// The smallest power of two s >= 2^-126 with amax <= 127 s, from amax's bits: 127 = 1.984375 * 2^6.
__device__ __forceinline__ float scale_for(uint32_t amax) {
    if (amax < 0x00800000u) return 0.f;
    const int e = int(amax >> 23) - ((amax & 0x7FFFFFu) <= 0x7E0000u ? 6 : 5);
    return __uint_as_float(uint32_t(e < 1 ? 1 : e) << 23);
}

// A block's scales, and the call's n rows of it from token `first` on, of which each warp holds its tasks' (keys, then values; task
// warp + 8 k in x[k]).  amax, in shared memory: bits of the largest key and value among them; all threads of the CTA come here.
template <int D>
__device__ __forceinline__ void finish_block(unsigned char* rec, int first, int n, const uint32_t* amax, const float (&x)[kAppendTasks][D / 32], int lane, int warp) {
    constexpr int E = D / 32;
    float* scales = reinterpret_cast<float*>(rec + 2 * kKvBlock * D);
    float now[2];
    if (first > 0) {
        const float2 v = *reinterpret_cast<const float2*>(scales);
        now[0] = v.x;
        now[1] = v.y;
    } else {
        now[0] = now[1] = 0.f;
    }
    __syncthreads();  // amax
    bool grew = false;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const uint32_t had = __float_as_uint(now[w]);
        const float before = had & 0x80000000u ? 0.f : now[w];
        const bool spoilt = amax[w] >= kInfBits || (had & 0x7FFFFFFFu) >= kInfBits;
        const float s_new = spoilt ? __uint_as_float(kNanBits) : fmaxf(before, scale_for(amax[w]));
        if (first > 0 && (spoilt || s_new != before)) {  // the codes before, to the new scale
            grew = true;
            const float ratio = spoilt ? 0.f : fdiv(before, s_new);
            if (threadIdx.x < D) {
                uint4* at = reinterpret_cast<uint4*>(rec + w * kKvBlock * D) + threadIdx.x;
                uint4 q = *at;
                uint32_t* words = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t made = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float code = rintf(float(int(words[i] >> (8 * k) & 255u) - 128) * ratio);
                        made |= (uint32_t(int(code) + 128) & 255u) << (8 * k);
                    }
                    words[i] = made;
                }
                *at = q;
            }
        }
        now[w] = s_new;
    }
    if (grew) __syncthreads();  // their bytes share words with the new tokens'
    if (threadIdx.x == 0) *reinterpret_cast<float2*>(scales) = make_float2(now[0], now[1]);
#pragma unroll
    for (int k = 0; k < kAppendTasks; ++k) {
        const int task = warp + kAppendWarps * k;
        if (task >= 2 * n) break;
        const bool key = task < n;
        const int t = first + (key ? task : task - n);  // token of the block
        const float s_now = key ? now[0] : now[1];
        const uint32_t at = key ? ((t & 7) * 4 + (lane >> 3)) * 16 + (t >> 3) * 8 + (lane & 7)
                                : kKvBlock * D + ((lane >> 2) * 4 + (t & 7) / 2) * 16 + (lane & 3) * 4 + (t >> 3) * 2 + (t & 1);
        const bool valued = s_now > 0.f;  // neither 0 nor NaN
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int code = valued ? __float2int_rn(fdiv(x[k][i], s_now)) : 0;
            rec[at + 512 * i] = static_cast<unsigned char>(max(-127, min(127, code)) + 128);
        }
    }
}

template <typename K, typename... Args>
int launch_rows(K kernel, int rows, int heads, int threads, size_t smem, void* stream, Args... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(unsigned(rows), unsigned(heads));
    cfg.blockDim = dim3(unsigned(threads));
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return kv_status(cudaLaunchKernelEx(&cfg, kernel, args...));
}

// What is wrong with the rows of a call, or what the kernels take.
inline int kv_check_rows(const tetra_kv_rows& rows, const KvCache& c, int D, KvRows& p) {
    if (rows.half_type != 0 && rows.half_type != 1) return TETRA_ERR_SHAPE;
    if (!rows.k || !rows.v || !rows.q != !rows.q_out) return TETRA_ERR_NULL;
    const int64_t kv_row = int64_t(c.kv_heads) * D;
    if (rows.k_stride < kv_row || rows.v_stride < kv_row) return TETRA_ERR_SHAPE;
    if (rows.q && (rows.q_heads < 1 || rows.q_heads % c.kv_heads || rows.q_heads > 4096 || rows.q_stride < int64_t(rows.q_heads) * D))
        return TETRA_ERR_SHAPE;
    const size_t size = rows.half_type ? 2 : 4;
    if (!kv_aligned(rows.q, size) || !kv_aligned(rows.k, size) || !kv_aligned(rows.v, size) || !kv_aligned(rows.q_out, 2) ||
        !kv_aligned(rows.inv_freq, 8) || !kv_aligned(rows.q_weight, 4) || !kv_aligned(rows.k_weight, 4))
        return TETRA_ERR_ALIGN;
    if (!(rows.eps >= 0.)) return TETRA_ERR_SHAPE;
    p = KvRows{rows.q, rows.k, rows.v, static_cast<__half*>(rows.q_out), rows.inv_freq, rows.q_weight, rows.k_weight,
                   rows.q_stride, rows.k_stride, rows.v_stride, rows.eps, rows.q ? rows.q_heads / c.kv_heads : 0};
    return TETRA_OK;
}

}  // namespace
}  // namespace tetra
