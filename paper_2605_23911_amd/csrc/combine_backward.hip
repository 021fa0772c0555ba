// Gradients of the weighted combine y[t,:] = sum_i w[t,i] * p[row_of[t*k+i],:]  (Eq. 3):
//   dp[row_of[t*k+i],:] = w[t,i] dy[t,:]        dw[t,i] = <dy[t,:], p[row_of[t*k+i],:]>
#include "mma_tile.hpp"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

// p and dp may be one buffer.  One token per workgroup, up to eight slots at a time: dy's piece is read once for all of them, their rows' pieces are requested
// before the first is used.  Every dp row belongs to one slot, so nothing is added in memory; the dot products are summed in fp32 per
// thread (d / 2048 pieces of eight), over the wavefront and over the four wavefronts, always in the same order.
// Bound by memory: 4096 tokens x 8 x 7168, 1.0 GB, 193-205 us (4.9-5.2 TB/s, a copy's rate; 212 through the caches), 333 x 8 x 3584 9 us.
// STREAM (from 128 MiB of rows on, as in combine.hip): rows and their gradients pass the caches by.
template <int N, bool STREAM>
__device__ __forceinline__ void slots(const uint16_t* __restrict__ dy, const uint16_t* p, const int32_t* __restrict__ rows,
                                      const float* __restrict__ w, int d, uint16_t* dp, float* __restrict__ dw, float (*part)[8]) {
    size_t at[N];
    float wi[N], dot[N];
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = (size_t)rows[i] * d, wi[i] = w[i], dot[i] = 0.0f;
    for (int c = threadIdx.x * 8; c < d; c += kThreads * 8) {
        float v[8];
        u32x4_t row[N];
        const u32x4_t g = *reinterpret_cast<const u32x4_t*>(dy + c);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const u32x4_t* from = reinterpret_cast<const u32x4_t*>(p + at[i] + c);
            row[i] = STREAM ? __builtin_nontemporal_load(from) : *from;
        }
        unpack8(g, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float q[8], o[8];
            unpack8(row[i], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dot[i] = fmaf(v[j], q[j], dot[i]);
                o[j] = wi[i] * v[j];
            }
            u32x4_t* to = reinterpret_cast<u32x4_t*>(dp + at[i] + c);
            if constexpr (STREAM) __builtin_nontemporal_store(pack8(o), to);
            else *to = pack8(o);
        }
    }
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int o = kWave / 2; o > 0; o >>= 1) dot[i] += __shfl_xor(dot[i], o, kWave);
        if (lane == 0) part[wave][i] = dot[i];
    }
    __syncthreads();
    if (threadIdx.x < N) {
        float sum = part[0][threadIdx.x];
#pragma unroll
        for (int v = 1; v < kWaves; ++v) sum += part[v][threadIdx.x];
        dw[threadIdx.x] = sum;
    }
    __syncthreads();
}

template <int K, bool STREAM>
__global__ __launch_bounds__(kThreads) void combine_backward_kernel(const uint16_t* __restrict__ dy, const uint16_t* p,
                                                                   const int32_t* __restrict__ row_of, const float* __restrict__ topk_w, int k, int d,
                                                                   uint16_t* dp, float* __restrict__ dw) {
    __shared__ float part[kWaves][8];
    const size_t t = blockIdx.x;
    dy += t * d;
    row_of += t * (K ? K : k);
    topk_w += t * (K ? K : k);
    dw += t * (K ? K : k);
    if constexpr (K > 0) {
        slots<K, STREAM>(dy, p, row_of, topk_w, d, dp, dw, part);
    } else {
        int i = 0;
        for (; i + 8 <= k; i += 8) slots<8, STREAM>(dy, p, row_of + i, topk_w + i, d, dp, dw + i, part);
        if (k & 4) slots<4, STREAM>(dy, p, row_of + i, topk_w + i, d, dp, dw + i, part), i += 4;
        if (k & 2) slots<2, STREAM>(dy, p, row_of + i, topk_w + i, d, dp, dw + i, part), i += 2;
        if (k & 1) slots<1, STREAM>(dy, p, row_of + i, topk_w + i, d, dp, dw + i, part);
    }
}

}  // namespace

hipError_t launch_combine_backward(const moe_config& c, const uint16_t* dy, const uint16_t* y_perm, const int32_t* row_of, const float* topk_w,
                                   uint16_t* dy_perm, float* d_topk_w, hipStream_t s) {
    const bool stream = (long long)c.T * c.k * c.d >= (1ll << 26);
    auto go = [&](auto k) {
        constexpr int K = decltype(k)::value;
        constexpr int kMost = 1 << 23;         // a launch has less than 2^32 threads
        for (int t = 0; t < c.T; t += kMost) {
            const size_t at = (size_t)t * c.k;
            hipLaunchKernelGGL((stream ? combine_backward_kernel<K, true> : combine_backward_kernel<K, false>), dim3(c.T - t < kMost ? c.T - t : kMost), dim3(kThreads), 0, s,
                               dy + (size_t)t * c.d, y_perm, row_of + at, topk_w + at, c.k, c.d, dy_perm, d_topk_w + at);
        }
    };
    using std::integral_constant;
    switch (c.k) {
        case 1: go(integral_constant<int, 1>{}); break;
        case 2: go(integral_constant<int, 2>{}); break;
        case 3: go(integral_constant<int, 3>{}); break;
        case 4: go(integral_constant<int, 4>{}); break;
        case 5: go(integral_constant<int, 5>{}); break;
        case 6: go(integral_constant<int, 6>{}); break;
        case 7: go(integral_constant<int, 7>{}); break;
        case 8: go(integral_constant<int, 8>{}); break;
        default: go(integral_constant<int, 0>{});
    }
    return hipGetLastError();
}

}  // namespace moe
