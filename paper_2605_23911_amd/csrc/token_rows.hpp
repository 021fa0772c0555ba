// Rows of tokens and rows of slots: y[t] = sum_i w[t,i] row(t,i) (gather) and row(t,i) = w[t,i] v[t] (scatter), each with the products
// <v[t], row(t,i)> where they are asked for, over slots of which some have no row.  And dropout, whose mask is a function of (seed, offset, element).
//
// A row is read and written through a buffer descriptor of its own, which is empty (range 0) where the slot has no row: loads from it give zeros, stores to it
// are dropped, neither goes to memory, and no branch stands between the loads of a token's rows.  The hardware also ends them at the row's last element.  What comes before them does wait: row numbers
// and weights are fetched slot by slot, each behind the one before (in dispatch's gradient 7 waits for two slots, 19 for eight).
#pragma once

#include "moe_internal.hpp"

namespace moe {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int kTokenThreads = 256;
constexpr int kTokenWaves = kTokenThreads / kWave;

// ---- dropout ----------------------------------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): key = the seed, counter = (block of eight
// elements, offset).  Element j of a block takes bits 16 j .. 16 j + 15 of the 128 and is dropped if they are below `limit` = 65536 p.
struct Dropout {
    const uint64_t* rng;      // device: seed, offset; null: nothing is dropped
    uint32_t limit;
    float scale;              // 65536 / (65536 - limit)
};

__device__ __forceinline__ u32x4_t philox(uint64_t seed, uint64_t block, uint64_t offset) {
    uint32_t x0 = (uint32_t)block, x1 = (uint32_t)(block >> 32), x2 = (uint32_t)offset, x3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)x0 * 0xD2511F53u, b = (uint64_t)x2 * 0xCD9E8D57u;
        x0 = (uint32_t)(b >> 32) ^ x1 ^ k0;
        x1 = (uint32_t)b;
        x2 = (uint32_t)(a >> 32) ^ x3 ^ k1;
        x3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4_t{x0, x1, x2, x3};
}

__device__ __forceinline__ float dropped(float v, u32x4_t bits, int j, const Dropout& p) {
    const uint32_t h = j & 1 ? bits[j / 2] >> 16 : bits[j / 2] & 0xffffu;
    return h >= p.limit ? v * p.scale : 0.0f;
}
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t block, uint64_t seed, uint64_t offset, const Dropout& p) {
    const u32x4_t bits = philox(seed, block, offset);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = dropped(v[j], bits, j, p);
}

// ---- rows -------------------------------------------------------------------------------
typedef __amdgpu_buffer_rsrc_t Row;
// base + at: wave-uniform
__device__ __forceinline__ Row row_at(const void* base, size_t bytes_in_front, bool there, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((char*)const_cast<void*>(base) + (there ? bytes_in_front : 0), 0, there ? bytes : 0, 0x00020000);
}
// eight elements at byte `at` of the row; NT: they pass the caches by
template <bool NT>
__device__ __forceinline__ u32x4_t read8(Row r, int at) { return __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, NT ? 2 : 0); }
template <bool NT>
__device__ __forceinline__ void write8(u32x4_t v, Row r, int at) { __builtin_amdgcn_raw_buffer_store_b128(v, r, at, 0, NT ? 2 : 0); }

__device__ __forceinline__ void floats8(u32x4_t p, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(p[i] << 16), v[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
}
__device__ __forceinline__ u32x4_t bf16s8(const float (&v)[8]) {
    return u32x4_t{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
}

__device__ __forceinline__ float wave_total(float v) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// Slots i0 .. i0 + N - 1 of a token (of its k): a slot without a row, or beyond k, has an empty one and the weight 0.
template <int N>
struct Slots {
    int32_t row[N];
    float w[N];
    bool any;
    // rows: how many there are; row numbers outside 0 .. rows - 1 mean none
    __device__ __forceinline__ void load(const int32_t* row_of, const float* weight, int i0, int k, long long rows) {
        any = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int32_t r = i0 + i < k ? __builtin_amdgcn_readfirstlane(row_of[i0 + i]) : -1;
            row[i] = r >= 0 && r < rows ? r : -1;
            w[i] = row[i] < 0 ? 0.0f : weight ? weight[i0 + i] : 1.0f;
            any |= row[i] >= 0;
        }
    }
    __device__ __forceinline__ Row at(const void* base, int i, int d) const { return row_at(base, (size_t)(uint32_t)(row[i] < 0 ? 0 : row[i]) * d * 2, row[i] >= 0, d * 2); }
};

// Adds up the dot products of a token's N slots over its threads (a wavefront, or the whole workgroup) and stores them, always in the same order; 0 for a slot
// without a row, whatever its zeros were multiplied with.
template <int N>
__device__ __forceinline__ void store_dots(float (&dot)[N], const Slots<N>& s, float (*part)[8], bool whole, int count, float* dw) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < N; ++i) dot[i] = s.row[i] >= 0 ? wave_total(dot[i]) : 0.0f;
    if (!whole) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (lane == i && i < count) dw[i] = dot[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (lane == 0) part[wave][i] = dot[i];
    __syncthreads();
    if ((int)threadIdx.x < count) {
        float sum = part[0][threadIdx.x];
#pragma unroll
        for (int v = 1; v < kTokenWaves; ++v) sum += part[v][threadIdx.x];
        dw[threadIdx.x] = sum;
    }
    __syncthreads();
}

}  // namespace

}  // namespace moe
