// The router's gradient: from those of the gate weights w[t,i] = gate(z[t])[idx[t,i]], z = x W_r^T + bias, to x, W_r and bias.
//   softmax over all experts   dz_e = p_e (G_e - sum_i p_i g_i),  p = softmax(z), G_e = sum of g over the slots that chose e
//   renormalised               dz_i = w_i (g_i - sum_j w_j g_j) for the chosen experts (no logits are needed)
//   sigmoid, normalised        the same times 1 - sigmoid(z_i)
//   dx = dz W_r,  dW_r = dz^T x,  dbias = sum_t dz
// Launches: logits in pieces of d (where needed), dz of a token by a wavefront, dx and dW_r (its sum over the tokens in pieces) side by side, the pieces' sum.
// dz enters the products as three bf16 numbers, all its 24 bits: with two, 16 bits, dx of a router whose rows have a large common part, and dW_r where tokens cancel, lose more
// than their own rounding to bf16.
#include <algorithm>

#include "mma_tile.hpp"

namespace moe {

namespace {

// Tiles of the two products, by the size of one of them, T d E (E in whole tiles of 64), up to 2^31 Low, from there to 2^32 Mid, above that Many; up to 64 tokens Few.
// Smaller tiles fill the CUs with fewer pieces to join and leave a shorter last round; larger ones read less from the caches.  dz, products and join, us, Low / Mid / Many, of the
// renormalised gate, two sets of inputs in turn:
// 256 experts of 7168, 768 tokens 27.6 / 36.5 / 35.1, 1024 32.8 / 36.5 / 36.8, 2048 54.6 / 53.2 / 52.3, 4096 117 / 97.3 / 83.1; 256 of 2048, 2048 27.7 / 29.2 / 33.3, 8192 67.8 / 59.4 / 64.7;
// 128 of 2048, 2048 22.5 / 23.9 / 24.3, 8192 43.6 / 45.4 / 49.9; 64 of 3584, 4096 29.3 / 31.7 / 31.0; 8 of 4096, 2048 19.1 / 19.9 / 20.1, 8192 48.3 / 53.6 / 43.8, 16384 93.4 / 108 / 82.9:
// up to 64 experts fill no more than half of Mid's tiles of dW_r, and it is left out.
typedef Pair Many;
typedef Shape<128, 128, 2, 2, 32, 2, 3, 60> Mid;
typedef Shape<64, 128, 1, 4, 32, 2, 3, 60> Low;
typedef Shape<64, 64, 2, 2, 64, 2, 2, 60> Few;
typedef Shape<64, 128, 1, 4, 64, 4, 1, 60> Slim;        // logits of few tokens
constexpr int kParts = 3;

struct RouteArgs {
    const uint16_t *x, *wr;
    const float* bias;
    const int32_t* idx;
    const float *w, *g;
    uint16_t* dx;
    void* dwr;
    float* dbias;
    int f32, add;
    float* part;       // [logit_pieces][T, Ep]
    uint16_t* dz;      // [T, kParts Ep]: dz rounded, of all experts; what that leaves, rounded; and once more
    float* bias_part;  // [dz_blocks][Ep]
    float* sums;       // [weight_pieces][E, d]
    int T, d, E, k, Ep, gating;
    int logit_pieces, weight_pieces, dz_blocks;
};

// Tile: BM tokens x BN experts, one piece of d.  4096 tokens x 256 experts of 7168: 25-30 us (0.50-0.60 PFLOP/s) with two sets of inputs in turn, x (59 MB) coming from memory; 22.4-24.4
// (0.62-0.67 PFLOP/s, matrix cores 22-24 % busy) with one set again and again, x in the caches.  Compared on such a set: four pieces 22.5, 2: 30, 3: 24.5, 6: 28, 8: 30; Small 22.5, Tall 23,
// Half 24.5, Wide 28, Pair 32, 64 x 256, 128 x 256 and 128 x 128 of four wavefronts 23-24.  Few experts take Flat.
// Products up to 2^31 take Slim, us, Small / Slim (Flat): 256 of 7168, 200 tokens 8.4 / 7.3 (7.0), 512 11.2 / 10.0 (10.6), 1024 11.4 / 10.4 (12.3), 4096 21.8 / 24.4; 128 of 2048, 4096 12.3 / 8.4 (10.9).
template <class S>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void route_logits_kernel(RouteArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    const int cols = (a.E + S::BN - 1) / S::BN, blocks = (a.T + S::BM - 1) / S::BM;
    const int t = xcd_tile(blockIdx.x, a.logit_pieces * blocks * cols);        // [piece][block of tokens][experts]: an XCD's tiles share W_r's piece and x's rows
    if (t < 0) return;
    const int piece = t / (blocks * cols), m0 = t / cols % blocks * S::BM, n0 = t % cols * S::BN;
    const int rows = a.T - m0 < S::BM ? a.T - m0 : S::BM, experts = a.E - n0 < S::BN ? a.E - n0 : S::BN;
    const int all = a.d / S::BK, each = (all + a.logit_pieces - 1) / a.logit_pieces, s0 = piece * each, s1 = s0 + each < all ? s0 + each : all;
    const int k0 = s0 * S::BK, k = (s1 - s0) * S::BK;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    typename S::template LoadA<true> la;
    typename S::template LoadB<true> lb;
    la.init(a.d, wave, lane);
    lb.init(a.d, wave, lane);
    by_height<S>(rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, true, true>(acc, Stream<true, S::BK>::make(a.x + (size_t)m0 * a.d + k0, a.d, rows, k, k0),
                                    Stream<true, S::BK>::make(a.wr + (size_t)n0 * a.d + k0, a.d, experts, k, k0), la, lb, s1 - s0, lds);
        by_rows<S, S::BN / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            if (r >= rows || n0 + c * 8 >= a.Ep) return;
            float* to = a.part + ((size_t)piece * a.T + m0 + r) * a.Ep + n0 + c * 8;
            *reinterpret_cast<f32x4*>(to) = *reinterpret_cast<const f32x4*>(row + c * 8);
            *reinterpret_cast<f32x4*>(to + 4) = *reinterpret_cast<const f32x4*>(row + c * 8 + 4);
        });
    });
}

constexpr int kDzThreads = 256, kDzWaves = kDzThreads / kWave;

__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}
__device__ __forceinline__ float wave_most(float v) {
#pragma unroll
    for (int o = kWave / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, kWave));
    return v;
}

// Slots' experts and gradients, 64 at a time: a lane each, handed to the others through a scalar register.  f(expert, -1 if it is outside 0 .. E - 1; w; g).
template <class F>
__device__ __forceinline__ void for_slots(const RouteArgs& a, size_t t, F&& f) {
    const int lane = threadIdx.x % kWave;
    for (int i0 = 0; i0 < a.k; i0 += kWave) {
        const size_t at = t * a.k + i0 + lane;
        const bool mine = i0 + lane < a.k;
        const int32_t id = mine ? a.idx[at] : -1;
        const float w = mine ? a.w[at] : 0.0f, g = mine ? a.g[at] : 0.0f;
        const int e = (uint32_t)id < (uint32_t)a.E ? id : -1, n = a.k - i0 < kWave ? a.k - i0 : kWave;
        for (int i = 0; i < n; ++i)
            f(__builtin_amdgcn_readlane(e, i), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), i)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(g), i)));
    }
}

// Q numbers of a lane in one access.
template <int Q>
struct Lot;
template <>
struct Lot<1> { typedef float f; typedef uint16_t h; };
template <>
struct Lot<2> { typedef float f __attribute__((ext_vector_type(2))); typedef uint16_t h __attribute__((ext_vector_type(2))); };
template <>
struct Lot<4> { typedef float f __attribute__((ext_vector_type(4))); typedef uint16_t h __attribute__((ext_vector_type(4))); };
template <class V>
__device__ __forceinline__ auto part_of(const V& v, int q) {
    if constexpr (sizeof(V) <= 4 && !std::is_same<V, Lot<2>::h>::value) return v;
    else return v[q];
}

// dz of a token by a wavefront, experts Q lane .. Q lane + Q - 1 in a lane.  The workgroup's share of dbias is summed on the way.  A slot whose expert is outside
// 0 .. E - 1 has no part in anything.
// A weight next to one leaves little of g - c: for the expert of the largest logit, the slot of the largest weight, the difference is formed as (sum of the others' weights) g -
// (sum of the others' w g) instead, which nothing cancels in, so that dz is off as if every g were off by a few of its own roundings.  (With g - c for all, dz of an expert
// with a weight of 1 - 10^-6 was off by several percent.)  The others' sum and 1 - w differ by the weights' own rounding where they add up to one; a slot without an expert has its
// share of the rest.
// Bound by latency: one load of the pieces of the logits, the exchanges between lanes, one store; 4.5 us for a token, 9 for 4096 x 256.
template <int Q>
__global__ __launch_bounds__(kDzThreads) void route_dz_kernel(RouteArgs a) {
    typedef typename Lot<Q>::f Floats;
    typedef typename Lot<Q>::h Halves;
    __shared__ float bias_sum[kDzWaves][Q * kWave];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, e0 = lane * Q;
    const bool held = e0 < a.Ep;          // whole lots: Ep is a multiple of 32
    float bias_acc[Q], bias[Q];
    bool in[Q];                           // the lane's q-th expert exists
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        in[q] = e0 + q < a.E;
        bias_acc[q] = 0.0f;
        bias[q] = a.bias && in[q] ? a.bias[e0 + q] : 0.0f;
    }
    for (int t = blockIdx.x * kDzWaves + wave; t < a.T; t += a.dz_blocks * kDzWaves) {
        float z[Q], dz[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) z[q] = dz[q] = 0.0f;
        if (a.gating != MOE_GATE_SOFTMAX_RENORM) {
            const char* from = reinterpret_cast<const char*>(a.part + (size_t)t * a.Ep + (held ? e0 : 0));
            const size_t each = (size_t)a.T * a.Ep * sizeof(float);
            constexpr int AHEAD = 8;
            for (int p0 = 0; p0 < a.logit_pieces; p0 += AHEAD) {
                Floats v[AHEAD];
#pragma unroll
                for (int p = 0; p < AHEAD; ++p) v[p] = held && p0 + p < a.logit_pieces ? *reinterpret_cast<const Floats*>(from + (p0 + p) * each) : Floats(0.0f);
#pragma unroll
                for (int p = 0; p < AHEAD; ++p)
#pragma unroll
                    for (int q = 0; q < Q; ++q) z[q] += part_of(v[p], q);
            }
#pragma unroll
            for (int q = 0; q < Q; ++q) z[q] += bias[q];
        }
        if (a.gating == MOE_GATE_SOFTMAX) {
            float most = -INFINITY, sum = 0.0f, c = 0.0f, p[Q], top_p = 0.0f, top_g = 0.0f;
            bool top[Q], mine = false;                     // the expert of the largest logit, the first of several
            for_slots(a, t, [&](int e, float, float g) {
#pragma unroll
                for (int q = 0; q < Q; ++q)
                    if (e == e0 + q) dz[q] += g;
            });
#pragma unroll
            for (int q = 0; q < Q; ++q)
                if (in[q]) most = fmaxf(most, z[q]);
            most = wave_most(most);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                top[q] = in[q] && z[q] == most && !mine;
                mine |= top[q];
            }
            const unsigned long long tops = __ballot(mine);
            const int at = tops ? __builtin_ctzll(tops) : 0;        // none: the logits are all NaN
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                top[q] &= lane == at;
                p[q] = in[q] ? expf(z[q] - most) : 0.0f;
                if (top[q]) {
                    top_p = p[q];
                    top_g = dz[q];
                } else {
                    sum += p[q];
                    c = fmaf(p[q], dz[q], c);
                }
            }
            top_p = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top_p), at));
            top_g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(top_g), at));
            sum = wave_add(sum);
            c = wave_add(c);
            const float all = sum + top_p, top_dz = fmaf(sum, top_g, -c) / all;
            c = fmaf(top_p, top_g, c) / all;
#pragma unroll
            for (int q = 0; q < Q; ++q) dz[q] = in[q] ? p[q] / all * (top[q] ? top_dz : dz[q] - c) : 0.0f;
        } else {
            float top_w = 0.0f, top_g = 0.0f, sum = 0.0f, c = 0.0f;      // the slot of the largest weight; sums over the others
            int top = -1, i = 0;
            bool whole = true;                             // every slot has an expert
            for_slots(a, t, [&](int e, float w, float g) {
                if (e >= 0) {
                    const bool more = w > top_w;
                    const float low_w = more ? top_w : w, low_g = more ? top_g : g;
                    sum += low_w;
                    c = fmaf(low_w, low_g, c);
                    if (more) {
                        top_w = w;
                        top_g = g;
                        top = i;
                    }
                } else {
                    whole = false;
                }
                ++i;
            });
            const float rest = 1.0f - top_w, rounding = (a.k + 4) * 0x1p-24f;
            const float top_dz = fmaf(whole && fabsf(sum - rest) <= rounding ? sum : rest, top_g, -c);
            c = fmaf(top_w, top_g, c);
            i = 0;
            for_slots(a, t, [&](int e, float w, float g) {
                const float v = w * (i == top ? top_dz : g - c);
#pragma unroll
                for (int q = 0; q < Q; ++q)
                    if (e == e0 + q) dz[q] += v;
                ++i;
            });
            if (a.gating == MOE_GATE_SIGMOID_NORM) {
#pragma unroll
                for (int q = 0; q < Q; ++q) dz[q] = dz[q] != 0.0f ? dz[q] / (1.0f + expf(z[q])) : 0.0f;
            }
        }
        uint16_t* to = a.dz + (size_t)t * kParts * a.Ep + e0;
        float left[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            bias_acc[q] += dz[q];
            left[q] = dz[q];
        }
#pragma unroll
        for (int h = 0; h < kParts; ++h) {
            Halves out;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const uint16_t v = float_to_bf16_bits(left[q]);
                if constexpr (Q == 1) out = v;
                else out[q] = v;
                left[q] -= bf16_bits_to_float(v);
            }
            if (held) *reinterpret_cast<Halves*>(to + h * a.Ep) = out;
        }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) bias_sum[wave][e0 + q] = bias_acc[q];
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kDzThreads) {
        float v = bias_sum[0][e];
#pragma unroll
        for (int i = 1; i < kDzWaves; ++i) v += bias_sum[i][e];
        a.bias_part[(size_t)blockIdx.x * a.Ep + e] = v;
    }
}

// Tile of dx = dz W_r, dz's parts one after the other in each step.
template <class S>
__device__ __forceinline__ void dx_tile(const RouteArgs& a, int m0, int n0, char* lds) {
    const int rows = a.T - m0 < S::BM ? a.T - m0 : S::BM, ld = kParts * a.Ep;
    const int wave = __builtin_amdgcn_readfirstlane(body_thread() / kWave), lane = body_thread() % kWave;
    typename S::template LoadA<true> la;
    typename S::template LoadB<false> lb;
    la.init(ld, wave, lane);
    lb.init(a.d, wave, lane);
    by_height<S>(rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, true, false>(acc, Stream<true, S::BK>::make(a.dz + (size_t)m0 * ld, ld, rows, a.Ep), Stream<false, S::BK>::make(a.wr, a.d, n0, a.E), la, lb,
                                     a.Ep / S::BK, lds, (uint32_t)a.Ep * 2);
        by_rows_bf16<S, MB>(acc, lds, [&](int r, int c, u32x4_t v) {
            if (r < rows && n0 + c * 8 < a.d) *reinterpret_cast<u32x4_t*>(a.dx + (size_t)(m0 + r) * a.d + n0 + c * 8) = v;
        });
    });
}

// Eight elements of dW_r, on top of what it holds or not.
__device__ __forceinline__ void store_weights(const RouteArgs& a, size_t at, float (&sum)[8]) {
    float v[8];
    if (a.f32) {
        float* to = reinterpret_cast<float*>(a.dwr) + at;
        if (a.add) {
            load8(to, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
        *reinterpret_cast<f32x4*>(to) = f32x4{sum[0], sum[1], sum[2], sum[3]};
        *reinterpret_cast<f32x4*>(to + 4) = f32x4{sum[4], sum[5], sum[6], sum[7]};
    } else {
        u32x4_t* to = reinterpret_cast<u32x4_t*>(reinterpret_cast<uint16_t*>(a.dwr) + at);
        if (a.add) {
            unpack8(*to, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
        *to = pack8(sum);
    }
}

// dbias of sixteen experts, from the sums of the workgroups that formed dz; by any number of threads that is a multiple of sixteen, up to 512.
constexpr int kBiasExperts = 16;
template <int THREADS>
__device__ __forceinline__ void bias_group(const RouteArgs& a, int group, float (*part)[kBiasExperts]) {
    constexpr int SEGS = THREADS / kBiasExperts;
    const int mine = threadIdx.x % kBiasExperts, e = group * kBiasExperts + mine, seg = threadIdx.x / kBiasExperts;
    float v = 0.0f;
    if (e < a.E) {
#pragma unroll 8
        for (int b = seg; b < a.dz_blocks; b += SEGS) v += a.bias_part[(size_t)b * a.Ep + e];
    }
    part[seg][mine] = v;
    __syncthreads();
    if (seg == 0 && e < a.E) {
        float sum = a.add ? a.dbias[e] : 0.0f;
        for (int i = 0; i < SEGS; ++i) sum += part[i][mine];
        a.dbias[e] = sum;
    }
}
__host__ __device__ inline int bias_groups(const RouteArgs& a) { return a.dbias ? (a.E + kBiasExperts - 1) / kBiasExperts : 0; }

// Tile of dW_r = dz^T x over one piece of the tokens, dz's parts one after the other in each step.
template <class S>
__device__ __forceinline__ void dw_tile(const RouteArgs& a, int piece, int m0, int n0, char* lds) {
    const int all = (a.T + S::BK - 1) / S::BK, each = (all + a.weight_pieces - 1) / a.weight_pieces, s0 = piece * each, s1 = s0 + each < all ? s0 + each : all;
    const int t0 = s0 * S::BK, tokens = a.T - t0 < (s1 - s0) * S::BK ? a.T - t0 : (s1 - s0) * S::BK, ld = kParts * a.Ep;
    const int wave = __builtin_amdgcn_readfirstlane(body_thread() / kWave), lane = body_thread() % kWave;
    typename S::template LoadA<false> la;
    typename S::template LoadB<false> lb;
    la.init(ld, wave, lane);
    lb.init(a.d, wave, lane);
    by_height<S>(a.E - m0, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, false, false>(acc, Stream<false, S::BK>::make(a.dz + (size_t)t0 * ld, ld, m0, tokens), Stream<false, S::BK>::make(a.x + (size_t)t0 * a.d, a.d, n0, tokens),
                                      la, lb, s1 - s0, lds, (uint32_t)a.Ep * 2);
        by_rows<S, S::BN / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            if (m0 + r >= a.E || n0 + c * 8 >= a.d) return;
            const size_t at = (size_t)(m0 + r) * a.d + n0 + c * 8;
            if (a.weight_pieces == 1) {
                float v[8];
                load8(row + c * 8, v);
                return store_weights(a, at, v);
            }
            float* to = a.sums + (size_t)piece * a.E * a.d + at;
            *reinterpret_cast<f32x4*>(to) = *reinterpret_cast<const f32x4*>(row + c * 8);
            *reinterpret_cast<f32x4*>(to + 4) = *reinterpret_cast<const f32x4*>(row + c * 8 + 4);
        });
    });
}

// Both products in one launch, and dbias.  The tiles of dW_r, which are several times as long, come first: one per CU at most (weight_pieces_of), whose other workgroups
// take tiles of dx; in turn with them a CU gets two (4096 x 256 x 7168: 92 us instead of 74).
// Two long steps per ring: a step holds all parts of dz and the panel that they are multiplied with, which is loaded once and read from LDS once.  Mixtral-sized weights' gradients
// have the same layouts (both operands with k across the rows).  4096 tokens x 256 experts of 7168: 90 GFLOP in 78 us (1.15 PFLOP/s; matrix
// cores 56 % busy at 1.94 GHz, 23 % of the wave cycles waits; with two parts for dx 75 GFLOP in 70).
// How it got there, with two parts for dx, us: dx and dW_r one after the other 95 (two parts for dW_r, too), in one launch 86, part by part through all steps 83, one tile of dW_r per
// CU 74, shared panels 70.
template <class S>
constexpr int products_per_cu() { return 160 * 1024 / Parted<S, kParts, 2>::kLds < S::PER ? 160 * 1024 / Parted<S, kParts, 2>::kLds : S::PER; }
template <class S>
__global__ __launch_bounds__(S::THREADS, (products_per_cu<S>() * S::WAVES / 4)) void route_products_kernel(RouteArgs a) {
    using P = Parted<S, kParts, 2>;
    __shared__ __attribute__((aligned(1024))) char lds[P::kLds];
    const int cols = (a.d + S::BN - 1) / S::BN, heads = (a.E + S::BM - 1) / S::BM, blocks = (a.T + S::BM - 1) / S::BM;
    const int weights = a.dwr ? a.weight_pieces * cols * heads : 0, rows = a.dx ? blocks * cols : 0, ids_w = (weights + 7) / 8 * 8, ids_r = (rows + 7) / 8 * 8;
    const int id = blockIdx.x;
    if (id >= ids_w + ids_r) return bias_group<S::THREADS>(a, id - ids_w - ids_r, reinterpret_cast<float(*)[kBiasExperts]>(lds));
    if (id < ids_w) {
        const int t = xcd_tile(id, weights);
        if (t >= 0) dw_tile<P>(a, t / (cols * heads), t % heads * S::BM, t / heads % cols * S::BN, lds);
        return;
    }
    const int t = xcd_tile(id - ids_w, rows);
    if (t < 0) return;
    int m, n;
    patch(t, blocks, cols, m, n);
    dx_tile<P>(a, m * S::BM, n * S::BN, lds);
}

// The pieces of dW_r, eight elements per thread, in their order: 7 us for four of 256 x 7168 (37 MB), 4 for small ones.
__global__ __launch_bounds__(256) void route_join_kernel(RouteArgs a) {
    const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8, n = (size_t)a.E * a.d;
    if (at >= n) return;
    float sum[8], v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
#pragma unroll 4
    for (int p = 0; p < a.weight_pieces; ++p) {
        load8(a.sums + p * n + at, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    store_weights(a, at, sum);
}

// dbias where there is nothing else to do.
__global__ __launch_bounds__(256) void route_bias_kernel(RouteArgs a) {
    __shared__ float part[256 / kBiasExperts][kBiasExperts];
    bias_group<256>(a, blockIdx.x, part);
}

bool few_tokens(const moe_config& c) { return c.T <= Few::BM; }
// Experts rounded up to whole steps of the products' reduction.
static_assert(Mid::BK == Many::BK && Low::BK == Many::BK, "one padding");
int padded(const moe_config& c) { return few_tokens(c) ? (c.E + Few::BK - 1) / Few::BK * Few::BK : (c.E + Many::BK - 1) / Many::BK * Many::BK; }
bool few_experts(const moe_config& c) { return c.E <= Flat::BM; }

constexpr int kMostPieces = 16;
template <class S>
int logit_pieces_of(const moe_config& c) {
    const long long tiles = (long long)((c.T + S::BM - 1) / S::BM) * ((c.E + S::BN - 1) / S::BN), most = c.d / S::BK / 4;
    long long n = tiles > 0 ? 256 * S::PER / tiles : 1;
    if (n > kMostPieces) n = kMostPieces;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}
long long size_of_product(const moe_config& c) { return (long long)c.T * c.d * ((c.E + 63) / 64 * 64); }
bool low(const moe_config& c) { return size_of_product(c) <= 1LL << 31; }
bool mid(const moe_config& c) { return size_of_product(c) <= 1LL << 32 && c.E > 64; }
int logit_pieces(const moe_config& c) {
    if (c.gating == MOE_GATE_SOFTMAX_RENORM) return 0;
    return few_experts(c) ? logit_pieces_of<Flat>(c) : low(c) ? logit_pieces_of<Slim>(c) : logit_pieces_of<Small>(c);
}
// Pieces of the tokens that dW_r is summed over: one tile of it per CU, beside which the CU's other workgroups take tiles of dx; no shorter than four steps.
template <class S>
int weight_pieces_of(const moe_config& c) {
    const long long tiles = (long long)((c.d + S::BN - 1) / S::BN) * ((c.E + S::BM - 1) / S::BM), most = c.T / (4 * S::BK);
    long long n = 256 / tiles;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}
int weight_pieces(const moe_config& c) {
    return few_tokens(c) ? weight_pieces_of<Few>(c) : low(c) ? weight_pieces_of<Low>(c) : mid(c) ? weight_pieces_of<Mid>(c) : weight_pieces_of<Many>(c);
}
int dz_blocks(const moe_config& c) {
    const int n = (c.T + kDzWaves - 1) / kDzWaves;
    return n < 1024 ? n : 1024;
}

// The size never falls as T grows, so that a workspace for the most tokens does for fewer: rows as wide as for the few; the logits' tiles, as many as the CUs hold where they are cut
// into pieces, at their most.  (The pieces of dW_r only grow in number, as its tiles grow.)
struct RouteSpace {
    size_t part, dz, bias, sums, total;
};
template <class S>
constexpr size_t tiles_of_all_cus() { return (size_t)256 * S::PER * S::BM * S::BN; }
RouteSpace space(const moe_config& c) {
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const size_t T = c.T, Ep = (c.E + Few::BK - 1) / Few::BK * Few::BK, full = few_experts(c) ? tiles_of_all_cus<Flat>() : tiles_of_all_cus<Small>();
    static_assert(tiles_of_all_cus<Slim>() <= tiles_of_all_cus<Small>() && Few::BK % Many::BK == 0, "room for both");
    RouteSpace s;
    s.part = take(logit_pieces(c) > 0 ? std::max(T * Ep, std::min(kMostPieces * T * Ep, full)) * sizeof(float) : 0);
    s.dz = take(T * kParts * Ep * sizeof(uint16_t));
    s.bias = take((size_t)dz_blocks(c) * Ep * sizeof(float));
    s.sums = take(weight_pieces(c) > 1 ? (size_t)weight_pieces(c) * c.E * c.d * sizeof(float) : 0);
    s.total = at;
    return s;
}

template <class S>
void go_logits(const RouteArgs& a, hipStream_t s) {
    const long long tiles = (long long)a.logit_pieces * ((a.T + S::BM - 1) / S::BM) * ((a.E + S::BN - 1) / S::BN);
    hipLaunchKernelGGL(route_logits_kernel<S>, dim3(xcd_grid(tiles)), dim3(S::THREADS), 0, s, a);
}
template <class S>
void go_products(const RouteArgs& a, hipStream_t s) {
    const long long cols = (a.d + S::BN - 1) / S::BN, weights = a.dwr ? a.weight_pieces * cols * ((a.E + S::BM - 1) / S::BM) : 0, rows = a.dx ? cols * ((a.T + S::BM - 1) / S::BM) : 0;
    const dim3 grid(xcd_grid(weights) + xcd_grid(rows) + bias_groups(a));
    hipLaunchKernelGGL(route_products_kernel<S>, grid, dim3(S::THREADS), 0, s, a);
}

}  // namespace

size_t route_backward_workspace_bytes(const moe_config& c) { return space(c).total; }

hipError_t launch_route_backward(const moe_config& c, const RouteGrad& p, hipStream_t s) {
    const RouteSpace at = space(c);
    RouteArgs a{p.x, p.wr, p.bias, p.idx, p.w, p.g, p.dx, p.dwr, p.dbias, p.f32, p.add, (float*)(p.workspace + at.part), (uint16_t*)(p.workspace + at.dz),
                (float*)(p.workspace + at.bias), (float*)(p.workspace + at.sums), c.T, c.d, c.E, c.k, padded(c), c.gating,
                logit_pieces(c), c.T > 0 ? weight_pieces(c) : 0, dz_blocks(c)};
    const bool add_nothing = c.T == 0 && p.add;
    if (add_nothing || (!(p.dx && c.T > 0) && !p.dwr && !p.dbias)) return hipSuccess;
    const unsigned joins = (unsigned)(((size_t)c.E * c.d / 8 + 255) / 256);
    if (c.T == 0) {            // sums over nothing
        if (p.dwr) hipLaunchKernelGGL(route_join_kernel, dim3(joins), dim3(256), 0, s, a);
        if (p.dbias) hipLaunchKernelGGL(route_bias_kernel, dim3(bias_groups(a)), dim3(256), 0, s, a);
        return hipGetLastError();
    }
    if (a.logit_pieces > 0) {
        if (few_experts(c)) go_logits<Flat>(a, s);
        else if (low(c)) go_logits<Slim>(a, s);
        else go_logits<Small>(a, s);
    }
    if (a.Ep <= kWave) hipLaunchKernelGGL(route_dz_kernel<1>, dim3(a.dz_blocks), dim3(kDzThreads), 0, s, a);
    else if (a.Ep <= 2 * kWave) hipLaunchKernelGGL(route_dz_kernel<2>, dim3(a.dz_blocks), dim3(kDzThreads), 0, s, a);
    else hipLaunchKernelGGL(route_dz_kernel<4>, dim3(a.dz_blocks), dim3(kDzThreads), 0, s, a);
    if (!p.dx && !p.dwr) hipLaunchKernelGGL(route_bias_kernel, dim3(bias_groups(a)), dim3(256), 0, s, a);
    else if (few_tokens(c)) go_products<Few>(a, s);
    else if (low(c)) go_products<Low>(a, s);
    else if (mid(c)) go_products<Mid>(a, s);
    else go_products<Many>(a, s);
    if (p.dwr && a.weight_pieces > 1) hipLaunchKernelGGL(route_join_kernel, dim3(joins), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace moe
