// The gated feed-forward block for training, over expert-contiguous rows (one expert: a dense block).
//   forward   g = x Wg^T, u = x Wu^T, both kept; h = SiLU(g) (.) u                                  (Eq. 4)
//   backward  dh = dy Wd;  dg = dh u SiLU'(g), du = dh SiLU(g), h again from g and u                (launch 1)
//             dx = dg Wg + du Wu                                                                    (launch 2)
//             dWg = dg^T x, dWu = du^T x, dWd = dy^T h, per expert                                  (launch 3)
// with SiLU(g) = g s, SiLU'(g) = s (1 + g (1 - s)), s = 1 / (1 + exp(-g)).
#include "mma_tile.hpp"

namespace moe {

namespace {

// s = sigmoid(g); exp(-g) = inf gives 0.  The exponential's argument g log2(e) is rounded, so its relative error grows with the gate: with v_exp_f32 and v_rcp_f32 at
// 1 ulp each s is off by ((2 |g| + 2)(1 - s) + 3) 2^-24 of itself at most, 2^-16 at g = -88, below which s (under 2^-126) is zero.  What is formed from
// s is rounded to bf16, 2^-8.
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

struct GatedArgs {
    const uint16_t *x, *wg, *wu;
    const int32_t* offsets;
    uint16_t *g, *u, *h;
    int E, d, F;
};

// Tile: BM rows x BN / 2 features of both projections: the first half of B's rows are the gate's, the second the up projection's,
// so that one copy of the token tile in LDS feeds both and the activation needs nothing but the tile.  g and u pass the caches by: the backward pass
// reads them much later.  Mixtral shape, 8192 rows 2030-2200 us (0.9 PFLOP/s).  Bound by waits (the ring holds two steps): the
// wavefronts spend 49 % of their cycles on them and the matrix cores are 54 % busy at 1.6 GHz, where the inference pair's row-major kernel (which stores h alone) is at 17 % and
// 66 % at the same clock: 1630-1720 us, of which the 0.46 GB of g and u that are stored beside it here would explain 95.  512 tokens 490 / 365, 16 tokens 362 / 295.
template <class S>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void gated_keep_kernel(GatedArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    constexpr int FB = S::BN / 2;
    RowTile t;
    if (!find_tile(a.offsets, a.E, S::BM, (a.F + FB - 1) / FB, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int f0 = t.n * FB, features = a.F - f0 < FB ? a.F - f0 : FB;
    const bool up = wave >= S::WAVES / 2;
    typename S::template LoadA<true> la;
    typename S::template LoadB<true> lb;
    la.init(a.d, wave, lane);
    lb.init(a.d, wave, lane, up ? FB : 0);
    by_height<S>(t.rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, true, true>(acc, Stream<true, S::BK>::make(a.x + (size_t)t.row0 * a.d, a.d, t.rows, a.d),
                                Stream<true, S::BK>::make((up ? a.wu : a.wg) + ((size_t)t.e * a.F + f0) * a.d, a.d, features, a.d), la, lb, a.d / S::BK, lds);
        by_rows<S, FB / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            if (r >= t.rows || c * 8 >= features) return;
            float g[8], u[8], h[8];
            load8(row + c * 8, g);
            load8(row + FB + c * 8, u);
    #pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = g[i] * sigmoid(g[i]) * u[i];
            const size_t at = (size_t)(t.row0 + r) * a.F + f0 + c * 8;
            __builtin_nontemporal_store(pack8(g), reinterpret_cast<u32x4_t*>(a.g + at));
            __builtin_nontemporal_store(pack8(u), reinterpret_cast<u32x4_t*>(a.u + at));
            *reinterpret_cast<u32x4_t*>(a.h + at) = pack8(h);
        });
    });
}

struct GradArgs {
    const uint16_t *x, *wg, *wu, *wd, *g, *u, *dy;
    const int32_t* offsets;
    uint16_t *dg, *du, *h, *dx;
    void *dwg, *dwu, *dwd;     // bf16 or fp32; null: not wanted
    int E, d, F;
    int f32, add;              // weight gradients in fp32; added to what is there
    float* sums;               // [pieces][R, d] of dx, where its sum is cut (rows_pieces)
    int pieces, R;
};

// dh = dy Wd, and from the tile's dh and the kept g and u: dg, du and h.  dg and du are rounded to bf16, as the operands that the
// products of launches 2 and 3 take; g and u are the rounded values that the forward pass kept.  Mixtral shape, 8192 rows 1090 us (0.88 PFLOP/s, with
// 1.2 GB of g, u, dg, du and h read and written beside it).
template <class S>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void gated_grad_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    RowTile t;
    if (!find_tile(a.offsets, a.E, S::BM, (a.F + S::BN - 1) / S::BN, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int f0 = t.n * S::BN;
    typename S::template LoadA<true> la;
    typename S::template LoadB<false> lb;
    la.init(a.d, wave, lane);
    lb.init(a.F, wave, lane);
    by_height<S>(t.rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, true, false>(acc, Stream<true, S::BK>::make(a.dy + (size_t)t.row0 * a.d, a.d, t.rows, a.d),
                                 Stream<false, S::BK>::make(a.wd + (size_t)t.e * a.d * a.F, a.F, f0, a.d), la, lb, a.d / S::BK, lds);
        struct Kept {
            u32x4_t g, u;
        };
        auto kept = [&](int r, int c) {
            const size_t at = (size_t)(t.row0 + (r < t.rows ? r : 0)) * a.F + (f0 + c * 8 < a.F ? f0 + c * 8 : f0);
            return Kept{*reinterpret_cast<const u32x4_t*>(a.g + at), *reinterpret_cast<const u32x4_t*>(a.u + at)};
        };
        by_rows<S, S::BN / 8>(acc, lds, kept, [&](int r, int c, const float* row, const Kept& k) {
            if (r >= t.rows || f0 + c * 8 >= a.F) return;
            const size_t at = (size_t)(t.row0 + r) * a.F + f0 + c * 8;
            float dh[8], g[8], u[8], dg[8], du[8], h[8];
            unpack8(k.g, g);
            unpack8(k.u, u);
            load8(row + c * 8, dh);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float s = sigmoid(g[i]), act = g[i] * s;
                dg[i] = dh[i] * u[i] * (s + act * (1.0f - s));
                du[i] = dh[i] * act;
                h[i] = act * u[i];
            }
            *reinterpret_cast<u32x4_t*>(a.dg + at) = pack8(dg);
            *reinterpret_cast<u32x4_t*>(a.du + at) = pack8(du);
            *reinterpret_cast<u32x4_t*>(a.h + at) = pack8(h);
        });
    });
}

// dx = dg Wg + du Wu: one sum over 2 F.  Mixtral shape, 8192 rows 1850-1950 us (1.0 PFLOP/s; one expert 1490, 1.29).
// CUT: one of `pieces` pieces of that sum (the grid's y) as fp32, for sum_pieces_kernel to add up.
template <class S, bool CUT = false>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void rows_grad_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    RowTile t;
    if (!find_tile(a.offsets, a.E, S::BM, (a.d + S::BN - 1) / S::BN, t)) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int n0 = t.n * S::BN;
    typename S::template LoadA<true> la;
    typename S::template LoadB<false> lb;
    la.init(a.F, wave, lane);
    lb.init(a.d, wave, lane);
    by_height<S>(t.rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        const int all = a.F / S::BK, each = CUT ? (2 * all + a.pieces - 1) / a.pieces : 2 * all, from = CUT ? blockIdx.y * each : 0;
#pragma unroll 1
        for (int m = 0; m < 2; ++m) {              // the gate's part, then the up projection's
            const int s0 = from - m * all > 0 ? from - m * all : 0, end = from + each - m * all, s1 = end < all ? end : all, k0 = s0 * S::BK, k = (s1 - s0) * S::BK;
            multiply<S, MB, true, false>(acc, Stream<true, S::BK>::make((m ? a.du : a.dg) + (size_t)t.row0 * a.F + k0, a.F, t.rows, k, k0),
                                         Stream<false, S::BK>::make((m ? a.wu : a.wg) + ((size_t)t.e * a.F + k0) * a.d, a.d, n0, k), la, lb, s1 - s0, lds);
        }
        if constexpr (CUT) {
            by_rows<S, S::BN / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
                if (r >= t.rows || n0 + c * 8 >= a.d) return;
                float* to = a.sums + ((size_t)blockIdx.y * a.R + t.row0 + r) * a.d + n0 + c * 8;
                *reinterpret_cast<f32x4*>(to) = *reinterpret_cast<const f32x4*>(row + c * 8);
                *reinterpret_cast<f32x4*>(to + 4) = *reinterpret_cast<const f32x4*>(row + c * 8 + 4);
            });
            return;
        }
        by_rows_bf16<S, MB>(acc, lds, [&](int r, int c, u32x4_t v) {
            if (r < t.rows && n0 + c * 8 < a.d) *reinterpret_cast<u32x4_t*>(a.dx + (size_t)(t.row0 + r) * a.d + n0 + c * 8) = v;
        });
    });
}

// dx from the pieces of its sum, in their order; rows behind the last expert stay.
__global__ __launch_bounds__(256) void sum_pieces_kernel(GradArgs a) {
    const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8, n = (size_t)a.R * a.d;
    if (at >= (size_t)a.offsets[a.E] * a.d) return;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    for (int p = 0; p < a.pieces; ++p) {
        float v[8];
        load8(a.sums + p * n + at, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    *reinterpret_cast<u32x4_t*>(a.dx + at) = pack8(sum);
}

// dW[m, n] = sum over the expert's rows of P[row, m] Q[row, n] for the three matrices in one launch (the tails of three would add
// up): tiles [expert][matrix][patch].  An expert without rows gets zeros.  Results pass the caches by.  Mixtral shape, 8192 rows 2720-2850 us (1.03
// PFLOP/s, 2.75 GB written); 64 experts of 250 rows, 3584 x 2560, at skew 1 1480 us, of which 3.5 GB written are 600.  Written / added to, bf16 2830 / 3280 and 1510 / 2560,
// fp32 3460 / 4050 and 2200 / 3350: what is added to is read item by item where it is stored, and passes through the caches.
template <class S>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void weights_grad_kernel(GradArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    const int tm_f = (a.F + S::BM - 1) / S::BM, tn_d = (a.d + S::BN - 1) / S::BN;     // gate, up: [F, d]
    const int tm_d = (a.d + S::BM - 1) / S::BM, tn_f = (a.F + S::BN - 1) / S::BN;     // down: [d, F]
    const int n_g = a.dwg ? tm_f * tn_d : 0, n_u = a.dwu ? tm_f * tn_d : 0, n_d = a.dwd ? tm_d * tn_f : 0, each = n_g + n_u + n_d;
    int t = xcd_run_tile(blockIdx.x, a.E * each);
    if (t < 0) return;
    const int e = t / each;
    t -= e * each;
    const int which = t < n_g ? 0 : t < n_g + n_u ? 1 : 2;
    t -= which == 0 ? 0 : which == 1 ? n_g : n_g + n_u;
    int tm, tn;
    patch(t, which < 2 ? tm_f : tm_d, which < 2 ? tn_d : tn_f, tm, tn);
    const int M = which < 2 ? a.F : a.d, N = which < 2 ? a.d : a.F, m0 = tm * S::BM, n0 = tn * S::BN;
    const uint16_t* P = which == 0 ? a.dg : which == 1 ? a.du : a.dy;
    const uint16_t* Q = which < 2 ? a.x : a.h;
    const int row0 = a.offsets[e], rows = a.offsets[e + 1] - row0;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    typename S::template LoadA<false> la;
    typename S::template LoadB<false> lb;
    la.init(M, wave, lane);
    lb.init(N, wave, lane);
    by_height<S>(M - m0, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        multiply<S, MB, false, false>(acc, Stream<false, S::BK>::make(P + (size_t)row0 * M, M, m0, rows), Stream<false, S::BK>::make(Q + (size_t)row0 * N, N, n0, rows),
                                  la, lb, (rows + S::BK - 1) / S::BK, lds);
        void* const out = which == 0 ? a.dwg : which == 1 ? a.dwu : a.dwd;
        if (!a.f32 && !a.add) {
            by_rows_bf16<S, MB>(acc, lds, [&](int r, int c, u32x4_t v) {
                if (m0 + r >= M || n0 + c * 8 >= N) return;
                u32x4_t* dst = reinterpret_cast<u32x4_t*>(reinterpret_cast<uint16_t*>(out) + ((size_t)e * M + m0 + r) * N + n0 + c * 8);
                __builtin_nontemporal_store(v, dst);
            });
            return;
        }
        by_rows<S, S::BN / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            if (m0 + r >= M || n0 + c * 8 >= N) return;
            const size_t at = ((size_t)e * M + m0 + r) * N + n0 + c * 8;
            float v[8];
            load8(row + c * 8, v);
            if (a.f32) {
                float* dst = reinterpret_cast<float*>(out) + at;
                if (a.add) {
                    float o[8];
                    load8(dst, o);
    #pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += o[i];
                }
                *reinterpret_cast<f32x4*>(dst) = f32x4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(dst + 4) = f32x4{v[4], v[5], v[6], v[7]};
            } else {
                u32x4_t* dst = reinterpret_cast<u32x4_t*>(reinterpret_cast<uint16_t*>(out) + at);
                if (a.add) {
                    float o[8];
                    unpack8(*dst, o);
    #pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] += o[i];
                }
                *dst = pack8(v);
            }
        });
    });
}

__global__ __launch_bounds__(256) void zero_kernel(u32x4_t* p, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = u32x4_t{0, 0, 0, 0};
}

template <class S>
void go_keep(const GatedArgs& a, const moe_config& c, hipStream_t s) {
    const long long tiles = most_blocks(c, S::BM) * ((a.F + S::BN / 2 - 1) / (S::BN / 2));
    hipLaunchKernelGGL(gated_keep_kernel<S>, dim3(16 + xcd_grid(tiles)), dim3(S::THREADS), 0, s, a);
}
template <class S>
void go_gated_grad(const GradArgs& a, const moe_config& c, hipStream_t s) {
    hipLaunchKernelGGL(gated_grad_kernel<S>, dim3(16 + xcd_grid(most_blocks(c, S::BM) * ((a.F + S::BN - 1) / S::BN))), dim3(S::THREADS), 0, s, a);
}
template <class S>
void go_rows_grad(const GradArgs& a, const moe_config& c, hipStream_t s) {
    hipLaunchKernelGGL(rows_grad_kernel<S>, dim3(16 + xcd_grid(most_blocks(c, S::BM) * ((a.d + S::BN - 1) / S::BN))), dim3(S::THREADS), 0, s, a);
}
template <class S>
void go_weights_grad(const GradArgs& a, hipStream_t s) {
    const long long fd = (long long)((a.F + S::BM - 1) / S::BM) * ((a.d + S::BN - 1) / S::BN), df = (long long)((a.d + S::BM - 1) / S::BM) * ((a.F + S::BN - 1) / S::BN);
    hipLaunchKernelGGL(weights_grad_kernel<S>, dim3(xcd_run_grid(a.E * ((a.dwg ? fd : 0) + (a.dwu ? fd : 0) + (a.dwd ? df : 0)))), dim3(S::THREADS), 0, s, a);
}

// Which tiles for rows x N results, from the mean number of rows per expert (the host does not know more): 0 the large ones, 1 Tall, 2 Small.
// Tall where an expert may have more than one block of 128 rows: Mixtral shape, backward, us, with / without it: 512 tokens (128 +- 11 rows per expert) 1454 /
// 1649, 1024 2160 / 2335; at 16 rows per expert it gains nothing (8 experts of 256 x 512, 64 tokens 25.3 / 22.5).
template <class S>
int tiles_for(const moe_config& c, long long N) {
    const long long R = (long long)c.T * c.k, active = R < c.E ? R : c.E, rows = (R + active - 1) / active;
    const bool even = active == 1;
    const long long large = cost<S>(active, rows, N, even), tall = cost<Tall>(active, rows, N, even), small = cost<Small>(active, rows, N, even);
    if (large <= small && (large <= tall || rows <= 64)) return 0;
    return rows > 64 && tall <= small ? 1 : 2;
}

// Pieces that the sum of dx (2 F long) is cut into: where the small tiles are for fewer than half of the CUs (a dense block of few rows, a narrow layer),
// no shorter than sixteen steps (the launch that adds them up takes about 4 us).  Backward pass, us, one sum / cut: dense 2048 x 5632, 1 row 85 / 54, 100 rows
// 111 / 71, 500 143 / 108, 768 x 6848, 11 rows 84 / 34; Mixtral shape, 1 token 719 / 623.
int rows_pieces(const moe_config& c) {
    const long long R = (long long)c.T * c.k, active = R < c.E ? R : c.E, rows = active > 0 ? (R + active - 1) / active : 0;
    const long long tiles = active * ((rows + Small::BM - 1) / Small::BM) * ((c.d + Small::BN - 1) / Small::BN);
    if (tiles == 0 || tiles >= 128) return 1;
    long long n = 256 / tiles;
    const long long most = 2ll * c.F / Small::BK / 16;
    if (n > 16) n = 16;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}

// Weight gradients, n matrices of every expert: Small instead of Pair.
bool small_weight_tiles(const moe_config& c, int n) { return cost<Small>((long long)n * c.E, c.F, c.d) < cost<Pair>((long long)n * c.E, c.F, c.d); }

}  // namespace

size_t rows_grad_bytes(const moe_config& c) {
    const int n = rows_pieces(c);
    return n > 1 ? (size_t)n * c.T * c.k * c.d * sizeof(float) : 0;
}

hipError_t launch_gated_keep(const moe_config& c, const uint16_t* x_rows, const int32_t* offsets, const uint16_t* wg, const uint16_t* wu,
                             uint16_t* g, uint16_t* u, uint16_t* h, hipStream_t s) {
    const GatedArgs a{x_rows, wg, wu, offsets, g, u, h, c.E, c.d, c.F};
    switch (tiles_for<Wide>(c, 2ll * c.F)) {
        case 0: go_keep<Wide>(a, c, s); break;
        case 1: go_keep<Tall>(a, c, s); break;
        default: go_keep<Small>(a, c, s);
    }
    return hipGetLastError();
}

hipError_t launch_ffn_backward(const moe_config& c, const FfnGrad& p, hipStream_t s) {
    const GradArgs a{p.x, p.wg, p.wu, p.wd, p.g, p.u, p.dy, p.offsets, p.dg, p.du, p.h, p.dx, p.dwg, p.dwu, p.dwd, c.E, c.d, c.F, p.f32, p.add, p.sums, rows_pieces(c), c.T * c.k};
    const bool weights = p.dwg || p.dwu || p.dwd;
    if (!(weights && !(c.T == 0 && p.add)) && !(p.dx && c.T > 0)) return hipSuccess;      // nothing is wanted
    if (c.T == 0) {            // no rows: weight gradients of zero, unless they are added to
        const size_t n = (size_t)c.E * c.d * c.F * (p.f32 ? 4 : 2) / 16;
        for (void* w : {p.dwg, p.dwu, p.dwd})
            if (w && !p.add) hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(n / 256 + 1 < 4096 ? n / 256 + 1 : 4096)), dim3(256), 0, s, (u32x4_t*)w, n);
        return hipGetLastError();
    }
    switch (tiles_for<Deep>(c, c.F)) {
        case 0: go_gated_grad<Deep>(a, c, s); break;
        case 1: go_gated_grad<Tall>(a, c, s); break;
        default: go_gated_grad<Small>(a, c, s);
    }
    if (p.dx && a.pieces > 1) {
        const long long tiles = most_blocks(c, Small::BM) * ((a.d + Small::BN - 1) / Small::BN);
        hipLaunchKernelGGL((rows_grad_kernel<Small, true>), dim3(16 + xcd_grid(tiles), a.pieces), dim3(Small::THREADS), 0, s, a);
        hipLaunchKernelGGL(sum_pieces_kernel, dim3((unsigned)(((size_t)a.R * a.d / 8 + 255) / 256)), dim3(256), 0, s, a);
    } else if (p.dx) {
        switch (tiles_for<Deep>(c, c.d)) {
            case 0: go_rows_grad<Deep>(a, c, s); break;
            case 1: go_rows_grad<Tall>(a, c, s); break;
            default: go_rows_grad<Small>(a, c, s);
        }
    }
    if (weights) {
        const int n = (p.dwg != nullptr) + (p.dwu != nullptr) + (p.dwd != nullptr);
        if (small_weight_tiles(c, n)) go_weights_grad<Small>(a, s);
        else go_weights_grad<Pair>(a, s);
    }
    return hipGetLastError();
}

}  // namespace moe

// Test hook (host arithmetic only, not part of include/moe.h): the tiles that a call takes for one of its products.
// product 0: the forward pass's pair, 1: dh, 2: dx, 3: the weight gradients (all three).  0: the large tiles, 1: Tall, 2: Small, 3: Small with the sum in pieces.
extern "C" __attribute__((visibility("default"))) int32_t moe_test_train_tiles(const moe_config* c, int32_t product) {
    using namespace moe;
    switch (product) {
        case 0: return tiles_for<Wide>(*c, 2ll * c->F);
        case 1: return tiles_for<Deep>(*c, c->F);
        case 2: return rows_pieces(*c) > 1 ? 3 : tiles_for<Deep>(*c, c->d);
        default: return small_weight_tiles(*c, 3) ? 2 : 0;
    }
}
