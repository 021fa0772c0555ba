// Low-rank adapters of many requests at once beside a shared projection:
//   y[t] = (base[t] +) x[t] W^T + scale[a] (x[t] A[a]^T) B[a]^T,   a = adapter_of[t]
// and the gated pair of two such projections of one input, h = SiLU(gate) (.) up.
// Always two launches: v[t] = scale[a] x[t] A[a]^T has to be whole before it meets B.
//   prompts         low_rank_kernel forms v; adapter_rows_kernel takes v[t] B[a]^T as `rank` more elements of the projection's reduction, so
//                   the result is rounded once and never read back.
//   decode batches  adapter_part_kernel forms v and x W^T side by side, in pieces of K where there are few tiles; adapter_join_kernel adds
//                   v B^T to the sums.  (And projections with few tiles.)
// Tokens stay in the caller's order: a block of tokens goes through the adapters that occur in it one after the other, the other
// tokens' v masked to zero.  Tokens of a request lie together in a prompt (one adapter per block); in a decode batch every adapter is
// needed anyway.
#include "mma_tile.hpp"

namespace moe {

namespace {

struct AdapterArgs {
    const uint16_t* x;                // [T, K]
    const uint16_t *w[2], *a[2], *b[2];   // [N, K], [n, rank, K], [n, N, rank]; the gated pair has two of each
    const float* scale;               // [n] or null
    const int32_t* of;                // [T]
    const uint16_t* base;             // [T, N] or null
    float* v;                         // [parts][matrices][T][rank] partial sums over K
    float* sums;                      // [splits][matrices][T][N] the projection's, where its launch has too few tiles (adapter_part_kernel)
    int splits;
    uint16_t* y;                      // [T, N]
    int T, N, K, n, rank;
    int parts, lists;                 // pieces of K that v is summed in; adapters' workgroups per block of tokens
};

constexpr int kThreads = 512, kWaves = kThreads / kWave;       // of the kernels that are not tiled

__device__ __forceinline__ bf16x8 zeros8() { return bf16x8{0, 0, 0, 0, 0, 0, 0, 0}; }
// Adapter of a token; -1 where it has none (an id outside 0 .. n - 1 means that too).
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int t) {
    const int a = t < p.T ? p.of[t] : -1;
    return a >= 0 && a < p.n ? a : -1;
}

// v: a workgroup takes 32 tokens, one piece of K, and of the adapters that occur in the block every lists-th.  Its eight wavefronts split the
// piece again and are joined through LDS.  Bound by the latency of a few dependent loads: 4096 tokens of K = 4096, two adapters of rank 16 22 us,
// 1999 of 2048, rank 32 12 us (x read at 1.5 and 0.7 TB/s).
template <int RB, int MATS>
__global__ __launch_bounds__(kThreads) void low_rank_kernel(AdapterArgs p) {
    __shared__ float part[kWaves][32][RB * 32 + 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, r = lane & 31, half = lane >> 5;
    const int block = blockIdx.x / (p.lists * p.parts), rest = blockIdx.x % (p.lists * p.parts), list = rest / p.parts, piece = rest % p.parts;
    const int t0 = block * 32, t = t0 + r;
    const int steps = p.K / 16, each = (steps + p.parts * kWaves - 1) / (p.parts * kWaves);
    const int s0 = (piece * kWaves + wave) * each, s1 = s0 + each < steps ? s0 + each : steps;
    const int id = adapter_of(p, t);
    unsigned long long left = __ballot(id >= 0) & 0xffffffffull;
    const uint16_t* x = p.x + (size_t)(t < p.T ? t : p.T - 1) * p.K + half * 8;
    for (int i = 0; left != 0; ++i) {
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const bool mine = id == a;
        left &= ~__ballot(mine);
        if (i % p.lists != list) continue;
        f32x16 acc[MATS][RB];
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[m][b][q] = 0.0f;
        const uint16_t* rows[MATS][RB];
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int row = b * 32 + r;
                rows[m][b] = p.a[m] + ((size_t)a * p.rank + (row < p.rank ? row : p.rank - 1)) * p.K + half * 8;
            }
        // U steps' loads are under way at once; those past the end are zeros on both sides
        constexpr int LOADS = 1 + MATS * RB, U = LOADS <= 3 ? 8 : LOADS <= 5 ? 4 : 2;
        for (int s = s0; s < s1; s += U) {
            bf16x8 fx[U], fa[U][MATS][RB];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int at = (s + i < s1 ? s + i : s1 - 1) * 16;
                fx[i] = *reinterpret_cast<const bf16x8*>(x + at);
#pragma unroll
                for (int m = 0; m < MATS; ++m)
#pragma unroll
                    for (int b = 0; b < RB; ++b) fa[i][m][b] = *reinterpret_cast<const bf16x8*>(rows[m][b] + at);
            }
            __builtin_amdgcn_sched_barrier(0);     // else the compiler waits for each load before it issues the next, to save registers
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const bool in = s + i < s1;
                const bf16x8 vx = in ? fx[i] : zeros8();
#pragma unroll
                for (int m = 0; m < MATS; ++m)
#pragma unroll
                    for (int b = 0; b < RB; ++b) acc[m][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(in ? fa[i][m][b] : zeros8(), vx, acc[m][b], 0, 0, 0);
            }
        }
        const float scale = p.scale ? p.scale[a] : 1.0f;
        const unsigned here = (unsigned)__ballot(mine);          // the block's tokens with this adapter
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            __syncthreads();
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int q = 0; q < 16; ++q) part[wave][r][b * 32 + (q / 4) * 8 + half * 4 + q % 4] = acc[m][b][q];
            __syncthreads();
            for (int j = threadIdx.x; j < 32 * p.rank; j += kThreads) {
                const int row = j / p.rank, c = j % p.rank;
                if (!((here >> row) & 1)) continue;
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += part[w][row][c];
                p.v[(((size_t)piece * MATS + m) * p.T + t0 + row) * p.rank + c] = sum * scale;
            }
        }
    }
}

// Takes over what an adapter adds for the lanes whose token (a lane holds one token's results) has it: a masked zero times an infinity or a
// NaN in another request's adapter would be NaN.
template <class V>
__device__ __forceinline__ void keep_mine(V& acc, V with, bool mine) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(V) / 4); ++i) acc[i] = mine ? with[i] : acc[i];
}

// Eight elements of a token's v, the pieces' sum, as two bf16 numbers each: rounded once, v would add 2^-8 of the adapter's part to the error, as much as
// the result's own rounding; with what the first leaves it is 2^-16, for one more multiplication per `rank` elements of the reduction.
struct Pair8 {
    u32x4_t hi, lo;
};
__device__ __forceinline__ Pair8 low_rank8(const AdapterArgs& p, int mats, int m, int t, int c) {
    float sum[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
    for (int q = 0; q < p.parts; ++q) {
        float v[8];
        load8(p.v + (((size_t)q * mats + m) * p.T + t) * p.rank + c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    Pair8 r;
    r.hi = pack8(sum);
    unpack8(r.hi, hi);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = fabsf(hi[i]) < INFINITY ? sum[i] - hi[i] : 0.0f;     // an infinity stays one
    r.lo = pack8(sum);
    return r;
}

__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

constexpr int kMaxRank = 128, kPiece = 64;         // of the rank, at a time


// Many tokens: tiles of the projection as in ffn_train.hip, then the adapters of the tile's tokens, 64 of the rank at a time.  4096 tokens of six
// prompts, 4096 -> 2 x 14336, rank 16 770-840 us (1.15-1.25 PFLOP/s; matrix cores 61 % busy at 1.8 GHz, the wavefronts wait for 46 % of their cycles); 1999 tokens, 2048 ->
// 7168 64 us.  Where a block holds many adapters they are what takes the time, two multiplications per 16 of the rank for each (splits, below).
template <class S, int MATS>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void adapter_rows_kernel(AdapterArgs p) {
    constexpr int FB = S::BN / MATS, kRow = 2 * kPiece * 2 + 16, kV = MATS * S::BM * kRow;   // bytes of a token's v in LDS: a piece of the rank
    __shared__ __attribute__((aligned(1024))) char lds[(S::kLds > kV ? S::kLds : kV) + S::BM * 4];
    const int tm_n = (p.T + S::BM - 1) / S::BM, tn_n = (p.N + FB - 1) / FB;
    const int t = xcd_tile(blockIdx.x, tm_n * tn_n);
    if (t < 0) return;
    int tm, tn;
    patch(t, tm_n, tn_n, tm, tn);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
    const int t0 = tm * S::BM, rows = p.T - t0 < S::BM ? p.T - t0 : S::BM, n0 = tn * FB, cols = p.N - n0 < FB ? p.N - n0 : FB;
    int32_t* const ids = reinterpret_cast<int32_t*>(lds + (S::kLds > kV ? S::kLds : kV));
    for (int i = tid; i < S::BM; i += S::THREADS) ids[i] = adapter_of(p, t0 + i);
    __syncthreads();           // without a shared projection nothing else stands between this and the reads
    by_height<S>(rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        {
            const bool second = MATS == 2 && wave >= S::WAVES / 2;
            typename S::template LoadA<true> la;
            typename S::template LoadB<true> lb;
            la.init(p.K, wave, lane);
            lb.init(p.K, wave, lane, second ? FB : 0);
            const uint16_t* w = second ? p.w[1] : p.w[0];
            multiply<S, MB, true, true>(acc, Stream<true, S::BK>::make(p.x + (size_t)t0 * p.K, p.K, rows, p.K), Stream<true, S::BK>::make(w + (size_t)n0 * p.K, p.K, cols, p.K),
                                    la, lb, w ? p.K / S::BK : 0, lds);
        }
        // What the rest derives from the thread's number is worked out here, not held in registers through the reduction.
        const int tid2 = body_thread(), lane2 = tid2 % kWave;
        const int r = lane2 & 31, half = lane2 >> 5, c0 = wn * S::NB * 32, m2 = MATS == 2 && c0 >= FB ? 1 : 0;
        int id[MB];
#pragma unroll
        for (int m = 0; m < MB; ++m) id[m] = ids[(wm * MB + m) * 32 + r];
        uint32_t brow[S::NB];              // byte offset of the lane's row of B
#pragma unroll
        for (int n = 0; n < S::NB; ++n) {
            const int col = n0 + c0 - m2 * FB + n * 32 + r;
            brow[n] = (uint32_t)((col < p.N ? col : p.N - 1) * p.rank + half * 8) * 2u;
        }
#pragma unroll 1
        for (int base = 0; base < p.rank; base += kPiece) {
            // the tile's v, this piece of the rank
            const int chunks = (p.rank - base < kPiece ? p.rank - base : kPiece) / 8;
            for (int j = tid2; j < MATS * S::BM * chunks; j += S::THREADS) {
                const int c = j % chunks, row = j / chunks % S::BM, m = j / chunks / S::BM;
                if (ids[row] >= 0) {
                    const Pair8 v = low_rank8(p, MATS, m, t0 + row, base + c * 8);
                    char* to = lds + (m * S::BM + row) * kRow + c * 16;
                    *reinterpret_cast<u32x4_t*>(to) = v.hi;
                    *reinterpret_cast<u32x4_t*>(to + kPiece * 2) = v.lo;
                }
            }
            __syncthreads();
            // The adapters of the wavefront's tokens; the next one's piece of B is under way while one is multiplied.
            unsigned left[MB], here[MB];
#pragma unroll
            for (int m = 0; m < MB; ++m) left[m] = (unsigned)__ballot(id[m] >= 0);
            int a = -1;
            bf16x8 fb[kPiece / 16][S::NB];
            auto next = [&] {
                a = -1;
#pragma unroll
                for (int m = MB - 1; m >= 0; --m)
                    if (left[m]) a = __builtin_amdgcn_readlane(id[m], __builtin_ctz(left[m]));
                if (a < 0) return;
#pragma unroll
                for (int m = 0; m < MB; ++m) {
                    here[m] = (unsigned)__ballot(id[m] == a);
                    left[m] &= ~here[m];
                }
#pragma unroll
                for (int q = 0; q < kPiece / 16; ++q)
#pragma unroll
                    for (int n = 0; n < S::NB; ++n)
                        fb[q][n] = base + q * 16 + half * 8 < p.rank ? *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(p.b[m2] + (size_t)a * p.N * p.rank + base + q * 16) + brow[n]) : zeros8();
            };
            next();
            while (a >= 0) {
                const int a0 = a;
                unsigned h0[MB];
                bf16x8 f0[kPiece / 16][S::NB];
#pragma unroll
                for (int m = 0; m < MB; ++m) h0[m] = here[m];
#pragma unroll
                for (int q = 0; q < kPiece / 16; ++q)
#pragma unroll
                    for (int n = 0; n < S::NB; ++n) f0[q][n] = fb[q][n];
                next();
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < kPiece / 16; ++q) {
                    if (base + q * 16 >= p.rank) break;
                    const bool in = base + q * 16 + half * 8 < p.rank;
#pragma unroll
                    for (int m = 0; m < MB; ++m) {
                        if (!h0[m]) continue;
                        const bool mine = id[m] == a0;
                        const char* from = lds + (m2 * S::BM + (wm * MB + m) * 32 + r) * kRow + (q * 16 + half * 8) * 2;
                        const bf16x8 hi = in && mine ? *reinterpret_cast<const bf16x8*>(from) : zeros8();
                        const bf16x8 lo = in && mine ? *reinterpret_cast<const bf16x8*>(from + kPiece * 2) : zeros8();
#pragma unroll
                        for (int n = 0; n < S::NB; ++n) {
                            const f32x16 some = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f0[q][n], lo, acc[n][m], 0, 0, 0);
                            keep_mine<f32x16>(acc[n][m], __builtin_amdgcn_mfma_f32_32x32x16_bf16(f0[q][n], hi, some, 0, 0, 0), mine);
                        }
                    }
                }
            }
            __syncthreads();
        }
        by_rows<S, FB / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            if (r >= rows || c * 8 >= cols) return;
            float v[8];
            load8(row + c * 8, v);
            const size_t at = (size_t)(t0 + r) * p.N + n0 + c * 8;
            if constexpr (MATS == 2) {
                float u[8];
                load8(row + FB + c * 8, u);
    #pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = silu(v[i]) * u[i];
            } else if (p.base) {
                float o[8];
                unpack8(*reinterpret_cast<const u32x4_t*>(p.base + at), o);
    #pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += o[i];
            }
            *reinterpret_cast<u32x4_t*>(p.y + at) = pack8(v);
        });
    });
}

// The j-th adapter, counted from 0, that occurs among up to 128 tokens from t0; -1: fewer occur.
__device__ __forceinline__ int occurring(const AdapterArgs& p, int t0, int rows, int j, int lane) {
    const int a0 = lane < rows ? adapter_of(p, t0 + lane) : -1, a1 = lane + kWave < rows ? adapter_of(p, t0 + lane + kWave) : -1;
    unsigned long long left0 = __ballot(a0 >= 0), left1 = __ballot(a1 >= 0);
    for (;;) {
        if ((left0 | left1) == 0) return -1;
        const int a = left0 ? __builtin_amdgcn_readlane(a0, __builtin_ctzll(left0)) : __builtin_amdgcn_readlane(a1, __builtin_ctzll(left1));
        if (j-- == 0) return a;
        left0 &= ~__ballot(a0 == a);
        left1 &= ~__ballot(a1 == a);
    }
}

// Decode batches, and projections with too few tiles for the CUs: the fp32 sums of x W^T over one of `splits` pieces of K, and in the same launch
// v, one tile per adapter that occurs (its A takes W's place, the rows that have it are kept).  Bound by streaming W and A, of which a CU's
// three workgroups have 96 KiB under way: 14336 -> 4096 for one token 22 us (5.4 TB/s), 4096 -> 2 x 14336 for 48 tokens with 48 adapters of rank 64
// 67-75 us (4 TB/s; tiles of 128 features, one workgroup per CU 87, two 83).
template <class S, int MATS>
__global__ __launch_bounds__(S::THREADS, S::SIMD_WAVES) void adapter_part_kernel(AdapterArgs p) {
    constexpr int FB = S::BN / MATS;
    static_assert(S::BM <= 2 * kWave, "occurring");
    __shared__ __attribute__((aligned(1024))) char lds[S::kLds];
    const int tn_n = p.w[0] ? (p.N + FB - 1) / FB : 0, tn_r = (p.rank + FB - 1) / FB, low = p.lists * tn_r, per = low + tn_n;
    const int piece = blockIdx.x % p.splits, t = blockIdx.x / p.splits, tm = t / per;
    int tn = t - tm * per;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
    const int t0 = tm * S::BM, rows = p.T - t0 < S::BM ? p.T - t0 : S::BM;
    const bool second = MATS == 2 && wave >= S::WAVES / 2;
    const uint16_t* w = second ? p.w[1] : p.w[0];
    int a = -1, N = p.N;
    float* out = p.sums;
    float scale = 1.0f;
    if (tn < low) {                    // an adapter's tile
        a = occurring(p, t0, rows, tn / tn_r, lane);
        if (a < 0) return;
        tn %= tn_r;
        N = p.rank;
        w = (second ? p.a[1] : p.a[0]) + (size_t)a * p.rank * p.K;
        out = p.v;
        if (p.scale) scale = p.scale[a];
    } else {
        tn -= low;
    }
    const int n0 = tn * FB, cols = N - n0 < FB ? N - n0 : FB;
    const int all = p.K / S::BK, each = (all + p.splits - 1) / p.splits, s0 = piece * each < all ? piece * each : all, steps = all - s0 < each ? all - s0 : each;
    by_height<S>(rows, [&](auto height) {
        constexpr int MB = decltype(height)::value;
        Acc<S, MB> acc;
        clear<S, MB>(acc);
        typename S::template LoadA<true> la;
        typename S::template LoadB<true> lb;
        la.init(p.K, wave, lane);
        lb.init(p.K, wave, lane, second ? FB : 0);
        const int k0 = s0 * S::BK;      // the panels start at k0; their rows still end where the tile's do
        multiply<S, MB, true, true>(acc, Stream<true, S::BK>::make(p.x + (size_t)t0 * p.K + k0, p.K, rows, steps * S::BK, k0),
                                    Stream<true, S::BK>::make(w + (size_t)n0 * p.K + k0, p.K, cols, steps * S::BK, k0), la, lb, steps, lds);
        by_rows<S, S::BN / 8>(acc, lds, AheadNothing{}, [&](int r, int c, const float* row, Nothing) {
            const int m = MATS == 2 && c * 8 >= FB ? 1 : 0, col = c * 8 - m * FB;
            if (r >= rows || col >= cols) return;
            if (a >= 0 && adapter_of(p, t0 + r) != a) return;
            float* to = out + (((size_t)piece * MATS + m) * p.T + t0 + r) * N + n0 + col;
            float v[8];
            load8(row + c * 8, v);
            *reinterpret_cast<f32x4*>(to) = f32x4{v[0] * scale, v[1] * scale, v[2] * scale, v[3] * scale};
            *reinterpret_cast<f32x4*>(to + 4) = f32x4{v[4] * scale, v[5] * scale, v[6] * scale, v[7] * scale};
        });
    });
}

// Adds adapter_part_kernel's sums and the adapters' part.  A workgroup takes up to 64 tokens (MB blocks of 16) and NB blocks of 16 features (of each
// matrix); its eight wavefronts share the adapters that occur and are joined through LDS.  Bound by reading B: 48 adapters of rank 64, 2 x 14336
// features 43 us (4.1 TB/s); one token, 4096 features 6.5 us, a launch.
template <int MB, int NB, int MATS>
__global__ __launch_bounds__(kThreads, 4) void adapter_join_kernel(AdapterArgs p) {
    constexpr int kRow = kMaxRank * 4 + 16, kV = MATS * MB * 16 * kRow, kPart = kWaves / 2 * MATS * NB * MB * 64 * 16;
    __shared__ __attribute__((aligned(1024))) char lds[kPart > kV ? kPart : kV];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave, r = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x * (NB * 16), t0 = blockIdx.y * (MB * 16);
    f32x4 acc[MATS][NB][MB];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int b = 0; b < MB; ++b) acc[m][n][b] = f32x4{0, 0, 0, 0};
    // v of all tokens as bf16
    const int chunks = p.rank / 8;
    for (int j = tid; j < MATS * MB * 16 * chunks; j += kThreads) {
        const int c = j % chunks, t = j / chunks % (MB * 16), m = j / chunks / (MB * 16);
        if (adapter_of(p, t0 + t) >= 0) {
            const Pair8 v = low_rank8(p, MATS, m, t0 + t, c * 8);
            char* to = lds + (m * MB * 16 + t) * kRow + c * 16;
            *reinterpret_cast<u32x4_t*>(to) = v.hi;
            *reinterpret_cast<u32x4_t*>(to + kMaxRank * 2) = v.lo;
        }
    }
    __syncthreads();
    const int id = lane < MB * 16 ? adapter_of(p, t0 + lane) : -1;
    int idb[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) idb[b] = __shfl(id, b * 16 + r, kWave);
    // This wavefront's adapters: every eighth of those that occur, 32 of the rank at a time; the next piece of B is under way meanwhile.
    unsigned long long left = __ballot(id >= 0), here = 0;
    int a = -1, c = 0, seen = 0;
    auto next = [&] {
        c += 32;
        if (a >= 0 && c < p.rank) return;
        a = -1;
        c = 0;
        while (left != 0 && a < 0) {
            const int first = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
            here = __ballot(id == first);
            left &= ~here;
            if (seen++ % kWaves == wave) a = first;
        }
    };
    bf16x8 fb[MATS][NB];
    auto load = [&] {
        const bool in = c + quad * 8 < p.rank;
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const char* base = reinterpret_cast<const char*>(p.b[m] + ((size_t)a * p.N + n0 + n * 16) * p.rank + c);
                fb[m][n] = in ? *reinterpret_cast<const bf16x8*>(base + (uint32_t)(r * p.rank + quad * 8) * 2u) : zeros8();
            }
    };
    next();
    if (a >= 0) load();
    while (a >= 0) {
        const int a0 = a, c0 = c;
        const unsigned long long h0 = here;
        bf16x8 f0[MATS][NB];
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n) f0[m][n] = fb[m][n];
        next();
        if (a >= 0) load();
        __builtin_amdgcn_sched_barrier(0);
        const bool in = c0 + quad * 8 < p.rank;
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            if (!((h0 >> (b * 16)) & 0xffff)) continue;
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
                const bool mine = idb[b] == a0;
                const char* from = lds + (m * MB * 16 + b * 16 + r) * kRow + (c0 + quad * 8) * 2;
                const bf16x8 hi = in && mine ? *reinterpret_cast<const bf16x8*>(from) : zeros8();
                const bf16x8 lo = in && mine ? *reinterpret_cast<const bf16x8*>(from + kMaxRank * 2) : zeros8();
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    const f32x4 some = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0[m][n], lo, acc[m][n][b], 0, 0, 0);
                    keep_mine<f32x4>(acc[m][n][b], __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0[m][n], hi, some, 0, 0, 0), mine);
                }
            }
        }
    }
    __syncthreads();
    // join: the upper four wavefronts hand theirs to the lower four, whose sums are added by whoever stores (half the LDS, hence two workgroups per CU)
    constexpr int kJoin = kWaves / 2;
    f32x4* const part = reinterpret_cast<f32x4*>(lds);       // [wave][matrix][n][b][lane]
    f32x4* const mine = part + (size_t)(wave % kJoin) * MATS * NB * MB * 64 + lane;
    if (wave >= kJoin) {
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int b = 0; b < MB; ++b) mine[((m * NB + n) * MB + b) * 64] = acc[m][n][b];
    }
    __syncthreads();
    if (wave < kJoin) {
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int b = 0; b < MB; ++b) {
                    const f32x4 o = mine[((m * NB + n) * MB + b) * 64];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][n][b][i] += o[i];
                    mine[((m * NB + n) * MB + b) * 64] = acc[m][n][b];
                }
    }
    __syncthreads();
    for (int j = tid; j < NB * MB * 64; j += kThreads) {
        const int l = j % 64, b = j / 64 % MB, n = j / 64 / MB, t = t0 + b * 16 + (l & 15), col = n0 + n * 16 + (l >> 4) * 4;
        if (t >= p.T) continue;
        f32x4 v[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            v[m] = part[((m * NB + n) * MB + b) * 64 + l];
#pragma unroll
            for (int w = 1; w < kJoin; ++w) {
                const f32x4 o = part[(((w * MATS + m) * NB + n) * MB + b) * 64 + l];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[m][i] += o[i];
            }
        }
        const size_t at = (size_t)t * p.N + col;
        for (int q = 0; q < (p.w[0] ? p.splits : 0); ++q)
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
                const f32x4 o = *reinterpret_cast<const f32x4*>(p.sums + ((size_t)q * MATS + m) * p.T * p.N + at);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[m][i] += o[i];
            }
        if constexpr (MATS == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] = silu(v[0][i]) * v[1][i];
        } else if (p.base) {
            const uint2 o = *reinterpret_cast<const uint2*>(p.base + at);
            v[0][0] += __uint_as_float(o.x << 16), v[0][1] += __uint_as_float(o.x & 0xffff0000u);
            v[0][2] += __uint_as_float(o.y << 16), v[0][3] += __uint_as_float(o.y & 0xffff0000u);
        }
        *reinterpret_cast<uint2*>(p.y + at) = make_uint2(pack2_bf16(v[0][0], v[0][1]), pack2_bf16(v[0][2], v[0][3]));
    }
}

// Pieces of K and workgroups per block of 32 tokens of low_rank_kernel, for about 512 workgroups.  In a prompt a block has one or two adapters: K is
// cut first, into up to eight pieces (which the projection's kernel adds up), no finer than 64 elements per wavefront.
struct Split {
    int blocks, lists, parts;
};
Split split(const moe_adapter_config& c) {
    Split s;
    s.blocks = (c.T + 31) / 32;
    const int most = c.adapters < 32 ? c.adapters : 32;
    s.parts = 1;
    while (s.parts < 8 && s.blocks * s.parts < 512 && c.K >= s.parts * 2 * kWaves * 64) s.parts *= 2;
    s.lists = s.blocks * s.parts * 2 <= 512 ? 512 / (s.blocks * s.parts) : 1;
    if (s.lists > most) s.lists = most;
    return s;
}

template <int MATS>
void low_rank(const AdapterArgs& p, unsigned grid, hipStream_t s) {
    const int rb = (p.rank + 31) / 32;
    if (rb == 1) hipLaunchKernelGGL((low_rank_kernel<1, MATS>), dim3(grid), dim3(kThreads), 0, s, p);
    else if (rb == 2) hipLaunchKernelGGL((low_rank_kernel<2, MATS>), dim3(grid), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((low_rank_kernel<4, MATS>), dim3(grid), dim3(kThreads), 0, s, p);
}

template <int MB, int MATS>
void join(const AdapterArgs& p, hipStream_t s) {
    hipLaunchKernelGGL((adapter_join_kernel<MB, 2, MATS>), dim3(p.N / 32, (p.T + MB * 16 - 1) / (MB * 16)), dim3(kThreads), 0, s, p);
}

// adapter_part_kernel's workgroups per piece of K: the projection's tiles and, per block of tokens, at most so many of adapters.
struct PartGrid {
    long long blocks, main, low;
    int lists, slots;            // adapters per block of tokens at most; workgroups that run at once
};
template <class S>
PartGrid part_grid(const moe_adapter_config& c, int mats) {
    const int FB = S::BN / mats, block = c.T < S::BM ? c.T : S::BM;
    PartGrid g;
    g.blocks = (c.T + S::BM - 1) / S::BM;
    g.main = g.blocks * ((c.N + FB - 1) / FB);
    g.lists = c.adapters < block ? c.adapters : block;
    g.low = g.blocks * g.lists * ((c.rank + FB - 1) / FB);
    g.slots = 256 * S::PER;
    return g;
}
PartGrid part_grid(const moe_adapter_config& c, int mats) { return c.T <= Flat::BM ? part_grid<Flat>(c, mats) : part_grid<Half>(c, mats); }
// Pieces of K for adapter_part_kernel; 0: one launch does the projection and the adapters (adapter_rows_kernel).  The former for up to 128 tokens, whose
// adapters its launch and the join take side by side, and where there are tiles for fewer than half of the CUs.  us, adapter_rows_kernel / adapter_part_kernel and join:
//   4096 -> 2 x 14336, 48 tokens, adapters of rank 64 of their own 122 / 110;  2048 -> 2048, 512 tokens, 64 adapters of rank 128 190 / 61;
//   4096 -> 2 x 14336, 512 tokens: one adapter of rank 16 111 / 200, eight prompts' of rank 128 218 / 256, 64 scattered adapters of rank 64 423 / 432, of rank 128 742 / 719;
//   14336 -> 4096, 512 tokens: one adapter of rank 16 96 / 104, eight prompts' of rank 64 125 / 156, 64 scattered adapters of rank 16 201 / 187, of rank 128 671 / 294.
// Neither the number of adapters nor the rank is in the rule: a narrow projection of more than 128 tokens that has 128 tiles or more takes up to 2.5 times as long as it
// would need where many adapters are scattered over the tokens.
int splits(const moe_adapter_config& c, int mats) {
    const PartGrid g = part_grid(c, mats);
    if (c.T > Half::BM && g.main >= 128) return 0;
    long long n = g.slots / (g.main + g.low), most = c.K / 64 / 4;       // no fewer than four steps each
    if (n > 8) n = 8;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}
template <class S, int MATS>
void part(const AdapterArgs& p, hipStream_t s) {
    constexpr int FB = S::BN / MATS;
    const long long per = (long long)p.lists * ((p.rank + FB - 1) / FB) + (p.w[0] ? (p.N + FB - 1) / FB : 0);
    hipLaunchKernelGGL((adapter_part_kernel<S, MATS>), dim3((unsigned)((p.T + S::BM - 1) / S::BM * per * p.splits)), dim3(S::THREADS), 0, s, p);
}

template <class S, int MATS>
void many(const AdapterArgs& p, hipStream_t s) {
    const long long tiles = (long long)((p.T + S::BM - 1) / S::BM) * ((p.N + S::BN / MATS - 1) / (S::BN / MATS));
    hipLaunchKernelGGL((adapter_rows_kernel<S, MATS>), dim3(xcd_grid(tiles)), dim3(S::THREADS), 0, s, p);
}

// Tiles of adapter_rows_kernel: 0 Wide, 1 Tall, 2 Small.
// us, without / with Tall: gated 4096 -> 2 x 14336, 200 tokens 84 / 69; 14336 -> 4096, 2048 tokens 265 / 229; 7168 -> 2048, 3000 129 / 108; others even
int rows_tiles(const moe_adapter_config& c, int mats) {
    const long long N = (long long)c.N * mats, wide = cost<Wide>(1, c.T, N), tall = cost<Tall>(1, c.T, N), small = cost<Small>(1, c.T, N);
    return wide <= tall && wide <= small ? 0 : tall <= small ? 1 : 2;
}

template <int MATS>
hipError_t launch(AdapterArgs p, const moe_adapter_config& c, hipStream_t s) {
    p.splits = splits(c, MATS);
    if (p.splits > 0) {
        p.parts = p.splits;
        p.lists = part_grid(c, MATS).lists;
        if (p.T <= Flat::BM) part<Flat, MATS>(p, s);
        else part<Half, MATS>(p, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        switch (p.T > 48 ? 4 : (p.T + 15) / 16) {
            case 1: join<1, MATS>(p, s); break;
            case 2: join<2, MATS>(p, s); break;
            case 3: join<3, MATS>(p, s); break;
            default: join<4, MATS>(p, s);
        }
        return hipGetLastError();
    }
    const Split sp = split(c);
    p.parts = sp.parts;
    p.lists = sp.lists;
    low_rank<MATS>(p, (unsigned)(sp.blocks * sp.lists * sp.parts), s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    switch (rows_tiles(c, MATS)) {
        case 0: many<Wide, MATS>(p, s); break;
        case 1: many<Tall, MATS>(p, s); break;
        default: many<Small, MATS>(p, s);
    }
    return hipGetLastError();
}

// v: as many pieces as the path of either entry point has
size_t low_rank_bytes(const moe_adapter_config& c) {
    int pieces = 1;
    for (int mats = 1; mats <= 2; ++mats) {
        const int n = splits(c, mats) > 0 ? splits(c, mats) : split(c).parts;
        if (n > pieces) pieces = n;
    }
    return ((size_t)pieces * 2 * c.T * c.rank * sizeof(float) + 255) / 256 * 256;
}

}  // namespace

size_t adapter_workspace_bytes(const moe_adapter_config& c) {
    if (c.T == 0) return 0;
    const int one = splits(c, 1), two = splits(c, 2);
    return low_rank_bytes(c) + (size_t)(one > 2 * two ? one : 2 * two) * c.T * c.N * sizeof(float);
}

hipError_t launch_adapter(const moe_adapter_config& c, int mats, const uint16_t* x, const uint16_t* const w[2], const uint16_t* const a[2],
                          const uint16_t* const b[2], const float* scale, const int32_t* adapter_of, const uint16_t* base, uint16_t* y, float* v,
                          hipStream_t s) {
    const AdapterArgs p{x, {w[0], w[1]}, {a[0], a[1]}, {b[0], b[1]}, scale, adapter_of, base, v, (float*)((char*)v + low_rank_bytes(c)), 0, y, c.T, c.N, c.K, c.adapters, c.rank, 0, 0};
    return mats == 2 ? launch<2>(p, c, s) : launch<1>(p, c, s);
}

}  // namespace moe

// Test hook (host arithmetic only, not part of include/moe.h): the tiles of a call with `mats` matrices.
// 0: Wide, 1: Tall, 2: Small (adapter_rows_kernel); 3: Flat, 4: Half (adapter_part_kernel).
extern "C" __attribute__((visibility("default"))) int32_t moe_test_adapter_tiles(const moe_adapter_config* c, int32_t mats) {
    using namespace moe;
    return splits(*c, mats) > 0 ? (c->T <= Flat::BM ? 3 : 4) : rows_tiles(*c, mats);
}
