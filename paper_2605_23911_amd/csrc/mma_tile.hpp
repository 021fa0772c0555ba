// One tile of C[m, n] = sum_k A(m, k) B(n, k) on bf16 MFMA (gfx950), for the operators whose operands are not both stored with
// the reduction dimension contiguous: gradients with respect to rows (the weights' rows run along k), gradients with respect to
// weights (both operands' rows run along k), and the projections with row-major weights beside them.
//
// Both operands go global -> LDS by DMA from buffer descriptors, BK of k per step into a ring of buffers; a descriptor's range is the
// tile's own rows, so what lies beyond a ragged end (rows of the next expert, whatever they hold) arrives as zeros and needs no mask.
//   operand stored with k contiguous:   LDS rows of BK k (128 or 64 bytes), one ds_read_b128 per MFMA fragment.  Position p of row r
//       holds 16-byte chunk p ^ ((r >> 1) & 7) (BK 32: p ^ ((r >> 2) & 3)): sixteen lanes that read one chunk column of sixteen
//       rows hit all 64 banks once.
//   operand stored with m (n) contiguous: LDS rows of the tile's width, one per k; a fragment is two ds_read_b64_tr_b16, each of
//       which transposes 4 k x 16 m among sixteen lanes.  32-byte piece q of row k lies at q ^ 2 (k & 3) (two bits of it where the
//       row has only four pieces): the eight pieces that half a wavefront reads lie in different banks.
// The DMA fixes the order in LDS, so both permutations are applied to the source address and again by the reads.
// The first MFMA operand is B: a lane then holds four consecutive n of one row m (32x32 blocks, fp32 accumulators).
#pragma once

#include <type_traits>
#include <utility>

#include "lds_dma.hpp"
#include "moe_internal.hpp"

namespace moe {

namespace {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// The thread's number at the start of a body.  Opaque to the compiler, which would work out what all bodies of a kernel derive from it once, in
// front of them, and hold it in registers that the tallest body does not have.
__device__ __forceinline__ int body_thread() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
}

template <int... Is, class F>
__device__ __forceinline__ void static_for_impl(std::integer_sequence<int, Is...>, F&& f) {
    (f(std::integral_constant<int, Is>{}), ...);
}
// f(integral_constant<0>) ... f(integral_constant<N - 1>)
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(std::make_integer_sequence<int, N>{}, f);
}

// A buffer descriptor's parts; everything in it is the same for all lanes.
struct Panel {
    uint64_t base;
    uint32_t range;
    __device__ __forceinline__ i32x4 desc() const {
        return i32x4{__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32) & 0xffff),
                     __builtin_amdgcn_readfirstlane((int)range), 0x00020000};
    }
};

// An operand on its way through the reduction, a step of BK elements at a time: the next step's panel.
//   k contiguous: `rows` rows of `ld` elements; a step advances BK elements along them.
//   m contiguous: a step is BK rows (k) of `ld` elements; the last one may hold fewer.
// Past the last step panels are empty (range 0): loads from them leave zeros and fetch nothing.
template <bool KC, int BK>
struct Stream {
    uint64_t base;
    uint32_t range;       // KC: bytes from base to the end of the tile's last row
    uint32_t row_bytes;
    uint32_t skip;        // !KC: bytes of the row in front of the tile
    int left;             // elements of k still to come
    // k0: KC, p is that many elements into the rows
    __device__ static __forceinline__ Stream make(const uint16_t* p, int ld, int rows_or_m0, int k, int k0 = 0) {
        Stream s;
        s.row_bytes = (uint32_t)ld * 2u;
        s.left = k;
        if constexpr (KC) {
            s.base = (uint64_t)(uintptr_t)p;
            s.range = (uint32_t)rows_or_m0 * s.row_bytes - (uint32_t)k0 * 2u;
            s.skip = 0;
        } else {
            s.skip = (uint32_t)rows_or_m0 * 2u;
            s.base = (uint64_t)(uintptr_t)p + s.skip;
            s.range = 0;
        }
        return s;
    }
    __device__ __forceinline__ Panel next() {
        Panel p;
        p.base = base;
        if constexpr (KC) {
            p.range = left > 0 ? range : 0;
            base += BK * 2;
            range -= BK * 2;
        } else {
            const int n = left < BK ? left : BK;
            p.range = left > 0 ? (uint32_t)n * row_bytes - skip : 0;
            base += (uint64_t)BK * row_bytes;
        }
        left -= BK;
        return p;
    }
};

// Permutation of a row's chunks (k contiguous) or pieces, by the row's number in the panel.
template <int MN, bool KC, int BK>
__device__ __forceinline__ int swizzle(int r) {
    if constexpr (KC) return BK == 64 ? (r >> 1) & 7 : (r >> 2) & 3;
    else return MN >= 128 ? 2 * (r & 3) : (r & 2);
}

// What a wavefront loads of an operand's panel: N KiB of its MN x BK elements, and the lanes' byte offsets from the panel's start.
template <int MN, bool KC, int BK, int WAVES>
struct Loader {
    static constexpr int N = MN * BK / (512 * WAVES);
    uint32_t off[N];
    // first: KC only, the tile's row that the panel starts with (operands of two matrices: half of the rows each)
    __device__ __forceinline__ void init(int ld, int wave, int lane, int first = 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int u = wave * N + j;
            if constexpr (KC) {
                constexpr int C = BK / 8;          // 16-byte chunks of a row
                const int row = u * (64 / C) + lane / C, chunk = (lane % C) ^ swizzle<MN, KC, BK>(row);
                off[j] = (uint32_t)(row - first) * (uint32_t)ld * 2u + chunk * 16;
            } else {
                constexpr int W = MN * 2;          // bytes of an LDS row
                const int byte = u * 1024 + lane * 16, k = byte / W, piece = (byte % W) >> 5;
                off[j] = (uint32_t)k * (uint32_t)ld * 2u + (piece ^ swizzle<MN, KC, BK>(k)) * 32 + (byte & 16);
            }
        }
    }
    // the wavefront's J-th KiB
    template <int J>
    __device__ __forceinline__ void one(i32x4 desc, uint32_t lds, int wave) const { buffer_dma(off[J], desc, lds + wave * (N * 1024) + J * 1024); }
};

// What a lane reads: fragments of 32 rows (m or n) x 16 k, slot s of the step: element i of lane l is k = 16 s + 8 (l / 32) + i.
template <int MN, bool KC, int BK, int BLOCKS>
struct Reader {
    uint32_t at[KC ? BK / 16 : BLOCKS];
    __device__ __forceinline__ void init(int row0, int lane) {
        const int half = lane >> 5;
        if constexpr (KC) {
            const int r = lane & 31;
#pragma unroll
            for (int s = 0; s < BK / 16; ++s) at[s] = (uint32_t)((row0 + r) * BK * 2 + ((2 * s + half) ^ swizzle<MN, KC, BK>(r)) * 16);
        } else {
            constexpr int W = MN * 2;
            const int k = 8 * half + ((lane & 15) >> 2);
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const int piece = (row0 + b * 32) / 16 + ((lane >> 4) & 1);
                at[b] = (uint32_t)(k * W + (piece ^ swizzle<MN, KC, BK>(k)) * 32 + (lane & 3) * 8);
            }
        }
    }
    __device__ __forceinline__ bf16x8 read(const char* lds, int b, int s) const {
        if constexpr (KC) {
            return *reinterpret_cast<const bf16x8*>(lds + at[s] + b * (64 * BK));
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
            constexpr int W = MN * 2;
            const char* p = lds + at[b] + s * 16 * W;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * W));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// BM x BN tile by WM x WN wavefronts, BK elements of k per step, a ring of STAGES steps.
template <int BM_, int BN_, int WM_, int WN_, int BK_, int STAGES_, int PER_, int RATE_>
struct Shape {
    static constexpr int PER = PER_, RATE = RATE_;
    static constexpr int SIMD_WAVES = PER_ * WM_ * WN_ / 4;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = WAVES * kWave;
    static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;   // 32x32 blocks per wavefront
    static constexpr int kBufA = BM * BK * 2, kBuf = (BM + BN) * BK * 2, kRing = STAGES * kBuf;
    static constexpr int LD = BN + 4;                            // floats per staged row: 16 bytes more, which spreads the rows over the banks
    static constexpr int kPassRows = WM * 32;                    // rows staged at a time: one block of every wavefront row
    static constexpr int kStage = kPassRows * LD * 4;
    static constexpr int kTile = BM * (BN * 2 + 16);             // the whole tile as bf16
    static constexpr int kMost = kRing > kStage ? kRing : kStage, kLds = kMost > kTile ? kMost : kTile;
    template <bool KC> using LoadA = Loader<BM, KC, BK, WAVES>;
    template <bool KC> using LoadB = Loader<BN, KC, BK, WAVES>;
    static_assert(MB >= 1 && MB <= 4 && NB >= 1, "blocks");
};

// Both operands with k contiguous: rows of 128 bytes, whole lines.  Else four short steps, three of them under way (8192 rows, 28672 -> 4096, four
// steps of 32 / two of 64: 1840 / 2100 us; with k contiguous in both 2050 / 2010).
typedef Shape<256, 256, 2, 4, 64, 2, 1, 100> Wide;
typedef Shape<256, 256, 2, 4, 32, 4, 1, 100> Deep;
// Two workgroups per CU, one of which stores while the other multiplies: weight gradients, where a tile's reduction is as short as an expert
// has rows (250 rows of 64 experts, 2560 x 3584: 1470 us, Deep 1500, Wide 1560).
typedef Shape<128, 256, 1, 4, 32, 3, 2, 95> Pair;
// Few tiles: a quarter of the work each and three steps under way.
typedef Shape<128, 128, 2, 4, 64, 4, 1, 60> Small;
// Weights past up to 256 rows per expert in one block: half as wide as Deep, so twice as many tiles (tiles_for in ffn_train.hip).
typedef Shape<256, 128, 4, 2, 64, 3, 1, 75> Tall;
// Streaming weights past few rows: three (two) workgroups per CU, 96 (64) KiB under way.
typedef Shape<64, 64, 2, 2, 64, 3, 3, 60> Flat;
typedef Shape<128, 128, 2, 4, 64, 2, 2, 60> Half;

// A wavefront's results: MB blocks of 32 rows (up to the shape's: a tile of few rows takes a body with fewer), NB of 32 columns.
template <class S, int MB>
using Acc = f32x16[S::NB][MB];

template <class S, int MB>
__device__ __forceinline__ void clear(f32x16 (&acc)[S::NB][MB]) {
#pragma unroll
    for (int n = 0; n < S::NB; ++n)
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] = 0.0f;
}

// Calls body(integral_constant<MB>) with the fewest blocks per wavefront that hold `rows` rows: a ragged expert's last tile does not multiply
// rows that it does not have.
template <class S, class F>
__device__ __forceinline__ void by_height(int rows, F&& body) {
    using std::integral_constant;
    const int need = (rows + S::WM * 32 - 1) / (S::WM * 32);
    if constexpr (S::MB >= 4) if (need >= 4) return body(integral_constant<int, 4>{});
    if constexpr (S::MB >= 3) if (need == 3) return body(integral_constant<int, 3>{});
    if constexpr (S::MB >= 2) if (need == 2 || (S::MB == 2 && need > 2)) return body(integral_constant<int, 2>{});
    body(integral_constant<int, 1>{});
}

// acc += the tile's product over `steps` steps.  a, b: the operands' streams, loaders with the offsets set.
// Everything is put in its place by hand: a slot (16 of k) is MB x NB multiplications, and between them go the reads of the next slot's fragments,
// one or two after each, and the next step's loads, one after each from the last slot on.  In a burst the loads of all wavefronts
// queue up for longer than a slot takes, and the multiplications behind them wait.  A step's barrier stands in front of its last slot, whose
// multiplications cover the first reads of the next step.
// Ends with every wavefront past its last LDS read and nothing on its way into LDS.
template <class S, int MB, bool AKC, bool BKC>
__device__ __forceinline__ void multiply(f32x16 (&acc)[S::NB][MB], Stream<AKC, S::BK> a, Stream<BKC, S::BK> b, const typename S::template LoadA<AKC>& la,
                                         const typename S::template LoadB<BKC>& lb, int steps, char* lds) {
    constexpr int SLOTS = S::BK / 16, NA = S::template LoadA<AKC>::N, LOADS = NA + S::template LoadB<BKC>::N;     // loads per step and wavefront
    constexpr int READS = MB + S::NB, MFMAS = MB * S::NB, PER = (READS + MFMAS - 1) / MFMAS;
    // loads that go with the last slot (of the step after next), the rest with the first slots of the next step
    constexpr int SPREAD = S::STAGES > 2 ? SLOTS : SLOTS - 1;    // slots that loads are spread over
    constexpr int EACH = (LOADS + SPREAD - 1) / SPREAD;
    const int tid = body_thread(), wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
    Reader<S::BM, AKC, S::BK, MB> ra;
    Reader<S::BN, BKC, S::BK, S::NB> rb;
    ra.init(wm * MB * 32, lane);
    rb.init(wn * S::NB * 32, lane);
    const uint32_t at = (uint32_t)(uintptr_t)lds;
    bf16x8 fa[2][MB], fb[2][S::NB];
    i32x4 da, db;                                                // the step that is being loaded: descriptors, and where it goes
    uint32_t to = 0;
    auto begin = [&](uint32_t where) {
        da = a.next().desc();
        db = b.next().desc();
        to = at + where;
    };
    auto load = [&](auto piece) {
        constexpr int p = decltype(piece)::value;
        if constexpr (p < NA) la.template one<p>(da, to, wave);
        else if constexpr (p < LOADS) lb.template one<p - NA>(db, to + S::kBufA, wave);
    };
    auto read = [&](uint32_t from, int s, int set, int which) {
        if (which < S::NB) fb[set][which] = rb.read(lds + from + S::kBufA, which, s);
        else if (which < READS) fa[set][which - S::NB] = ra.read(lds + from, which - S::NB, s);
    };
    if (steps <= 0) return;
    // Steps 0 .. STAGES - 2 whole, and of the next one what the last slot of a step loads.
    begin(0);
    static_for<LOADS>(load);
#pragma unroll
    for (int i = 1; i < S::STAGES - 1; ++i) {
        begin(i * S::kBuf);
        static_for<LOADS>(load);
    }
    wait_vmcnt<(S::STAGES - 2) * LOADS>();
    asm volatile("s_barrier" ::: "memory");
    begin((S::STAGES - 1) * S::kBuf);
    static_for<EACH>(load);
#pragma unroll
    for (int w = 0; w < READS; ++w) read(0, 0, 0, w);
    uint32_t buf = 0;                                            // byte offset of the step that is read
    for (int i = 0; i < steps; ++i) {
        const uint32_t next = buf + S::kBuf == S::kRing ? 0 : buf + S::kBuf;
        static_for<SLOTS>([&](auto slot) {
            constexpr int s = decltype(slot)::value;
            constexpr bool last = s + 1 == SLOTS;
            if constexpr (last) {   // the next step has landed, and no wavefront reads this one any more
                begin(buf);
                wait_vmcnt<(S::STAGES - 2) * LOADS>();
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            constexpr int first = last ? 0 : (s + 1) * EACH;     // of the step's loads, those of this slot
            static_for<MFMAS>([&](auto mfma) {
                constexpr int j = decltype(mfma)::value, m = j / S::NB, n = j % S::NB;
#pragma unroll
                for (int q = 0; q < PER; ++q) read(last ? next : buf, last ? 0 : s + 1, (s + 1) & 1, j * PER + q);
                acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][n], fa[s & 1][m], acc[n][m], 0, 0, 0);
                if constexpr (j < EACH) load(std::integral_constant<int, first + j>{});
                if constexpr (j + 1 == MFMAS) static_for<(EACH > MFMAS ? EACH - MFMAS : 0)>([&](auto more) { load(std::integral_constant<int, first + MFMAS + decltype(more)::value>{}); });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        buf = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __forceinline__ u32x4_t pack8(const float (&v)[8]) {
    return u32x4_t{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
__device__ __forceinline__ void unpack8(u32x4_t p, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(p[i] << 16), v[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
}

// Hands the tile's fp32 results out by rows: f(row in the tile, group, the row's BN floats in LDS, what `ahead` gave) for GROUPS groups of columns per
// row.  Staged through LDS, one 32-row block of every wavefront row at a time, so that what f stores are whole rows.  ahead(row, group) loads what f
// needs beside them and is called a block earlier.
template <class S, int GROUPS, int MB, class A, class F>
__device__ __forceinline__ void by_rows(const f32x16 (&acc)[S::NB][MB], char* lds, A&& ahead, F&& f) {
    constexpr int ITEMS = S::kPassRows * GROUPS / S::THREADS;
    static_assert(S::kPassRows * GROUPS % S::THREADS == 0, "whole items");
    const int tid = body_thread(), wave = tid / kWave, lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
    auto row_of = [&](int item, int p) {
        const int r = (tid + item * S::THREADS) / GROUPS;
        return (r / 32) * (MB * 32) + p * 32 + (r & 31);
    };
    decltype(ahead(0, 0)) held[2][ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) held[0][i] = ahead(row_of(i, 0), (tid + i * S::THREADS) % GROUPS);
#pragma unroll
    for (int p = 0; p < MB; ++p) {
        if (p + 1 < MB) {
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) held[(p + 1) & 1][i] = ahead(row_of(i, p + 1), (tid + i * S::THREADS) % GROUPS);
        }
        float* row = reinterpret_cast<float*>(lds) + (size_t)(wm * 32 + (lane & 31)) * S::LD + wn * S::NB * 32 + (lane >> 5) * 4;
#pragma unroll
        for (int n = 0; n < S::NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(row + n * 32 + q * 8) = f32x4{acc[n][p][q * 4], acc[n][p][q * 4 + 1], acc[n][p][q * 4 + 2], acc[n][p][q * 4 + 3]};
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int j = tid + i * S::THREADS;
            f(row_of(i, p), j % GROUPS, reinterpret_cast<const float*>(lds) + (size_t)(j / GROUPS) * S::LD, held[p & 1][i]);
        }
        if (p + 1 < MB) __syncthreads();
    }
}
struct Nothing {};
struct AheadNothing {
    __device__ __forceinline__ Nothing operator()(int, int) const { return {}; }
};

// The same for results that need nothing but their rounding to bf16: the whole tile is staged at once, f(row, group of 8 columns, the eight values).
template <class S, int MB, class F>
__device__ __forceinline__ void by_rows_bf16(const f32x16 (&acc)[S::NB][MB], char* lds, F&& f) {
    constexpr int LD = S::BN * 2 + 16, GROUPS = S::BN / 8;
    static_assert(S::BM * LD <= S::kLds, "the tile fits");
    const int tid = body_thread(), wave = tid / kWave, lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int p = 0; p < MB; ++p) {
        char* row = lds + (wm * MB * 32 + p * 32 + (lane & 31)) * LD + wn * S::NB * 64 + (lane >> 5) * 8;
#pragma unroll
        for (int n = 0; n < S::NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint2*>(row + n * 64 + q * 16) =
                    make_uint2(pack2_bf16(acc[n][p][q * 4], acc[n][p][q * 4 + 1]), pack2_bf16(acc[n][p][q * 4 + 2], acc[n][p][q * 4 + 3]));
    }
    __syncthreads();
#pragma unroll 4
    for (int j = tid; j < S::WM * MB * 32 * GROUPS; j += S::THREADS) {
        const int r = j / GROUPS, g = j % GROUPS;
        f(r, g, *reinterpret_cast<const u32x4_t*>(lds + r * LD + g * 16));
    }
}

// Which of a launch's tiles a workgroup takes.  The hardware deals workgroups to the eight XCDs in turn.
// One run of consecutive tiles per XCD, so that tiles which share operands share an L2: for tiles that take the same time.
__device__ __forceinline__ int xcd_tile(int id, int total) {
    const int per = (total + 7) / 8, t = (id & 7) * per + (id >> 3);
    return (id >> 3) < per && t < total ? t : -1;
}
// Runs of 32 (what an XCD works on at a time) dealt to the XCDs in turn: for tiles of unequal length.
__device__ __forceinline__ int xcd_run_tile(int id, int total) {
    const int t = ((id >> 8) * 8 + (id & 7)) * 32 + ((id >> 3) & 31);
    return t < total ? t : -1;
}
inline unsigned xcd_grid(long long total) { return (unsigned)((total + 7) / 8 * 8); }
inline unsigned xcd_run_grid(long long total) { return (unsigned)((total + 255) / 256 * 256); }

// What a launch of `groups` times M x N results takes: rounds of tiles times a tile's area, at the shape's RATE (percent of the large ones').  A tile
// of few rows takes a body of its height, but no less than half of the large ones' for what it loads of B.
// `even`: every group has M rows; else M is their mean, and beyond half a block each has half a block more.
template <class S>
inline long long cost(long long groups, long long M, long long N, bool even = true) {
    const long long blocks = even ? groups * ((M + S::BM - 1) / S::BM) : 2 * M <= S::BM ? groups : (groups * (2 * M + S::BM) + 2 * S::BM - 1) / (2 * S::BM);
    const long long tiles = blocks * ((N + S::BN - 1) / S::BN), rows = (M + 63) / 64 * 64;
    const long long height = rows < S::BM ? (rows > 128 ? rows : S::BM < 128 ? S::BM : 128) : S::BM;
    return (tiles + 256 * S::PER - 1) / (256 * S::PER) * S::PER * height * S::BN * 100 / S::RATE;
}

// Order inside a rectangle of tiles: columns of up to G row tiles, so that what an XCD runs at one time is a square-ish patch.
__device__ __forceinline__ void patch(int t, int rows, int cols, int& m, int& n) {
    constexpr int G = 8;
    const int g = t / (G * cols), first = g * G, size = rows - first < G ? rows - first : G, rem = t - g * G * cols;
    n = rem / size;
    m = first + rem - n * size;
}

// Rows of expert-contiguous storage cut into blocks of BM per expert (Alg. 1), each with `cols` column tiles: the workgroup's tile, found from
// the offsets by every wavefront for itself (up to 256 experts: four per lane).  No list in memory, hence no launch that writes one.
// Whole blocks come first, then what is left of the experts, the taller ones (more than half a block) before the others: a launch then ends
// with its short tiles, where it would otherwise start another round of whole ones.  Where whole blocks are the rule the rest is dealt to
// the XCDs tile by tile, else (many experts of less than a block) in runs like the whole ones.
// 8 experts, 8192 rows, 14336 -> 4096: 448 whole tiles of 256 x 256, 64 nearly whole, two rounds, and 64 of a few rows.
struct RowTile {
    int e, row0, rows, n;      // expert, first row, rows in the tile, column tile
};
__device__ __forceinline__ int wave_sums(int v, int lane) {
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int up = __shfl_up(v, o, kWave);
        if (lane >= o) v += up;
    }
    return v;
}
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int E, int BM, int cols, RowTile& out) {
    const int lane = threadIdx.x % kWave;
    int start[5], count[3][4], sum[3] = {0, 0, 0}, inc[3], total[3];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const int e = lane * 4 + i;
        start[i] = offsets[e < E ? e : E];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int n = start[i + 1] - start[i], rest = n % BM;
        sum[0] += count[0][i] = n / BM;
        sum[1] += count[1][i] = rest > BM / 2;
        sum[2] += count[2][i] = rest > 0 && rest <= BM / 2;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        inc[k] = wave_sums(sum[k], lane);
        total[k] = __builtin_amdgcn_readlane(inc[k], kWave - 1);
    }
    // which class, and the place in it
    const bool deal = total[0] > total[1] + total[2];
    int id = blockIdx.x, k = -1, t = -1;
#pragma unroll
    for (int c = 0; c < 3; ++c) {
        const int n = total[c] * cols, ids = (n + 7) / 8 * 8;
        if (k < 0 && id < ids) {
            k = c;
            t = c > 0 && deal ? (id < n ? id : -1) : xcd_tile(id, n);
        }
        if (k < 0) id -= ids;
    }
    if (t < 0) return false;
    const int block = t / cols;                    // some block of the same expert
    const int upto = k == 0 ? inc[0] : k == 1 ? inc[1] : inc[2];
    const int owner = __builtin_ctzll(__ballot(upto > block));
    int before = upto - (k == 0 ? sum[0] : k == 1 ? sum[1] : sum[2]), e = 0, s = 0, n_e = 0, blocks = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int nb = k == 0 ? count[0][i] : k == 1 ? count[1][i] : count[2][i];
        if (!found && block < before + nb) found = true, e = lane * 4 + i, s = start[i], n_e = start[i + 1] - start[i], blocks = nb;
        if (!found) before += nb;
    }
    e = __builtin_amdgcn_readlane(e, owner);
    s = __builtin_amdgcn_readlane(s, owner);
    n_e = __builtin_amdgcn_readlane(n_e, owner);
    blocks = __builtin_amdgcn_readlane(blocks, owner);
    before = __builtin_amdgcn_readlane(before, owner);
    int m, n;
    patch(t - before * cols, blocks, cols, m, n);
    if (k > 0) m = n_e / BM;
    out.e = e;
    out.row0 = s + m * BM;
    out.rows = n_e - m * BM < BM ? n_e - m * BM : BM;
    out.n = n;
    return true;
}
// At most so many blocks: floor(R / BM) + min(E, R).
inline long long most_blocks(const moe_config& c, int BM) {
    const long long R = (long long)c.T * c.k;
    return R / BM + (R < c.E ? R : c.E);
}

}  // namespace

}  // namespace moe
