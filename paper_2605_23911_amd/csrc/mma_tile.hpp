// One tile of C[m, n] = sum_k A(m, k) B(n, k) on bf16 MFMA (gfx950), for the operators whose operands are not both stored with
// the reduction dimension contiguous: gradients with respect to rows (the weights' rows run along k), gradients with respect to
// weights (both operands' rows run along k), and the projections with row-major weights beside them.
//
// Both operands go global -> LDS by DMA from buffer descriptors, BK of k per step into a ring of buffers; a descriptor's range is the tile's own rows, so what lies beyond a ragged end (rows of the next
// expert, whatever they hold) arrives as zeros and needs no mask.
//   operand stored with k contiguous:   LDS rows of 64 k (128 bytes), one ds_read_b128 per MFMA fragment.  Position p of row r
//       holds 16-byte chunk p ^ ((r >> 1) & 7): sixteen lanes that read one chunk column of sixteen rows hit all 64 banks once.
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
typedef short s16x8 __attribute__((ext_vector_type(8)));

// The thread's number at the start of a body.  Opaque to the compiler, which would work out what all bodies of a kernel derive from it once, in
// front of them, and hold it in registers that the tallest body does not have.
__device__ __forceinline__ int body_thread() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
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
    __device__ static __forceinline__ Stream make(const uint16_t* p, int ld, int rows_or_m0, int k) {
        Stream s;
        s.row_bytes = (uint32_t)ld * 2u;
        s.left = k;
        if constexpr (KC) {
            s.base = (uint64_t)(uintptr_t)p;
            s.range = (uint32_t)rows_or_m0 * s.row_bytes;
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
    __device__ __forceinline__ void issue(const Panel& p, uint32_t lds, int wave) const { buffer_dma<N>(off, p.desc(), lds + wave * (N * 1024)); }
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
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BK = BK_, STAGES = STAGES_;
    static constexpr int WAVES = WM * WN, THREADS = WAVES * kWave;
    static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;   // 32x32 blocks per wavefront
    static constexpr int kBufA = BM * BK * 2, kBuf = (BM + BN) * BK * 2, kRing = STAGES * kBuf;
    static constexpr int LD = BN + 4;                            // floats per staged row: 16 bytes more, which spreads the rows over the banks
    static constexpr int kPassRows = WM * 32;                    // rows staged at a time: one block of every wavefront row
    static constexpr int kStage = kPassRows * LD * 4;
    static constexpr int kLds = kRing > kStage ? kRing : kStage;
    template <bool KC> using LoadA = Loader<BM, KC, BK, WAVES>;
    template <bool KC> using LoadB = Loader<BN, KC, BK, WAVES>;
    static_assert(MB >= 1 && MB <= 4 && NB >= 1, "blocks");
};

typedef Shape<256, 256, 2, 4, 64, 2, 1, 100> Wide;
typedef Shape<128, 256, 1, 4, 32, 3, 2, 95> Pair;
typedef Shape<128, 128, 2, 4, 64, 2, 2, 75> Half;

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
// The ring is always full: STAGES - 1 steps are under way while one is read.  The fragments of a slot are read while the slot before is
// multiplied; a step's barrier stands in front of its last slot's multiplications, which cover the first reads of the next step.
// Ends with every wavefront past its last LDS read and nothing on its way into LDS.
template <class S, int MB, bool AKC, bool BKC>
__device__ __forceinline__ void multiply(f32x16 (&acc)[S::NB][MB], Stream<AKC, S::BK> a, Stream<BKC, S::BK> b, const typename S::template LoadA<AKC>& la,
                                         const typename S::template LoadB<BKC>& lb, int steps, char* lds) {
    constexpr int SLOTS = S::BK / 16, LOADS = S::template LoadA<AKC>::N + S::template LoadB<BKC>::N;     // loads per step and wavefront
    constexpr int READS = (AKC ? 1 : 2) * MB + (BKC ? 1 : 2) * S::NB, MFMAS = MB * S::NB;
    const int tid = body_thread(), wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
    Reader<S::BM, AKC, S::BK, MB> ra;
    Reader<S::BN, BKC, S::BK, S::NB> rb;
    ra.init(wm * MB * 32, lane);
    rb.init(wn * S::NB * 32, lane);
    const uint32_t at = (uint32_t)(uintptr_t)lds;
    uint32_t buf = 0;                                            // byte offset of the step that is read
    bf16x8 fa[2][MB], fb[2][S::NB];
    auto load = [&](uint32_t to) {
        la.issue(a.next(), at + to, wave);
        lb.issue(b.next(), at + to + S::kBufA, wave);
    };
    auto read = [&](uint32_t from, int s, int set) {
#pragma unroll
        for (int n = 0; n < S::NB; ++n) fb[set][n] = rb.read(lds + from + S::kBufA, n, s);
#pragma unroll
        for (int m = 0; m < MB; ++m) fa[set][m] = ra.read(lds + from, m, s);
    };
    auto landed = [&] {       // the oldest step under way has landed, and no wavefront reads what it has read any more
        wait_vmcnt<(S::STAGES - 2) * LOADS>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    if (steps <= 0) return;
#pragma unroll
    for (int i = 0; i < S::STAGES; ++i) {
        if (i + 1 == S::STAGES) landed();
        load(i * S::kBuf);
    }
    read(0, 0, 0);
    for (int i = 0; i < steps; ++i) {
        const uint32_t next = buf + S::kBuf == S::kRing ? 0 : buf + S::kBuf;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            if (s + 1 < SLOTS) {
                read(buf, s + 1, (s + 1) & 1);
            } else {
                landed();
                read(next, 0, 0);
                load(buf);
            }
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int n = 0; n < S::NB; ++n) acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[s & 1][n], fa[s & 1][m], acc[n][m], 0, 0, 0);
            // one multiplication, then as many of the next slot's reads as keep the reads in front of the end
#pragma unroll
            for (int j = 0; j < MFMAS; ++j) {
                __builtin_amdgcn_sched_group_barrier(0x100, (READS + MFMAS - 1) / MFMAS, 0);
                __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            }
        }
        buf = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Hands the tile's fp32 results out by rows: f(row in the tile, group, the row's BN floats in LDS) for GROUPS groups of columns per row.  Staged
// through LDS, one 32-row block of every wavefront row at a time, so that what f stores are whole rows.
template <class S, int GROUPS, int MB, class F>
__device__ __forceinline__ void by_rows(const f32x16 (&acc)[S::NB][MB], char* lds, F&& f) {
    const int tid = body_thread(), wave = tid / kWave, lane = tid % kWave;
    const int wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
    for (int p = 0; p < MB; ++p) {
        float* row = reinterpret_cast<float*>(lds) + (size_t)(wm * 32 + (lane & 31)) * S::LD + wn * S::NB * 32 + (lane >> 5) * 4;
#pragma unroll
        for (int n = 0; n < S::NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(row + n * 32 + q * 8) = f32x4{acc[n][p][q * 4], acc[n][p][q * 4 + 1], acc[n][p][q * 4 + 2], acc[n][p][q * 4 + 3]};
        __syncthreads();
#pragma unroll 4
        for (int j = tid; j < S::kPassRows * GROUPS; j += S::THREADS) {
            const int r = j / GROUPS, g = j % GROUPS;
            f((r / 32) * (MB * 32) + p * 32 + (r & 31), g, reinterpret_cast<const float*>(lds) + (size_t)r * S::LD);
        }
        if (p + 1 < MB) __syncthreads();
    }
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

// Which of a launch's `total` tiles a workgroup takes: the hardware deals workgroups to the eight XCDs in turn, and here every XCD gets
// one run of consecutive tiles, so that tiles which share operands share an L2.  -1: none.
__device__ __forceinline__ int xcd_tile(int total) {
    const int per = (total + 7) / 8, x = blockIdx.x & 7, i = blockIdx.x >> 3;
    const int t = x * per + i;
    return i < per && t < total ? t : -1;
}
inline unsigned xcd_grid(long long total) { return (unsigned)((total + 7) / 8 * 8); }

// What a launch of M x N results takes by rounds of tiles, in units of a result: rounds times what a CU works on at a time.  PER: workgroups per CU;
// RATE: how fast the shape multiplies where rounds are full, in percent of Wide.
template <class S>
inline long long cost(long long M, long long N) {
    const long long tiles = ((M + S::BM - 1) / S::BM) * ((N + S::BN - 1) / S::BN);
    return (tiles + 256 * S::PER - 1) / (256 * S::PER) * S::PER * S::BM * S::BN * 100 / S::RATE;
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
struct RowTile {
    int e, row0, rows, n;      // expert, first row, rows in the tile, column tile
};
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int E, int BM, int cols, RowTile& out) {
    const int lane = threadIdx.x % kWave;
    int start[5], nb[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const int e = lane * 4 + i;
        start[i] = offsets[e < E ? e : E];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += nb[i] = (start[i + 1] - start[i] + BM - 1) / BM;
    int inc = sum;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int up = __shfl_up(inc, o, kWave);
        if (lane >= o) inc += up;
    }
    const int total = __shfl(inc, kWave - 1, kWave) * cols;
    const int t = xcd_tile(total);
    if (t < 0) return false;
    const int block = t / cols;                    // some block of the same expert
    const unsigned long long hit = __ballot(inc > block);
    const int owner = __builtin_ctzll(hit);
    int before = inc - sum, e = 0, s = 0, n_e = 0, blocks = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (!found && block < before + nb[i]) found = true, e = lane * 4 + i, s = start[i], n_e = start[i + 1] - start[i], blocks = nb[i];
        if (!found) before += nb[i];
    }
    e = __builtin_amdgcn_readlane(e, owner);
    s = __builtin_amdgcn_readlane(s, owner);
    n_e = __builtin_amdgcn_readlane(n_e, owner);
    blocks = __builtin_amdgcn_readlane(blocks, owner);
    before = __builtin_amdgcn_readlane(before, owner);
    int m, n;
    patch(t - before * cols, blocks, cols, m, n);
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
