// Tokens sorted by expert, their rows' way back, and the gradients of both, where not every slot has a row.
//   slot j = t k + i has a row iff e = idx[j] - first is in 0 .. E - 1 and fewer than `capacity` slots in front of j chose e (its rank)
//   counts[e] = slots that chose e;  offsets = exclusive sums of min(counts, capacity);  row(j) = offsets[e] + rank
//   dispatch   rows[row(t,i)] = (w[t,i]) x[t]          its gradient  dx[t] = (base[t] +) sum_i (w[t,i]) drows[row(t,i)],  dw[t,i] = <x[t], drows[row(t,i)]>
//   collect    y[t] = (residual[t] +) D(sum_i (w[t,i]) rows[row(t,i)])
//              its gradient  v = D(dy[t]), drows[row(t,i)] = (w[t,i]) v,  dw[t,i] = <v, rows[row(t,i)]>
// Each pass moves every row once, so all four are bound by memory from about a thousand rows on, the small ones by a launch's 2-5 us.  No atomics on memory: results are
// bit-reproducible.
#include <type_traits>

#include "token_rows.hpp"

namespace moe {

namespace {

constexpr int kChunk = 1024;              // slots per workgroup of the count and the tables
constexpr int kMostSlots = 1024;          // of a workgroup that moves rows
constexpr int kNarrow = 256;              // width up to which lanes of a wavefront take several tokens
constexpr int kBins = 512;                // counters in LDS: as many copies of the experts' as fit, so that one wavefront's slots rarely meet

struct DispatchArgs {
    const uint16_t* x;
    const int32_t* idx;
    const float* w;
    int32_t *counts, *offsets, *row_of, *src_of;
    uint16_t* rows;
    int32_t* hist;            // [chunks, E]; null: every workgroup counts all slots itself
    int T, d, k, E, first, capacity;
    int per;                  // tokens per workgroup
    int chunks;
    bool summed;              // hist holds the counts of all chunks in front, counts the totals
};

__device__ __forceinline__ int local_expert(const DispatchArgs& a, long long j) {
    const int e = (int)((uint32_t)a.idx[j] - (uint32_t)a.first);      // wraps for ids below first
    return (uint32_t)e < (uint32_t)a.E ? e : -1;
}

// Slots j0 .. j1 - 1 into the bins; those from `split` on into the second half.  Sixteen ids per thread are requested before the first is counted, and what is no slot of an
// expert here goes to a bin of the lane's own behind the others: no branch that a wavefront takes by its ids (with such branches 4096 slots took a workgroup 4.8 us, so 1.8).
template <int THREADS>
__device__ __forceinline__ void count_slots(const DispatchArgs& a, long long j0, long long j1, long long split, int copies, int* bins) {
    constexpr int AHEAD = 16;
    const int mine = (threadIdx.x & (copies - 1)) * a.E, none = 2 * kBins + threadIdx.x % kWave;
    for (long long at = j0; at < j1; at += AHEAD * THREADS) {
        const int32_t* idx = a.idx + at;
        const int n = j1 - at < AHEAD * THREADS ? (int)(j1 - at) : AHEAD * THREADS, half = split - at < n ? (int)(split - at) : n;     // may be negative
        int id[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int j = threadIdx.x + i * THREADS;
            if (i * THREADS < n) id[i] = idx[j < n ? j : n - 1];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int j = threadIdx.x + i * THREADS;
            const uint32_t e = (uint32_t)id[i] - (uint32_t)a.first;
            if (i * THREADS < n) atomicAdd(&bins[j < n && e < (uint32_t)a.E ? (j >= half ? kBins : 0) + mine + (int)e : none], 1);
        }
    }
}
__device__ __forceinline__ int bin_copies(int E) {
    int n = 32;
    while (n * E > kBins) n >>= 1;
    return n;
}
__device__ __forceinline__ int bin_total(const int* bins, int copies, int E, int e) {
    int n = 0;
#pragma unroll 8
    for (int c = 0; c < copies; ++c) n += bins[c * E + e];
    return n;
}

// What each chunk of 1024 slots has of every expert, for calls in which counting all slots in every workgroup takes longer than a launch: 3.4-4.8 us at 32768 slots.
__global__ __launch_bounds__(kTokenThreads) void count_chunks_kernel(DispatchArgs a) {
    __shared__ int bins[2 * kBins + kWave];
    const int copies = bin_copies(a.E);
    for (int i = threadIdx.x; i < copies * a.E; i += kTokenThreads) bins[i] = 0;
    __syncthreads();
    const long long R = (long long)a.T * a.k, j0 = (long long)blockIdx.x * kChunk, j1 = j0 + kChunk < R ? j0 + kChunk : R;
    count_slots<kTokenThreads>(a, j0, j1, j1, copies, bins);
    __syncthreads();
    if ((int)threadIdx.x < a.E) a.hist[(size_t)blockIdx.x * a.E + threadIdx.x] = bin_total(bins, copies, a.E, threadIdx.x);
}

// Exclusive sums over the chunks, 64 experts per workgroup: each wavefront takes a run of chunks, first its total, then, with those of the wavefronts in
// front, the sums.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void sum_chunks_kernel(DispatchArgs a) {
    __shared__ int part[kSumThreads / kWave][kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, e = blockIdx.x * kWave + lane;
    const int each = (a.chunks + kSumThreads / kWave - 1) / (kSumThreads / kWave), c0 = wave * each, c1 = c0 + each < a.chunks ? c0 + each : a.chunks;
    int n = 0;
    if (e < a.E) {
#pragma unroll 8
        for (int c = c0; c < c1; ++c) n += a.hist[(size_t)c * a.E + e];
    }
    part[wave][lane] = n;
    __syncthreads();
    if (e >= a.E) return;
    int at = 0, all = 0;
    for (int w = 0; w < kSumThreads / kWave; ++w) {
        if (w < wave) at += part[w][lane];
        all += part[w][lane];
    }
    if (wave == 0) a.counts[e] = all;
    for (int c = c0; c < c1; ++c) {
        const int m = a.hist[(size_t)c * a.E + e];
        a.hist[(size_t)c * a.E + e] = at;
        at += m;
    }
}

// in[t] (after dropout, where there is any) times a slot's weight into its row.  Slots i0 .. of the token; DOT: and <in[t], row of `with`>.
// PAST: the rows pass the caches by, 1: those written, 2: those read, too.
struct ScatterArgs {
    const uint16_t* in;
    const uint16_t* with;
    uint16_t* out;
    int d;
    bool scaled;              // false: rows are copies
    Dropout p;
};
template <int N, bool DOT, int PAST>
__device__ __forceinline__ void scatter_slots(const ScatterArgs& a, const Slots<N>& s, int t, int lane, int threads, uint64_t seed, uint64_t offset, float (&dot)[N]) {
    const Row in = row_at(a.in, (size_t)t * a.d * 2, s.any, a.d * 2);
    Row out[N], with[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out[i] = s.at(a.out, i, a.d);
        if constexpr (DOT) with[i] = s.at(a.with, i, a.d);
        dot[i] = 0.0f;
    }
    for (int c = lane * 8; c < a.d; c += threads * 8) {
        const u32x4_t raw = read8<false>(in, c * 2);
        u32x4_t other[N];
        if constexpr (DOT) {
#pragma unroll
            for (int i = 0; i < N; ++i) other[i] = read8<PAST == 2>(with[i], c * 2);
        }
        float v[8];
        floats8(raw, v);
        if (a.p.rng) drop8(v, ((uint64_t)t * a.d + c) / 8, seed, offset, a.p);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (DOT) {
                float q[8];
                floats8(other[i], q);
#pragma unroll
                for (int j = 0; j < 8; ++j) dot[i] = fmaf(v[j], q[j], dot[i]);
            }
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = s.w[i] * v[j];
            write8<PAST >= 1>(a.scaled ? bf16s8(o) : raw, out[i], c * 2);
        }
    }
}

// Where every expert's slots go on from: before[e] slots in front of the workgroup's own, start[e] the expert's first row.  All of it from LDS counts of all slots, or, with
// `hist`, of the slots between the chunk's start and the workgroup's own and the chunks' counts.  The first workgroup writes counts and offsets.
template <int THREADS>
struct Places {
    int bins[2 * kBins + kWave];
    int next[kMaxExperts], start[kMaxExperts], sums[THREADS / kWave];

    __device__ __forceinline__ void find(const DispatchArgs& a, long long s0) {
        const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave, copies = bin_copies(a.E), chunk = (int)(s0 / kChunk);
        const long long R = (long long)a.T * a.k;
        for (int i = tid; i < copies * a.E; i += THREADS) bins[i] = bins[kBins + i] = 0;
        __syncthreads();
        if (a.hist) count_slots<THREADS>(a, (long long)chunk * kChunk, s0, s0, copies, bins);
        else count_slots<THREADS>(a, 0, R, s0, copies, bins);
        __syncthreads();
        int total = 0, before = 0;
        if (tid < a.E) {
            before = bin_total(bins, copies, a.E, tid);
            if (!a.hist) total = before + bin_total(bins + kBins, copies, a.E, tid);
            else if (a.summed) before += a.hist[(size_t)chunk * a.E + tid], total = a.counts[tid];
            else {
#pragma unroll 16
                for (int c = 0; c < a.chunks; ++c) {
                    const int n = a.hist[(size_t)c * a.E + tid];
                    total += n;
                    before += c < chunk ? n : 0;
                }
            }
        }
        const int most = a.capacity ? a.capacity : 0x7fffffff, kept = total < most ? total : most;
        int upto = kept;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int up = __shfl_up(upto, o, kWave);
            if (lane >= o) upto += up;
        }
        if (lane == kWave - 1) sums[wave] = upto;
        __syncthreads();
        for (int w = 0; w < wave && w < kMaxExperts / kWave; ++w) upto += sums[w];
        if (tid < a.E) {
            next[tid] = before;
            start[tid] = upto - kept;
            if (blockIdx.x == 0) {
                if (!a.summed) a.counts[tid] = total;
                a.offsets[tid] = upto - kept;
                if (tid == a.E - 1) a.offsets[a.E] = upto;
            }
        }
        __syncthreads();
    }
};

// Of the wavefront's lanes, those whose slot chose the same expert (they agree in all eight bits; e < 0: none).
__device__ __forceinline__ unsigned long long same_expert(int e) {
    unsigned long long same = __ballot(e >= 0);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const unsigned long long has = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? has : ~has;
    }
    return same;
}
__device__ __forceinline__ int in_front(unsigned long long lanes, int lane) { return __popcll(lanes & ((1ull << lane) - 1)); }

// The tables alone, 1024 slots per workgroup, a slot per thread.  A wavefront ranks its 64 slots among themselves, a sum over the wavefronts' counts does the rest (one wavefront
// after the other 15 us).  Bound by latency: 4.2 us at 2 slots, 5.3 at 4096, 8 at 32768.
constexpr int kTableThreads = kChunk, kTableWaves = kTableThreads / kWave;
__global__ __launch_bounds__(kTableThreads) void tables_kernel(DispatchArgs a) {
    __shared__ Places<kTableThreads> places;
    __shared__ int count[kTableWaves][kMaxExperts];      // of every wavefront; then of those in front of it
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const long long R = (long long)a.T * a.k, s0 = (long long)blockIdx.x * kChunk, j = s0 + tid;
    const int e = j < R ? local_expert(a, j) : -1;
    for (int i = tid; i < kTableWaves * kMaxExperts; i += kTableThreads) (&count[0][0])[i] = 0;
    places.find(a, s0);
    const unsigned long long same = same_expert(e);
    const int rank = in_front(same, lane);
    if (e >= 0 && rank == 0) count[wave][e] = __popcll(same);
    __syncthreads();
    if (tid < a.E) {
        int n = places.next[tid];
#pragma unroll
        for (int w = 0; w < kTableWaves; ++w) {
            const int m = count[w][tid];
            count[w][tid] = n;
            n += m;
        }
    }
    __syncthreads();
    if (j >= R) return;
    const int r = e >= 0 ? count[wave][e] + rank : 0, most = a.capacity ? a.capacity : 0x7fffffff, row = e >= 0 && r < most ? places.start[e] + r : -1;
    a.row_of[j] = row;
    if (row >= 0) a.src_of[row] = (int32_t)j;
}

// What the lanes of a wavefront did to LDS so far comes before what they do from here on.
__device__ __forceinline__ void order_lanes() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Tables and rows: a workgroup takes `per` tokens, finds out where its slots go, ranks them, and moves its tokens' rows: less than four tokens one after the other, more a
// wavefront each, narrow ones (d up to kNarrow, half a wavefront's loads) a few lanes each.  One launch for tables and rows, since a launch of its own for the rows takes 3 us more
// than it saves (24576 slots x 2048 31.3 / 28.6 us).  x is read once, not once per slot.  1 token 4.5 us, 1024 x 2 x 4096 8; 4096 x 8 x 7168, 0.39 GB written, 82 us (5.5 TB/s).
// What comes before the rows, of a workgroup's time: 0.2 us to clear the bins, 1-2 to count, 0.4-1.6 for the totals, 0.6 for the sums, 0.6 for the ranks.  Not kept: x (1 token 4.5 us,
// so 6.1), the chunks' counts and the workgroup's own ids (even or 0.2 us more) requested before the count.
template <int N, bool NT, bool NARROW>
__global__ __launch_bounds__(kTokenThreads) void dispatch_kernel(DispatchArgs a) {
    __shared__ Places<kTokenThreads> places;
    __shared__ int row[kMostSlots];
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const long long R = (long long)a.T * a.k, s0 = (long long)blockIdx.x * a.per * a.k, s1 = s0 + (long long)a.per * a.k < R ? s0 + (long long)a.per * a.k : R;
    places.find(a, s0);
    if (wave == 0) {
        const int most = a.capacity ? a.capacity : 0x7fffffff;
        for (long long j0 = s0; j0 < s1; j0 += kWave) {
            const long long j = j0 + lane;
            const int e = j < s1 ? local_expert(a, j) : -1;
            const unsigned long long same = same_expert(e);
            const int rank = in_front(same, lane), base = e >= 0 ? places.next[e] : 0;
            order_lanes();                 // every lane has read the count before the first of its expert advances it
            if (e >= 0 && rank == 0) places.next[e] = base + __popcll(same);
            order_lanes();
            const int r = e >= 0 && base + rank < most ? places.start[e] + base + rank : -1;
            if (j < s1) {
                row[j - s0] = r;
                a.row_of[j] = r;
                if (r >= 0) a.src_of[r] = (int32_t)j;
            }
        }
    }
    __syncthreads();
    const int tokens = (int)((s1 - s0) / a.k), first = (int)(s0 / a.k);
    if constexpr (NARROW) {
        const int lots = a.d / 8;
        for (int q = tid; q < tokens * lots; q += kTokenThreads) {
            const int t = q / lots, c = q - t * lots;
            const u32x4_t raw = *reinterpret_cast<const u32x4_t*>(a.x + ((size_t)first * lots + q) * 8);
            float v[8], o[8];
            floats8(raw, v);
            for (int i = 0; i < a.k; ++i) {
                const int r = row[t * a.k + i];
                if (r < 0) continue;
                const float w = a.w ? a.w[s0 + t * a.k + i] : 1.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = w * v[j];
                *reinterpret_cast<u32x4_t*>(a.rows + (size_t)r * a.d + c * 8) = a.w ? bf16s8(o) : raw;
            }
        }
    } else {
        const ScatterArgs to{a.x, nullptr, a.rows, a.d, a.w != nullptr, {}};
        const bool whole = a.per < kTokenWaves;
        for (int t = whole ? 0 : wave; t < tokens; t += whole ? 1 : kTokenWaves) {
            for (int i0 = 0; i0 < a.k; i0 += N) {
                Slots<N> s;
                s.load(row + t * a.k, a.w ? a.w + (size_t)(first + t) * a.k : nullptr, i0, a.k, R);
                float dot[N];
                scatter_slots<N, false, NT ? 1 : 0>(to, s, first + t, whole ? tid : lane, whole ? kTokenThreads : kWave, 0, 0, dot);
            }
        }
    }
}

struct CollectArgs {
    ScatterArgs to;           // of the gradient
    const uint16_t *rows, *add, *x;
    const int32_t* row_of;
    const float* w;
    uint16_t* y;
    float* dw;
    Dropout p;
    int T, d, k, t0;
    bool whole;               // a workgroup per token, else a wavefront
};

__device__ __forceinline__ int my_token(const CollectArgs& a) {
    return a.t0 + (a.whole ? (int)blockIdx.x : (int)blockIdx.x * kTokenWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
}

// y[t] = (add[t] +) D(sum_i w[t,i] row(t,i)), and with DOT <x[t], row(t,i)>, in slot order.  A token's rows are requested before the first is used.  Bound by memory: 4096 x 8 x
// 7168 97-98 us (0.59 GB, 6.0 TB/s), with dropout the same; 512 x 8 x 7168 13.1, 64 x 2 x 4096 3.1.
// B batches of N slots, all requested before the first is used; B = 0: any number of batches, over which the columns run for the sum and which run over the columns for the dot
// products.
template <int N, bool DOT, bool NT, int B>
__global__ __launch_bounds__(kTokenThreads) void gather_kernel(CollectArgs a) {
    __shared__ float part[kTokenWaves][8];
    const int t = my_token(a);
    if (t >= a.T) return;
    const int lane = a.whole ? threadIdx.x : threadIdx.x % kWave, threads = a.whole ? kTokenThreads : kWave;
    const long long R = (long long)a.T * a.k;
    const int32_t* row_of = a.row_of + (size_t)t * a.k;
    const float* w = a.w ? a.w + (size_t)t * a.k : nullptr;
    const Row add = row_at(a.add, (size_t)t * a.d * 2, a.add != nullptr, a.d * 2), y = row_at(a.y, (size_t)t * a.d * 2, true, a.d * 2);
    const uint64_t seed = a.p.rng ? a.p.rng[0] : 0, offset = a.p.rng ? a.p.rng[1] : 0;
    constexpr int HELD = B ? B : 1;
    Slots<N> s[HELD];
    float dot[HELD][N];
    bool any = false;
#pragma unroll
    for (int b = 0; b < B; ++b) {
        s[b].load(row_of, w, b * N, a.k, R);
        any |= s[b].any;
    }
#pragma unroll
    for (int b = 0; b < HELD; ++b)
#pragma unroll
        for (int i = 0; i < N; ++i) dot[b][i] = 0.0f;
    const Row x = row_at(a.x, (size_t)t * a.d * 2, DOT && any, a.d * 2);
    for (int c = lane * 8; c < a.d; c += threads * 8) {
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
        const u32x4_t more = read8<false>(add, c * 2);
        auto request = [&](const Slots<N>& from, u32x4_t (&v)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = read8<NT>(from.at(a.rows, i, a.d), c * 2);
        };
        auto take = [&](const Slots<N>& from, const u32x4_t (&v)[N], const u32x4_t& with, float (&dots)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float q[8];
                floats8(v[i], q);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum[j] = fmaf(from.w[i], q[j], sum[j]);
                if constexpr (DOT && B > 0) {
                    float o[8];
                    floats8(with, o);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dots[i] = fmaf(o[j], q[j], dots[i]);
                }
            }
        };
        u32x4_t with = {0, 0, 0, 0};
        if constexpr (DOT && B > 0) with = read8<false>(x, c * 2);
        if constexpr (B == 1) {
            u32x4_t v[N];
            request(s[0], v);
            take(s[0], v, with, dot[0]);
        } else if constexpr (B > 1) {
            u32x4_t v[HELD][N];
#pragma unroll
            for (int b = 0; b < B; ++b) request(s[b], v[b]);
#pragma unroll
            for (int b = 0; b < B; ++b) take(s[b], v[b], with, dot[b]);
        } else {
            for (int i0 = 0; i0 < a.k; i0 += N) {
                u32x4_t v[N];
                s[0].load(row_of, w, i0, a.k, R);
                request(s[0], v);
                take(s[0], v, with, dot[0]);
            }
        }
        if (a.p.rng) drop8(sum, ((uint64_t)t * a.d + c) / 8, seed, offset, a.p);
        float o[8];
        floats8(more, o);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += o[j];
        write8<false>(bf16s8(sum), y, c * 2);
    }
    if constexpr (DOT && B > 0) {
#pragma unroll
        for (int b = 0; b < B; ++b) store_dots<N>(dot[b], s[b], part, a.whole, a.k - b * N < N ? a.k - b * N : N, a.dw + (size_t)t * a.k + b * N);
    }
    if constexpr (DOT && B == 0) {         // the rows once more, a batch of slots at a time
        for (int i0 = 0; i0 < a.k; i0 += N) {
            s[0].load(row_of, w, i0, a.k, R);
            const Row in = row_at(a.x, (size_t)t * a.d * 2, s[0].any, a.d * 2);
#pragma unroll
            for (int i = 0; i < N; ++i) dot[0][i] = 0.0f;
            for (int c = lane * 8; c < a.d; c += threads * 8) {
                float o[8];
                floats8(read8<false>(in, c * 2), o);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    float q[8];
                    floats8(read8<false>(s[0].at(a.rows, i, a.d), c * 2), q);
#pragma unroll
                    for (int j = 0; j < 8; ++j) dot[0][i] = fmaf(o[j], q[j], dot[0][i]);
                }
            }
            store_dots<N>(dot[0], s[0], part, a.whole, a.k - i0 < N ? a.k - i0 : N, a.dw + (size_t)t * a.k + i0);
        }
    }
}

// The gradient of collect: rows read (DOT) and their gradients written.  Bound by memory where there is much: 4096 x 8 x 7168, 1.0 GB, 192-215 us (4.6-5.2 TB/s; a copy 4.9).  1999 x 8 x 3584 with
// 0.14 GB 31: the slots' numbers and weights fetched one after the other, and five wavefronts per SIMD (84 registers, 78 scalars spilled into lanes of them), 1.6 rounds.
template <int N, bool DOT, int PAST>
__global__ __launch_bounds__(kTokenThreads) void scatter_kernel(CollectArgs a) {
    __shared__ float part[kTokenWaves][8];
    const int t = my_token(a);
    if (t >= a.T) return;
    const int lane = a.whole ? threadIdx.x : threadIdx.x % kWave, threads = a.whole ? kTokenThreads : kWave;
    const uint64_t seed = a.to.p.rng ? a.to.p.rng[0] : 0, offset = a.to.p.rng ? a.to.p.rng[1] : 0;
    for (int i0 = 0; i0 < a.k; i0 += N) {
        Slots<N> s;
        s.load(a.row_of + (size_t)t * a.k, a.w ? a.w + (size_t)t * a.k : nullptr, i0, a.k, (long long)a.T * a.k);
        float dot[N];
        scatter_slots<N, DOT, PAST>(a.to, s, t, lane, threads, seed, offset, dot);
        if constexpr (DOT) store_dots<N>(dot, s, part, a.whole, a.k - i0 < N ? a.k - i0 : N, a.dw + (size_t)t * a.k + i0);
    }
}

// NARROW rows (d up to 256): `lots` = d / 8 lanes per token, as many tokens as fit into a wavefront; the other lanes idle.  16384 tokens of 8 slots, d = 8, the way back and
// its gradient, a wavefront per token / so: 11.2 / 7.3 and 29.6 / 7.7 us, of 4 slots, d = 64 8.2 / 7.1 and 16.6 / 7.6 (what a call takes on the host).
struct NarrowPlace {
    int t, c, lot;             // token (0 where the lane idles), first column, the lane's place among the token's
    bool there;
};
__device__ __forceinline__ NarrowPlace narrow_place(const CollectArgs& a) {
    const int lots = a.d / 8, fit = kWave / lots, lane = threadIdx.x % kWave, mine = lane / lots, lot = lane - mine * lots;
    const long long t = a.t0 + ((long long)blockIdx.x * kTokenWaves + threadIdx.x / kWave) * fit + mine;
    const bool there = mine < fit && t < a.T;
    return {there ? (int)t : 0, lot * 8, lot, there};
}
// Sum over the token's lanes, in its first one, always in the same order.
__device__ __forceinline__ float narrow_total(float v, int lot, int lots) {
#pragma unroll
    for (int o = kWave / 4; o > 0; o >>= 1) {
        const float up = __shfl_down(v, o, kWave);
        if (lot + o < lots) v += up;
    }
    return v;
}

template <int N, bool DOT>
__global__ __launch_bounds__(kTokenThreads) void narrow_gather_kernel(CollectArgs a) {
    const NarrowPlace m = narrow_place(a);
    const int lots = a.d / 8;
    const size_t at = (size_t)m.t * a.d + m.c;
    const long long R = (long long)a.T * a.k;
    const u32x4_t none = {0, 0, 0, 0};
    const u32x4_t more = m.there && a.add ? *reinterpret_cast<const u32x4_t*>(a.add + at) : none, with = DOT && m.there ? *reinterpret_cast<const u32x4_t*>(a.x + at) : none;
    float sum[8], x[8];
    floats8(with, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.0f;
    for (int i0 = 0; i0 < a.k; i0 += N) {
        u32x4_t v[N];
        float w[N];
        bool has[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const size_t slot = (size_t)m.t * a.k + i0 + i;
            const int32_t r = m.there && i0 + i < a.k ? a.row_of[slot] : -1;
            has[i] = r >= 0 && r < R;
            w[i] = has[i] ? a.w ? a.w[slot] : 1.0f : 0.0f;
            v[i] = has[i] ? *reinterpret_cast<const u32x4_t*>(a.rows + (size_t)r * a.d + m.c) : none;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float q[8], dot = 0.0f;
            floats8(v[i], q);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sum[j] = fmaf(w[i], q[j], sum[j]);
                if constexpr (DOT) dot = fmaf(x[j], q[j], dot);
            }
            if constexpr (DOT) {
                dot = narrow_total(dot, m.lot, lots);
                if (m.there && m.lot == 0 && i0 + i < a.k) a.dw[(size_t)m.t * a.k + i0 + i] = has[i] ? dot : 0.0f;
            }
        }
    }
    if (!m.there) return;
    if (a.p.rng) drop8(sum, at / 8, a.p.rng[0], a.p.rng[1], a.p);
    float o[8];
    floats8(more, o);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += o[j];
    *reinterpret_cast<u32x4_t*>(a.y + at) = bf16s8(sum);
}

template <int N, bool DOT>
__global__ __launch_bounds__(kTokenThreads) void narrow_scatter_kernel(CollectArgs a) {
    const NarrowPlace m = narrow_place(a);
    const int lots = a.d / 8;
    const size_t at = (size_t)m.t * a.d + m.c;
    const long long R = (long long)a.T * a.k;
    const u32x4_t none = {0, 0, 0, 0}, raw = m.there ? *reinterpret_cast<const u32x4_t*>(a.to.in + at) : none;
    float v[8];
    floats8(raw, v);
    if (a.to.p.rng) drop8(v, at / 8, a.to.p.rng[0], a.to.p.rng[1], a.to.p);
    for (int i0 = 0; i0 < a.k; i0 += N) {
        u32x4_t with[N];
        int32_t r[N];
        float w[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const size_t slot = (size_t)m.t * a.k + i0 + i;
            const int32_t n = m.there && i0 + i < a.k ? a.row_of[slot] : -1;
            r[i] = n >= 0 && n < R ? n : -1;
            w[i] = r[i] >= 0 && a.w ? a.w[slot] : 1.0f;
            if constexpr (DOT) with[i] = r[i] >= 0 ? *reinterpret_cast<const u32x4_t*>(a.to.with + (size_t)r[i] * a.d + m.c) : none;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (DOT) {
                float q[8], dot = 0.0f;
                floats8(with[i], q);
#pragma unroll
                for (int j = 0; j < 8; ++j) dot = fmaf(v[j], q[j], dot);
                dot = narrow_total(dot, m.lot, lots);
                if (m.there && m.lot == 0 && i0 + i < a.k) a.dw[(size_t)m.t * a.k + i0 + i] = r[i] >= 0 ? dot : 0.0f;
            }
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = w[i] * v[j];
            if (r[i] >= 0) *reinterpret_cast<u32x4_t*>(a.to.out + (size_t)r[i] * a.d + m.c) = a.to.scaled ? bf16s8(o) : raw;
        }
    }
}

// Sixteen bits per element, so that one call of the generator serves the eight elements of a load and stays below memory's time: 4096 x 7168 with a residual 26.5-30 us
// (176 MB, 5.9-6.6 TB/s), with the generator called twice 32.
template <bool ADD>
__global__ __launch_bounds__(kTokenThreads) void dropout_kernel(const uint16_t* x, const uint16_t* add, uint16_t* y, long long n, Dropout p) {
    const uint64_t seed = p.rng ? p.rng[0] : 0, offset = p.rng ? p.rng[1] : 0;
    for (long long b = (long long)blockIdx.x * kTokenThreads + threadIdx.x; b * 8 < n; b += (long long)gridDim.x * kTokenThreads) {
        float v[8], o[8];
        if (b * 8 + 8 <= n) {
            floats8(reinterpret_cast<const u32x4_t*>(x)[b], v);
            if (p.rng) drop8(v, b, seed, offset, p);
            if constexpr (ADD) {
                floats8(reinterpret_cast<const u32x4_t*>(add)[b], o);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] += o[j];
            }
            reinterpret_cast<u32x4_t*>(y)[b] = bf16s8(v);
        } else {                           // the last, partial block
            const u32x4_t bits = philox(seed, b, offset);
            for (int j = 0; b * 8 + j < n; ++j) {
                float q = bf16_bits_to_float(x[b * 8 + j]);
                if (p.rng) q = ((j & 1 ? bits[j / 2] >> 16 : bits[j / 2] & 0xffffu) >= p.limit) ? q * p.scale : 0.0f;
                if constexpr (ADD) q += bf16_bits_to_float(add[b * 8 + j]);
                y[b * 8 + j] = float_to_bf16_bits(q);
            }
        }
    }
}

// Slots up to which every workgroup counts them all (of the workgroups that move rows, of those that write the tables); beyond, a launch before counts them by chunks.  Rows, us, all
// counted / by chunks: 8192 slots x 2048 14.3 / 15.9, x 7168 27.9 / 30.8, 12000 x 7168 40.9 / 43.0, 16384 x 2048 22.5 / 20.7, 32768 x 512 27.5 / 16.6; tables: 32768 slots 9.0 / 9.7,
// 65536 13.5 / 9.6.
constexpr int kCountAllRows = 8192, kCountAll = 32768;
constexpr int kSumInside = 64;            // chunks up to which a workgroup adds their counts up

int chunks_of(const moe_dispatch_config& c) { return (int)(((long long)c.T * c.k + kChunk - 1) / kChunk); }

// From 128 MiB of rows on, half of the Infinity Cache, they pass the caches by: 448 MiB, us, cached / past the caches, collect 120 / 99, its gradient 217 / 205, dispatch 105 / 85.
// Below, dispatch's rows are read next: 94 MiB 28.5 / 30.1 alone, 64 MiB 34.8 / 38.8 with a collect of them.
bool passes_caches(const moe_dispatch_config& c) { return (long long)c.T * c.k * c.d >= (1ll << 26); }
// The gradient of collect, which reads as much as it writes, writes past them from 64 MiB on: 94 MiB 42 / 35.5 us alone.  In a step, where its rows are not in the caches, it
// takes longer and the block's gradient behind it less: together 304 / 303.5, 82 MiB 397 / 393, 109 MiB 515 / 507.
int passes_caches_gradient(const moe_dispatch_config& c) {
    const long long n = (long long)c.T * c.k * c.d;
    return n >= (1ll << 26) ? 2 : n >= (1ll << 25) ? 1 : 0;
}

// go(integral_constant<slots per batch>): a token's slots in the fewest batches of up to eight, all of one size.  Batches of 4 and 8 with empty rows cost 1-3 % at 3, 5, 6 and 7
// slots and 1-13 % at 9 to 15.
template <class F>
void by_slots(int k, F&& go) {
    using std::integral_constant;
    const int batches = (k + 7) / 8;
    switch ((k + batches - 1) / batches) {
        case 1: go(integral_constant<int, 1>{}); break;
        case 2: go(integral_constant<int, 2>{}); break;
        case 3: go(integral_constant<int, 3>{}); break;
        case 4: go(integral_constant<int, 4>{}); break;
        case 5: go(integral_constant<int, 5>{}); break;
        case 6: go(integral_constant<int, 6>{}); break;
        case 7: go(integral_constant<int, 7>{}); break;
        default: go(integral_constant<int, 8>{});
    }
}

// Tokens of one launch: it has less than 2^32 threads.  A wavefront per token up to 1024 columns, two loads of it, else a workgroup: us, a wavefront / a workgroup, collect
// 16384 x 2 x 1024 21.7 / 22.8, 8192 x 2 x 2048 22.0 / 21.6, 512 x 3 x 7168 10.4 / 8.0; its gradient 16384 x 2 x 1024 34.5 / 42.9, 8192 x 2 x 2048 35.7 / 32.9.
template <class F>
void by_launch(CollectArgs a, F&& go) {
    a.whole = a.d > 1024;
    const int each = a.whole ? 1 : kTokenWaves * (a.d <= kNarrow ? kWave / (a.d / 8) : 1);       // tokens per workgroup
    const int step = (1 << 23) * (each < 64 ? each : 64) / each * each;      // whole workgroups: a token of two launches would be added to twice where y is the residual
    for (long long t = 0; t < a.T; t += step) {
        a.t0 = (int)t;
        const long long n = a.T - t < step ? a.T - t : step;
        go(a, dim3((unsigned)((n + each - 1) / each)));
    }
}

}  // namespace

size_t dispatch_workspace_bytes(const moe_dispatch_config& c) {
    return (long long)c.T * c.k > kCountAllRows ? (size_t)chunks_of(c) * c.E * sizeof(int32_t) : 0;
}

static hipError_t launch_gather(const moe_dispatch_config& c, CollectArgs a, hipStream_t s) {
    const bool nt = passes_caches(c);
    by_slots(c.k, [&](auto n) {
        constexpr int N = decltype(n)::value;
        by_launch(a, [&](const CollectArgs& b, dim3 grid) {
            if (c.d <= kNarrow) {
                if (b.dw) hipLaunchKernelGGL((narrow_gather_kernel<N, true>), grid, dim3(kTokenThreads), 0, s, b);
                else hipLaunchKernelGGL((narrow_gather_kernel<N, false>), grid, dim3(kTokenThreads), 0, s, b);
                return;
            }
            auto go = [&](auto dot, auto batches) {
                constexpr bool DOT = decltype(dot)::value;
                constexpr int B = decltype(batches)::value;
                if (nt) hipLaunchKernelGGL((gather_kernel<N, DOT, true, B>), grid, dim3(kTokenThreads), 0, s, b);
                else hipLaunchKernelGGL((gather_kernel<N, DOT, false, B>), grid, dim3(kTokenThreads), 0, s, b);
            };
            auto with_dots = [&](auto batches) {
                if (b.dw) go(std::true_type{}, batches);
                else go(std::false_type{}, batches);
            };
            using std::integral_constant;
            if constexpr (N >= 5) {
                if (c.k > 2 * N) return with_dots(integral_constant<int, 0>{});
                if (c.k > N) return with_dots(integral_constant<int, 2>{});
            }
            with_dots(integral_constant<int, 1>{});
        });
    });
    return hipGetLastError();
}

static Dropout dropout_of(float p, const void* rng) {
    const uint32_t limit = (uint32_t)((double)p * 65536.0 + 0.5);
    return {limit ? (const uint64_t*)rng : nullptr, limit, 65536.0f / (float)(65536u - limit)};
}

hipError_t launch_dispatch_backward(const moe_dispatch_config& c, const uint16_t* x, const uint16_t* drows, const int32_t* row_of, const float* topk_w,
                                    const uint16_t* base, uint16_t* dx, float* d_topk_w, hipStream_t s) {
    return launch_gather(c, CollectArgs{{}, drows, base, x, row_of, topk_w, dx, d_topk_w, {}, c.T, c.d, c.k, 0, false}, s);
}

hipError_t launch_collect(const moe_dispatch_config& c, const uint16_t* rows, const int32_t* row_of, const float* topk_w, const uint16_t* residual, float p,
                          const void* rng, uint16_t* y, hipStream_t s) {
    return launch_gather(c, CollectArgs{{}, rows, residual, nullptr, row_of, topk_w, y, nullptr, dropout_of(p, rng), c.T, c.d, c.k, 0, false}, s);
}

static hipError_t launch_scatter(const moe_dispatch_config& c, const ScatterArgs& to, const int32_t* row_of, const float* topk_w, float* d_topk_w, hipStream_t s) {
    const CollectArgs a{to, nullptr, nullptr, nullptr, row_of, topk_w, nullptr, d_topk_w, {}, c.T, c.d, c.k, 0, false};
    const int past = d_topk_w ? passes_caches_gradient(c) : passes_caches(c);
    by_slots(c.k, [&](auto n) {
        constexpr int N = decltype(n)::value;
        by_launch(a, [&](const CollectArgs& b, dim3 grid) {
            auto go = [&](auto dot) {
                constexpr bool DOT = decltype(dot)::value;
                if (c.d <= kNarrow) hipLaunchKernelGGL((narrow_scatter_kernel<N, DOT>), grid, dim3(kTokenThreads), 0, s, b);
                else if (past == 2) hipLaunchKernelGGL((scatter_kernel<N, DOT, DOT ? 2 : 1>), grid, dim3(kTokenThreads), 0, s, b);
                else if (past == 1) hipLaunchKernelGGL((scatter_kernel<N, DOT, 1>), grid, dim3(kTokenThreads), 0, s, b);
                else hipLaunchKernelGGL((scatter_kernel<N, DOT, 0>), grid, dim3(kTokenThreads), 0, s, b);
            };
            if (b.dw) go(std::true_type{});
            else go(std::false_type{});
        });
    });
    return hipGetLastError();
}

hipError_t launch_collect_backward(const moe_dispatch_config& c, const uint16_t* dy, const uint16_t* rows, const int32_t* row_of, const float* topk_w, float p,
                                   const void* rng, uint16_t* drows, float* d_topk_w, hipStream_t s) {
    const Dropout drop = dropout_of(p, rng);
    return launch_scatter(c, {dy, rows, drows, c.d, topk_w != nullptr || drop.rng != nullptr, drop}, row_of, topk_w, d_topk_w, s);
}

hipError_t launch_dispatch(const moe_dispatch_config& c, const uint16_t* x, const int32_t* topk_idx, const float* topk_w, int32_t* counts, int32_t* offsets,
                           int32_t* row_of, int32_t* src_of, uint16_t* rows, int32_t* hist, hipStream_t s) {
    DispatchArgs a{x, topk_idx, topk_w, counts, offsets, row_of, src_of, rows, nullptr, c.T, c.d, c.k, c.E, c.first, c.capacity, 1, chunks_of(c), false};
    if ((long long)c.T * c.k > (rows ? kCountAllRows : kCountAll)) {
        a.hist = hist;
        a.summed = a.chunks > kSumInside;
        hipLaunchKernelGGL(count_chunks_kernel, dim3(a.chunks), dim3(kTokenThreads), 0, s, a);
        if (a.summed) hipLaunchKernelGGL(sum_chunks_kernel, dim3((c.E + kWave - 1) / kWave), dim3(kSumThreads), 0, s, a);
    }
    if (!rows || c.T == 0) {
        hipLaunchKernelGGL(tables_kernel, dim3(a.chunks > 0 ? a.chunks : 1), dim3(kTableThreads), 0, s, a);
        return hipGetLastError();
    }
    a.per = (c.T + 1023) / 1024;           // about a thousand workgroups, of a thousand slots at most
    if (a.per > kMostSlots / c.k) a.per = kMostSlots / c.k;
    const dim3 grid((unsigned)(((long long)c.T + a.per - 1) / a.per));
    const bool nt = passes_caches(c);
    by_slots(c.k, [&](auto n) {
        constexpr int N = decltype(n)::value;
        if (c.d <= kNarrow) hipLaunchKernelGGL((dispatch_kernel<1, false, true>), grid, dim3(kTokenThreads), 0, s, a);
        else if (nt) hipLaunchKernelGGL((dispatch_kernel<N, true, false>), grid, dim3(kTokenThreads), 0, s, a);
        else hipLaunchKernelGGL((dispatch_kernel<N, false, false>), grid, dim3(kTokenThreads), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_dropout(long long n, const uint16_t* x, const uint16_t* residual, float p, const void* rng, uint16_t* y, hipStream_t s) {
    const Dropout drop = dropout_of(p, rng);
    const long long groups = (n + 8ll * kTokenThreads - 1) / (8ll * kTokenThreads);
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192));
    if (residual) hipLaunchKernelGGL(dropout_kernel<true>, grid, dim3(kTokenThreads), 0, s, x, residual, y, n, drop);
    else hipLaunchKernelGGL(dropout_kernel<false>, grid, dim3(kTokenThreads), 0, s, x, residual, y, n, drop);
    return hipGetLastError();
}

}  // namespace moe

// Test hook (exported, not declared in include/moe.h): the launches that T tokens of width d take, on the host.  out[i] = {first token, workgroups}; returns how many there are, or -1 if
// that is more than `capacity`.
extern "C" __attribute__((visibility("default"))) int32_t moe_test_token_launches(int32_t T, int32_t d, int32_t capacity, int32_t* out) {
    moe::CollectArgs a{};
    a.T = T;
    a.d = d;
    int32_t n = 0;
    moe::by_launch(a, [&](const moe::CollectArgs& b, dim3 grid) {
        if (n < capacity) out[2 * n] = b.t0, out[2 * n + 1] = (int32_t)grid.x;
        ++n;
    });
    return n <= capacity ? n : -1;
}
