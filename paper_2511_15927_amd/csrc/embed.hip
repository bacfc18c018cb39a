// Token table: rows of it by id, and its gradient by sorted ids.
#include "model_ops.h"

namespace bm {

// out[row] = scale * table[id].  A copy: bound by the rows written (and those of the table that are read).  `lanes` threads to a row, 16
// bytes of the wider type a thread, so that a row's accesses are one run and a workgroup takes several short rows.  8 x 8192 rows of
// 2048: fp32 to bf16 65 us, bf16 50, fp32 96 (537 MB written, 5.6 TB/s); 16 x 32 rows 3.3 us, the launch and two loads one after the other.
struct EmbedArgs {
    const int64_t* ids;
    long long ids_sb, ids_st;
    const void* table;
    RowView out;
    unsigned rows, L;
    int d, vocab, lanes;
    float scale;
};
constexpr int kRowAhead = 2;   // pieces that a thread has in flight
template <typename TT, typename IO, int N, bool kPast>
__device__ __forceinline__ void embed_rows(const EmbedArgs& a)
{
    const unsigned per = 256 / a.lanes, lane = threadIdx.x % a.lanes;
    for (unsigned row = blockIdx.x * per + threadIdx.x / a.lanes; row < a.rows; row += gridDim.x * per) {
        const unsigned b = row / a.L, t = row - b * a.L;
        const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
        const bool known = id >= 0 && id < a.vocab;
        const typename TT::T* const from = static_cast<const typename TT::T*>(a.table) + (known ? id : 0) * a.d;
        typename IO::T* const to = static_cast<typename IO::T*>(a.out.p) + row_offset(a.out, b, t);
        for (int first = lane * N; first < a.d; first += a.lanes * N * kRowAhead) {
            Piece<TT, N> p[kRowAhead];
#pragma unroll
            for (int k = 0; k < kRowAhead; k++) p[k] = load_clamped<TT, N>(from, first + k * a.lanes * N, a.d);
#pragma unroll
            for (int k = 0; k < kRowAhead; k++) {
                const int at = first + k * a.lanes * N;
                settle(p[k], at, a.d, typename TT::T(0));
                float f[N];
#pragma unroll
                for (int i = 0; i < N; i++) f[i] = known ? a.scale * p[k][i] : 0.0f;
                store_piece_of<IO, kPast>(to, at, a.d, f);
            }
        }
    }
}
template <typename TT, typename IO, bool kPast>
__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs a)
{
    constexpr int N = kPieceOf<TT> < kPieceOf<IO> ? kPieceOf<TT> : kPieceOf<IO>;
    if (a.d >= N) embed_rows<TT, IO, N, kPast>(a);
    else embed_rows<TT, IO, 1, kPast>(a);
}

// ---- gradient ----
//
// dtable[v] = scale * sum of dout over the places with id v.  The places are sorted by (id, place); a sum then is over neighbours, in a
// fixed order, without atomics, and however many places share an id (in a noised sequence half of them are the mask token) they are
// summed by as many waves as they have slices.  Sorting: chunks of up to 4096 in a workgroup's registers, then merges of eight runs at a time, each
// place counting by binary search what precedes it in the other seven.  It moves 8 bytes a place and occupies few CUs for 10 to 20 us;
// meanwhile the other workgroups of its launches clear the table, half of it each, so that only rows of ids that occur are left to
// write.  (Looking up which rows are absent instead, after the sort, writes those rows once and not twice, but hides nothing.)
// What bounds it are the bytes, 412 MB of zeros, 135 MB of dout and 53 MB of rows at 8 x 4096 tokens of 2048 channels and 50304 ids: 126 us
// (sort 38 and merge 36 with the clearing in them, sums 46, join 7; 4.8 TB/s); for few tokens the four launches.

// Places sorted by one workgroup, 2048 or 4096 by the bits that the ids leave of a 32-bit key, four neighbouring ones a lane.
constexpr int kChunkBits = 11, kLargeChunkBits = 12, kSortKeys = 4;
constexpr int kMaxVocab = (1 << 21) - 1;
constexpr int kMaxWidth = 1 << 20;
constexpr int kMergeRuns = 8, kFewRuns = 4;
constexpr unsigned kMergeSamples = 256, kMergeWindow = 8;   // (a chunk: samples x window, or twice that)

struct EmbedClear {
    float* p;
    long long n;
    unsigned first_wg;   // of the launch; the workgroups before it sort
    int past;            // stores go past the caches
};
// Floats that a workgroup of kThreads clears.
constexpr int kClearFloats = 32768;
template <int kThreads, bool kPast>
__device__ __forceinline__ void clear_part_as(const EmbedClear& c)
{
    const long long from = (long long)(blockIdx.x - c.first_wg) * kClearFloats;
    const int n = (int)min((long long)kClearFloats, c.n - from);
    const float zero[4] = {};
    float* const p = c.p + from;
#pragma unroll 8
    for (int at = threadIdx.x * 4; at + 4 <= n; at += kThreads * 4) store_piece<IoF32, kPast>(p + at, zero);
    const int rest = n & ~3;
    if (rest + (int)threadIdx.x < n) p[rest + threadIdx.x] = 0.0f;
}
template <int kThreads>
__device__ __forceinline__ void clear_part(const EmbedClear& c)
{
    if (c.past) clear_part_as<kThreads, true>(c);
    else clear_part_as<kThreads, false>(c);
}

struct EmbedSortArgs {
    const int64_t* ids;
    long long ids_sb, ids_st;
    unsigned rows, L;
    int vocab;
    unsigned* id;     // sorted within each chunk; ids outside [0, vocab) are `vocab`
    unsigned* place;
    unsigned* n_spans;   // two counts, set to 0
    EmbedClear clear;
};
// The value of the lane whose number differs in bit kXor.
template <int kXor>
__device__ __forceinline__ unsigned from_lane(unsigned v)
{
#define BM_DPP(ctrl) (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, true)
    if constexpr (kXor == 1) {
        return BM_DPP(0xB1);    // quad_perm 1 0 3 2
    } else if constexpr (kXor == 2) {
        return BM_DPP(0x4E);    // quad_perm 2 3 0 1
    } else if constexpr (kXor == 4) {
        v = BM_DPP(0x141);      // row_half_mirror: differs in bits 0 to 2
        return BM_DPP(0x1B);    // quad_perm 3 2 1 0
    } else if constexpr (kXor == 8) {
        return BM_DPP(0x128);   // row_ror 8
    } else if constexpr (kXor == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
#undef BM_DPP
}
// One step of a bitonic sort of the workgroup's keys, four neighbours a lane: keys kStep apart are put in order, ascending where the bit
// kSize of their place is clear.
template <int kChunk, int kSize, int kStep>
__device__ __forceinline__ void sort_step(unsigned (&key)[kSortKeys], unsigned (*across)[kChunk])
{
    const unsigned first = threadIdx.x * kSortKeys;
    if constexpr (kStep < kSortKeys) {
#pragma unroll
        for (int k = 0; k < kSortKeys; k++)
            if (!(k & kStep)) {
                const unsigned x = key[k], y = key[k + kStep];
                const bool up = ((first + k) & kSize) == 0;
                key[k] = up ? min(x, y) : max(x, y);
                key[k + kStep] = up ? max(x, y) : min(x, y);
            }
    } else {
        const bool low = ((first & kStep) == 0) == ((first & kSize) == 0);   // (steps of a lane or more: the same for its four keys)
        unsigned other[kSortKeys];
        if constexpr (kStep < 64 * kSortKeys) {
#pragma unroll
            for (int k = 0; k < kSortKeys; k++) other[k] = from_lane<kStep / kSortKeys>(key[k]);
        } else {
            // two buffers in turn, so that one barrier a step is enough: the number of such steps before this one says which
            constexpr int kBlock = 64 * kSortKeys, kLevel = __builtin_ctz(kSize / kBlock), kWithin = __builtin_ctz(kSize / kStep) - 1;
            constexpr int kTurn = (kLevel * (kLevel - 1) / 2 + kWithin) & 1;
            unsigned* const b = across[kTurn];
#pragma unroll
            for (int k = 0; k < kSortKeys; k++) b[first + k] = key[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kSortKeys; k++) other[k] = b[(first ^ kStep) + k];
        }
#pragma unroll
        for (int k = 0; k < kSortKeys; k++) key[k] = low ? min(key[k], other[k]) : max(key[k], other[k]);
    }
}
template <int kChunk, int kSize, int kStep>
__device__ __forceinline__ void sort_steps(unsigned (&key)[kSortKeys], unsigned (*across)[kChunk])
{
    sort_step<kChunk, kSize, kStep>(key, across);
    if constexpr (kStep > 1) sort_steps<kChunk, kSize, kStep / 2>(key, across);
    else if constexpr (kSize < kChunk) sort_steps<kChunk, kSize * 2, kSize>(key, across);
}

template <int kBits>
__global__ __launch_bounds__((1 << kBits) / kSortKeys) void embed_sort_kernel(const EmbedSortArgs a)
{
    constexpr int kChunk = 1 << kBits, kSortThreads = kChunk / kSortKeys;
    if (blockIdx.x >= a.clear.first_wg) {
        clear_part<kSortThreads>(a.clear);
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) a.n_spans[threadIdx.x] = 0;
    __shared__ __align__(16) unsigned across[2][kChunk];
    const unsigned base = blockIdx.x << kBits, first = threadIdx.x * kSortKeys;
    unsigned key[kSortKeys];
#pragma unroll
    for (int k = 0; k < kSortKeys; k++) {
        key[k] = ~0u;
        const unsigned row = base + first + k;
        if (row < a.rows) {
            const unsigned b = row / a.L, t = row - b * a.L;
            const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
            key[k] = (unsigned)(id >= 0 && id < a.vocab ? id : a.vocab) << kBits | (first + k);
        }
    }
    sort_steps<kChunk, 2, 1>(key, across);
#pragma unroll
    for (int k = 0; k < kSortKeys; k++) {
        const unsigned row = base + first + k;
        if (row < a.rows) {
            a.id[row] = key[k] >> kBits;
            a.place[row] = base + (key[k] & (kChunk - 1));
        }
    }
}

// Runs of `run` sorted places each, kRuns of them merged into one.
struct EmbedMergeArgs {
    const unsigned *id, *place;
    unsigned *to_id, *to_place;
    unsigned rows, run;
    EmbedClear clear;
};
template <int kRuns>
__global__ __launch_bounds__(256) void embed_merge_kernel(const EmbedMergeArgs a)
{
    if (blockIdx.x >= a.clear.first_wg) {
        clear_part<256>(a.clear);
        return;
    }
    // (a run's places are whole workgroups)
    __shared__ unsigned sample[kRuns * kMergeSamples];
    const unsigned run = a.run, r = blockIdx.x * 256 / run, first = r / kRuns * kRuns;
#pragma unroll
    for (int q = 0; q < kRuns; q++) {
        const unsigned long long at = (unsigned long long)(first + q) * run + (threadIdx.x + 1) * (run / kMergeSamples) - 1;
        sample[q * kMergeSamples + threadIdx.x] = a.id[at < a.rows ? at : 0];   // (beyond the list: not looked at)
    }
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    const unsigned id = i < a.rows ? a.id[i] : 0, place = i < a.rows ? a.place[i] : 0;
    __syncthreads();
    if (i >= a.rows) return;
    unsigned below[kRuns], len[kRuns];
#pragma unroll
    for (int q = 0; q < kRuns; q++) {
        const unsigned long long start = (unsigned long long)(first + q) * run;
        len[q] = first + q == r || start >= a.rows ? 0u : min(run, a.rows - (unsigned)start);
        below[q] = 0;
    }
    // the last of every 256th part of each run, in shared memory, gives the first eight bits of a place
    const unsigned part = run / kMergeSamples;
    const auto precedes = [&](int q, unsigned other) { return first + q < r ? other <= id : other < id; };   // (equal ids keep the order of their places)
#pragma unroll
    for (unsigned step = kMergeSamples / 2; step > 0; step /= 2) {
#pragma unroll
        for (int q = 0; q < kRuns; q++) {
            const unsigned other = sample[q * kMergeSamples + below[q] + step - 1];
            if ((below[q] + step) * part <= len[q] && precedes(q, other)) below[q] += step;
        }
    }
#pragma unroll
    for (int q = 0; q < kRuns; q++) {   // (255 parts at most so far)
        const unsigned other = sample[q * kMergeSamples + below[q]];
        if ((below[q] + 1) * part <= len[q] && precedes(q, other)) below[q]++;
        below[q] *= part;
    }
    // long runs: halves of a part, all runs' loads of a step in flight at once, down to eight places; those are looked at together
    for (unsigned step = part / 2; step >= kMergeWindow; step /= 2) {
        unsigned other[kRuns];
#pragma unroll
        for (int q = 0; q < kRuns; q++) other[q] = a.id[below[q] + step <= len[q] ? (first + q) * run + below[q] + step - 1 : i];
#pragma unroll
        for (int q = 0; q < kRuns; q++)
            if (below[q] + step <= len[q] && precedes(q, other[q])) below[q] += step;
    }
    unsigned window[kRuns][kMergeWindow];
#pragma unroll
    for (int q = 0; q < kRuns; q++) {   // (the lists are as long as whole chunks; a run that is not there: this place's own)
        const unsigned at = below[q] < len[q] ? (first + q) * run + below[q] : i & ~(kMergeWindow - 1u);
        __builtin_memcpy(window[q], __builtin_assume_aligned(a.id + at, 16), sizeof window[q]);
    }
#pragma unroll
    for (int q = 0; q < kRuns; q++) {
        unsigned count = 0;
#pragma unroll
        for (unsigned k = 0; k < kMergeWindow; k++) count += below[q] + k < len[q] && precedes(q, window[q][k]);
        below[q] += count;
    }
    unsigned to = first * run + (i - r * run);
#pragma unroll
    for (int q = 0; q < kRuns; q++) to += below[q];
    a.to_id[to] = id;
    a.to_place[to] = place;
}

// A wave sums a slice of neighbouring places over 512 channels, eight a lane.  A run of one id that lies within the slice gives its row of
// dtable; what a run that goes on into the next slice, or came from the one before, adds up to here is left in the slice's two slots
// for embed_join_kernel, and such a run is put on a list (whose order says nothing about any sum).
constexpr int kMaxSlice = 64;
constexpr int kSumCols = 512;
constexpr unsigned kShortSpan = 16;   // slices that a short run reaches into at most
struct EmbedSpan {
    unsigned slice, last, id;   // the run of `id` starts in `slice` and ends in `last`
};
struct EmbedSumArgs {
    const unsigned *id, *place;
    RowView dout;
    float* dtable;
    float* slots;   // [slices][2][d]: of the run that came into the slice, of the one that starts in it and goes on
    unsigned* n_spans;
    EmbedSpan* span;   // lists of runs that span slices: short ones, and after `slices` entries long ones
    unsigned rows, L;
    int d, vocab, slice, col_blocks;
    unsigned slices;
    float scale;
};
// A lane's eight of the wave's 512 channels from `col`: two groups of four.  N 8: neighbours, one load of bf16; what is stored goes through
// pairs of lanes, so that each pair writes 32 bytes side by side.  N 4: one group in each half, two loads of fp32.  N 1: rows of
// fewer channels than that, one a lane.
template <typename IO, int N, bool kPast>
__device__ __forceinline__ void sum_slice(const EmbedSumArgs& a, unsigned slice, int block, int lane)
{
    constexpr int kLoads = N == 8 ? 1 : N == 4 ? 2 : 1;   // pieces a row and lane
    const int col = block * kSumCols + lane * N;
    const unsigned i0 = slice * a.slice, n = min((unsigned)a.slice, a.rows - i0);
    // a lane's place of the slice: its id and where its row of dout starts
    unsigned my_id = ~0u;
    long long my_row = 0;
    if ((unsigned)lane < n) {
        my_id = a.id[i0 + lane];
        const unsigned place = a.place[i0 + lane], b = place / a.L;
        my_row = row_offset(a.dout, b, place - b * a.L);
    }
    const unsigned before = i0 > 0 ? a.id[i0 - 1] : ~0u, after = i0 + n < a.rows ? a.id[i0 + n] : ~0u;
    const typename IO::T* const dout = static_cast<const typename IO::T*>(a.dout.p);
    unsigned cur = __builtin_amdgcn_readlane(my_id, 0);
    bool came = cur == before;
    float acc[kLoads][N] = {};
    auto flush = [&](bool goes_on) {
        if (cur >= (unsigned)a.vocab) return;
        const bool slot = came || goes_on;
        float* const to = slot ? a.slots + ((long long)slice * 2 + (came ? 0 : 1)) * a.d : a.dtable + (long long)cur * a.d;
        const float scale = slot ? 1.0f : a.scale;
        if constexpr (N == 8) {
            float x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float lo = scale * acc[0][i], hi = scale * acc[0][4 + i];
                const float other = __uint_as_float(from_lane<1>(__float_as_uint(lane & 1 ? lo : hi)));
                x[i] = lane & 1 ? other : lo;
                y[i] = lane & 1 ? hi : other;
            }
            const int at = block * kSumCols + (lane & ~1) * 8 + (lane & 1) * 4;
            store_piece_of<IoF32>(to, at, a.d, x);
            store_piece_of<IoF32>(to, at + 8, a.d, y);
        } else {
#pragma unroll
            for (int h = 0; h < kLoads; h++) {
                float x[N];
#pragma unroll
                for (int i = 0; i < N; i++) x[i] = scale * acc[h][i];
                store_piece_of<IoF32>(to, col + h * 64 * N, a.d, x);
            }
        }
    };
    constexpr int kAhead = 8;
    for (unsigned e = 0; e < n; e += kAhead) {
        Piece<IO, N> p[kAhead][kLoads];
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            const unsigned at = min(e + j, n - 1);   // (past the slice: its last row again, not added)
            const unsigned lo = __builtin_amdgcn_readlane((unsigned)my_row, at), hi = __builtin_amdgcn_readlane((unsigned)(my_row >> 32), at);
            const typename IO::T* const row = dout + (long long)((unsigned long long)hi << 32 | lo);
#pragma unroll
            for (int h = 0; h < kLoads; h++) p[j][h] = load_clamped<IO, N, kPast>(row, col + h * 64 * N, a.d);
        }
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            if (e + j < n) {
                const unsigned id = __builtin_amdgcn_readlane(my_id, e + j);
                if (id != cur) {
                    flush(false);
                    cur = id;
                    came = false;
#pragma unroll
                    for (int h = 0; h < kLoads; h++)
#pragma unroll
                        for (int i = 0; i < N; i++) acc[h][i] = 0.0f;
                }
#pragma unroll
                for (int h = 0; h < kLoads; h++) {
                    settle(p[j][h], col + h * 64 * N, a.d, typename IO::T(0));
#pragma unroll
                    for (int i = 0; i < N; i++) acc[h][i] += p[j][h][i];
                }
            }
        }
    }
    flush(cur == after);
    if (block == 0 && !came && cur == after && cur < (unsigned)a.vocab) {
        // the last slice that the run goes into: 64 slices are looked at together
        unsigned last = slice + 1;
        for (unsigned range = a.slices - last; range > 1;) {
            const unsigned step = (range + 63) / 64, at = last + lane * step;
            const bool there = lane * step < range;
            const unsigned count = __popcll(__ballot(there && a.id[there ? (unsigned long long)at * a.slice : i0] == cur));   // (the first lanes)
            range = min(step, range - (count - 1) * step);
            last += (count - 1) * step;
        }
        const bool long_run = last > slice + kShortSpan;
        if (lane == 0) a.span[(long_run ? a.slices : 0) + atomicAdd(a.n_spans + long_run, 1u)] = EmbedSpan{slice, last, cur};
    }
}
template <typename IO, bool kPast>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedSumArgs a)
{
    const unsigned w = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64), slice = w / a.col_blocks;
    if (slice >= a.slices) return;
    const int block = w - slice * a.col_blocks, lane = threadIdx.x % 64;
    if (a.d >= kPieceOf<IO>) sum_slice<IO, kPieceOf<IO>, kPast>(a, slice, block, lane);
    else sum_slice<IO, 1, kPast>(a, slice, block, lane);
}

// The rows of runs that span slices.  256 channels of a short run: a wave adds up its slots.  Of a long run: a workgroup, each of its
// groups of lanes a share of the slots.
constexpr int kJoinWaves = 16, kJoinCols = 256, kShortGroups = 256, kLongGroups = 32;
struct EmbedJoinArgs {
    const float* slots;
    float* dtable;
    const unsigned* n_spans;
    const EmbedSpan* span;
    unsigned slices, short_groups, lanes;   // lanes: that a long run's slot takes, fewer where rows are short
    int d, col_blocks;
    float scale;
};
// kAt a time, N neighbours of each slot from `col`: slots first, first + step, ... up to last.
template <int N, int kAt>
__device__ __forceinline__ void add_slots(float (&acc)[N], const EmbedJoinArgs& a, int col, unsigned first, unsigned last, unsigned step)
{
    for (unsigned s = first; s <= last; s += kAt * step) {
        Piece<IoF32, N> p[kAt];
#pragma unroll
        for (int j = 0; j < kAt; j++) p[j] = load_clamped<IoF32, N>(a.slots + (long long)min(s + j * step, last) * 2 * a.d, col, a.d);
#pragma unroll
        for (int j = 0; j < kAt; j++) {
            settle(p[j], col, a.d, 0.0f);
            if (s + j * step <= last)
#pragma unroll
                for (int i = 0; i < N; i++) acc[i] += p[j][i];
        }
    }
}
template <int N>
__device__ __forceinline__ void join_runs(const EmbedJoinArgs& a)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const auto start = [&](float (&acc)[N], const EmbedSpan& span, int col) {   // what the run's first slice left
        const Piece<IoF32, N> p = load_piece_of<IoF32, N>(a.slots + ((long long)span.slice * 2 + 1) * a.d, col, a.d, 0.0f);
#pragma unroll
        for (int i = 0; i < N; i++) acc[i] = p[i];
    };
    if (blockIdx.x < a.short_groups) {
        const unsigned n = a.n_spans[0];
        for (unsigned long long w = blockIdx.x * kJoinWaves + wave; w < (unsigned long long)n * a.col_blocks; w += a.short_groups * kJoinWaves) {
            const unsigned k = w / a.col_blocks;
            const EmbedSpan span = a.span[k];
            const int col = (int)(w - (unsigned long long)k * a.col_blocks) * kJoinCols + lane * N;
            float acc[N];
            start(acc, span, col);
            add_slots<N, 4>(acc, a, col, span.slice + 1, span.last, 1);
#pragma unroll
            for (int i = 0; i < N; i++) acc[i] *= a.scale;
            store_piece_of<IoF32>(a.dtable + (long long)span.id * a.d, col, a.d, acc);
        }
        return;
    }
    __shared__ float sum[kJoinWaves * 64 * N];
    const unsigned n = a.n_spans[1], first = blockIdx.x - a.short_groups;
    for (unsigned long long w = first; w < (unsigned long long)n * a.col_blocks; w += gridDim.x - a.short_groups) {
        const unsigned k = w / a.col_blocks;
        const EmbedSpan span = a.span[a.slices + k];
        const int block = (int)(w - (unsigned long long)k * a.col_blocks), col = block * kJoinCols + (int)(threadIdx.x % a.lanes) * N;
        float acc[N] = {};
        if (threadIdx.x < a.lanes) start(acc, span, col);
        add_slots<N, 8>(acc, a, col, span.slice + 1 + threadIdx.x / a.lanes, span.last, 64 * kJoinWaves / a.lanes);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; i++) sum[threadIdx.x * N + i] = acc[i];
        __syncthreads();
        const int width = a.lanes * N, c = block * kJoinCols + threadIdx.x;
        if ((int)threadIdx.x < width && c < a.d) {
            float f = 0.0f;
#pragma unroll 16
            for (int i = threadIdx.x; i < kJoinWaves * 64 * N; i += width) f += sum[i];
            a.dtable[(long long)span.id * a.d + c] = a.scale * f;
        }
    }
}
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(const EmbedJoinArgs a)
{
    if (a.d >= 4) join_runs<4>(a);
    else join_runs<1>(a);
}

namespace {

int check_embed(const bimamba_embed_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_embed_desc) || d->d_model < 1 || d->vocab < 1 || !std::isfinite(d->scale)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->table_dtype) || !known_dtype(d->io_dtype) || d->vocab > kMaxVocab || d->d_model > kMaxWidth) return BIMAMBA_ERR_UNSUPPORTED;
    return BIMAMBA_OK;
}

// Places to a slice: as many as 64, fewer where that leaves the chip short of two waves per SIMD.
struct EmbedPlan {
    unsigned rows, chunk, chunks, slices;
    int slice, col_blocks;
    size_t list, slots, total;   // bytes of one list of ids or places, of the slots, and of the workspace
};
EmbedPlan plan_embed(const bimamba_embed_desc* d)
{
    EmbedPlan p{};
    p.rows = (unsigned)((long long)d->batch * d->seqlen);
    // (up to 4096 places then need no merge: 3711 of them, 740 channels, 38 -> 34 us in all)
    p.chunk = d->vocab < 1 << (32 - kLargeChunkBits) && p.rows > 1u << kChunkBits ? 1u << kLargeChunkBits : 1u << kChunkBits;
    p.chunks = (p.rows + p.chunk - 1) / p.chunk;
    p.col_blocks = (d->d_model + kSumCols - 1) / kSumCols;
    p.slice = kMaxSlice;
    while (p.slice > 8 && (long long)(p.rows / p.slice) * p.col_blocks < 8 * cu_count()) p.slice /= 2;
    p.slices = (p.rows + p.slice - 1) / p.slice;
    p.list = (size_t)p.chunks * p.chunk * 4;   // (whole chunks: a merge reads eight places at a time)
    p.slots = ((size_t)p.slices * 2 * d->d_model * sizeof(float) + 15) / 16 * 16;
    p.total = 4 * p.list + p.slots + 16 + 2 * (size_t)p.slices * sizeof(EmbedSpan);   // (and the lists of runs that span slices, after their lengths)
    return p;
}

template <typename TT, typename IO>
void launch_embed(const EmbedArgs& a, unsigned grid, hipStream_t st)
{
    if (past_caches((double)a.rows * a.d * (sizeof(typename TT::T) + sizeof(typename IO::T)))) hipLaunchKernelGGL((embed_kernel<TT, IO, true>), dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((embed_kernel<TT, IO, false>), dim3(grid), dim3(256), 0, st, a);
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

int bimamba_embed(const bimamba_embed_desc* d, const bimamba_tokens* tokens, const void* table, const bimamba_tensor* out,
                  void* hip_stream)
{
    int rc = check_embed(d);
    if (rc) return rc;
    if (!tokens || !out) return BIMAMBA_ERR_NULL_POINTER;
    if (d->batch == 0 || d->seqlen == 0) return BIMAMBA_OK;
    if (!table) return BIMAMBA_ERR_NULL_POINTER;
    Bytes ids, to;
    if ((rc = check_tokens(tokens, d->batch, d->seqlen, &ids))) return rc;
    if ((rc = check_view(out, d->batch, d->seqlen, d->d_model, d->io_dtype, true, &to))) return rc;
    if (!aligned_to(table, dtype_bytes(d->table_dtype))) return BIMAMBA_ERR_MISALIGNED;
    if (meet(to, ids) || meet(to, bytes_of(table, (long long)d->vocab * d->d_model, dtype_bytes(d->table_dtype)))) return BIMAMBA_ERR_ALIAS;
    EmbedArgs a{tokens->ptr, tokens->stride_batch, tokens->stride_token, table, row_view(out), (unsigned)(d->batch * (long long)d->seqlen),
                (unsigned)d->seqlen, d->d_model, d->vocab, 256, d->scale};
    const bool tb = d->table_dtype == BIMAMBA_BF16, ib = d->io_dtype == BIMAMBA_BF16;
    while (a.lanes > 1 && (a.lanes / 2) * (tb && ib ? 8 : 4) * kRowAhead >= d->d_model) a.lanes /= 2;
    const unsigned per = 256 / a.lanes, want = (a.rows + per - 1) / per, grid = want < 1u << 20 ? want : 1u << 20;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    if (tb && ib) launch_embed<IoBF16, IoBF16>(a, grid, st);
    else if (tb) launch_embed<IoBF16, IoF32>(a, grid, st);
    else if (ib) launch_embed<IoF32, IoBF16>(a, grid, st);
    else launch_embed<IoF32, IoF32>(a, grid, st);
    return launches.status();
}

size_t bimamba_embed_bwd_workspace_bytes(const bimamba_embed_desc* d) { return check_embed(d) ? 0 : plan_embed(d).total; }

int bimamba_embed_bwd(const bimamba_embed_desc* d, const bimamba_tokens* tokens, const bimamba_tensor* dout, float* dtable,
                      void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_embed(d);
    if (rc) return rc;
    if (!tokens || !dout || !dtable) return BIMAMBA_ERR_NULL_POINTER;
    if (!aligned_to(dtable, 4)) return BIMAMBA_ERR_MISALIGNED;
    const EmbedPlan p = plan_embed(d);
    if ((unsigned long long)p.slices * p.col_blocks >= 1u << 25) return BIMAMBA_ERR_UNSUPPORTED;   // (a grid holds 2^32 threads)
    const Bytes table = bytes_of(dtable, (long long)d->vocab * d->d_model, 4);
    if (p.rows > 0) {
        Bytes ids, from;
        if ((rc = check_tokens(tokens, d->batch, d->seqlen, &ids))) return rc;
        if ((rc = check_view(dout, d->batch, d->seqlen, d->d_model, d->io_dtype, false, &from))) return rc;
        if ((rc = check_workspace(workspace, workspace_bytes, p.total))) return rc;
        const Bytes ws = bytes_of(workspace, p.total, 1);
        if (meet(table, ids) || meet(table, from) || meet(table, ws) || meet(ws, ids) || meet(ws, from)) return BIMAMBA_ERR_ALIAS;
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    char* const ws = static_cast<char*>(workspace);
    unsigned *id = reinterpret_cast<unsigned*>(ws), *place = reinterpret_cast<unsigned*>(ws + p.list);
    unsigned *to_id = reinterpret_cast<unsigned*>(ws + 2 * p.list), *to_place = reinterpret_cast<unsigned*>(ws + 3 * p.list);
    float* const slots = reinterpret_cast<float*>(ws + 4 * p.list);
    unsigned* const n_spans = reinterpret_cast<unsigned*>(ws + 4 * p.list + p.slots);
    EmbedSpan* const span = reinterpret_cast<EmbedSpan*>(ws + 4 * p.list + p.slots + 16);
    // the table is cleared beside the sort and, where there is one, the first merge
    const long long all = (long long)d->vocab * d->d_model;
    const bool past = past_caches(4.0 * all + (double)p.rows * d->d_model * dtype_bytes(d->io_dtype));   // (8 x 4096 tokens, 412 MB: 143 -> 128 us)
    const long long half = p.rows > p.chunk ? (all / 2 + kClearFloats - 1) / kClearFloats * kClearFloats : all, early = half < all ? half : all;
    const auto wgs = [](long long n) { return (unsigned)((n + kClearFloats - 1) / kClearFloats); };
    const EmbedSortArgs sa{tokens->ptr, tokens->stride_batch, tokens->stride_token, p.rows, (unsigned)d->seqlen, d->vocab, id, place,
                           n_spans, EmbedClear{dtable, early, p.chunks, past}};
    if (p.chunk == 1u << kChunkBits) hipLaunchKernelGGL(embed_sort_kernel<kChunkBits>, dim3(p.chunks + wgs(early)), dim3(p.chunk / kSortKeys), 0, st, sa);
    else hipLaunchKernelGGL(embed_sort_kernel<kLargeChunkBits>, dim3(p.chunks + wgs(early)), dim3(p.chunk / kSortKeys), 0, st, sa);
    if (p.rows == 0) return launches.status();
    long long left = all - early;
    for (unsigned long long run = p.chunk; run < p.rows; run *= kMergeRuns) {
        const unsigned merge_wgs = (p.rows + 255) / 256;
        const EmbedMergeArgs ma{id, place, to_id, to_place, p.rows, (unsigned)run, EmbedClear{dtable + early, left, merge_wgs, past}};
        // (few runs, less to look at: 16384 places, four runs 7.7 us; 32768, eight runs 11.8)
        if (run * kFewRuns >= p.rows) hipLaunchKernelGGL(embed_merge_kernel<kFewRuns>, dim3(merge_wgs + wgs(left)), dim3(256), 0, st, ma);
        else hipLaunchKernelGGL(embed_merge_kernel<kMergeRuns>, dim3(merge_wgs + wgs(left)), dim3(256), 0, st, ma);
        left = 0;
        unsigned* const i = id;
        unsigned* const q = place;
        id = to_id, place = to_place;
        to_id = i, to_place = q;
    }
    const EmbedSumArgs a{id, place, row_view(dout), dtable, slots, n_spans, span, p.rows, (unsigned)d->seqlen, d->d_model, d->vocab, p.slice, p.col_blocks,
                         p.slices, d->scale};
    const unsigned sum_wgs = (unsigned)(((unsigned long long)p.slices * p.col_blocks + 3) / 4);
    const bool bf16 = d->io_dtype == BIMAMBA_BF16;
    if (bf16 && past) hipLaunchKernelGGL((embed_sum_kernel<IoBF16, true>), dim3(sum_wgs), dim3(256), 0, st, a);
    else if (bf16) hipLaunchKernelGGL((embed_sum_kernel<IoBF16, false>), dim3(sum_wgs), dim3(256), 0, st, a);
    else if (past) hipLaunchKernelGGL((embed_sum_kernel<IoF32, true>), dim3(sum_wgs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((embed_sum_kernel<IoF32, false>), dim3(sum_wgs), dim3(256), 0, st, a);
    if (p.slices > 1) {
        EmbedJoinArgs ja{slots, dtable, n_spans, span, p.slices, kShortGroups, 64, d->d_model, 0, d->scale};
        while (ja.lanes > 4 && ja.lanes / 2 * 4 >= (unsigned)d->d_model) ja.lanes /= 2;
        ja.col_blocks = (d->d_model + kJoinCols - 1) / kJoinCols;
        const unsigned long long most = ((unsigned long long)p.slices * ja.col_blocks + kJoinWaves - 1) / kJoinWaves;
        if (ja.short_groups > most) ja.short_groups = (unsigned)most;
        const unsigned long_groups = p.slices - 1 > kShortSpan ? kLongGroups : 1;   // (one: for none)
        hipLaunchKernelGGL(embed_join_kernel, dim3(ja.short_groups + long_groups), dim3(64 * kJoinWaves), 0, st, ja);
    }
    return launches.status();
}

}  // extern "C"
