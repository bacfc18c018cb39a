// Token table: rows of it by id, and its gradient by sorted ids.
#include "model_ops.h"

namespace bm {

// out[row] = scale * table[id].  A copy: bound by the rows written (and those of the table that are read).  `lanes` threads to a row,
// eight elements a thread, so that a row's accesses are one run and a workgroup takes several short rows.
struct EmbedArgs {
    const int64_t* ids;
    long long ids_sb, ids_st;
    const void* table;
    RowView out;
    unsigned rows, L;
    int d, vocab, lanes;
    float scale;
};
template <typename TT, typename IO>
__global__ __launch_bounds__(256) void embed_kernel(const EmbedArgs a)
{
    const unsigned per = 256 / a.lanes, lane = threadIdx.x % a.lanes;
    for (unsigned row = blockIdx.x * per + threadIdx.x / a.lanes; row < a.rows; row += gridDim.x * per) {
        const unsigned b = row / a.L, t = row - b * a.L;
        const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
        const bool known = id >= 0 && id < a.vocab;
        const typename TT::T* const from = static_cast<const typename TT::T*>(a.table) + (known ? id : 0) * a.d;
        typename IO::T* const to = static_cast<typename IO::T*>(a.out.p) + row_offset(a.out, b, t);
        for (int at = lane * kPiece; at < a.d; at += a.lanes * kPiece) {
            float f[kPiece] = {};
            if (known) {
                const Piece<TT> p = load_piece_of<TT>(from, at, a.d, typename TT::T(0));
#pragma unroll
                for (int i = 0; i < kPiece; i++) f[i] = a.scale * p[i];
            }
            store_piece_of<IO>(to, at, a.d, f);
        }
    }
}

// ---- gradient ----
//
// dtable[v] = scale * sum of dout over the places with id v.  The places are sorted by (id, place); a sum then is over neighbours, in a
// fixed order, without atomics, and however many places share an id (in a noised sequence half of them are the mask token) they are
// summed by as many waves as they have slices.  Sorting: chunks of 2048 in shared memory, then merges of sixteen runs at a time, each
// place counting by binary search what precedes it in the other fifteen.  It moves 8 bytes a place; the rows of dout and of dtable
// are what bounds the call.

constexpr int kChunkBits = 11, kChunk = 1 << kChunkBits;   // places sorted by one workgroup: 21 + 11 bits of a key
constexpr int kMaxVocab = (1 << 21) - 1;
constexpr int kMaxWidth = 1 << 20;
constexpr int kMergeRuns = 16;

struct EmbedSortArgs {
    const int64_t* ids;
    long long ids_sb, ids_st;
    unsigned rows, L;
    int vocab;
    unsigned* id;     // sorted within each chunk; ids outside [0, vocab) are `vocab`
    unsigned* place;
};
__global__ __launch_bounds__(1024) void embed_sort_kernel(const EmbedSortArgs a)
{
    __shared__ unsigned key[kChunk];
    const unsigned base = blockIdx.x << kChunkBits;
    for (unsigned i = threadIdx.x; i < kChunk; i += 1024) {
        unsigned k = ~0u;
        const unsigned row = base + i;
        if (row < a.rows) {
            const unsigned b = row / a.L, t = row - b * a.L;
            const long long id = a.ids[b * a.ids_sb + t * a.ids_st];
            k = (unsigned)(id >= 0 && id < a.vocab ? id : a.vocab) << kChunkBits | i;
        }
        key[i] = k;
    }
    for (int size = 2; size <= kChunk; size *= 2) {
        for (int step = size / 2; step > 0; step /= 2) {
            __syncthreads();
            const int i = 2 * threadIdx.x - (threadIdx.x & (step - 1)), j = i + step;   // a pair `step` apart
            const unsigned x = key[i], y = key[j];
            if ((x > y) == ((i & size) == 0)) {
                key[i] = y;
                key[j] = x;
            }
        }
    }
    __syncthreads();
    for (unsigned i = threadIdx.x; i < kChunk && base + i < a.rows; i += 1024) {
        const unsigned k = key[i];
        a.id[base + i] = k >> kChunkBits;
        a.place[base + i] = base + (k & (kChunk - 1));
    }
}

// Runs of `run` sorted places each, sixteen of them merged into one.
struct EmbedMergeArgs {
    const unsigned *id, *place;
    unsigned *to_id, *to_place;
    unsigned rows, run;
};
__global__ __launch_bounds__(256) void embed_merge_kernel(const EmbedMergeArgs a)
{
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i >= a.rows) return;
    const unsigned run = a.run, r = i / run, first = r / kMergeRuns * kMergeRuns;
    const unsigned id = a.id[i], place = a.place[i];
    unsigned below[kMergeRuns], len[kMergeRuns];
#pragma unroll
    for (int q = 0; q < kMergeRuns; q++) {
        const unsigned long long start = (unsigned long long)(first + q) * run;
        len[q] = first + q == r || start >= a.rows ? 0u : min(run, a.rows - (unsigned)start);
        below[q] = 0;
    }
    for (unsigned step = run; step > 0; step /= 2) {
#pragma unroll
        for (int q = 0; q < kMergeRuns; q++) {
            const unsigned at = below[q] + step;
            if (at <= len[q]) {
                const unsigned other = a.id[(first + q) * run + at - 1];
                if (first + q < r ? other <= id : other < id) below[q] = at;   // (equal ids keep the order of their places)
            }
        }
    }
    unsigned to = first * run + (i - r * run);
#pragma unroll
    for (int q = 0; q < kMergeRuns; q++) to += below[q];
    a.to_id[to] = id;
    a.to_place[to] = place;
}

// A wave sums a slice of neighbouring places over 512 channels, eight a lane.  A run of one id that lies within the slice gives its
// row of dtable; what a run that goes on into the next slice, or came from the one before, adds up to here is left in the slice's two
// slots for embed_join_kernel.  Other workgroups of the launch write the rows whose ids do not occur.
constexpr int kMaxSlice = 64;
constexpr int kSumCols = 64 * kPiece;
constexpr int kZeroRows = 8;   // rows of the table that a wave looks up and, where they are absent, clears
struct EmbedSumArgs {
    const unsigned *id, *place;
    RowView dout;
    float* dtable;
    float* slots;   // [slices][2][d]: of the run that came into the slice, of the one that starts in it and goes on
    unsigned rows, L;
    int d, vocab, slice, col_blocks;
    unsigned slices, sum_wgs;
    float scale;
};
template <typename IO>
__global__ __launch_bounds__(256) void embed_sum_kernel(const EmbedSumArgs a)
{
    const int lane = threadIdx.x % 64;
    const unsigned wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    if (blockIdx.x >= a.sum_wgs) {   // rows of ids that do not occur
        const unsigned v0 = ((blockIdx.x - a.sum_wgs) * 4 + wave) * kZeroRows;
        bool absent = false;
        if (lane < kZeroRows && v0 + lane < (unsigned)a.vocab) {
            const unsigned v = v0 + lane;
            unsigned lo = 0, hi = a.rows;
            while (lo < hi) {
                const unsigned mid = lo + (hi - lo) / 2;
                if (a.id[mid] < v) lo = mid + 1;
                else hi = mid;
            }
            absent = lo >= a.rows || a.id[lo] != v;
        }
        unsigned long long todo = __ballot(absent);
        const float zero[kPiece] = {};
        while (todo) {
            const int k = __builtin_ctzll(todo);
            todo &= todo - 1;
            float* const row = a.dtable + (long long)(v0 + k) * a.d;
            for (int at = lane * kPiece; at < a.d; at += kSumCols) store_piece_of<IoF32>(row, at, a.d, zero);
        }
        return;
    }
    const unsigned w = blockIdx.x * 4 + wave, slice = w / a.col_blocks;
    if (slice >= a.slices) return;
    const int col = (w - slice * a.col_blocks) * kSumCols + lane * kPiece;
    const bool mine = col < a.d;
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
    float acc[kPiece] = {};
    auto flush = [&](bool goes_on) {
        if (cur >= (unsigned)a.vocab || !mine) return;
        if (came || goes_on) {
            store_piece_of<IoF32>(a.slots + ((long long)slice * 2 + (came ? 0 : 1)) * a.d, col, a.d, acc);
        } else {
            float f[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; i++) f[i] = a.scale * acc[i];
            store_piece_of<IoF32>(a.dtable + (long long)cur * a.d, col, a.d, f);
        }
    };
    constexpr int kAhead = 8;
    for (unsigned e = 0; e < n; e += kAhead) {
        Piece<IO> p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; j++) {
            const unsigned lo = __builtin_amdgcn_readlane((unsigned)my_row, e + j), hi = __builtin_amdgcn_readlane((unsigned)(my_row >> 32), e + j);
            if (e + j < n && mine)
                p[j] = load_piece_of<IO>(dout + (long long)((unsigned long long)hi << 32 | lo), col, a.d, typename IO::T(0));
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
                    for (int i = 0; i < kPiece; i++) acc[i] = 0.0f;
                }
                if (mine)
#pragma unroll
                    for (int i = 0; i < kPiece; i++) acc[i] += p[j][i];
            }
        }
    }
    flush(cur == after);
}

// The rows of runs that span slices: the workgroup of the slice in which a run starts adds up its slots, 256 channels at a time, the
// waves a share of the slices each.
constexpr int kJoinWaves = 8, kJoinCols = 256;
struct EmbedJoinArgs {
    const unsigned* id;
    const float* slots;
    float* dtable;
    unsigned rows;
    int d, vocab, slice;
    float scale;
};
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(const EmbedJoinArgs a)
{
    const unsigned slice = blockIdx.x, i0 = slice * a.slice, i1 = i0 + a.slice;   // (the last slice has no workgroup)
    const unsigned v = a.id[i1 - 1];
    if (v >= (unsigned)a.vocab || a.id[i1] != v || (a.id[i0] == v && i0 > 0 && a.id[i0 - 1] == v)) return;
    unsigned lo = i1 + 1, hi = a.rows;   // where the run ends
    while (lo < hi) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (a.id[mid] == v) lo = mid + 1;
        else hi = mid;
    }
    const unsigned last = (lo - 1) / a.slice;   // slices slice + 1 .. last came into it
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, col = blockIdx.y * kJoinCols + lane * 4;
    __shared__ float sum[kJoinWaves][kJoinCols];
    float acc[4] = {};
    auto add = [&](const float* row) {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (col + i < a.d) acc[i] += row[col + i];
    };
    if (wave == 0) add(a.slots + ((long long)slice * 2 + 1) * a.d);
#pragma unroll 4
    for (unsigned s = slice + 1 + wave; s <= last; s += kJoinWaves) add(a.slots + (long long)s * 2 * a.d);
#pragma unroll
    for (int i = 0; i < 4; i++) sum[wave][lane * 4 + i] = acc[i];
    __syncthreads();
    const int c = blockIdx.y * kJoinCols + threadIdx.x;
    if (threadIdx.x < kJoinCols && c < a.d) {
        float f = 0.0f;
#pragma unroll
        for (int k = 0; k < kJoinWaves; k++) f += sum[k][threadIdx.x];
        a.dtable[(long long)v * a.d + c] = a.scale * f;
    }
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
    unsigned rows, chunks, slices;
    int slice, col_blocks;
    size_t list, total;   // bytes of one list of ids or places, and of the workspace
};
EmbedPlan plan_embed(const bimamba_embed_desc* d)
{
    EmbedPlan p{};
    p.rows = (unsigned)((long long)d->batch * d->seqlen);
    p.chunks = (p.rows + kChunk - 1) / kChunk;
    p.col_blocks = (d->d_model + kSumCols - 1) / kSumCols;
    p.slice = kMaxSlice;
    while (p.slice > 8 && (long long)(p.rows / p.slice) * p.col_blocks < 8 * cu_count()) p.slice /= 2;
    p.slices = (p.rows + p.slice - 1) / p.slice;
    p.list = ((size_t)p.rows * 4 + 15) / 16 * 16;
    p.total = 4 * p.list + (size_t)p.slices * 2 * d->d_model * sizeof(float);
    return p;
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
    while (a.lanes > 1 && (a.lanes / 2) * kPiece >= d->d_model) a.lanes /= 2;
    const unsigned per = 256 / a.lanes, want = (a.rows + per - 1) / per, grid = want < 1u << 20 ? want : 1u << 20;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const bool tb = d->table_dtype == BIMAMBA_BF16, ib = d->io_dtype == BIMAMBA_BF16;
    if (tb && ib) hipLaunchKernelGGL((embed_kernel<IoBF16, IoBF16>), dim3(grid), dim3(256), 0, st, a);
    else if (tb) hipLaunchKernelGGL((embed_kernel<IoBF16, IoF32>), dim3(grid), dim3(256), 0, st, a);
    else if (ib) hipLaunchKernelGGL((embed_kernel<IoF32, IoBF16>), dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((embed_kernel<IoF32, IoF32>), dim3(grid), dim3(256), 0, st, a);
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
    if (p.rows > 0) {
        const EmbedSortArgs sa{tokens->ptr, tokens->stride_batch, tokens->stride_token, p.rows, (unsigned)d->seqlen, d->vocab, id, place};
        hipLaunchKernelGGL(embed_sort_kernel, dim3(p.chunks), dim3(1024), 0, st, sa);
        for (unsigned long long run = kChunk; run < p.rows; run *= kMergeRuns) {
            const EmbedMergeArgs ma{id, place, to_id, to_place, p.rows, (unsigned)run};
            hipLaunchKernelGGL(embed_merge_kernel, dim3((p.rows + 255) / 256), dim3(256), 0, st, ma);
            unsigned* const i = id;
            unsigned* const q = place;
            id = to_id, place = to_place;
            to_id = i, to_place = q;
        }
    }
    EmbedSumArgs a{id, place, row_view(dout), dtable, slots, p.rows, (unsigned)d->seqlen, d->d_model, d->vocab, p.slice, p.col_blocks,
                   p.slices, 0, d->scale};
    a.sum_wgs = (unsigned)(((unsigned long long)p.slices * p.col_blocks + 3) / 4);
    const unsigned zero_wgs = (d->vocab + 4 * kZeroRows - 1) / (4 * kZeroRows);
    if (d->io_dtype == BIMAMBA_BF16) hipLaunchKernelGGL(embed_sum_kernel<IoBF16>, dim3(a.sum_wgs + zero_wgs), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(embed_sum_kernel<IoF32>, dim3(a.sum_wgs + zero_wgs), dim3(256), 0, st, a);
    if (p.slices > 1) {
        const EmbedJoinArgs ja{id, slots, dtable, p.rows, d->d_model, d->vocab, p.slice, d->scale};
        hipLaunchKernelGGL(embed_join_kernel, dim3(p.slices - 1, (d->d_model + kJoinCols - 1) / kJoinCols), dim3(64 * kJoinWaves), 0, st, ja);
    }
    return launches.status();
}

}  // extern "C"
