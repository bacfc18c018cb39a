// The gated linear recurrence h = a h + u, channel by channel, in either direction along the sequence, and its gradients.
#include "slot_sums.h"

namespace bm {

// The sequence is cut into pieces of kW waves times kT tokens, a workgroup each for the channels of one wave, whose tokens stay in
// registers.  A wave first runs its tokens from a state of zero, which gives the state E that they add and the factor P that they put
// on what enters; the pairs are exchanged through shared memory, folded onto the state that enters the piece, and the tokens run again
// from there: the activations are read once.  (32 tokens of a wave stay as they were read, and their gates are formed twice: what they take in
// registers is half.)  What enters a piece comes from those before it.  A workgroup publishes its piece's (P, E),
// looks back, and then publishes what leaves the piece as (0, h).  A pair is one word of 64
// bits, written and read whole, so that no fence is needed; a word of ones says that nothing is there yet.  Pieces are handed out by a
// counter in the order of the walk, all channels and sequences of a step before the next step: a workgroup waits for pieces of its own channels
// only, which were handed out before its own to workgroups that run, so every wait ends.
//
// Everything is in fp32: a, u, the states; y is rounded once.  1 - a is formed beside a from the same exponential, not as a difference, so
// that it loses no digits where a is near 1.  fp32 activations: with e = exp(-|v|), sigmoid(|v|) = 1 - e / (1 + e) and sigmoid(-|v|) = e / (1 + e),
// a off by half a unit of its last place where it is near 1.  bf16 ones: with e = exp(-v), a = 1 / (1 + e) and 1 - a = e a, without a
// selection; a is off by two units there (the sum's and the reciprocal's, 2^-23).  With the 2^-24 that a step's own rounding may take, a channel that
// remembers M tokens turns that into 1.5 M 2^-23 of its state at most, where half a unit of a would leave 0.75 M 2^-23: at 1000 tokens a twentieth of
// what y loses as it is rounded, at 20000 as much; the states, dh_in and dbias are not rounded and carry it.  (8 x 8192 tokens of 4096 channels:
// 356 us with selections, 332 without; fp32 the same.)
constexpr int kKeep = BIMAMBA_RECURRENCE_KEEP;   // steps between two kept states

enum Gate { kLog, kSigmoid };

struct RecurArgs {
    RowView x, g, add, y;    // add.p null: none
    RowView dy, dx, dg;      // gradients
    const float* bias;       // null: 0
    const int64_t* lengths;  // null: L
    const float* enter;      // [batch][d], null: 0; the state before the first step (gradients: that of the state after the last)
    float* leave;            // [batch][d] or null: the state after the last (gradients: that of the state before the first)
    float* states;           // [batch][ceil(L / kKeep)][d] or null
    float* dbias;            // [batch * pieces][d] or null
    unsigned long long* slots;   // [batch][pieces][d], with several pieces: what enters the first one, then what each leaves, in the order of the walk
    unsigned* ticket;        // [kXcds]
    int L, d, pieces, reverse, batch, queues, look;   // look: pieces before its own that a workgroup looks at
};

// The tokens that the steps of a walk take.
struct Places {
    int len, reverse;
    __device__ __forceinline__ Places(const RecurArgs& a, int b) : len(a.L), reverse(a.reverse)
    {
        if (a.lengths) len = __builtin_amdgcn_readfirstlane((int)max(0ll, min((long long)a.L, (long long)a.lengths[b])));
    }
    // One that may be read for step s: beyond the end some other one.
    __device__ __forceinline__ int readable(int s) const
    {
        const int k = min(s, len - 1);
        return max(0, reverse ? len - 1 - k : k);
    }
    // The one that step s writes.
    __device__ __forceinline__ int written(int s) const { return reverse && s < len ? len - 1 - s : s; }
};

// A lane's channels of the rows that a wave's steps take.  Lanes beyond the last channels take those along with their owner, and store nothing;
// where the last lane's channels would reach beyond the row it takes the row's last ones and stores those that are its own.
// kWhole: every lane owns all of its channels and all steps lie within the sequence; nothing is clamped, and there is no branch.  Rows are
// wave-uniform pointers and lanes unsigned 32-bit offsets, kept narrow where they are used, so that the accesses take a scalar base:
// sixteen tokens of two tensors in flight otherwise hold sixty registers of addresses.
template <typename IO, int kC, int kT, bool kPast, bool kWhole>
struct Steps {
    typedef typename IO::T T;
    typedef Piece<IO, kC> Raw;
    const Places& places;
    int b, s0, L, at, own;   // own: the first channel that is the lane's, at + kC if none is
    unsigned off;            // bytes
    __device__ __forceinline__ Steps(const Places& places, int b, int s0, int L, int first, int lane, int d)
        : places(places), b(b), s0(s0), L(L), at(min(first + lane * kC, d - kC)), own(min(first + lane * kC, d)), off((unsigned)at * (unsigned)sizeof(T)) {}
    static __device__ __forceinline__ char* row(const RowView& v, int b, int t) { return static_cast<char*>(v.p) + row_offset(v, b, t) * (long long)sizeof(T); }
    __device__ __forceinline__ unsigned narrow() const
    {
        unsigned o = off;
        asm volatile("" : "+v"(o));
        return o;
    }
    __device__ __forceinline__ bool inside(int i) const { return kWhole || s0 + i < places.len; }
    __device__ __forceinline__ bool idle() const { return !kWhole && s0 >= places.len; }   // (the whole wave)
    __device__ __forceinline__ void load(Raw (&r)[kT], const RowView& v) const
    {
        const char* p = row(v, b, places.readable(s0));
        const long long step = (places.reverse ? -v.st : v.st) * (long long)sizeof(T);
#pragma unroll
        for (int i = 0; i < kT; i++) {
            if constexpr (!kWhole) p = row(v, b, places.readable(s0 + i));
            r[i] = load_piece<IO, kC, kPast>(reinterpret_cast<const T*>(p + narrow()));
            if constexpr (kWhole) p += step;
        }
    }
    __device__ __forceinline__ void store(const RowView& v, int i, const float (&f)[kC]) const
    {
        if constexpr (kWhole) {
            store_piece<IO, kPast>(reinterpret_cast<T*>(row(v, b, places.written(s0)) + (places.reverse ? -i : i) * v.st * (long long)sizeof(T) + narrow()), f);
        } else if (s0 + i < L) {
            T* const to = reinterpret_cast<T*>(row(v, b, places.written(s0 + i)) + narrow());
            if (own == at) store_piece<IO, kPast>(to, f);
            else if (kC == 2 && own == at + 1) to[kC - 1] = io_value<IO>(f[kC - 1]);
        }
    }
    __device__ __forceinline__ void load_params(float (&f)[kC], const float* p) const
    {
#pragma unroll
        for (int j = 0; j < kC; j++) f[j] = 0.0f;
        if (p) {
            const Piece<IoF32, kC> v = load_piece<IoF32, kC>(p + at);
#pragma unroll
            for (int j = 0; j < kC; j++) f[j] = v[j];
        }
    }
    __device__ __forceinline__ bool has(int j) const { return kWhole || at + j >= own; }
    __device__ __forceinline__ void store_params(float* p, const float (&f)[kC]) const
    {
#pragma unroll
        for (int j = 0; j < kC; j++)
            if (has(j)) p[at + j] = f[j];
    }
};

// a, and for a sigmoid gate 1 - a, for a log gate the factor that da / dg is (a, or 0 where g > 0 was cut).
template <typename IO, int kGate>
__device__ __forceinline__ void gate_of(float g, float bias, float& a, float& q)
{
    if constexpr (kGate == kSigmoid && sizeof(typename IO::T) == 4) {
        const float v = g + bias, e = __builtin_amdgcn_exp2f(-kLog2e * fabsf(v)), low = e * __builtin_amdgcn_rcpf(1.0f + e), high = 1.0f - low;
        a = v > 0.0f ? high : low;
        q = v > 0.0f ? low : high;
    } else if constexpr (kGate == kSigmoid) {   // (e is cut at 2^126, and a at 2^-126; a NaN stays one)
        const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(-kLog2e * (g + bias), 126.0f));
        a = __builtin_amdgcn_rcpf(1.0f + e);
        q = e * a;
    } else {
        a = __builtin_amdgcn_exp2f(kLog2e * (g > 0.0f ? 0.0f : g));   // (a NaN stays one)
        q = g > 0.0f ? 0.0f : a;
    }
}

// Keeps a raw piece as it is: what was made of it before is not kept in registers for later.
template <typename Raw>
__device__ __forceinline__ void hold(Raw& r)
{
    if constexpr (sizeof r == 4) {
        unsigned bits = __builtin_bit_cast(unsigned, r);
        asm volatile("" : "+v"(bits));
        r = __builtin_bit_cast(Raw, bits);
    }
}

template <int kC>
struct Link {
    float p[kC], e[kC];
};

constexpr unsigned kNothing = ~0u;
__device__ __forceinline__ void publish(unsigned long long* to, float p, float e)
{
    const unsigned hi = p != p ? 0x7fc00000u : __float_as_uint(p);
    __hip_atomic_store(to, (unsigned long long)hi << 32 | __float_as_uint(e), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// What a link makes of the state that enters it.  (One that nothing passes ends there, so that the word (0, h) stands for the state h itself.)
__device__ __forceinline__ float through(float p, float e, float h) { return p == 0.0f ? e : p * h + e; }

// Waits for the words of pieces that lie `stride` slots apart, of `end`'s for those of the state that it leaves, a lane for those of its own channels:
// one that the tile before owns (a last tile of a single channel takes it along) is another chain's, which no order of the queues ties to this
// one's pieces, and nothing is made of it.  (Were the words not to come, which would be a mistake here, the walk would go on with a NaN, not stand still.)
template <int kC, int kN, typename At>
__device__ __forceinline__ void await(Link<kC> (&links)[kN], int n, const unsigned long long* from, long long stride, int end, const At& steps)
{
    unsigned long long word[kN][kC];
    const auto there = [&](int k, int j) {
        const unsigned hi = (unsigned)(word[k][j] >> 32);
        return !steps.has(j) || (min(k, n - 1) == end ? hi == 0 : hi != kNothing);
    };
    int tries = 1 << 22;
    for (;;) {
        bool all = true;
#pragma unroll
        for (int k = 0; k < kN; k++)
#pragma unroll
            for (int j = 0; j < kC; j++)
                word[k][j] = __hip_atomic_load(from + min(k, n - 1) * stride + steps.at + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int k = 0; k < kN; k++)
#pragma unroll
            for (int j = 0; j < kC; j++) all &= there(k, j);
        if (__all(all) || --tries == 0) break;
        __builtin_amdgcn_s_sleep(1);
    }
#pragma unroll
    for (int k = 0; k < kN; k++)
#pragma unroll
        for (int j = 0; j < kC; j++) {
            links[k].p[j] = there(k, j) ? __uint_as_float((unsigned)(word[k][j] >> 32)) : 0.0f;
            links[k].e[j] = there(k, j) ? __uint_as_float((unsigned)word[k][j]) : __builtin_nanf("");
        }
}
// Chains (the channels of a wave, of one sequence) are handed out from one queue or from eight, each a run of neighbouring ones for the
// workgroups of one XCD (and, when that is empty, for the others): the first chain of queue q.  (A launch has fewer than 2^26 chains.)
constexpr unsigned kXcds = 8;
__device__ __forceinline__ unsigned queue_of(unsigned chains, unsigned q, unsigned queues) { return queues == 1 ? q * chains : q * chains / kXcds; }
// Before the pieces: nothing is there but what enters the first one.  (The state that enters is read here only: it may be the one that the
// last piece replaces.)
constexpr int kCleared = 8;   // words of a thread
__global__ __launch_bounds__(256) void recur_clear_kernel(const RecurArgs r)
{
    const long long n = (long long)r.pieces * r.d, first = blockIdx.x * (256ll * kCleared) + threadIdx.x;
    const int b = blockIdx.y;
    if (first < kXcds && b == 0) r.ticket[first] = 0;
#pragma unroll
    for (int k = 0; k < kCleared; k++) {
        const long long i = first + k * 256;
        if (i < n) r.slots[b * n + i] = i < r.d ? (r.enter ? __float_as_uint(r.enter[(long long)b * r.d + i]) : 0) : ~0ull;
    }
}

// What a workgroup's waves share.
template <int kC, int kT, int kW>
struct PieceShared {
    static constexpr bool kOnly = kT * kW <= 32;        // (short sequences: there is one piece)
    static constexpr int kMostLooked = kW < 8 ? 8 : kW;   // pieces before its own that a workgroup looks at
    Link<kC> part[kW][64], seen[kOnly ? 1 : kMostLooked][64];
    float before[kW][kC][64];                      // (gradients)
    int turn;
    unsigned chain;
};
// Which piece it is, of how many channels and where.
struct PieceOf {
    int turn, b, first;
    template <typename Shared>
    __device__ __forceinline__ PieceOf(const RecurArgs& r, int channels, Shared& sh)
    {
        const unsigned tiles = (r.d + channels - 1) / channels, chains = tiles * r.batch;
        unsigned chain = blockIdx.x;
        turn = 0;
        if (!Shared::kOnly && r.pieces > 1) {
            if (threadIdx.x == 0) {
                // (there are as many pieces as workgroups, and each takes one: a queue that is not empty is found)
                constexpr int kXccId = 20 | 3 << 11;   // (hardware register XCC_ID, four bits)
                unsigned q = r.queues > 1 ? __builtin_amdgcn_s_getreg(kXccId) % kXcds : 0, n, of;
                for (;; q = q + 1 == (unsigned)r.queues ? 0 : q + 1) {
                    of = queue_of(chains, q + 1, r.queues) - queue_of(chains, q, r.queues);
                    n = atomicAdd(r.ticket + q, 1u);
                    if (n < of * r.pieces) break;
                }
                sh.turn = n / of;
                sh.chain = queue_of(chains, q, r.queues) + n % of;
            }
            __syncthreads();
            turn = __builtin_amdgcn_readfirstlane(sh.turn), chain = __builtin_amdgcn_readfirstlane(sh.chain);
        }
        b = chain / tiles;
        first = chain % tiles * channels;
    }
};
// What enters the piece: the state that the r.look-th piece before it leaves, and the links of those between, folded in the order of the walk.
// The state that a piece leaves is this same fold, one link further, so its bits do not depend on how far back the look went or on
// which of the words were there.  A sequence of one piece has read what enters it beside its tokens, before a barrier: the same memory may
// be written at its end.
template <int kC, int kT, int kW, typename At>
__device__ __forceinline__ void look_back(float (&carry)[kC], const At& steps, const RecurArgs& r, const PieceOf& piece, int w, int lane, PieceShared<kC, kT, kW>& sh)
{
    const unsigned long long* const slots = r.slots + (long long)piece.b * r.pieces * r.d;
    const int look = min(r.look, piece.turn + 1);   // (slot `turn` is what the piece before this one leaves, slot 0 what enters the first one)
    constexpr int kN = PieceShared<kC, kT, kW>::kMostLooked / kW;   // of one wave
    const int n = (look - w + kW - 1) / kW;
    if (n > 0) {
        Link<kC> links[kN];
        await<kC, kN>(links, n, slots + (long long)(piece.turn - w) * r.d, -(long long)kW * r.d, (look - 1) % kW == w ? n - 1 : -1, steps);
#pragma unroll
        for (int k = 0; k < kN; k++)
            if (k < n) sh.seen[w + k * kW][lane] = links[k];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kC; j++) carry[j] = sh.seen[look - 1][lane].e[j];
#pragma unroll 1
    for (int k = look - 2; k >= 0; k--) {
        const Link<kC> link = sh.seen[k][lane];
#pragma unroll
        for (int j = 0; j < kC; j++) carry[j] = through(link.p[j], link.e[j], carry[j]);
    }
}
// What the piece leaves: to those after it, or, from the last one, to the caller.
template <int kC, typename At>
__device__ __forceinline__ void leave(const Link<kC>& all, const float (&carry)[kC], const At& steps, const RecurArgs& r, const PieceOf& piece)
{
    float end[kC];
#pragma unroll
    for (int j = 0; j < kC; j++) end[j] = through(all.p[j], all.e[j], carry[j]);
    if (piece.turn == r.pieces - 1) {
        if (r.leave) steps.store_params(r.leave + (long long)piece.b * r.d, end);
        return;
    }
    unsigned long long* const to = r.slots + ((long long)piece.b * r.pieces + piece.turn + 1) * r.d + steps.at;
#pragma unroll
    for (int j = 0; j < kC; j++)
        if (steps.has(j)) publish(to + j, 0.0f, end[j]);
}
template <int kC, typename At>
__device__ __forceinline__ void announce(const Link<kC>& all, const At& steps, const RecurArgs& r, const PieceOf& piece)
{
    if (r.look < 2 || piece.turn == 0 || piece.turn == r.pieces - 1) return;   // (the first one's end is known at once, the last one's no piece asks for)
    unsigned long long* const to = r.slots + ((long long)piece.b * r.pieces + piece.turn + 1) * r.d + steps.at;
#pragma unroll
    for (int j = 0; j < kC; j++)
        if (steps.has(j)) publish(to + j, all.p[j], all.e[j]);
}

template <typename IO, int kGate, int kC, int kT, int kW, bool kPast, bool kWhole>
__device__ __forceinline__ void recur_piece(const RecurArgs& r, const Places& places, const PieceOf& piece, int w, int lane, PieceShared<kC, kT, kW>& sh)
{
    const int s0 = (piece.turn * kW + w) * kT;
    const Steps<IO, kC, kT, kPast, kWhole> steps(places, piece.b, s0, r.L, piece.first, lane, r.d);
    Piece<IO, kC> x[kT], g[kT], add[kT];
    constexpr bool kAgain = kT > 16;
    float bias[kC] = {}, a[kAgain ? 1 : kT][kC], u[kAgain ? 1 : kT][kC], h[kC];
    const auto gates = [&](int i, float (&at)[kC], float (&ut)[kC]) {
#pragma unroll
        for (int j = 0; j < kC; j++) {
            float q;
            gate_of<IO, kGate>(g[i][j], bias[j], at[j], q);
            ut[j] = kGate == kSigmoid ? q * x[i][j] : x[i][j];
            if (!steps.inside(i)) at[j] = 1.0f, ut[j] = 0.0f;
        }
    };
    if (r.pieces == 1) steps.load_params(h, r.enter ? r.enter + (long long)piece.b * r.d : nullptr);
#pragma unroll
    for (int i = 0; i < kT; i++) add[i] = Piece<IO, kC>{};
    Link<kC> mine;
#pragma unroll
    for (int j = 0; j < kC; j++) mine.p[j] = 1.0f, mine.e[j] = 0.0f;
    if (steps.idle()) {
#pragma unroll
        for (int i = 0; i < kT; i++) {
            x[i] = g[i] = Piece<IO, kC>{};
            if constexpr (!kAgain)
#pragma unroll
                for (int j = 0; j < kC; j++) a[i][j] = 1.0f, u[i][j] = 0.0f;
        }
    } else {
        steps.load(x, r.x);
        steps.load(g, r.g);
        steps.load_params(bias, r.bias);
        if (!kAgain && r.add.p) steps.load(add, r.add);
#pragma unroll
        for (int i = 0; i < kT; i++) {
            float at[kC], ut[kC];
            gates(i, at, ut);
#pragma unroll
            for (int j = 0; j < kC; j++) {
                if constexpr (!kAgain) a[i][j] = at[j], u[i][j] = ut[j];
                mine.e[j] = at[j] * mine.e[j] + ut[j];
                mine.p[j] *= at[j];
            }
        }
        if (kAgain && r.add.p) steps.load(add, r.add);
    }
    Link<kC> all = mine, before;
    if constexpr (kW > 1) {
        sh.part[w][lane] = mine;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kC; j++) all.p[j] = before.p[j] = 1.0f, all.e[j] = before.e[j] = 0.0f;
#pragma unroll 2
        for (int k = 0; k < kW; k++) {   // (all of it unrolled: the links' registers cost a quarter of the waves)
            const Link<kC> link = sh.part[k][lane];
#pragma unroll
            for (int j = 0; j < kC; j++) {
                all.e[j] = link.p[j] * all.e[j] + link.e[j];
                all.p[j] *= link.p[j];
                if (k + 1 == w) before.p[j] = all.p[j], before.e[j] = all.e[j];
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < kC; j++) before.p[j] = 1.0f, before.e[j] = 0.0f;
    }
    if (!PieceShared<kC, kT, kW>::kOnly && w == 0) announce(all, steps, r, piece);
    if (!PieceShared<kC, kT, kW>::kOnly && r.pieces > 1) look_back<kC, kT, kW>(h, steps, r, piece, w, lane, sh);
    if (w == 0) leave(all, h, steps, r, piece);
#pragma unroll
    for (int j = 0; j < kC; j++) h[j] = before.p[j] * h[j] + before.e[j];
    if (r.states && s0 % kKeep == 0 && s0 < r.L) steps.store_params(r.states + ((long long)piece.b * ((r.L + kKeep - 1) / kKeep) + s0 / kKeep) * r.d, h);
#pragma unroll
    for (int i = 0; i < kT; i++) {
        float f[kC], at[kC], ut[kC];
        if constexpr (kAgain) {
            hold(x[i]), hold(g[i]);
            gates(i, at, ut);
        }
#pragma unroll
        for (int j = 0; j < kC; j++) {
            if constexpr (!kAgain) at[j] = a[i][j], ut[j] = u[i][j];
            h[j] = at[j] * h[j] + ut[j];
            f[j] = steps.inside(i) ? h[j] + add[i][j] : 0.0f;
        }
        steps.store(r.y, i, f);
    }
}
template <typename IO, int kGate, int kC, int kT, int kW, bool kPast>
__global__ __launch_bounds__(64 * kW, kT * kW > 32 ? 4 : 1) void recur_kernel(const RecurArgs r)
{
    __shared__ PieceShared<kC, kT, kW> sh;
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const PieceOf piece(r, 64 * kC, sh);
    const Places places(r, piece.b);
    if (piece.first + 64 * kC <= r.d && (piece.turn + 1) * kW * kT <= places.len) recur_piece<IO, kGate, kC, kT, kW, kPast, true>(r, places, piece, w, lane, sh);
    else recur_piece<IO, kGate, kC, kT, kW, kPast, false>(r, places, piece, w, lane, sh);
}

// dh_s = dy_s + a_{s+1} dh_{s+1} is the same recurrence from the other end: what enters a wave's tokens is q = a dh of the token after
// them, and they leave Q + P q; the pieces go from the last one to the first.  The states in front of a wave's tokens are folded from the kept
// one before them, so that x, g and dy are read once and dx and dg written.  Between the two runs a token keeps a, the factors that dx
// and dg are of dh, and dy as it was read, not the states.  dbias is summed by lane over the wave's tokens, then over the waves and the
// pieces in a fixed order.
template <typename IO, int kGate, int kC, int kT, int kW, bool kPast, bool kWhole>
__device__ __forceinline__ void recur_bwd_piece(const RecurArgs& r, const Places& places, const PieceOf& piece, int w, int lane, PieceShared<kC, kT, kW>& sh)
{
    const int seg = r.pieces - 1 - piece.turn, base = seg * kW * kT, s0 = base + w * kT, kept = (r.L + kKeep - 1) / kKeep, first = min(s0 / kKeep, kept - 1);
    const Steps<IO, kC, kT, kPast, kWhole> steps(places, piece.b, s0, r.L, piece.first, lane, r.d);
    Piece<IO, kC> x[kT], g[kT], dy[kT];
    float bias[kC], dbias[kC], h[kC], dh[kC], a[kT][kC], q[kT][kC];
    steps.load_params(h, r.states + ((long long)piece.b * kept + first) * r.d);
    if (r.pieces == 1) steps.load_params(dh, r.enter ? r.enter + (long long)piece.b * r.d : nullptr);
    Link<kC> mine;   // (P, Q)
    float e[kC];
#pragma unroll
    for (int j = 0; j < kC; j++) mine.p[j] = 1.0f, mine.e[j] = e[j] = dbias[j] = 0.0f;
    if (steps.idle()) {
#pragma unroll
        for (int i = 0; i < kT; i++) {
            x[i] = dy[i] = Piece<IO, kC>{};
#pragma unroll
            for (int j = 0; j < kC; j++) a[i][j] = 1.0f, q[i][j] = 0.0f;
        }
    } else {
        steps.load(x, r.x);
        steps.load(g, r.g);
        steps.load(dy, r.dy);
        steps.load_params(bias, r.bias);
#pragma unroll
        for (int i = 0; i < kT; i++)
#pragma unroll
            for (int j = 0; j < kC; j++) {
                gate_of<IO, kGate>(g[i][j], bias[j], a[i][j], q[i][j]);
                if (!steps.inside(i)) a[i][j] = 1.0f, q[i][j] = 0.0f, x[i].v[j] = dy[i].v[j] = 0;
                e[j] = a[i][j] * e[j] + (kGate == kSigmoid ? q[i][j] * x[i][j] : x[i][j]);
                mine.p[j] *= a[i][j];
            }
#pragma unroll
        for (int i = kT - 1; i >= 0; i--)
#pragma unroll
            for (int j = 0; j < kC; j++) mine.e[j] = a[i][j] * (dy[i][j] + mine.e[j]);
    }
    Link<kC> all = mine, behind;
#pragma unroll
    for (int j = 0; j < kC; j++) behind.p[j] = 1.0f, behind.e[j] = 0.0f;
    if constexpr (kW > 1) {
        sh.part[w][lane] = mine;
#pragma unroll
        for (int j = 0; j < kC; j++) sh.before[w][j][lane] = e[j];
        __syncthreads();
        const int w0 = (first * kKeep - base) / kT;   // (the wave that starts at the kept state)
#pragma unroll 1
        for (int k = w0; k < w; k++) {
            const Link<kC> link = sh.part[k][lane];
#pragma unroll
            for (int j = 0; j < kC; j++) h[j] = link.p[j] * h[j] + sh.before[k][j][lane];
        }
#pragma unroll
        for (int j = 0; j < kC; j++) all.p[j] = 1.0f, all.e[j] = 0.0f;
#pragma unroll 2
        for (int k = kW - 1; k >= 0; k--) {
            const Link<kC> link = sh.part[k][lane];
#pragma unroll
            for (int j = 0; j < kC; j++) {
                all.e[j] = link.p[j] * all.e[j] + link.e[j];
                all.p[j] *= link.p[j];
                if (k - 1 == w) behind.p[j] = all.p[j], behind.e[j] = all.e[j];
            }
        }
    }
    if (!PieceShared<kC, kT, kW>::kOnly && w == 0) announce(all, steps, r, piece);
    float c[kT][kC];
#pragma unroll
    for (int i = 0; i < kT; i++) {
        hold(x[i]);
#pragma unroll
        for (int j = 0; j < kC; j++) {
            const float v = x[i][j];
            c[i][j] = kGate == kSigmoid ? q[i][j] * (h[j] - v) * a[i][j] : h[j] * q[i][j];
            h[j] = a[i][j] * h[j] + (kGate == kSigmoid ? q[i][j] * v : v);
        }
    }
    if (!PieceShared<kC, kT, kW>::kOnly && r.pieces > 1) look_back<kC, kT, kW>(dh, steps, r, piece, w, lane, sh);
    if (w == 0) leave(all, dh, steps, r, piece);
#pragma unroll
    for (int j = 0; j < kC; j++) dh[j] = behind.p[j] * dh[j] + behind.e[j];
#pragma unroll
    for (int i = kT - 1; i >= 0; i--) {
        float dx[kC], dg[kC];
        hold(dy[i]);
#pragma unroll
        for (int j = 0; j < kC; j++) {
            const float d = dy[i][j] + dh[j];
            dh[j] = a[i][j] * d;
            dx[j] = kGate == kSigmoid ? d * q[i][j] : d;
            dg[j] = d * c[i][j];
            if (!steps.inside(i)) dx[j] = dg[j] = 0.0f;
            dbias[j] += dg[j];
        }
        steps.store(r.dx, i, dx);
        steps.store(r.dg, i, dg);
    }
    if (r.dbias) {
        if constexpr (kW > 1) {
            __syncthreads();   // (`before` has been read)
#pragma unroll
            for (int j = 0; j < kC; j++) sh.before[w][j][lane] = dbias[j];
            __syncthreads();
            if (w == 0)
#pragma unroll
                for (int k = 1; k < kW; k++)
#pragma unroll
                    for (int j = 0; j < kC; j++) dbias[j] += sh.before[k][j][lane];
        }
        if (w == 0) steps.store_params(r.dbias + ((long long)piece.b * r.pieces + seg) * r.d, dbias);
    }
}
template <typename IO, int kGate, int kC, int kT, int kW, bool kPast>
__global__ __launch_bounds__(64 * kW) void recur_bwd_kernel(const RecurArgs r)
{
    __shared__ PieceShared<kC, kT, kW> sh;
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const PieceOf piece(r, 64 * kC, sh);
    const Places places(r, piece.b);
    if (piece.first + 64 * kC <= r.d && (r.pieces - piece.turn) * kW * kT <= places.len) recur_bwd_piece<IO, kGate, kC, kT, kW, kPast, true>(r, places, piece, w, lane, sh);
    else recur_bwd_piece<IO, kGate, kC, kT, kW, kPast, false>(r, places, piece, w, lane, sh);
}

namespace {

constexpr int kMaxWidth = 65536;

int check_recurrence(const bimamba_recurrence_desc* d)
{
    if (!d) return BIMAMBA_ERR_NULL_POINTER;
    if (d->struct_size != sizeof(bimamba_recurrence_desc) || d->d_inner < 1 || (d->reverse != 0 && d->reverse != 1)) return BIMAMBA_ERR_BAD_SHAPE;
    if (const int rc = check_rows(d->batch, d->seqlen)) return rc;
    if (!known_dtype(d->io_dtype) || (d->gate != BIMAMBA_GATE_LOG && d->gate != BIMAMBA_GATE_SIGMOID)) return BIMAMBA_ERR_UNSUPPORTED;
    if (d->batch > 65535 || d->d_inner > kMaxWidth) return BIMAMBA_ERR_UNSUPPORTED;
    // (a grid holds 2^32 threads: up to four tokens are one wave's, else a piece has four waves for each 64 steps at most)
    const long long pieces = ((d->seqlen + 63ll) / 64) * d->batch * ((d->d_inner + 63) / 64);
    return d->seqlen > 4 && pieces >= 1ll << 23 ? BIMAMBA_ERR_UNSUPPORTED : BIMAMBA_OK;
}

// Tokens of a wave in a piece, waves of one, channels of a lane.  Short sequences go in one piece of as few registers as hold it, since its
// time is that of one load after the other (16 x 32 tokens of 4096 channels: 8 x 4 4.4 us, 16 x 8 9.2).  Two channels a lane take fewer
// instructions for a byte, one spreads the work over twice the waves.  What there is to spread is the number n of pieces of 128 tokens of 64
// channels, what has to follow one another a chain's pieces.
//   Forward (bf16, us, one channel and two): 64 x 128 tokens of 2048 channels (n = 2048) 21.3, 22.5; 128 x 128 of 4096 (8192) 83, 75.
// Up to 256 tokens in one piece, of 16 x 16 with one channel and of 32 x 8 with two: 4 x 200 of 4096 (512) 10.5, 14.5; 16 x 256 of 2048 (1024) 15.1,
// 14.1; 32 x 256 (2048) 27.6, 23.2; in two of 16 x 8 64 x 256 of 4096 (8192) 97, in one 87; fp32 64 x 200 of 2048 79, 72.
// Longer ones with one channel in pieces of 16 x 16 and of 16 x 8, and with two of 16 x 8 and 32 x 8: 700 of 512 (48) 11.7, 8.6, 11.3, -; 2048 of 2048
// (512) 13.4, 17.5, 15.0, -; 8192 of 2048 (2048) 34.2, 39.4, 37.6, 39.0; 8 x 2048 of 4096 (8192) 116, 119, 102, 91; 8 x 4096 (16384) 216, -, 169, 172;
// 8 x 8192 with add -, -, 373, 379; 64 x 600 of 2048 (10240), whose last piece is not filled, 172, -, 120, 130; in few chains, 65536 of 512 (4096)
// 61, -, 117, 77; of 1024 122, -, 133, 109; of 2048 227, -, 185, 174; where a chain's pieces are most of it, 8192 of 64 (64) 13.5, 14.8; 4096 of 512
// (256) 11.9, 12.5; 2048 of 512 (128) 10.5, 9.3.
//   The gradients hold half as much again, so with two channels two workgroups of eight waves no longer fit a CU.  One channel 16 x 16 and 16 x 8,
// two channels 16 x 8 and 16 x 4: 700 of 512 15.3, 10.0, 13.2, 12.5; 2048 of 2048 16.7, 20.0, 17.9, 22.4; 8192 of 2048 46.9, 45.1, 48.4, 51.6;
// 8 x 2048 of 4096 170, 160, 161, 150; in few chains, 65536 of 512 98, 99, 116, 192, of 256 51, 77, 110, 179.  fp32 has one channel a lane:
// 4 x 8192 of 4096 16 x 16 544, 16 x 8 503, 16 x 4 506; forward 321, 302, 430.
struct RecurPlan {
    int tokens, waves, pieces;
    int channels;
    unsigned tiles;
};
RecurPlan plan_recurrence(const bimamba_recurrence_desc* d, bool back)
{
    RecurPlan p{};
    const int L = d->seqlen;
    const auto pieces = [&](int steps) { return (L + steps - 1) / steps; };
    const auto tiles = [&](int channels) { return (d->d_inner + 64 * channels - 1) / (64 * channels); };
    const long long cus = cu_count(), chains = (long long)tiles(1) * d->batch, n = chains * pieces(128);
    const bool some = n <= 8 * cus, one = back ? some || chains <= cus / 4 : L <= 128 ? some : L <= 256 ? n <= 2 * cus : some || chains <= cus / 32;
    p.channels = d->io_dtype == BIMAMBA_BF16 && d->d_inner > 64 && (L <= 64 || !one) ? 2 : 1;
    p.tiles = tiles(p.channels);
    const bool far = n > cus || pieces(128) >= 32;
    const bool words = p.channels == 2 || d->io_dtype == BIMAMBA_F32;   // (of 32 bits, as 32 tokens take it)
    p.tokens = 16, p.waves = 8;
    if (L == 1 && !back) p.tokens = 1, p.waves = 1;
    else if (L <= 4) p.tokens = 4, p.waves = 1;
    else if (L <= 32) p.tokens = 8, p.waves = 4;
    else if (L <= 64 || (back && p.channels == 2)) p.waves = 4;
    else if (L <= 128) p.waves = 8;
    else if (back) p.waves = far && (n <= 4 * cus || chains <= cus / 32) ? 16 : 8;
    else if (L <= 256) one || !words ? p.waves = 16 : p.tokens = 32;
    else if (p.channels == 1) p.waves = far && one ? 16 : 8;
    else if (16 * pieces(256) <= 9 * pieces(128) && (n <= 32 * cus || chains <= cus / 2)) p.tokens = 32;
    p.pieces = pieces(p.tokens * p.waves);
    return p;
}

size_t slots_bytes(const bimamba_recurrence_desc* d, const RecurPlan& p)   // (and the tickets)
{
    return p.pieces > 1 ? (size_t)d->batch * p.pieces * d->d_inner * 8 + kXcds * 4 : 0;
}

// False: there is no kernel for the plan's pieces.
template <typename IO, int kGate, int kC, bool kPast>
bool launch_pieces(const RecurPlan& p, RecurArgs a, bool back, hipStream_t st)
{
    // How far a workgroup looks back: what a hop from one state to the next takes has to pass over as many pieces of a sequence as are done
    // meanwhile, the more the fewer sequences and channels there are; each piece looked at costs words to read.  65536 tokens of 2048
    // channels in pieces of 16 x 8: 8 pieces 190 us, 4 199, 2 262; 8 x 8192 of 4096: 1 piece 322 us, 8 345.
    // (Of the gradients' pieces of four waves there are twice as many: 2 x 16384 of 4096, 2 pieces 273 us, 4 264.)
    const int look = (int)((p.waves <= 4 ? 2u : 1u) * cu_count() / (2u * p.tiles * (unsigned)a.batch));
    const int most = p.waves < 8 ? 8 : p.waves;
    a.look = look < 1 ? 1 : look > most ? most : look;
    if (p.pieces > 1) hipLaunchKernelGGL(recur_clear_kernel, dim3((unsigned)(((long long)p.pieces * a.d + 256 * kCleared - 1) / (256 * kCleared)), a.batch), dim3(256), 0, st, a);
    const dim3 grid(p.tiles * (unsigned)a.batch * p.pieces), wg(64 * p.waves);
    bool launched = false;
    const auto form = [&](auto tokens, auto waves) {
        constexpr int kT = decltype(tokens)::value, kW = decltype(waves)::value;
        constexpr bool kBack = kT > 1 && (kC == 1 ? kT < 32 : kT * kW <= 64);   // (there are gradients of such pieces)
        if (p.tokens != kT || p.waves != kW || (back && !kBack)) return;
        if (!back) hipLaunchKernelGGL((recur_kernel<IO, kGate, kC, kT, kW, kPast>), grid, wg, 0, st, a);
        else if constexpr (kBack) hipLaunchKernelGGL((recur_bwd_kernel<IO, kGate, kC, kT, kW, kPast>), grid, wg, 0, st, a);
        launched = true;
    };
    using std::integral_constant;
    const integral_constant<int, 1> n1{};
    const integral_constant<int, 4> n4{};
    const integral_constant<int, 8> n8{};
    const integral_constant<int, 16> n16{};
    const integral_constant<int, 32> n32{};
    if constexpr (!kPast || kC == 2 || sizeof(typename IO::T) == 4) {   // (up to four tokens of 64 channels: the caches hold all that 65535 sequences move)
        form(n1, n1);
        form(n4, n1);
    }
    form(n8, n4);
    form(n16, n4);
    form(n16, n8);
    if constexpr (kC == 1) form(n16, n16);
    if constexpr (sizeof(Piece<IO, kC>) == 4) form(n32, n8);
    return launched;
}
template <typename IO, int kC>
bool launch_gate(const bimamba_recurrence_desc* d, const RecurPlan& p, const RecurArgs& a, bool on_lines, bool back, hipStream_t st)
{
    const bool past = a.queues == 1 && on_lines && past_caches((back ? 5.0 : 3.0) * d->batch * d->seqlen * d->d_inner * sizeof(typename IO::T));
    if (d->gate == BIMAMBA_GATE_SIGMOID) return past ? launch_pieces<IO, kSigmoid, kC, true>(p, a, back, st) : launch_pieces<IO, kSigmoid, kC, false>(p, a, back, st);
    return past ? launch_pieces<IO, kLog, kC, true>(p, a, back, st) : launch_pieces<IO, kLog, kC, false>(p, a, back, st);
}
// Where rows do not start at cache lines the pieces of neighbouring channels share lines: they are read and written through the caches, and, with
// more chains than workgroups in hand, by workgroups of one XCD, which share a cache.  29 x 2478 tokens of 2248 channels, past the
// caches 306 us, through them 266, and with a queue for each XCD 249, gradients 542, 450, 381.  (With few chains the queues only
// keep them apart: one sequence of 65536 x 2040 231 us, with eight queues 314; and rows that start at lines have nothing to share:
// 65536 x 2048 189 and 238.)
bool on_lines(const RowView& v, size_t elem)
{
    return !v.p || (reinterpret_cast<uintptr_t>(v.p) % 128 == 0 && v.sb * (long long)elem % 128 == 0 && v.st * (long long)elem % 128 == 0);
}
bool launch(const bimamba_recurrence_desc* d, const RecurPlan& p, RecurArgs& a, bool back, hipStream_t st)
{
    const size_t elem = dtype_bytes(d->io_dtype);
    bool lines = true;
    for (const RowView* v : {&a.x, &a.g, &a.add, &a.y, &a.dy, &a.dx, &a.dg}) lines = lines && on_lines(*v, elem);
    a.queues = !lines && p.tiles * (unsigned)a.batch >= (unsigned)cu_count() ? kXcds : 1;
    if (d->io_dtype == BIMAMBA_F32) return launch_gate<IoF32, 1>(d, p, a, lines, back, st);
    return p.channels == 2 ? launch_gate<IoBF16, 2>(d, p, a, lines, back, st) : launch_gate<IoBF16, 1>(d, p, a, lines, back, st);
}

// An fp32 or int64 array, none if p is null.
int check_array(const void* p, long long count, size_t elem, Bytes* r)
{
    if (!aligned_to(p, elem)) return BIMAMBA_ERR_MISALIGNED;
    *r = bytes_of(p, count, elem);
    return BIMAMBA_OK;
}

}  // namespace
}  // namespace bm

using namespace bm;

extern "C" {

size_t bimamba_recurrence_workspace_bytes(const bimamba_recurrence_desc* d)
{
    if (check_recurrence(d) || d->batch == 0 || d->seqlen == 0) return 0;
    return slots_bytes(d, plan_recurrence(d, false));
}

int bimamba_recurrence(const bimamba_recurrence_desc* d, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                       const bimamba_tensor* add, const int64_t* lengths, const float* h_in, const bimamba_tensor* y, float* h_out,
                       float* states, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_recurrence(d);
    if (rc) return rc;
    if (!x || !g || !y) return BIMAMBA_ERR_NULL_POINTER;
    if (bias && d->gate != BIMAMBA_GATE_SIGMOID) return BIMAMBA_ERR_UNSUPPORTED;
    if (d->batch == 0) return BIMAMBA_OK;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    const size_t elem = dtype_bytes(io);
    const RecurPlan p = L ? plan_recurrence(d, false) : RecurPlan{};
    const size_t need = bimamba_recurrence_workspace_bytes(d);
    Bytes bx{}, bg{}, badd{}, by{}, bbias, blen, bin, bout, bkept;
    if (L) {
        if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (rc = check_view(g, Bt, L, D, io, false, &bg)) || (rc = check_view(y, Bt, L, D, io, true, &by)))
            return rc;
        if (add && (rc = check_view(add, Bt, L, D, io, false, &badd))) return rc;
    }
    if ((rc = check_array(bias, D, 4, &bbias)) || (rc = check_array(lengths, Bt, 8, &blen)) || (rc = check_array(h_in, (long long)Bt * D, 4, &bin)) ||
        (rc = check_array(h_out, (long long)Bt * D, 4, &bout)) || (rc = check_array(states, (long long)Bt * ((L + kKeep - 1) / kKeep) * D, 4, &bkept)))
        return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1);
    if (L) {
        if (views_meet(y, D, by, x, D, bx, Bt, elem, elem) || views_meet(y, D, by, g, D, bg, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        const bool same = add && add->ptr == y->ptr && add->stride_batch == y->stride_batch && add->stride_token == y->stride_token;
        if (add && !same && views_meet(y, D, by, add, D, badd, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes written[] = {by, bout, bkept, ws}, read[] = {bbias, blen, bin, bx, bg, badd};
    for (int i = 0; i < 4; i++) {
        for (int j = 0; j < (i == 0 ? 3 : 6); j++)
            if (meet(written[i], read[j]) && !(i == 1 && j == 2 && h_in == h_out)) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j])) return BIMAMBA_ERR_ALIAS;
    }
    RecurArgs a{};
    a.x = row_view(x), a.g = row_view(g), a.y = row_view(y);
    if (add) a.add = row_view(add);
    a.bias = bias, a.lengths = lengths, a.enter = h_in, a.leave = h_out, a.states = states;
    a.ticket = static_cast<unsigned*>(workspace), a.slots = static_cast<unsigned long long*>(workspace) + 4;
    a.L = L, a.d = D, a.pieces = p.pieces, a.reverse = d->reverse, a.batch = Bt;
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    if (L) {
        if (!launch(d, p, a, false, st)) return BIMAMBA_ERR_UNSUPPORTED;
    } else if (h_out && h_out != h_in) {
        // (no token: the state goes through; a sum of one slot, or of none)
        launch_slot_sum(SlotSumArgs{{const_cast<float*>(h_in), nullptr}, {h_out, nullptr}, h_in ? 1 : 0, D, D}, Bt, st);
    }
    return launches.status();
}

size_t bimamba_recurrence_bwd_workspace_bytes(const bimamba_recurrence_desc* d)
{
    if (check_recurrence(d) || d->batch == 0 || d->seqlen == 0) return 0;
    const RecurPlan p = plan_recurrence(d, true);
    const long long slots = (long long)d->batch * p.pieces;
    const size_t sums = d->gate == BIMAMBA_GATE_SIGMOID && slots > 1 ? (size_t)slots * d->d_inner * sizeof(float) : 0;
    return slots_bytes(d, p) + sums;
}

int bimamba_recurrence_bwd(const bimamba_recurrence_desc* d, const bimamba_tensor* x, const bimamba_tensor* g, const float* bias,
                           const int64_t* lengths, const float* states, const bimamba_tensor* dy, const float* dh_out,
                           const bimamba_tensor* dx, const bimamba_tensor* dg, float* dbias, float* dh_in,
                           void* workspace, size_t workspace_bytes, void* hip_stream)
{
    int rc = check_recurrence(d);
    if (rc) return rc;
    if (!x || !g || !dy || !dx || !dg) return BIMAMBA_ERR_NULL_POINTER;
    if ((bias || dbias) && d->gate != BIMAMBA_GATE_SIGMOID) return BIMAMBA_ERR_UNSUPPORTED;
    const int Bt = d->batch, L = d->seqlen, D = d->d_inner, io = d->io_dtype;
    const bool rows = Bt && L;
    const size_t elem = dtype_bytes(io);
    const RecurPlan p = rows ? plan_recurrence(d, true) : RecurPlan{};
    const size_t need = bimamba_recurrence_bwd_workspace_bytes(d);
    Bytes bx{}, bg{}, by{}, bdx{}, bdg{}, bbias, blen, bkept, bout, bdb, bin;
    if (rows) {
        if (!states) return BIMAMBA_ERR_NULL_POINTER;
        if ((rc = check_view(x, Bt, L, D, io, false, &bx)) || (rc = check_view(g, Bt, L, D, io, false, &bg)) ||
            (rc = check_view(dy, Bt, L, D, io, false, &by)) || (rc = check_view(dx, Bt, L, D, io, true, &bdx)) ||
            (rc = check_view(dg, Bt, L, D, io, true, &bdg)))
            return rc;
    }
    if ((rc = check_array(bias, D, 4, &bbias)) || (rc = check_array(lengths, Bt, 8, &blen)) ||
        (rc = check_array(states, (long long)Bt * ((L + kKeep - 1) / kKeep) * D, 4, &bkept)) || (rc = check_array(dh_out, (long long)Bt * D, 4, &bout)) ||
        (rc = check_array(dbias, D, 4, &bdb)) || (rc = check_array(dh_in, (long long)Bt * D, 4, &bin)))
        return rc;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const Bytes ws = bytes_of(need ? workspace : nullptr, need, 1);
    if (rows) {
        const bimamba_tensor *const in[] = {x, g, dy}, *const out[] = {dx, dg};
        const Bytes bin3[] = {bx, bg, by}, bout2[] = {bdx, bdg};
        for (int i = 0; i < 2; i++)
            for (int j = 0; j < 3; j++)
                if (views_meet(out[i], D, bout2[i], in[j], D, bin3[j], Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
        if (views_meet(dx, D, bdx, dg, D, bdg, Bt, elem, elem)) return BIMAMBA_ERR_ALIAS;
    }
    const Bytes written[] = {bdx, bdg, bdb, bin, ws}, read[] = {bbias, blen, bkept, bout, bx, bg, by};
    for (int i = 0; i < 5; i++) {
        for (int j = 0; j < (i < 2 ? 4 : 7); j++)
            if (meet(written[i], read[j]) && !(i == 3 && j == 3 && dh_in == dh_out)) return BIMAMBA_ERR_ALIAS;
        for (int j = 0; j < i; j++)
            if (meet(written[i], written[j]) && !(i == 1 && j == 0)) return BIMAMBA_ERR_ALIAS;
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
    const Launches launches;
    const long long slots = rows ? (long long)Bt * p.pieces : 0;
    if (rows) {
        RecurArgs a{};
        a.x = row_view(x), a.g = row_view(g), a.dy = row_view(dy), a.dx = row_view(dx), a.dg = row_view(dg);
        a.bias = bias, a.lengths = lengths, a.enter = dh_out, a.leave = dh_in, a.states = const_cast<float*>(states);
        a.ticket = static_cast<unsigned*>(workspace), a.slots = static_cast<unsigned long long*>(workspace) + 4;
        float* const sums = static_cast<float*>(workspace) + slots_bytes(d, p) / sizeof(float);
        a.dbias = dbias ? slots > 1 ? sums : dbias : nullptr;
        a.L = L, a.d = D, a.pieces = p.pieces, a.reverse = d->reverse, a.batch = Bt;
        if (!launch(d, p, a, true, st)) return BIMAMBA_ERR_UNSUPPORTED;
        if (dbias && slots > 1) launch_slot_sum(SlotSumArgs{{sums, nullptr}, {dbias, nullptr}, slots, D, D}, 1, st);
    } else {
        if (Bt && dh_in && dh_in != dh_out) launch_slot_sum(SlotSumArgs{{const_cast<float*>(dh_out), nullptr}, {dh_in, nullptr}, dh_out ? 1 : 0, D, D}, Bt, st);
        if (dbias) launch_slot_sum(SlotSumArgs{{nullptr, nullptr}, {dbias, nullptr}, 0, D, D}, 1, st);
    }
    return launches.status();
}

}  // extern "C"
