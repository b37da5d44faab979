// s4c_token_logprobs, s4c_tree_logprobs: what a distribution over the vocabulary says of the tokens that were given or emitted --
// their log probability, the distribution's entropy and its best alternatives -- from logits in memory.
//
// With m = max_v x_v, y_v = (x_v - m) / tau and S = sum_v exp(y_v):
//     log p(t) = y_t - ln S,   H = ln S - (sum_v exp(y_v) y_v) / S,
// sums of differences against a logit of the row: in the stream against a reference that lies at most 8 powers of two below the maximum (ln S is up to 5.5 more
// than against the maximum itself, its rounding 2^-24 of that), in extreme rows against the maximum.
//
// HBM-bound: every logit is read once, by a stream that no barrier interrupts (2048 x 128256 bf16 rows: 93 us, 87 % of the copy bandwidth, and 106
// with eight alternatives; one row of 32000 float32 logits 4.6 us, and 7.2).  A block (a cluster of up to eight for few rows) takes a
// row; its threads keep running sums S = sum 2^y and E = sum 2^y y against a reference of their own, y = x log2(e) / tau - M, and raise M only
// when a vector's maximum passes it by 2^8 (exact in any case; it spares the rescaling of nearly every vector).  Elements travel in pairs
// (f32x2 arithmetic).  At the end threads, warps, blocks are joined in a fixed order.
//
// Alternatives.  About the top-th greatest of the threads' maxima is a bound that at least `top` logits reach, and few more do.  A thread knows the
// batch that held its maximum and the maximum of its other batches, so that the few threads at or above the bound read one batch again (or,
// for the fewer ones with more, the block reads all of theirs).  Candidates find their ranks by counting, the best `top` go to the
// first block, where an entry's rank is its place in its own list and, by bisection, in the others.  A row whose candidates overflow
// (thousands of equal logits, say) finds its bound by bisection over all logits' ordered bits instead.  Greater logits first, then lower
// tokens: one 64-bit key, so that ranks are unique and do not hang on timing.
#include <algorithm>

#include "row_softmax.cuh"

namespace s4c {

using namespace rows;

constexpr int kLpMaxTop = 64;
constexpr int kLpCandidates = 1024;
// Threads of a block and blocks of an SM, for long, medium and short rows (see lp_launch)
constexpr int kLpThreads = 256, kLpBlocks = 4, kLpMedium = 128, kLpMediumBlocks = 8, kLpShort = 64, kLpShortBlocks = 16;
constexpr int kLpMediumRow = 6144, kLpMediumFew = 768, kLpShortRow = 384;  // vectors of such a row at most (Few: in calls of no more rows than SMs)
constexpr int kLpBatch = 4;       // vectors that a thread takes at once
constexpr int kLpRing = 2;        // batches on their way or in hand
constexpr float kLpSlack = 8.0f;  // how far (log2) a maximum may pass the reference of a running sum

struct LpParams {
    const void* logits;
    long long stride;          // elements between rows
    const int32_t* tokens;     // [R], or [B,T] of a walk
    const int32_t* path;       // [B, entries] of a walk; NULL: plain rows
    const int32_t* accept_len;
    const int32_t* next_token;
    int entries, T, V, top;
    float scale, inv_scale;    // log2(e) / temperature, and its reciprocal
    double exact;              // log2(e) / temperature, where it or its reciprocal is too small for float32 too
    float* logprob;
    float* entropy;
    int32_t* top_token;
    float* top_logprob;
    int32_t* status;
};

// Where a row of the call lies and which token it is asked for.
struct LpRow {
    long long row;  // the logits row
    int token;      // the token; -1: none (the row is not read)
    int flags;      // S4C_SEQ_* that make the whole row undefined
};

// Emission j of sequence b: the distribution after node path[j], and the token that followed it -- the next node's, or next_token behind
// the path's end.  Every thread of the block gets the same answer.
__device__ __forceinline__ LpRow lp_row(const LpParams& p, int r) {
    LpRow w;
    if (!p.path) {
        w.row = r;
        w.token = p.tokens ? p.tokens[r] : INT_MAX;  // (INT_MAX: nothing asked for, the row's own values only)
        w.flags = 0;
        return w;
    }
    const int b = r / p.entries, j = r - b * p.entries;
    const int a = p.accept_len[b];
    const int32_t* path = p.path + (size_t)b * p.entries;
    w.row = 0, w.token = -1, w.flags = 0;
    if (a < 0) return w;  // a sequence that the walk skipped
    if (a >= p.entries) {
        w.flags = S4C_SEQ_DEPTH;
        return w;
    }
    bool bad = false;
    for (int i = threadIdx.x & 31; i <= a; i += 32) bad = bad || path[i] >= p.T || (i == 0 ? path[i] != 0 : path[i] <= path[i - 1]);
    if (__any_sync(0xffffffffu, bad)) {
        w.flags = S4C_SEQ_BAD_PATH;
        return w;
    }
    if (j > a) return w;
    w.row = (long long)b * p.T + path[j];
    w.token = j < a ? p.tokens[(size_t)b * p.T + path[j + 1]] : p.next_token[b];
    if (w.token < 0) w.token = p.V;  // an emitted token has to be one: flagged as out of range
    return w;
}

// Logit and token as one number: greater logits are greater, of equal ones (zeros of both signs are) the lower token.
__device__ __forceinline__ uint32_t lp_order(float x) {
    uint32_t b = __float_as_uint(x);
    b = b << 1 ? b : 0u;
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint64_t lp_key(float x, int token) { return ((uint64_t)lp_order(x) << 32) | (0xffffffffu - (uint32_t)token); }
__device__ __forceinline__ int lp_token(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float lp_logit(uint64_t key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}

template <int S>
struct alignas(16) LpShared {
    uint4 ring[kLpRing * kLpBatch * S];  // the stream's; then, from its start, the candidates
    uint64_t list[kMaxCluster][kLpMaxTop];  // the first block's: every block's best, best first
    float4 part[kMaxCluster];               // the first block's: every block's maximum, M, S, E
    int listed[kMaxCluster];
    float best[S];                 // the threads' maxima
    float4 warp[S / 32];
    int found, count[2];
    int wides, wide[S];            // threads with candidates in more batches than one
    __device__ __forceinline__ uint64_t* candidates() { return reinterpret_cast<uint64_t*>(ring); }
};

// Where the candidates overflow: the top-th greatest logit and, among its equals, the highest token that still belongs, by bisection.  About fifty passes
// over the block's share: 2048 x 128256 bf16 rows filled with -1e4 but for three tokens, five alternatives, 9.5 ms (three alternatives, or a fill
// of -Inf, which is no candidate: 100 us); 26 x 32000 float32 170 us.
template <typename T, int S>
struct LpExactly {
    // How many of the block's logits pass `f(ordered bits, token)`; -Inf and NaN never do.  `turn` alternates between calls.
    template <typename F>
    __device__ __forceinline__ static int count(const Row<T>& row, const Share& mine, LpShared<S>& sh, int turn, F f) {
        int c = 0;
        for (int i = mine.begin + (int)threadIdx.x; i < mine.end; i += blockDim.x) {
            float x[Vec<T>::E];
            Vec<T>::unpack(row.load(i), x);
#pragma unroll
            for (int j = 0; j < Vec<T>::E; ++j)
                if (x[j] > -INFINITY && f(lp_order(x[j]), row.first(i) + j)) ++c;
        }
        c = __reduce_add_sync(0xffffffffu, c);
        if (threadIdx.x == 0) sh.count[turn ^ 1] = 0;  // (the last call's: everybody has read it before the barrier that this call began behind)
        if ((threadIdx.x & 31) == 0) atomicAdd(&sh.count[turn], c);
        __syncthreads();
        c = sh.count[turn];
        __syncthreads();
        return c;
    }
    // Collects exactly `top` candidates (the block has at least as many logits above -Inf).
    __device__ __noinline__ static void collect(const Row<T> row, const Share mine, LpShared<S>& sh, int top) {
        int turn = 0;
        __syncthreads();
        if (threadIdx.x == 0) sh.count[0] = sh.count[1] = 0;
        __syncthreads();
        uint32_t lo = 0, hi = 0xffffffffu;  // the greatest u that at least `top` logits reach
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2 + 1;
            if (count(row, mine, sh, turn, [&](uint32_t u, int) { return u >= mid; }) >= top)
                lo = mid;
            else
                hi = mid - 1;
            turn ^= 1;
        }
        const int above = count(row, mine, sh, turn, [&](uint32_t u, int) { return u > lo; });
        turn ^= 1;
        int first = 0, last = row.V - 1;  // the least token with enough equals up to it
        while (first < last) {
            const int mid = first + (last - first) / 2;
            if (count(row, mine, sh, turn, [&](uint32_t u, int t) { return u == lo && t <= mid; }) >= top - above)
                last = mid;
            else
                first = mid + 1;
            turn ^= 1;
        }
        if (threadIdx.x == 0) sh.found = 0;
        __syncthreads();
        for (int i = mine.begin + (int)threadIdx.x; i < mine.end; i += blockDim.x) {
            float x[Vec<T>::E];
            Vec<T>::unpack(row.load(i), x);
#pragma unroll
            for (int j = 0; j < Vec<T>::E; ++j) {
                const uint32_t u = lp_order(x[j]);
                const int t = row.first(i) + j;
                if (x[j] > -INFINITY && (u > lo || (u == lo && t <= first))) sh.candidates()[atomicAdd(&sh.found, 1)] = lp_key(x[j], t);
            }
        }
        __syncthreads();
    }
};

// Running sums of 2^y and 2^y y, y = x c - M, in pairs.
template <typename T>
struct LpSums {
    F2 S = 0, E = 0;      // (bits of two zeros)
    float M = -INFINITY;  // nothing above -Inf so far
    float minus = -300.0f;  // -M; terms of 2^-300 = 0 before there is one
    uint32_t low = 0;     // elements below it are taken as it: 2^y is 0 there, and y stays finite (-Inf times 0 would not be a 0)
    __device__ __forceinline__ void raise(float to, float inv_c) {
        const float d = fmaxf(M - to, -200.0f), f = exp2_fast(d);  // y becomes y + d: S -> S 2^d, E -> (E + S d) 2^d
        E = mul2(fma2(S, f2(d, d), E), f2(f, f)), S = mul2(S, f2(f, f));
        if (f == 0.0f) S = E = 0;  // (sums against a reference so far down that its rounding made them infinite)
        const float at = to * inv_c;  // the reference as a logit, give or take roundings
        M = to, minus = -to, low = Vec<T>::low(at - fmaxf(190.0f * inv_c, fabsf(at) * 1e-6f));
    }
    template <int N>
    __device__ __forceinline__ void take(const uint4 (&v)[N], float max, float c, float inv_c) {
        const float top = __fmul_rn(max, c);  // (rounded as it will be subtracted)
        if (top > M + kLpSlack) raise(top, inv_c);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            F2 x[Vec<T>::E / 2];
            Vec<T>::pairs(v[k], low, x);
#pragma unroll
            for (int j = 0; j < Vec<T>::E / 2; ++j) {
                const F2 y = fma2(x[j], f2(c, c), f2(minus, minus)), t = exp2_2(y);
                S = add2(S, t), E = fma2(t, y, E);
            }
        }
    }
};
// (M, S, E) against another, greater or equal reference
__device__ __forceinline__ void lp_move(float M, float& S, float& E, float to) {
    const float d = fmaxf(M - to, -200.0f), f = exp2_fast(d);
    E = f == 0.0f ? 0.0f : (E + S * d) * f, S = f == 0.0f ? 0.0f : S * f;
}

// Rows whose greatest logit times log2(e) / tau has a rounding of more than a few powers of two, or leaves float32, and temperatures at which
// the clamp of LpSums does (beyond 1e-30 .. 1e30): S and E by differences against the exact maximum, in float64, all of the row by one block.
template <typename T, int S>
__device__ __noinline__ void lp_extreme(const Row<T> row, LpShared<S>& sh, float m, double c, float& sum, float& weighted) {
    float s = 0.0f, e = 0.0f;
    for (int i = threadIdx.x; i < row.n; i += blockDim.x) {
        float x[Vec<T>::E];
        Vec<T>::unpack(row.load(i), x);
#pragma unroll
        for (int j = 0; j < Vec<T>::E; ++j) {
            const float y = (float)fmax(((double)x[j] - m) * c, -200.0), t = exp2_fast(y);
            s += t, e += t * y;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o), e += __shfl_xor_sync(0xffffffffu, e, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.warp[threadIdx.x >> 5] = make_float4(s, e, 0.0f, 0.0f);
    __syncthreads();
    sum = 0.0f, weighted = 0.0f;
    for (int w = 0; w < (int)blockDim.x >> 5; ++w) sum += sh.warp[w].x, weighted += sh.warp[w].y;
}

template <typename T, int S, int BLOCKS>
__global__ void __launch_bounds__(S, BLOCKS)
logprobs_kernel(const LpParams p, int cluster, int per) {
    __shared__ LpShared<S> sh;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (cluster > 1) cluster_arrive_relaxed();  // this block has started
    const int r = cluster_index(), rank = cluster_rank();
    constexpr int warps = S / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const LpRow w = lp_row(p, r);
    const int top = p.top;
    auto undefined = [&](float v, int flags) {  // a row without values: 0 where it is not asked for, NaN where it is flagged
        if (tid == 0) {
            if (p.logprob) p.logprob[r] = v;
            if (p.entropy) p.entropy[r] = v;
            if (p.status) p.status[r] = flags;
        }
        for (int j = tid; j < top; j += blockDim.x) p.top_token[(size_t)r * top + j] = -1, p.top_logprob[(size_t)r * top + j] = -INFINITY;
    };
    if (w.token == -1 || w.flags) {
        if (rank == 0) undefined(w.flags ? NAN : 0.0f, w.flags);
        if (cluster > 1) cluster_wait();
        return;
    }
    const Row<T> row(const_cast<T*>(static_cast<const T*>(p.logits)) + w.row * p.stride, p.V);
    const Share mine(row.n, rank, per);
    const uint4* vectors = row.vectors();
    const float c = p.scale, inv_c = p.inv_scale;

    // ---- the stream: sums, the batch with the thread's maximum, and the maximum of its other batches.  A ring of batches in shared memory keeps
    // kLpRing - 1 of them on their way while one is summed; a thread's copies are for that thread alone, so that no barrier is needed.
    LpSums<T> sums;
    float mt = -INFINITY, others = -INFINITY;
    int at_max = -1;
    auto take = [&](int i, const auto& v) {
        const float max = Vec<T>::max(v);
        sums.take(v, max, c, inv_c);
        others = fmaxf(others, fminf(mt, max));
        if (max > mt) at_max = i;
        mt = max_nan(mt, max);
    };
    {
        const uint32_t slot = (uint32_t)__cvta_generic_to_shared(sh.ring) + (uint32_t)tid * 16u;
        const uint4* own = sh.ring + tid;
        auto request = [&](int i, int stage) {
#pragma unroll
            for (int k = 0; k < kLpBatch; ++k)
                if (i + k * S < mine.e) copy16(slot + (uint32_t)(stage * kLpBatch + k) * (S * 16u), vectors + i + k * S);
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        int i = mine.b + tid;
#pragma unroll
        for (int d = 0; d < kLpRing; ++d) request(i + d * (kLpBatch * S), d);
        for (int stage = 0; i < mine.e; i += kLpBatch * S) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kLpRing - 1) : "memory");
            uint4 v[kLpBatch];
            if (i + (kLpBatch - 1) * S < mine.e) {
#pragma unroll
                for (int k = 0; k < kLpBatch; ++k) v[k] = own[(stage * kLpBatch + k) * S];
            } else {
#pragma unroll
                for (int k = 0; k < kLpBatch; ++k) {
                    v[k] = none<T>();
                    if (i + k * S < mine.e) v[k] = own[(stage * kLpBatch + k) * S];
                }
            }
            take(i, v);
            request(i + kLpRing * (kLpBatch * S), stage);
            if (++stage == kLpRing) stage = 0;
        }
        if (warp == 0 && (mine.begin == 0 || mine.end == row.n)) {
            const int edge = mine.edge(row.n, tid);
            uint4 v[1] = {none<T>()};
            if (edge >= 0) v[0] = row.load(edge);
            take(-1, v);
        }
    }

    // ---- the warps' sums, the threads' maxima
    if (tid == 0) sh.found = sh.wides = 0;
    sh.best[tid] = mt;
    float M = warp_max(sums.M);
    float s = lo(sums.S) + hi(sums.S), e = lo(sums.E) + hi(sums.E);
    lp_move(sums.M, s, e, M);
    s = warp_sum(s), e = warp_sum(e);
    if (lane == 0) sh.warp[warp] = make_float4(M, s, e, 0.0f);
    __syncthreads();
    float m = -INFINITY, bound = -INFINITY;
    {
        uint32_t u[S / 32];
#pragma unroll
        for (int k = 0; k < S / 32; ++k) {
            const float b = sh.best[lane + 32 * k];
            m = max_nan(m, b), u[k] = lp_order(b);
        }
        m = warp_max_nan(m);
        if (top > 0) {
            // about the top-th greatest of the threads' maxima, not above it: at least `top` logits reach it, and few more do
            uint32_t least = u[0], most = u[0];
#pragma unroll
            for (int k = 1; k < S / 32; ++k) least = min(least, u[k]), most = max(most, u[k]);
            least = __reduce_min_sync(0xffffffffu, least), most = __reduce_max_sync(0xffffffffu, most);
            while (least < most) {
                const uint32_t mid = least + (most - least) / 2 + 1;
                int n = 0;
#pragma unroll
                for (int k = 0; k < S / 32; ++k) n += u[k] >= mid;
                n = __reduce_add_sync(0xffffffffu, n);
                if (n < top) {
                    most = mid - 1;
                } else {
                    least = mid;
                    if (n <= top + top / 8 + 1) break;
                }
            }
            bound = lp_logit((uint64_t)least << 32);
        }
    }

    // ---- candidates at or above the bound: those of a thread's best batch, which it reads again, or of all its batches, which the block reads for it
    auto look = [&](int i, const uint4& v) {  // vector i
        float x[Vec<T>::E];
        Vec<T>::unpack(v, x);
#pragma unroll
        for (int j = 0; j < Vec<T>::E; ++j)
            if (x[j] >= bound && x[j] > -INFINITY) {
                const int place = atomicAdd(&sh.found, 1);
                if (place < kLpCandidates) sh.candidates()[place] = lp_key(x[j], row.first(i) + j);
            }
    };
    if (top > 0 && mt >= bound && mt > -INFINITY) {
        if (others >= bound && others > -INFINITY) {
            sh.wide[atomicAdd(&sh.wides, 1)] = tid;
        } else if (at_max >= 0) {
            uint4 v[kLpBatch];
#pragma unroll
            for (int k = 0; k < kLpBatch; ++k) {
                v[k] = none<T>();
                if (at_max + k * S < mine.e) v[k] = load16(vectors + at_max + k * S);
            }
#pragma unroll
            for (int k = 0; k < kLpBatch; ++k) look(at_max + k * S, v[k]);
        }
        const int i = mine.edge(row.n, tid);
        if (i >= 0) look(i, row.load(i));
    }
    if (cluster > 1) cluster_wait();  // (the first block has started)
    if (warp == 0) {
        const float4 o = lane < warps ? sh.warp[lane] : make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
        M = o.x, s = o.y, e = o.z;
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
        lp_move(o.x, s, e, M);
#pragma unroll
        for (int d = 4; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d), e += __shfl_xor_sync(0xffffffffu, e, d);
        if (lane == 0) peer_store(peer_address(&sh.part[rank], 0), make_float4(m, M, s, e));
    }
    if (top > 0) {
        __syncthreads();
        if (sh.wides) {
            const int each = (mine.e - mine.b + S - 1) / S, all = sh.wides * each;  // vectors of a thread
            for (int q = tid; q < all; q += kLpBatch * S) {
                int i[kLpBatch];
                uint4 v[kLpBatch];
#pragma unroll
                for (int k = 0; k < kLpBatch; ++k) {
                    const int n = q + k * S, whose = n / each;
                    i[k] = n < all ? mine.b + sh.wide[whose] + (n - whose * each) * S : INT_MAX;
                    v[k] = none<T>();
                    if (i[k] < mine.e) v[k] = load16(vectors + i[k]);
                }
#pragma unroll
                for (int k = 0; k < kLpBatch; ++k) look(i[k], v[k]);
            }
            __syncthreads();
        }
        int found = sh.found;
        if (found > kLpCandidates) {
            LpExactly<T, S>::collect(row, mine, sh, top);
            found = sh.found;
        }
        if (tid == 0) peer_store(peer_address(&sh.listed[rank], 0), min(found, top));
        for (int i = tid; i < found; i += blockDim.x) {
            const uint64_t key = sh.candidates()[i];
            int place = 0;
            for (int j = 0; j < found; ++j) place += sh.candidates()[j] > key;
            if (place < top) peer_store(peer_address(&sh.list[rank][place], 0), key);
        }
    }
    if (cluster > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (rank) return;

    // ---- the first block joins the blocks
    m = M = -INFINITY, s = e = 0.0f;
    for (int b = 0; b < cluster; ++b) m = max_nan(m, sh.part[b].x), M = fmaxf(M, sh.part[b].y);
    if (!usable(m)) return undefined(NAN, S4C_SEQ_NONFINITE);
    const bool extreme = !(fabsf(m) < 1e37f) || !(fabsf(m * c) < 1e8f) || !(c > 1e-30f && c < 1e30f);
    if (extreme) {
        lp_extreme(row, sh, m, p.exact, s, e);
    } else {
        for (int b = 0; b < cluster; ++b) {
            float4 q = sh.part[b];
            lp_move(q.y, q.z, q.w, M);
            s += q.z, e += q.w;
        }
    }
    if (tid >= max(1, cluster * top)) return;
    const float ln_s = ln_series(s);
    // (in float64: x c may leave float32 where the log probability does not)
    auto logprob = [&](float x) { return (float)((extreme ? ((double)x - m) * p.exact : (double)x * c - M) * kLn2 - ln_s); };
    const bool in_range = w.token >= 0 && w.token < p.V;
    if (tid == 0) {
        if (p.logprob) p.logprob[r] = in_range ? logprob(Vec<T>::get(row.x + w.token)) : NAN;
        if (p.entropy) p.entropy[r] = ln_s - __fdividef(e, s) * (float)kLn2;
        if (p.status) p.status[r] = p.tokens && !in_range ? S4C_SEQ_TOKEN_RANGE : 0;
    }
    if (top == 0) return;
    int total = 0;
    for (int b = 0; b < cluster; ++b) total += sh.listed[b];
    for (int i = tid; i < cluster * top; i += blockDim.x) {
        const int b = i / top, j = i - b * top;
        if (j >= sh.listed[b]) continue;
        const uint64_t key = sh.list[b][j];
        int place = j;
        for (int o = 0; o < cluster; ++o) {
            if (o == b) continue;
            int first = 0, last = sh.listed[o];  // how many of the other list's keys are greater
            while (first < last) {
                const int mid = (first + last) >> 1;
                if (sh.list[o][mid] > key)
                    first = mid + 1;
                else
                    last = mid;
            }
            place += first;
        }
        if (place < top) {
            p.top_token[(size_t)r * top + place] = lp_token(key);
            p.top_logprob[(size_t)r * top + place] = logprob(lp_logit(key));
        }
    }
    for (int j = total + tid; j < top; j += blockDim.x) p.top_token[(size_t)r * top + j] = -1, p.top_logprob[(size_t)r * top + j] = -INFINITY;
}

template <typename T>
static s4c_status lp_launch(const LpParams& p, long long rows, cudaStream_t stream) {
    const long long n = ((long long)p.V * (long long)sizeof(T) + 15) / 16 + 1;  // vectors, wherever a row starts
    // Few long rows are shared out, two blocks of 32 KB at least to an SM; where lists of alternatives have to be joined, among four.  (128256
    // float32 logits, none of them in L2, without and with twenty alternatives: one row by one block 22.5 / 24.6 us, by four 14.3 / 16.4, by
    // eight 12.3 / 16.4; 144 rows by a block each 30.7 / 34.8 us, by two 26.6 / 32.8, by four 30.7 / 36.9; the 80 that a walk through 16
    // paths of up to 9 emits of them 24.6 / 28.7, 20.5 / 24.6, 20.5 / 26.6.  576 rows of 32000: 28.7 / 32.8 us by a block each, 32.8 / 41.0 by two:
    // what a block does besides its stream is more than it saves.)
    const int cluster = (int)std::max(1ll, std::min({p.top ? 4ll : (long long)kMaxCluster, 2 * kSMs / rows, n / 2048}));
    const int per = (int)((n + cluster - 1) / cluster);
    // Shorter rows by fewer threads each and more rows at once: what a block does behind its stream is the same for every warp.  (4000 bf16 rows, five
    // alternatives, by 64 / 128 / 256 threads, each call on rows that are not in L2: V = 2000 29 / 32 / 64 us, 4000 35 / 33 / 57, 16384 52 / 51 / 68,
    // 32000 75 / 67 / 84; 1777 of 50001 53 / 51 / 51, 2368 of 128256 120 / 116 / 114.  140 rows of 32000: 15 / 12 / 11.  More than a quarter as many alternatives as threads lie far below the
    // threads' maxima: 4000 x 2000, 64 alternatives, rows in L2, 150 / 52 / 86 us.)
    if (n <= kLpShortRow && p.top <= kLpShort / 4) return row_launch(logprobs_kernel<T, kLpShort, kLpShortBlocks>, p, rows, 1, (int)n, kLpShort, 0, stream);
    if (n <= (rows > kSMs ? kLpMediumRow : kLpMediumFew))
        return row_launch(logprobs_kernel<T, kLpMedium, kLpMediumBlocks>, p, rows, 1, (int)n, kLpMedium, 0, stream);
    return row_launch(logprobs_kernel<T, kLpThreads, kLpBlocks>, p, rows, cluster, per, kLpThreads, 0, stream);
}

}  // namespace s4c

extern "C" s4c_status s4c_token_logprobs(const void* logits, long long row_stride, const int32_t* tokens, int R, int V, s4c_dtype dt,
                                         float temperature, int top, float* logprob, float* entropy, int32_t* top_token, float* top_logprob,
                                         int32_t* status, s4c_stream_t stream_) {
    using namespace s4c;
    if (R == 0 && V >= 1) return S4C_OK;
    if (!logits || (logprob && !tokens) || (top > 0 && (!top_token || !top_logprob))) return S4C_ERR_NULL;
    if (R < 0 || R > S4C_MAX_LOGITS_ROWS || V < 1 || V > S4C_MAX_LOGITS_COLUMNS || row_stride < V || top < 0 || !(temperature > 0.0f) || !(temperature < INFINITY) ||
        !(kLog2E / temperature < INFINITY))
        return S4C_ERR_SHAPE;
    if (dt != S4C_F32 && dt != S4C_BF16) return S4C_ERR_DTYPE;
    if (top > kLpMaxTop) return S4C_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(logits) % dtype_size(dt)) return S4C_ERR_ALIGN;
    const LpParams p = {logits, row_stride, tokens, nullptr, nullptr, nullptr, 0, 0, V, top, kLog2E / temperature, temperature / kLog2E, 1.4426950408889634 / temperature, logprob, entropy, top_token, top_logprob, status};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return dt == S4C_F32 ? lp_launch<float>(p, R, stream) : lp_launch<__nv_bfloat16>(p, R, stream);
}

extern "C" s4c_status s4c_tree_logprobs(const void* logits, const int32_t* tokens, const int32_t* path, const int32_t* accept_len,
                                        const int32_t* next_token, int B, int T, int V, int max_depth, s4c_dtype dt, float temperature, int top,
                                        float* logprob, float* entropy, int32_t* top_token, float* top_logprob, int32_t* status,
                                        s4c_stream_t stream_) {
    using namespace s4c;
    if (B == 0 && V >= 1) return S4C_OK;
    if (!logits || !tokens || !path || !accept_len || !next_token || !logprob || (top > 0 && (!top_token || !top_logprob))) return S4C_ERR_NULL;
    if (B < 0 || T < 1 || T > S4C_MAX_T || V < 1 || V > S4C_MAX_LOGITS_COLUMNS || max_depth < 0 || max_depth >= S4C_MAX_T || top < 0 || !(temperature > 0.0f) || !(temperature < INFINITY) ||
        !(kLog2E / temperature < INFINITY) || (long long)B * (max_depth + 1) > S4C_MAX_LOGITS_ROWS)
        return S4C_ERR_SHAPE;
    if (dt != S4C_F32 && dt != S4C_BF16) return S4C_ERR_DTYPE;
    if (top > kLpMaxTop) return S4C_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(logits) % dtype_size(dt)) return S4C_ERR_ALIGN;
    const LpParams p = {logits, V, tokens, path, accept_len, next_token, max_depth + 1, T, V, top, kLog2E / temperature, temperature / kLog2E, 1.4426950408889634 / temperature, logprob, entropy, top_token, top_logprob, status};
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    return dt == S4C_F32 ? lp_launch<float>(p, (long long)B * (max_depth + 1), stream) : lp_launch<__nv_bfloat16>(p, (long long)B * (max_depth + 1), stream);
}
