// s4c_distill_topk, s4c_distill_topk_backward: a drafter head's logits z against the target's top choices (t_j, l_j), j < K, and against
// labels, where there are some:
//     q = softmax(l / tau) over the entries that are there,  p = softmax(z / tau),  p1 = softmax(z),
//     loss = w_t tau^2 sum_j q_j (ln q_j - ln p(t_j)) - w_l ln p1(c),
//     d loss / d z_v = w_t tau (p_v - sum_{j: t_j = v} q_j) + w_l (p1_v - [v = c]).
// The gradient is dense in p and p1 and sparse in q: a pass over the row writes a exp((z_v - m) / tau) + b exp(z_v - m), and the
// at most K + 1 places that q and the label touch are written once more, behind a barrier.
//
// Loss and gradient in one call read and write every logit once (4096 x 128256 bf16 rows, K = 100: 440 to 475 us from GPU to GPU, 68 to 73 % of the copy
// bandwidth; the exponentials take 59 % of their unit, all instructions 55 % of their slots).  A cluster of up to eight blocks takes a row; its logits are
// copied to shared memory (cp.async, each thread's vectors for that thread alone, so that no barrier stands between a copy and its use), summed
// there against running references, and read from there once more for the gradient.  The blocks exchange (m, S, S1) through each
// other's shared memory.  The teacher's K entries are one warp's work, beside the stream.  The loss alone streams (2048 x 128256:
// 86 us, 94 % of the copy bandwidth), and so does the backward pass, whose blocks start from the row's saved (m, 1/S, 1/S1): 167 us, 96 %.
#include <algorithm>
#include <type_traits>

#include "row_softmax.cuh"

namespace s4c {

using namespace rows;

constexpr int kDsMaxTeach = 128;
constexpr int kDsBatch = 4;             // vectors that a thread takes at once
constexpr float kDsSlack = 8.0f;        // how far (log2) a maximum may pass the reference of a running sum
// Threads of a block's stream (one warp more has the teacher) and blocks of an SM, where the row is kept in shared memory, where it is streamed,
// and for short rows.  What a warp does besides its stream is a third of its instructions where the row is kept, so few warps are better
// there (4096 x 128256 bf16, loss and gradient: 256 threads 513 us, 192 495 us, 128 438 us when they were compared); a stream wants more of them
// (the loss alone 107 us with 6 x 128 threads for 2048 rows, 87 us with 5 x 256); a short row is two warps' (8000 x 4000, not in L2: 62 us by 8 x 64, 78 by
// 16 x 32).
constexpr int kDsKept = 128, kDsKeptBlocks = 6, kDsStreamed = 256, kDsStreamedBlocks = 5, kDsShort = 64, kDsShortBlocks = 8;
// Vectors of a block's share of a kept row, as far as eight blocks suffice: 34 KB, the most that leaves room for six blocks of an SM.  (2000 x 65536
// bf16, loss and gradient: 128 us by five blocks of 2048 vectors at most, 114 us by four of 2049; 132 us by 1536)
constexpr int kDsSlice = 2144;
// Vectors of a short row at most, and in calls of no more rows than SMs (not in L2: 30 x 8000 8.4 us as short rows, 5.8 us by blocks of a cluster;
// 2000 x 5000 22 us as short rows, 27 us as kept ones)
constexpr int kDsShortRow = 1024, kDsShortFew = 512;
// How 2^(x log2 e), of the label's term, comes from 2^(x log2 e / tau): there is none or it is the same, by an exponential of its own, or squared once
// or twice (tau = 2 or 4: two exponentials per logit and pass bound the kernel otherwise -- 2048 x 32000 bf16 rows with labels, tau = 2: 84 us by
// exponentials of their own, 70 us squared)
enum { kDsOne = 0, kDsTwo = -1, kDsSquare = 1, kDsFourth = 2 };
enum { kDsSkip = 0, kDsRow = 1, kDsBad = 2 };  // what stats[3] says of a row: nothing to learn from, a loss, undefined

struct DsParams {
    const void* logits;
    long long stride;
    const int32_t* teacher_token;  // [R,K]
    const float* teacher_logit;    // [R,K]
    int K;
    const int32_t* labels;         // [R] or NULL
    float inv_tau, scale, scale1;  // 1 / tau; log2(e) / tau; log2(e)
    int power;                     // kDsOne ...
    double w_teach;                // w_t tau^2 (which may leave float32 where the loss does not)
    float w_label;                 // w_l
    float g_teach;                 // w_t tau
    int V;
    float* loss;
    float* stats;                  // [R,4]: m, 1/S (0 without a teacher), 1/S1 (0 without a label), kDs*
    void* grad;                    // [R,V], rows grad_stride apart, or NULL
    long long grad_stride;
    const float* row_scale;        // [R] or NULL
    int32_t* status;
};

struct DsShared {
    // a row's teacher, entry K the label: q (-1: not there), ln q, the student's logit
    float q[kDsMaxTeach + 1];
    float log_q[kDsMaxTeach];
    float x[kDsMaxTeach + 1];
    // those of this block's share, in order
    int own_token[kDsMaxTeach + 1];
    float own_q[kDsMaxTeach + 1];  // -1: the label
    float own_x[kDsMaxTeach + 1];
    int owned, taught, labelled, flags;
    float4 warp[kDsStreamed / 32];  // a warp's maximum, reference, S, S1
    float4 part[2][kMaxCluster];  // every block's; [1]: S, S1 against the row's maximum, for extreme rows
};

// The teacher of row r, by one warp, in two steps: what it says and the student's logits there are asked for beside the stream, and looked at when
// the stream's sums have met (a gather behind a load is as long as the whole stream otherwise).  Between the two lies a barrier that
// orders the reads before any gradient that is written over the logits.
template <typename T>
struct DsTeacher {
    static constexpr int N = kDsMaxTeach / 32;
    int tok[N], label;
    float l[N];
    T x[N], label_x;
    __device__ __forceinline__ void ask(const DsParams& p, int r, const Row<T>& row, DsShared& t) {
        const int lane = threadIdx.x & 31;
        int flags = 0;
        bool any = false;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int j = lane + 32 * k;
            tok[k] = -1, l[k] = -INFINITY;
            if (j < p.K) tok[k] = p.teacher_token[(size_t)r * p.K + j], l[k] = p.teacher_logit[(size_t)r * p.K + j];
        }
        label = p.labels ? p.labels[r] : -1;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (tok[k] != -1 && (tok[k] < 0 || tok[k] >= p.V)) flags |= S4C_SEQ_TOKEN_RANGE, tok[k] = -1;
            if (tok[k] != -1 && !(l[k] < INFINITY)) flags |= S4C_SEQ_NONFINITE, tok[k] = -1;
            if (tok[k] == -1 || l[k] == -INFINITY) tok[k] = -1, l[k] = -INFINITY;
            any = any || tok[k] >= 0;
            if (tok[k] >= 0) x[k] = row.x[tok[k]];
        }
        if (label != -1 && (label < 0 || label >= p.V)) flags |= S4C_SEQ_TOKEN_RANGE, label = -1;
        if (label >= 0) label_x = row.x[label];
        flags = __reduce_or_sync(0xffffffffu, flags);
        any = __any_sync(0xffffffffu, any);
        if (lane == 0) t.taught = any, t.labelled = label >= 0, t.flags = flags;
    }
    // q, and what of it belongs to the block's share of the row
    __device__ __forceinline__ void learn(const DsParams& p, const Row<T>& row, const Share& mine, DsShared& t) {
        const int lane = threadIdx.x & 31;
        float lm = -INFINITY, total = 0.0f, e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) lm = fmaxf(lm, l[k]);
        lm = warp_max(lm);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (32 * k >= p.K) break;
            l[k] = tok[k] >= 0 ? (l[k] - lm) * p.scale : -INFINITY;  // log2 of q S
            e[k] = exp2_fast(l[k]);
            total += e[k];
        }
        total = warp_sum(total);
        const float inv_total = 1.0f / total, ln_total = ln_series(total);
        auto owns = [&](int token) {
            const int i = token < 0 ? -1 : (int)(((unsigned)token + row.lead) / Vec<T>::E);  // its vector
            return i >= mine.begin && i < mine.end;
        };
        int owned = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (32 * k >= p.K) break;
            const int j = lane + 32 * k;
            const float q = e[k] * inv_total, z = tok[k] >= 0 ? Vec<T>::get(&x[k]) : 0.0f;
            if (j < p.K) t.q[j] = tok[k] >= 0 ? q : -1.0f, t.log_q[j] = fmaf(l[k], (float)kLn2, -ln_total), t.x[j] = z;
            const uint32_t who = __ballot_sync(0xffffffffu, owns(tok[k]));
            if (owns(tok[k])) {
                const int at = owned + __popc(who & ((1u << lane) - 1));
                t.own_token[at] = tok[k], t.own_q[at] = q, t.own_x[at] = z;
            }
            owned += __popc(who);
        }
        if (lane == 0) {
            const float z = label >= 0 ? Vec<T>::get(&label_x) : 0.0f;
            t.x[p.K] = z;
            if (owns(label)) t.own_token[owned] = label, t.own_q[owned] = -1.0f, t.own_x[owned] = z, ++owned;
            t.owned = owned;
        }
        __syncwarp();
    }
};

// Both steps at once, where the row is streamed (a teacher that lives across the barrier costs the stream's few registers: 2048 x 128256 bf16 backward
// 169 us so, 199 us in two steps); `mine`: the block's share of the row.
template <typename T>
__device__ __forceinline__ void ds_teach(const DsParams& p, int r, const Row<T>& row, const Share& mine, DsShared& t) {
    constexpr int N = kDsMaxTeach / 32;
    const int lane = threadIdx.x & 31;
    int tok[N], flags = 0;
    float l[N], x[N], lm = -INFINITY, total = 0.0f, e[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int j = lane + 32 * k;
        tok[k] = -1, l[k] = -INFINITY;
        if (j < p.K) tok[k] = p.teacher_token[(size_t)r * p.K + j], l[k] = p.teacher_logit[(size_t)r * p.K + j];
    }
    int label = p.labels ? p.labels[r] : -1;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (32 * k >= p.K) break;
        if (tok[k] != -1 && (tok[k] < 0 || tok[k] >= p.V)) flags |= S4C_SEQ_TOKEN_RANGE, tok[k] = -1;
        if (tok[k] != -1 && !(l[k] < INFINITY)) flags |= S4C_SEQ_NONFINITE, tok[k] = -1;
        if (tok[k] == -1 || l[k] == -INFINITY) tok[k] = -1, l[k] = -INFINITY;
        lm = fmaxf(lm, l[k]);
    }
    if (label != -1 && (label < 0 || label >= p.V)) flags |= S4C_SEQ_TOKEN_RANGE, label = -1;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = tok[k] >= 0 ? Vec<T>::get(row.x + tok[k]) : 0.0f;
    const float label_x = label >= 0 ? Vec<T>::get(row.x + label) : 0.0f;
    lm = warp_max(lm);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (32 * k >= p.K) break;
        l[k] = tok[k] >= 0 ? (l[k] - lm) * p.scale : -INFINITY;  // log2 of q S
        e[k] = exp2_fast(l[k]);
        total += e[k];
    }
    total = warp_sum(total);
    const float inv_total = 1.0f / total, log2_total = (float)log2((double)total);
    auto owns = [&](int token) {
        const int i = token < 0 ? -1 : (int)(((unsigned)token + row.lead) / Vec<T>::E);  // its vector
        return i >= mine.begin && i < mine.end;
    };
    int owned = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (32 * k >= p.K) break;
        const int j = lane + 32 * k;
        const float q = e[k] * inv_total;
        if (j < p.K) t.q[j] = tok[k] >= 0 ? q : -1.0f, t.log_q[j] = (l[k] - log2_total) * (float)kLn2, t.x[j] = x[k];
        const uint32_t who = __ballot_sync(0xffffffffu, owns(tok[k]));
        if (owns(tok[k])) {
            const int at = owned + __popc(who & ((1u << lane) - 1));
            t.own_token[at] = tok[k], t.own_q[at] = q, t.own_x[at] = x[k];
        }
        owned += __popc(who);
    }
    flags = __reduce_or_sync(0xffffffffu, flags);
    if (lane == 0) {
        t.q[p.K] = label >= 0 ? 0.0f : -1.0f, t.x[p.K] = label_x;
        if (owns(label)) t.own_token[owned] = label, t.own_q[owned] = -1.0f, t.own_x[owned] = label_x, ++owned;
        t.owned = owned, t.taught = total > 0.0f, t.labelled = label >= 0, t.flags = flags;
    }
}

// What the gradient of a row is made of.
struct DsCoefs {
    float m, a, b;  // a 2^((z - m) scale) + b 2^((z - m) scale1)
    float wt, wl;   // what q and the label weigh, times the row's scale
};

// e^2, e^4
template <int P>
__device__ __forceinline__ F2 power_of(F2 e) {
    const F2 s = mul2(e, e);
    return P == kDsFourth ? mul2(s, s) : s;
}

// Vector i of a gradient row that is not aligned as its logits are, or sticks out of the row: element by element.
template <typename T>
__device__ __noinline__ void ds_by_element(T* g, int first, int V, const uint4 v) {
    constexpr int E = Vec<T>::E;
    float y[E];
    Vec<T>::unpack(v, y);
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (first + j >= 0 && first + j < V) Vec<T>::put(y[j], g + first + j);  // (exact: these are T's values)
}

// The dense part of the gradient: batches of vectors as `look` gives them.
template <int S, typename T, typename Look>
__device__ __forceinline__ void ds_dense(const DsParams& p, T* g, const Row<T>& row, const Share& mine, const DsCoefs& k, int kind, Look look) {
    constexpr int E = Vec<T>::E;
    const bool aligned = (int)(reinterpret_cast<uintptr_t>(g) & 15u) == row.lead * (int)sizeof(T);  // the gradient's vectors are the logits'
    uint4* vectors = reinterpret_cast<uint4*>(g - row.lead);
    auto store = [&](int i, const auto& v) {
        constexpr int N = sizeof(v) / sizeof(uint4);
        if (i < 0) {
            const int edge = mine.edge(row.n, threadIdx.x);
            if (edge >= 0) ds_by_element(g, row.first(edge), row.V, v[0]);
        } else if (aligned) {
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (i + n * S < mine.e) vectors[i + n * S] = v[n];
        } else {
            for (int n = 0; n < N; ++n)
                if (i + n * S < mine.e) ds_by_element(g, row.first(i + n * S), row.V, v[n]);
        }
    };
    if (kind != kDsRow) {
        F2 y[E / 2];
#pragma unroll
        for (int j = 0; j < E / 2; ++j) y[j] = kind == kDsBad ? f2(NAN, NAN) : f2(0.0f, 0.0f);
        const uint4 v[1] = {Vec<T>::pack(y)};
        for (int i = mine.b + (int)threadIdx.x; i < mine.e; i += S) store(i, v);
        store(-1, v);
        return;
    }
    const F2 minus = f2(-k.m, -k.m), c = f2(p.scale, p.scale), c1 = f2(p.scale1, p.scale1);
    auto pass = [&](auto power, float a) {
        constexpr int P = decltype(power)::value;
        look([&](int i, const auto& raw) {
            constexpr int N = sizeof(raw) / sizeof(uint4);
            uint4 v[N];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                F2 x[E / 2];
                Vec<T>::pairs(raw[n], x);
#pragma unroll
                for (int j = 0; j < E / 2; ++j) {
                    const F2 d = add2(x[j], minus), e = exp2_2(mul2(d, c));
                    x[j] = mul2(e, f2(a, a));
                    if constexpr (P != kDsOne) x[j] = fma2(P == kDsTwo ? exp2_2(mul2(d, c1)) : power_of<P>(e), f2(k.b, k.b), x[j]);
                }
                v[n] = Vec<T>::pack(x);
            }
            store(i, v);
        });
    };
    if (k.b == 0.0f || p.power == kDsOne)  // one exponential serves both terms
        pass(std::integral_constant<int, kDsOne>(), k.a + k.b);
    else if (p.power == kDsSquare)
        pass(std::integral_constant<int, kDsSquare>(), k.a);
    else if (p.power == kDsFourth)
        pass(std::integral_constant<int, kDsFourth>(), k.a);
    else
        pass(std::integral_constant<int, kDsTwo>(), k.a);
}

// The places that q and the label touch, behind a barrier that follows the dense part: a token's place by the first entry that names it.
template <typename T>
__device__ __forceinline__ void ds_sparse(const DsParams& p, T* g, const DsShared& t, const DsCoefs& k) {
    const int n = t.owned;
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
        const int tok = t.own_token[j];
        float off = 0.0f;
        bool first = true;
        for (int i = 0; i < n; ++i) {
            if (t.own_token[i] != tok) continue;
            first = first && i >= j;
            off += t.own_q[i] < 0.0f ? k.wl : k.wt * t.own_q[i];
        }
        if (!first) continue;
        const float d = t.own_x[j] - k.m;
        Vec<T>::put(k.a * exp2_fast(d * p.scale) + k.b * exp2_fast(d * p.scale1) - off, g + tok);
    }
}

// Running sums S = sum 2^(x c - M), S1 = sum 2^(x c1 - M1), in pairs; M and M1 are the reference logit's, which a vector's maximum raises where it
// passes it by kDsSlack (log2, at the larger scale).
template <int P>
struct DsSums {
    static constexpr bool TWO = P != kDsOne;
    F2 S = 0, S1 = 0;
    float ref = -INFINITY, minus = 0.0f, minus1 = 0.0f;
    float high = -INFINITY;  // ref at the larger scale
    template <typename T, int N>
    __device__ __forceinline__ void take(const uint4 (&v)[N], float max, float c, float c1) {
        const float cm = TWO ? fmaxf(c, c1) : c;
        if (max * cm > high + kDsSlack) {
            auto move = [&](float scale, float& minus, F2& sum) {
                const float to = __fmul_rn(max, scale), f = exp2_fast(fmaxf(-minus - to, -200.0f));  // (rounded as it will be subtracted)
                sum = f == 0.0f || ref == -INFINITY ? 0 : mul2(sum, f2(f, f));  // (0: also sums that a far reference's rounding made infinite)
                minus = -to;
            };
            move(c, minus, S);
            if (TWO) move(c1, minus1, S1);
            ref = max, high = max * cm;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            F2 x[Vec<T>::E / 2];
            Vec<T>::pairs(v[k], x);
#pragma unroll
            for (int j = 0; j < Vec<T>::E / 2; ++j) {
                const F2 e = exp2_2(fma2(x[j], f2(c, c), f2(minus, minus)));
                S = add2(S, e);
                // (a squared term has reference 2 M, which is what c1 = 2 c makes of the same logit, without another rounding)
                if (TWO) S1 = add2(S1, P == kDsTwo ? exp2_2(fma2(x[j], f2(c1, c1), f2(minus1, minus1))) : power_of<P>(e));
            }
        }
    }
};
// a sum against reference logit `from` against another, greater or equal one
__device__ __forceinline__ float ds_move(float sum, float from, float to, float c) {
    const float f = from > -INFINITY ? exp2_fast(fmaxf(__fmul_rn(from, c) - __fmul_rn(to, c), -200.0f)) : 0.0f;
    return f == 0.0f ? 0.0f : sum * f;
}

// One block's part of a row: its vectors, in shared memory from the first look on where RES.
template <typename T, int S, bool RES>
struct DsSlice {
    const Row<T>& row;
    const Share& share;
    uint4* kept;
    // requests the vectors, this thread's for this thread (two groups, so that the first can be summed while the second is on its way)
    __device__ __forceinline__ int half() const {
        return share.b + ((share.e - share.b) / 2 + kDsBatch * S - 1) / (kDsBatch * S) * (kDsBatch * S);
    }
    __device__ __forceinline__ void request() const {
        if (!RES) return;
        const uint4* vectors = row.vectors();
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(kept) - (uint32_t)share.begin * 16u;
        auto some = [&](int b, int e) {
            for (int i = b + (int)threadIdx.x; i < e; i += S)
                copy16(to + (uint32_t)i * 16u, vectors + i);
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        some(share.b, min(half(), share.e));
        some(half(), share.e);
        const int edge = share.edge(row.n, threadIdx.x);
        if (edge >= 0) kept[edge - share.begin] = row.load(edge);
    }
    template <typename F>
    __device__ __forceinline__ void look(F f, bool first) const {
        auto edge = [&](int i) { return RES ? kept[i - share.begin] : row.load(i); };
        const uint4* vectors = row.vectors();
        const int begin = share.begin, middle = half();
        auto at = [&](int i) {
            if (RES && first && i >= middle) asm volatile("cp.async.wait_group 0;" ::: "memory");
            return RES ? kept[i - begin] : load16(vectors + i);
        };
        if (RES && first) asm volatile("cp.async.wait_group 1;" ::: "memory");
        batches<T, kDsBatch>(share, row.n, S, at, edge, f);
    }
};

template <typename T, int P, bool RES, int S, int BLOCKS>
__global__ void __launch_bounds__(S + 32, BLOCKS)
distill_kernel(const DsParams p, int cluster, int per) {
    constexpr bool TWO = P != kDsOne;
    __shared__ DsShared t;
    extern __shared__ uint4 kept[];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (cluster > 1) cluster_arrive_relaxed();  // this block has started
    const int r = cluster_index(), rank = cluster_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool teacher = tid >= S;
    const Row<T> row(const_cast<T*>(static_cast<const T*>(p.logits)) + (long long)r * p.stride, p.V);
    const Share share(row.n, rank, per);
    const DsSlice<T, S, RES> mine{row, share, kept};
    const float c = p.scale, c1 = p.scale1;

    DsTeacher<T> asked;
    if (teacher) {
        if (RES)
            asked.ask(p, r, row, t);
        else
            ds_teach(p, r, row, share, t);
    } else {
        mine.request();
        DsSums<P> sums;
        float m = -INFINITY;
        mine.look([&](int, const auto& v) {
            const float max = Vec<T>::max(v);
            m = max_nan(m, max);
            sums.template take<T>(v, max, c, c1);
        }, true);
        m = warp_max_nan(m);
        const float ref = warp_max(sums.ref);
        const float s = warp_sum(ds_move(lo(sums.S) + hi(sums.S), sums.ref, ref, c));
        const float s1 = TWO ? warp_sum(ds_move(lo(sums.S1) + hi(sums.S1), sums.ref, ref, c1)) : 0.0f;
        if (lane == 0) t.warp[warp] = make_float4(m, ref, s, s1);
    }
    __syncthreads();

    // ---- every block gets every block's (m, reference, S, S1)
    // (m, reference, S, S1) of the first `n` entries, in lanes; every lane gets all of it
    auto join = [&](const float4* entry, int n) {
        const float4 o = lane < n ? entry[lane] : make_float4(-INFINITY, -INFINITY, 0.0f, 0.0f);
        const float m = warp_max_nan(o.x), ref = warp_max(o.y);
        float s = ds_move(o.z, o.y, ref, c), s1 = TWO ? ds_move(o.w, o.y, ref, c1) : 0.0f;
#pragma unroll
        for (int d = kMaxCluster / 2; d > 0; d >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, d);
            if (TWO) s1 += __shfl_xor_sync(0xffffffffu, s1, d);
        }
        return make_float4(m, ref, __shfl_sync(0xffffffffu, s, 0), TWO ? __shfl_sync(0xffffffffu, s1, 0) : 0.0f);
    };
    if (cluster > 1) cluster_wait();  // (they have started)
    if (warp == 0) {
        const float4 all = join(t.warp, S / 32);
        if (lane < cluster) peer_store(peer_address(&t.part[0][rank], lane), all);
    }
    auto meet = [&]() {
        if (cluster > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
    };
    meet();
    const float4 all = join(t.part[0], cluster);
    const float m = all.x, ref = all.y;
    float s = all.z, s1 = all.w;
    int kind = t.flags ? kDsBad : t.taught || t.labelled ? kDsRow : kDsSkip, flags = t.flags;
    if (kind == kDsRow && !usable(m)) flags = S4C_SEQ_NONFINITE, kind = kDsBad;
    if (usable(m) && (!(fabsf(m) < 1e37f) || !(fabsf(m * c) < 1e8f) || !(fabsf(m * c1) < 1e8f))) {
        // a product's rounding is worth powers of two, or leaves float32: sums by differences against the maximum
        s = s1 = 0.0f;
        if (!teacher)
            mine.look([&](int, const auto& v) {
                for (int k = 0; k < (int)(sizeof(v) / sizeof(uint4)); ++k) {
                    float x[Vec<T>::E];
                    Vec<T>::unpack(v[k], x);
#pragma unroll
                    for (int j = 0; j < Vec<T>::E; ++j) s += exp2_fast((x[j] - m) * c), s1 += exp2_fast((x[j] - m) * c1);
                }
            }, false);
        s = warp_sum(s), s1 = warp_sum(s1);
        if (lane == 0 && !teacher) t.warp[warp] = make_float4(s, s1, 0.0f, 0.0f);
        __syncthreads();
        s = s1 = 0.0f;
        for (int w = 0; w < S / 32; ++w) s += t.warp[w].x, s1 += t.warp[w].y;
        if (tid < cluster) peer_store(peer_address(&t.part[1][rank], tid), make_float4(s, s1, 0.0f, 0.0f));
        meet();
        s = s1 = 0.0f;
        for (int b = 0; b < cluster; ++b) s += t.part[1][b].x, s1 += t.part[1][b].y;
    } else {
        // against the maximum itself
        s *= exp2_fast((float)((double)__fmul_rn(ref, c) - (double)m * c));
        s1 = TWO ? s1 * exp2_fast((float)((double)__fmul_rn(ref, c1) - (double)m * c1)) : s;
    }
    const float inv_s = t.taught ? 1.0f / s : 0.0f, inv_s1 = t.labelled ? 1.0f / s1 : 0.0f;

    if (RES && teacher) asked.learn(p, row, share, t);
    if (rank == 0 && teacher) {
        float part = 0.0f;  // entry j: q (ln q - ln p); the label: -ln p1
        if (kind == kDsRow) {
            const float ln_s = ln_series(s);
            for (int j = lane; j < p.K; j += 32)
                if (t.q[j] > 0.0f) part += (float)(p.w_teach * t.q[j] * (t.log_q[j] - (((double)t.x[j] - m) * p.inv_tau - ln_s)));
            if (lane == 0 && t.labelled) part += (float)(p.w_label * (ln_series(s1) - ((double)t.x[p.K] - m)));
        }
        part = warp_sum(part);
        if (lane == 0) {
            p.loss[r] = kind == kDsBad ? NAN : part;
            if (p.stats) reinterpret_cast<float4*>(p.stats)[r] = kind == kDsRow ? make_float4(m, inv_s, inv_s1, kind) : make_float4(0, 0, 0, kind);
            if (p.status) p.status[r] = flags;
        }
    }
    if (!p.grad) return;
    T* g = static_cast<T*>(p.grad) + (long long)r * p.grad_stride;
    const float gs = p.row_scale ? p.row_scale[r] : 1.0f;
    const DsCoefs k = {m, gs * p.g_teach * inv_s, gs * p.w_label * inv_s1, gs * p.g_teach, gs * p.w_label};
    if (!teacher) ds_dense<S>(p, g, row, share, k, kind, [&](auto f) { mine.look(f, false); });
    __syncthreads();
    if (kind == kDsRow) ds_sparse(p, g, t, k);
}

template <typename T, int S, int BLOCKS>
__global__ void __launch_bounds__(S + 32, BLOCKS)
distill_backward_kernel(const DsParams p, int blocks, int per) {
    __shared__ DsShared t;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int r = blockIdx.x / blocks, rank = blockIdx.x - r * blocks;
    const Row<T> row(const_cast<T*>(static_cast<const T*>(p.logits)) + (long long)r * p.stride, p.V);
    const Share share(row.n, rank, per);
    const DsSlice<T, S, false> mine{row, share, nullptr};
    T* g = static_cast<T*>(p.grad) + (long long)r * p.grad_stride;
    const float4 st = reinterpret_cast<const float4*>(p.stats)[r];
    const float gs = p.row_scale[r];
    const DsCoefs k = {st.x, gs * p.g_teach * st.y, gs * p.w_label * st.z, gs * p.g_teach, gs * p.w_label};
    const int kind = (int)st.w;
    const bool in_place = p.grad == p.logits;  // the teacher's look at the logits comes before their gradient then
    if (threadIdx.x >= S) {
        ds_teach(p, r, row, share, t);
    }
    if (in_place) __syncthreads();
    if (threadIdx.x < S) ds_dense<S>(p, g, row, share, k, kind, [&](auto f) { mine.look(f, false); });
    __syncthreads();
    if (kind == kDsRow) ds_sparse(p, g, t, k);
}

template <typename T, int P>
static s4c_status ds_forward(const DsParams& p, long long rows, cudaStream_t stream) {
    const long long n = ((long long)p.V * (long long)sizeof(T) + 15) / 16 + 1;  // vectors, wherever a row starts
    if (n <= (rows > kSMs ? kDsShortRow : kDsShortFew))
        return row_launch(distill_kernel<T, P, true, kDsShort, kDsShortBlocks>, p, rows, 1, (int)n, kDsShort + 32, (size_t)n * 16, stream);
    // few rows are shared out to blocks with an SM of their own
    const long long spare = std::min(kSMs / rows, n / 512);
    if (p.grad) {
        const int cluster = (int)std::min((long long)kMaxCluster, std::max((n + kDsSlice - 1) / kDsSlice, 4 * spare)), per = (int)((n + cluster - 1) / cluster);
        const size_t smem = (size_t)per * 16;
        if (smem <= kMaxRowSmem)
            return row_launch(distill_kernel<T, P, true, kDsKept, kDsKeptBlocks>, p, rows, cluster, per, kDsKept + 32, smem, stream);
    }
    // the loss alone, and rows that eight blocks cannot keep (the second look at them comes from L2, or memory)
    const int cluster = (int)std::max(1ll, std::min((long long)kMaxCluster, p.grad ? kMaxCluster : spare));
    return row_launch(distill_kernel<T, P, false, kDsStreamed, kDsStreamedBlocks>, p, rows, cluster, (int)((n + cluster - 1) / cluster), kDsStreamed + 32, 0,
                      stream);
}
template <typename T>
static s4c_status ds_forward(const DsParams& p, long long rows, cudaStream_t stream) {
    return p.power == kDsOne      ? ds_forward<T, kDsOne>(p, rows, stream)
           : p.power == kDsSquare ? ds_forward<T, kDsSquare>(p, rows, stream)
           : p.power == kDsFourth ? ds_forward<T, kDsFourth>(p, rows, stream)
                                  : ds_forward<T, kDsTwo>(p, rows, stream);
}
template <typename T>
static s4c_status ds_backward(const DsParams& p, long long rows, cudaStream_t stream) {
    const long long n = ((long long)p.V * (long long)sizeof(T) + 15) / 16 + 1;
    if (n <= (rows > kSMs ? kDsShortRow : kDsShortFew)) return row_launch(distill_backward_kernel<T, kDsShort, kDsShortBlocks>, p, rows, 1, (int)n, kDsShort + 32, 0, stream, false);
    const int blocks = (int)((n + kDsSlice - 1) / kDsSlice);
    return row_launch(distill_backward_kernel<T, kDsStreamed, kDsStreamedBlocks>, p, rows, blocks, (int)((n + blocks - 1) / blocks), kDsStreamed + 32, 0, stream,
                      false);
}

// The rows of two arrays as byte ranges: whether they share any, unless they are the same rows.
static bool ds_overlaps(const void* a, long long a_stride, const void* b, long long b_stride, long long R, long long V, size_t size) {
    if (a == b && a_stride == b_stride) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + ((R - 1) * a_stride + V) * size, b1 = b0 + ((R - 1) * b_stride + V) * size;
    return a0 < b1 && b0 < a1;
}

static s4c_status ds_check(const void* logits, long long row_stride, const int32_t* teacher_token, const float* teacher_logit, int K, int R, int V,
                           s4c_dtype dt, float temperature, float teacher_weight, float label_weight, const void* grad, long long grad_stride) {
    if (!logits || (K > 0 && (!teacher_token || !teacher_logit))) return S4C_ERR_NULL;
    if (R < 0 || R > S4C_MAX_LOGITS_ROWS || V < 1 || V > S4C_MAX_LOGITS_COLUMNS || row_stride < V || K < 0 || !(temperature > 0.0f) || !(temperature < 1e18f) ||
        !(kLog2E / temperature < INFINITY) || !(fabsf(teacher_weight) < INFINITY) || !(fabsf(label_weight) < INFINITY) ||
        (grad && (grad_stride < V || !(fabsf(teacher_weight * temperature) < INFINITY))))
        return S4C_ERR_SHAPE;
    if (dt != S4C_F32 && dt != S4C_BF16) return S4C_ERR_DTYPE;
    if (K > kDsMaxTeach) return S4C_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(logits) % dtype_size(dt) || reinterpret_cast<uintptr_t>(grad) % dtype_size(dt)) return S4C_ERR_ALIGN;
    if (grad && ds_overlaps(logits, row_stride, grad, grad_stride, R, V, dtype_size(dt))) return S4C_ERR_SHAPE;
    return S4C_OK;
}

static DsParams ds_params(const void* logits, long long row_stride, const int32_t* teacher_token, const float* teacher_logit, int K, const int32_t* labels, int V,
                          float temperature, float teacher_weight, float label_weight, const float* row_scale, void* grad, long long grad_stride) {
    DsParams p = {};
    p.logits = logits, p.stride = row_stride, p.teacher_token = teacher_token, p.teacher_logit = teacher_logit, p.V = V;
    p.K = teacher_weight == 0.0f ? 0 : K, p.labels = label_weight == 0.0f ? nullptr : labels;  // (a term without weight is not looked at)
    p.inv_tau = 1.0f / temperature, p.scale = kLog2E / temperature, p.scale1 = kLog2E;
    p.w_teach = (double)teacher_weight * temperature * temperature, p.g_teach = teacher_weight * temperature, p.w_label = label_weight;
    p.power = !p.labels || temperature == 1.0f ? kDsOne : temperature == 2.0f ? kDsSquare : temperature == 4.0f ? kDsFourth : kDsTwo;
    p.row_scale = row_scale, p.grad = grad, p.grad_stride = grad_stride;
    return p;
}

}  // namespace s4c

extern "C" s4c_status s4c_distill_topk(const void* logits, long long row_stride, const int32_t* teacher_token, const float* teacher_logit, int K,
                                       const int32_t* labels, int R, int V, s4c_dtype dt, float temperature, float teacher_weight, float label_weight,
                                       float* loss, float* stats, const float* row_scale, void* grad, long long grad_stride, int32_t* status,
                                       s4c_stream_t stream) {
    using namespace s4c;
    if (R == 0 && V >= 1) return S4C_OK;
    if (!loss) return S4C_ERR_NULL;
    const s4c_status bad = ds_check(logits, row_stride, teacher_token, teacher_logit, K, R, V, dt, temperature, teacher_weight, label_weight, grad, grad_stride);
    if (bad != S4C_OK) return bad;
    if (!aligned16(stats)) return S4C_ERR_ALIGN;
    DsParams p = ds_params(logits, row_stride, teacher_token, teacher_logit, K, labels, V, temperature, teacher_weight, label_weight, row_scale, grad, grad_stride);
    p.loss = loss, p.stats = stats, p.status = status;
    return dt == S4C_F32 ? ds_forward<float>(p, R, static_cast<cudaStream_t>(stream))
                         : ds_forward<__nv_bfloat16>(p, R, static_cast<cudaStream_t>(stream));
}

extern "C" s4c_status s4c_distill_topk_backward(const void* logits, long long row_stride, const int32_t* teacher_token, const float* teacher_logit, int K,
                                                const int32_t* labels, int R, int V, s4c_dtype dt, float temperature, float teacher_weight,
                                                float label_weight, const float* stats, const float* grad_loss, void* grad, long long grad_stride,
                                                s4c_stream_t stream) {
    using namespace s4c;
    if (R == 0 && V >= 1) return S4C_OK;
    if (!stats || !grad_loss || !grad) return S4C_ERR_NULL;
    const s4c_status bad = ds_check(logits, row_stride, teacher_token, teacher_logit, K, R, V, dt, temperature, teacher_weight, label_weight, grad, grad_stride);
    if (bad != S4C_OK) return bad;
    if (!aligned16(stats)) return S4C_ERR_ALIGN;
    DsParams p = ds_params(logits, row_stride, teacher_token, teacher_logit, K, labels, V, temperature, teacher_weight, label_weight, grad_loss, grad, grad_stride);
    p.stats = const_cast<float*>(stats);
    return dt == S4C_F32 ? ds_backward<float>(p, R, static_cast<cudaStream_t>(stream))
                         : ds_backward<__nv_bfloat16>(p, R, static_cast<cudaStream_t>(stream));
}
