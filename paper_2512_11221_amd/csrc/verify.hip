// Verification of drafted tokens against the target's logits, from given random numbers.
//
// p = softmax(logits / T) behind a sequence's last token (the root) and behind each of its nodes.  The
// walk starts at the root and looks at the nodes in their order; one whose parent is the last
// accepted node, with token x, is accepted where
//     u q(x) W < w(x),   W = sum w,
// w = p at first.  Without draft probabilities q = 1 and a rejection sets w(x) = 0.  With them (row
// q of the parent) a rejection makes w = max(w / W - q, 0).  That has a closed form: after
// rejections w is max(p - c q, 0) up to a factor, with c the sum of the W so far (c' = c + W), since
//     max(p - c q, 0) / W - q = (p - (c + W) q) / W   where that is positive.
// So the state of a walk is three numbers and no vector.  Where nothing would remain, w stays.  The
// next token is the first whose running sum of w, in the vocabulary's order, passes u W.
// Greedy (T = 0): a node is accepted where its token has the largest logit, the lowest index among
// equals, and the next token is the one with the largest.
// Accepted or not, and which token: decisions on sums over a vocabulary whose neighbours lie 10^-6
// apart.  Exponentials (to 4e-14 of themselves) and sums are 64-bit, so that they do not hang on the order of summation.
//
// Launches: the sums of every row of logits, in parts of at most 64 to a row, and the walk, a workgroup to a
// sequence, which also draws the next token: the parts' sums say which part holds the drawn point, and
// only that one is read again.  The sums of 399 rows of 50257 logits (32 sequences of 9 to 17) take 22.1 us (3.6 TB/s; the
// 64-bit operations alone are 12 at the vector units' rate), of 48 rows of 128256 9.0; the walk, bound by round trips, 9 to
// 10.  Where the walk ends behind a rejection with draft probabilities the weights are other ones, whose sums a third
// launch forms; where such a rejection has a sibling to look at, the walk's workgroup forms them alone, 24 us a
// rejection over 128256 tokens.
#include "kernels.h"
#include "tiles.h"

namespace asrkf {
namespace {

constexpr int kThreads = 256;

// 2^x for x <= 0: 2^k (1 + f P(f)), k the nearest integer and f = x - k.  P interpolates (2^f - 1) / f at the
// nine Chebyshev nodes of [-1/2, 1/2], which leaves 3.7e-14 of the result; 2^0 is 1.  Below -1080,
// and at -infinity, it is 0.
__device__ __forceinline__ double exp2_64(double x) {
    x = fmax(x, -1080.0);
    const double k = rint(x), f = x - k;
    double r = 1.0203121063391729e-07;
    r = fma(r, f, 1.3255224878668817e-06);
    r = fma(r, f, 1.525268684626772e-05);
    r = fma(r, f, 0.00015403455852453838);
    r = fma(r, f, 0.0013333558179043112);
    r = fma(r, f, 0.009618129159402558);
    r = fma(r, f, 0.055504108664760424);
    r = fma(r, f, 0.2402265069581299);
    r = fma(r, f, 0.6931471805599453);
    r = fma(r, f, 1.0);
    return __builtin_ldexp(r, (int)k);
}
// e^((x - m) / T), inv_t = log2(e) / T.  The difference first: of products that are rounded each, what is left would be
// off by 2^-53 of m / T, which is 10^-9 of logits near 30 at T = 10^-6, and another factor in every part with a maximum of its own.
__device__ __forceinline__ double exp_of(float x, double inv_t, double m) { return exp2_64(((double)x - m) * inv_t); }

// Sums over a wave's lanes in six DPP steps: within rows of 16, then the rows before.  (Each is a
// few cycles where a permute through LDS is a round trip: the walk of 8 chains took 16.6 us with those.)
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double x) {
    const unsigned long long b = __double_as_longlong(x);
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xF, false);
    const unsigned hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xF, false);
    return __longlong_as_double(((unsigned long long)hi << 32) | lo);
}
__device__ __forceinline__ double running_sum(double x) {
    x += moved<0x111, 0xF>(x);                    // row_shr 1, 2, 4, 8: zeros come in
    x += moved<0x112, 0xF>(x);
    x += moved<0x114, 0xF>(x);
    x += moved<0x118, 0xF>(x);
    x += moved<0x142, 0xA>(x);                    // row_bcast 15 into rows 1 and 3
    x += moved<0x143, 0xC>(x);                    // row_bcast 31 into rows 2 and 3
    return x;
}
__device__ __forceinline__ double of_lane(double x, int i) {
    const unsigned long long b = __double_as_longlong(x);
    return __longlong_as_double(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(b >> 32), i) << 32) |
                                (unsigned)__builtin_amdgcn_readlane((int)b, i));
}
__device__ __forceinline__ double wave_sum(double x) { return of_lane(running_sum(x), 63); }

template <int CTRL, int ROWS>
__device__ __forceinline__ float max_moved(float x) {
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(x), __float_as_int(x), CTRL, ROWS, 0xF, false)));
}
__device__ __forceinline__ float wave_max(float x) {
    x = max_moved<0x111, 0xF>(x);
    x = max_moved<0x112, 0xF>(x);
    x = max_moved<0x114, 0xF>(x);
    x = max_moved<0x118, 0xF>(x);
    x = max_moved<0x142, 0xA>(x);
    x = max_moved<0x143, 0xC>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int min_moved(int x) {
    return min(x, __builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ int wave_min(int x) {
    x = min_moved<0x111, 0xF>(x);
    x = min_moved<0x112, 0xF>(x);
    x = min_moved<0x114, 0xF>(x);
    x = min_moved<0x118, 0xF>(x);
    x = min_moved<0x142, 0xA>(x);
    x = min_moved<0x143, 0xC>(x);
    return __builtin_amdgcn_readlane(x, 63);
}

constexpr int kNone = 0x7FFFFFFF;

__device__ __forceinline__ int nodes_of(const VerifyArgs& a, int b) {
    return a.count ? min(max(a.count[b], 0), a.N) : a.N;
}
// row 0: the root's, 1 + i: node i's
__device__ __forceinline__ const float* row_of(const VerifyArgs& a, int b, int row) {
    return row == 0 ? a.root + (size_t)b * a.V : a.logits + ((size_t)b * a.N + row - 1) * a.V;
}
__device__ __forceinline__ const float* draft_row(const VerifyArgs& a, int b, int row) {
    return a.probs + ((size_t)b * a.N + row) * a.V;
}

// Four values from any address, `fill` past the end.
__device__ __forceinline__ floatx4 load4(const float* x, int i, int end, float fill) {
    typedef float loose4 __attribute__((ext_vector_type(4), aligned(4)));
    floatx4 r = {fill, fill, fill, fill};
    if (i + 3 < end) {
        const loose4 v = *reinterpret_cast<const loose4*>(x + i);
        r = floatx4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (i + e < end) r[e] = x[i + e];
    }
    return r;
}

// ---- the sums of every row ----

// A workgroup's part: its maximum first, over the values it holds in registers, then (greedy) that
// maximum's first index, or the sum with one exponential to a value.
template <bool GREEDY>
__global__ void __launch_bounds__(kThreads)
verify_sums_kernel(VerifyArgs a) {
    constexpr int kWaves = kThreads / 64, kQuads = 4;
    __shared__ float top_lds[2][kWaves];
    __shared__ double sum_lds[kWaves];
    __shared__ int at_lds[kWaves], bad_lds[kWaves];
    const int sp = blockIdx.x, row = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nodes = nodes_of(a, b);
    if (row > nodes) return;
    const float* x = row_of(a, b, row);
    const int i0 = sp * a.part_len, i1 = min(a.V, i0 + a.part_len);
    int child = -1;                               // the token of a child of this row, a node to a lane of wave 0
    if (!GREEDY && wave == 0 && lane < nodes) {
        const int parent = a.parents[(size_t)b * a.N + lane], token = a.tokens[(size_t)b * a.N + lane];
        if (parent + 1 == row && lane >= row) child = token;
    }
    float m = -INFINITY;
    int at = kNone;
    double S = 0.0;                               // the thread's own values, against m
    bool bad = false;
    for (int j = i0, turn = 0; j < i1; j += kThreads * kQuads * 4, ++turn) {
        floatx4 v[kQuads];
#pragma unroll
        for (int u = 0; u < kQuads; ++u) v[u] = load4(x, j + (u * kThreads + threadIdx.x) * 4, i1, -INFINITY);
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < kQuads; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bad |= !(v[u][e] < INFINITY);
                top = fmaxf(top, v[u][e]);
            }
        top = wave_max(top);
        if (lane == 0) top_lds[turn & 1][wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, top_lds[turn & 1][w]);
        if (top > m) {
            if (!GREEDY && m > -INFINITY) S *= exp2_64(((double)m - top) * a.inv_t);
            m = top;
            at = kNone;
        }
        if constexpr (GREEDY) {
#pragma unroll
            for (int u = 0; u < kQuads; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (v[u][e] == m && top == m) at = min(at, j + (u * kThreads + (int)threadIdx.x) * 4 + e);
        } else if (m > -INFINITY && m < INFINITY) {
#pragma unroll
            for (int u = 0; u < kQuads; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) S += exp_of(v[u][e], a.inv_t, m);
        }
    }
    // what the walk looks up: the logit and the draft's probability of the children in this part
    if (!GREEDY && child >= i0 && child < i1)
        a.chance[(size_t)b * a.N + lane] = make_float2(x[child], a.probs ? draft_row(a, b, row)[child] : 1.f);
    if constexpr (GREEDY) at = wave_min(at);
    else S = wave_sum(S);
    const bool wave_bad = __any(bad);
    if (lane == 0) {
        sum_lds[wave] = S;
        at_lds[wave] = at;
        bad_lds[wave] = wave_bad;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        S = 0.0;
        int any_bad = 0;
        for (int w = 0; w < kWaves; ++w) {
            S += sum_lds[w];
            at = min(at, at_lds[w]);
            any_bad |= bad_lds[w];
        }
        a.part[((size_t)b * (a.N + 1) + row) * a.split + sp] = VerifyPart{S, m, any_bad ? -1 : at};
    }
}

// ---- the walk and the draw ----

// The weights max(e^((x - m) / T) scale - c q, 0) behind a row, and what a workgroup does with a range of them.
template <int THREADS>
struct Weights {
    static constexpr int kWaves = THREADS / 64;
    const float* x;
    const float* q;               // null: c is 0
    double inv_t, m, scale, c;
    int n_gone, gone;             // tokens without weight, one to a lane
    double* lds;                  // [kWaves]
    int* found;                   // LDS, [2]

    // of four tokens from v on
    __device__ __forceinline__ void four(floatx4 xv, floatx4 qv, double (&w)[4]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = exp_of(xv[e], inv_t, m) * scale;
            if (q) w[e] = fmax(w[e] - c * (double)qv[e], 0.0);
        }
    }
    __device__ __forceinline__ void leave_out(int v, double (&w)[4]) const {
        for (int i = 0; i < n_gone; ++i) {
            const int g = __builtin_amdgcn_readlane(gone, i) - v;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = g == e ? 0.0 : w[e];
        }
    }
    __device__ __forceinline__ double block_sum(double s) const {
        s = wave_sum(s);
        __syncthreads();                          // lds may still be read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.0;
        for (int w = 0; w < kWaves; ++w) s += lds[w];
        return s;
    }
    // of [i0, i1), in every thread; kQuads quads of a thread in flight
    template <int kQuads>
    __device__ __forceinline__ double sum(int i0, int i1) const {
        double s = 0.0;
        for (int j = i0; j < i1; j += THREADS * kQuads * 4) {
            floatx4 xv[kQuads], qv[kQuads];
#pragma unroll
            for (int u = 0; u < kQuads; ++u) {
                const int i = j + (u * THREADS + threadIdx.x) * 4;
                xv[u] = load4(x, i, i1, -INFINITY);
                qv[u] = q ? load4(q, i, i1, 0.f) : floatx4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int u = 0; u < kQuads; ++u) {
                double w[4];
                four(xv[u], qv[u], w);
                leave_out(j + (u * THREADS + (int)threadIdx.x) * 4, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) s += w[e];
            }
        }
        return block_sum(s);
    }
    // ... in a wave alone, in its lanes
    __device__ __forceinline__ double wave_sum_of(int i0, int i1) const {
        constexpr int kQuads = 8;
        double s = 0.0;
        for (int j = i0; j < i1; j += 64 * kQuads * 4) {
            floatx4 xv[kQuads];
#pragma unroll
            for (int u = 0; u < kQuads; ++u) xv[u] = load4(x, j + (u * 64 + (int)(threadIdx.x & 63)) * 4, i1, -INFINITY);
#pragma unroll
            for (int u = 0; u < kQuads; ++u) {
                double w[4];
                four(xv[u], floatx4{0.f, 0.f, 0.f, 0.f}, w);
                leave_out(j + (u * 64 + (int)(threadIdx.x & 63)) * 4, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) s += w[e];
            }
        }
        return wave_sum(s);
    }
    // The first token of [i0, i1) whose running sum passes point; where rounding leaves none, the last
    // of any weight; -1 without weights.  In every thread.
    __device__ __forceinline__ int find(int i0, int i1, double point) const {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (threadIdx.x == 0) {
            found[0] = kNone;
            found[1] = -1;
        }
        // a run of neighbouring tokens per thread, in whole quads
        const int per = ((i1 - i0 + THREADS - 1) / THREADS + 3) / 4 * 4;
        const int v0 = min(i1, i0 + (int)threadIdx.x * per), v1 = min(i1, v0 + per);
        auto quad = [&](int v, double (&w)[4]) __attribute__((always_inline)) {
            const floatx4 xv = load4(x, v, v1, -INFINITY), qv = q ? load4(q, v, v1, 0.f) : floatx4{0.f, 0.f, 0.f, 0.f};
            four(xv, qv, w);
            leave_out(v, w);
        };
        double mine = 0.0, first4[4] = {0.0, 0.0, 0.0, 0.0};
        if (v0 < v1) quad(v0, first4);
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += first4[e];
        for (int v = v0 + 4; v < v1; v += 4) {
            double w[4];
            quad(v, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) mine += w[e];
        }
        double run = running_sum(mine);
        __syncthreads();
        if (lane == 63) lds[wave] = run;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) run += w < wave ? lds[w] : 0.0;
        double before = run - mine;
        int first = kNone, last = -1;
        for (int v = v0; v < v1; v += 4) {
            double w[4];
            if (v == v0) for (int e = 0; e < 4; ++e) w[e] = first4[e];
            else quad(v, w);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                before += w[e];
                if (w[e] > 0.0) last = v + e;
                if (before > point && w[e] > 0.0 && first == kNone) first = v + e;
            }
        }
        // a wave's first and last are its first and last lane's that have one
        const uint64_t firsts = __ballot(first != kNone), lasts = __ballot(last >= 0);
        if (firsts && lane == __builtin_ctzll(firsts)) atomicMin(&found[0], first);
        if (lasts && lane == 63 - __builtin_clzll(lasts)) atomicMax(&found[1], last);
        __syncthreads();
        return found[0] != kNone ? found[0] : found[1];
    }
};

// The part that holds the point u W, from the parts' sums, one to a lane: the first whose running sum
// passes it; beyond the end (a random number of 1 and more) the last of any weight; -1 without weights.
// left: what is still to go within it.
__device__ __forceinline__ int part_of_point(double s, double u, double& left) {
    const double run = running_sum(s);
    const double point = u * of_lane(run, 63);
    const uint64_t past = __ballot(run > point), some = __ballot(s > 0.0);
    const int at = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : -1;
    left = of_lane(point - (run - s), max(at, 0));
    return at;
}

constexpr int kWalkThreads = 1024;

__global__ void __launch_bounds__(kWalkThreads)
verify_walk_kernel(VerifyArgs a) {
    __shared__ VerifyPart rows[kMaxDrafts + 1];
    __shared__ double share[kMaxDrafts + 1][kVerifySplitMax];    // of a row's sum, by part
    __shared__ double sums[kWalkThreads / 64];
    __shared__ int gone_lds[kMaxDrafts], found[2];
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const VerifyPart* parts = a.part + (size_t)b * (a.N + 1) * a.split;
    // a node to a lane, in every wave
    int parent = -2, token = -1;                  // -2: nobody's child; a token below 0 weighs nothing
    float u = 0.f, u_last = 0.f;
    float2 chance = make_float2(-INFINITY, 1.f);  // its logit and the draft's probability
    if (lane < a.N) {                             // (all of the first loads go out before the count is here)
        parent = a.parents[(size_t)b * a.N + lane];
        token = a.tokens[(size_t)b * a.N + lane];
    }
    VerifyPart mine{0.0, -INFINITY, kNone};       // (the first of the wave's rows, asked for before the tokens are here)
    if (lane < a.split && wave <= a.N) mine = parts[wave * a.split + lane];
    if (a.inv_t != 0.0) {
        if (lane < a.N) {
            u = a.u[(size_t)b * (a.N + 1) + lane];
            chance = a.chance[(size_t)b * a.N + lane];
        }
        u_last = a.u[(size_t)b * (a.N + 1) + a.N];
    }
    const int nodes = nodes_of(a, b);
    parent = parent >= -1 && parent < lane && lane < nodes ? parent : -2;
    token = (uint32_t)token < (uint32_t)a.V ? token : -1;
    for (int row = wave; row <= nodes; row += kWalkThreads / 64) {
        VerifyPart p = mine;
        if (row != wave) {
            p = VerifyPart{0.0, -INFINITY, kNone};
            if (lane < a.split) p = parts[row * a.split + lane];
        }
        const float m = wave_max(p.m);
        const bool none = __any(p.at < 0) || m == -INFINITY;
        if (a.inv_t == 0.0) {
            const int at = wave_min(p.m == m ? p.at : kNone);
            if (lane == 0) rows[row] = VerifyPart{0.0, m, none ? -1 : at};
        } else {
            const double s = p.m == -INFINITY || none ? 0.0 : p.S * exp2_64(((double)p.m - m) * a.inv_t);
            const double S = wave_sum(s);
            share[row][lane] = s / S;
            if (lane == 0) rows[row] = VerifyPart{S, m, none ? -1 : 0};
        }
    }
    __syncthreads();
    double mass = 0.0;                            // p(x) behind the parent
    if (parent >= -1 && token >= 0 && a.inv_t != 0.0) {
        const VerifyPart p = rows[parent + 1];
        if (p.at >= 0) mass = exp_of(chance.x, a.inv_t, p.m) / p.S;
    }
    const double q = chance.y;

    // the tokens of those nodes, one to a lane
    auto left_out = [&](uint64_t which) __attribute__((always_inline)) {
        if (wave == 0 && (which >> lane & 1)) gone_lds[__popcll(which & ((1ull << lane) - 1ull))] = token;
        __syncthreads();
        return lane < __popcll(which) ? gone_lds[lane] : -1;
    };

    int last = -1, n_path = 0;
    double W = 1.0, c = 0.0, c_before = -1.0;     // w = max(p - c q, 0), W its sum
    double W_summed = 1.0;                        // the sum that W was last formed as, before differences
    uint64_t rejected = 0, weighed = 0;           // since the last one kept; those of them that had a weight
    uint64_t todo = ~0ull;                        // nodes not looked at yet
    for (;;) {                                    // (the same in every wave)
        const uint64_t next = __ballot(parent == last) & todo;
        if (!next) break;
        const int i = __builtin_ctzll(next);
        todo = i < 63 ? ~0ull << (i + 1) : 0;
        const VerifyPart p = rows[last + 1];
        const int x = __builtin_amdgcn_readlane(token, i);
        bool yes = false;
        if (p.at >= 0 && x >= 0) {
            if (a.inv_t == 0.0) {
                yes = x == p.at;
            } else {
                const double qi = of_lane(q, i);
                double w = of_lane(mass, i);
                if (a.probs) w = fmax(w - c * qi, 0.0);
                else if (__ballot(token == x) & rejected) w = 0.0;         // a rejected sibling's token
                yes = (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(u), i)) * qi * W < w;
                if (!yes && !a.probs) {
                    W -= w;
                    weighed |= w > 0.0 ? 1ull << i : 0;
                    // The difference is off by 10^-13 of the sum, as the exponentials are.  Where next to nothing
                    // is left and another sibling asks, it is summed again, so that the last token of any weight is kept.
                    if (W < W_summed * 0x1p-10 && (__ballot(parent == last) & todo)) {
                        const Weights<kWalkThreads> rest{row_of(a, b, last + 1), nullptr, a.inv_t, p.m, 1.0 / p.S, 0.0, (int)__popcll(weighed),
                                                         left_out(weighed), sums, found};
                        W = W_summed = rest.template sum<4>(0, a.V);
                    }
                }
            }
        }
        if (yes) {
            if (threadIdx.x == 0) a.path[(size_t)b * a.N + n_path] = i;
            ++n_path;
            last = i;
            W = W_summed = 1.0;
            c = 0.0;
            rejected = weighed = 0;
            continue;
        }
        if (x >= 0) rejected |= 1ull << i;
        if (a.probs && p.at >= 0) {
            const double c2 = c + W;
            if (!(__ballot(parent == last) & todo)) {
                c_before = c;                     // nobody asks for the sum: the draw finds it
                c = c2;
                break;
            }
            const Weights<kWalkThreads> w{row_of(a, b, last + 1), draft_row(a, b, last + 1), a.inv_t, p.m, 1.0 / p.S, c2, 0, 0, sums, found};
            const double sum = w.template sum<4>(0, a.V);
            if (sum > 0.0) {
                c = c2;
                W = sum;
            }
        }
    }
    for (int i = n_path + threadIdx.x; i < a.N; i += kWalkThreads) a.path[(size_t)b * a.N + i] = -1;
    const VerifyPart p = rows[last + 1];
    if (threadIdx.x == 0) {
        a.n_path[b] = n_path;
        if (a.inv_t == 0.0 || p.at < 0) a.next[b] = p.at;
        if (a.probs) a.end[b] = VerifyEnd{1.0 / p.S, c, c_before, p.m, p.at < 0 || c == 0.0 ? -1 : last + 1};
    }
    if (a.inv_t == 0.0 || p.at < 0 || c != 0.0) return;

    // the draw from p without the rejected tokens
    const int n_gone = __popcll(weighed), gone = n_gone ? left_out(weighed) : -1;
    const Weights<kWalkThreads> w{row_of(a, b, last + 1), nullptr, a.inv_t, p.m, 1.0 / p.S, 0.0, n_gone, gone, sums, found};
    const double whole = share[last + 1][lane];
    double s = whole;
    for (uint64_t left = weighed; left; left &= left - 1) {
        const int i = __builtin_ctzll(left), sp = __builtin_amdgcn_readlane(token, i) / a.part_len;
        s -= lane == sp ? of_lane(mass, i) : 0.0;
    }
    // a part of which next to nothing is left is summed again without those tokens, a wave to a part (what
    // the difference is off by, 10^-13 of the whole, stays below 10^-10 of what is left)
    const uint64_t again = __ballot(s < whole * 0x1p-10);
    if (again) {
        __syncthreads();                          // every wave has read the shares that are replaced
        int turn = 0;
        for (uint64_t left = again; left; left &= left - 1, ++turn) {
            if (turn % (kWalkThreads / 64) != wave) continue;
            const int sp = __builtin_ctzll(left);
            const double sum = w.wave_sum_of(sp * a.part_len, min(a.V, (sp + 1) * a.part_len));
            if (lane == 0) share[last + 1][sp] = sum;
        }
        __syncthreads();
        s = again >> lane & 1 ? share[last + 1][lane] : s;
    }
    double left;
    const int sp = part_of_point(s, (double)u_last, left);
    // no weight is left only where a random number of 1 and more rejected the last token that had one: it is
    // the next one
    const int tok = sp < 0 ? __builtin_amdgcn_readlane(token, 63 - __builtin_clzll(weighed | 1))
                           : w.find(sp * a.part_len, min(a.V, (sp + 1) * a.part_len), left);
    if (threadIdx.x == 0) a.next[b] = tok;
}

// ---- the draw from what a rejection has left ----

__global__ void __launch_bounds__(kWalkThreads)
verify_rest_kernel(VerifyArgs a) {
    __shared__ double lds[kWalkThreads / 64];
    __shared__ int last_arrival, found[2];
    const int sp = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63;
    const VerifyEnd e = a.end[b];
    const double u = a.u[(size_t)b * (a.N + 1) + a.N];
    if (e.row < 0) return;
    Weights<kWalkThreads> w{row_of(a, b, e.row), draft_row(a, b, e.row), a.inv_t, e.m, e.scale, e.c, 0, 0, lds, found};
    {
        const double sum = w.template sum<1>(sp * a.part_len, min(a.V, (sp + 1) * a.part_len));
        if (threadIdx.x == 0) {
            __hip_atomic_store(a.sums + (size_t)b * a.split + sp, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            // the store has completed before the ticket is taken
            __builtin_amdgcn_s_waitcnt(0);
            last_arrival = __hip_atomic_fetch_add(a.ticket + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.split - 1;
            if (last_arrival) a.ticket[b] = 0;    // ready for the next launch
        }
        __syncthreads();
        if (!last_arrival) return;
    }
    const double s = lane < a.split ? __hip_atomic_load(a.sums + (size_t)b * a.split + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    double left;
    const int part = part_of_point(s, u, left);
    int i0 = part * a.part_len, i1 = min(a.V, (part + 1) * a.part_len);
    if (part < 0) {
        // nothing is left by the last rejection, which then changes nothing: the whole row with
        // the weights before it
        w.c = e.c_before;
        left = u * w.template sum<2>(0, a.V);
        i0 = 0;
        i1 = a.V;
    }
    const int tok = w.find(i0, i1, left);
    if (threadIdx.x == 0) a.next[b] = tok;
}

}  // namespace

// Parts of 4096 logits, as many as a workgroup's threads hold in registers; longer ones for
// vocabularies of more than 64 such parts, which the walk takes one to a lane.
int verify_part_len(int V) {
    const int most = kVerifySplitMax * 4096;
    return 4096 * ((V + most - 1) / most);
}

hipError_t launch_verify(const VerifyArgs& args, hipStream_t s) {
    VerifyArgs a = args;
    a.part_len = verify_part_len(a.V);
    a.split = (a.V + a.part_len - 1) / a.part_len;
    const dim3 grid(a.split, a.N + 1, a.B);
    if (a.inv_t == 0.0) hipLaunchKernelGGL(verify_sums_kernel<true>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(verify_sums_kernel<false>, grid, dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_walk_kernel, dim3(a.B), dim3(kWalkThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess || !a.probs) return e;
    hipLaunchKernelGGL(verify_rest_kernel, dim3(a.split, a.B), dim3(kWalkThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
