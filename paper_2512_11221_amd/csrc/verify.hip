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
// apart.  Exponentials and sums are 64-bit, so that they do not hang on the order of summation.
//
// Launches: the sums of every row of logits, in parts of at most 64 to a row, and the walk, a workgroup to a
// sequence, which also draws the next token: the parts' sums say which part holds the drawn point, and
// only that one is read again.  Where the walk ends behind a rejection with draft probabilities the
// weights are other ones, whose sums a third launch forms.
#include "kernels.h"
#include "tiles.h"

namespace asrkf {
namespace {

constexpr int kThreads = 256;

// 2^x for x <= 0, to 3e-15 of it: the nearest integer apart, the exponential's series on |y| <= ln 2 / 2.
__device__ __forceinline__ double exp2_64(double x) {
    x = fmax(x, -1080.0);                         // below: 0 (subnormals do not matter here); a NaN:
    const double k = rint(x);                     //   the caller's, who adds x to the sum
    const double y = (x - k) * 0.693147180559945309417;
    double r = fma(y, 1.0 / 39916800.0, 1.0 / 3628800.0);
    r = fma(y, r, 1.0 / 362880.0);
    r = fma(y, r, 1.0 / 40320.0);
    r = fma(y, r, 1.0 / 5040.0);
    r = fma(y, r, 1.0 / 720.0);
    r = fma(y, r, 1.0 / 120.0);
    r = fma(y, r, 1.0 / 24.0);
    r = fma(y, r, 1.0 / 6.0);
    r = fma(y, r, 0.5);
    r = fma(y, r, 1.0);
    r = fma(y, r, 1.0);
    return __builtin_ldexp(r, (int)k);
}

__device__ __forceinline__ double shfl_xor(double x, int o) {
    const unsigned long long b = __double_as_longlong(x);
    const unsigned lo = __shfl_xor((unsigned)b, o), hi = __shfl_xor((unsigned)(b >> 32), o);
    return __longlong_as_double(((unsigned long long)hi << 32) | lo);
}
__device__ __forceinline__ double shfl_up(double x, int o) {
    const unsigned long long b = __double_as_longlong(x);
    const unsigned lo = __shfl_up((unsigned)b, o), hi = __shfl_up((unsigned)(b >> 32), o);
    return __longlong_as_double(((unsigned long long)hi << 32) | lo);
}

__device__ __forceinline__ double wave_sum(double x) {
    for (int o = 1; o < 64; o <<= 1) x += shfl_xor(x, o);
    return x;
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

// A workgroup's part: its maximum first, over the values it holds in registers, then the sum with one
// exponential to a value.
__global__ void __launch_bounds__(kThreads)
verify_sums_kernel(VerifyArgs a) {
    constexpr int kWaves = kThreads / 64, kQuads = 4;
    __shared__ float top_lds[2][kWaves];
    __shared__ int at_lds[2][kWaves];
    __shared__ double sum_lds[kWaves];
    const int sp = blockIdx.x, row = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (row > nodes_of(a, b)) return;
    const float* x = row_of(a, b, row);
    const int i0 = sp * a.part_len, i1 = min(a.V, i0 + a.part_len);
    float m = -INFINITY;
    int at = kNone;
    double S = 0.0;                               // the thread's own values, against m
    bool bad = false;
    for (int j = i0, turn = 0; j < i1; j += kThreads * kQuads * 4, ++turn) {
        floatx4 v[kQuads];
#pragma unroll
        for (int u = 0; u < kQuads; ++u) v[u] = load4(x, j + (u * kThreads + threadIdx.x) * 4, i1, -INFINITY);
        float top = -INFINITY;
        int where = kNone;
#pragma unroll
        for (int u = 0; u < kQuads; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bad |= !(v[u][e] < INFINITY);
                if (v[u][e] > top) {              // the first of equals
                    top = v[u][e];
                    where = j + (u * kThreads + (int)threadIdx.x) * 4 + e;
                }
            }
        for (int o = 1; o < 64; o <<= 1) {
            const float y = __shfl_xor(top, o);
            const int z = __shfl_xor(where, o);
            where = y > top ? z : y == top ? min(where, z) : where;
            top = fmaxf(top, y);
        }
        if (lane == 0) {
            top_lds[turn & 1][wave] = top;
            at_lds[turn & 1][wave] = where;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float y = top_lds[turn & 1][w];
            const int z = at_lds[turn & 1][w];
            where = y > top ? z : y == top ? min(where, z) : where;
            top = fmaxf(top, y);
        }
        if (top > m) {
            S = m == -INFINITY ? 0.0 : S * exp2_64(((double)m - top) * a.inv_t);
            m = top;
            at = where;
        }
        if (a.inv_t != 0.0 && m > -INFINITY && m < INFINITY) {
#pragma unroll
            for (int u = 0; u < kQuads; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) S += v[u][e] == -INFINITY ? 0.0 : exp2_64(((double)v[u][e] - m) * a.inv_t);
        }
    }
    S = wave_sum(S);
    if (lane == 0) sum_lds[wave] = S;
    const bool any_bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        S = 0.0;
        for (int w = 0; w < kWaves; ++w) S += sum_lds[w];
        a.part[((size_t)b * (a.N + 1) + row) * a.split + sp] = VerifyPart{S, m, any_bad ? -1 : at};
    }
}

// ---- the walk and the draw ----

// e^((x - m) / T) scale - c q of a token, not below 0
__device__ __forceinline__ double weight_of(float x, float m, double inv_t, double scale, double c, double q) {
    return fmax(x == -INFINITY ? -c * q : exp2_64(((double)x - m) * inv_t) * scale - c * q, 0.0);
}

// The weights behind a row, and what a workgroup does with a range of them.
template <int THREADS>
struct Weights {
    static constexpr int kWaves = THREADS / 64;
    const float* x;
    const float* q;               // null: c is 0
    float m;
    double inv_t, scale, c;
    const int* gone;              // LDS: tokens without weight
    int n_gone;
    double* lds;                  // [kWaves + 1]
    int* found;                   // LDS, [2]

    __device__ __forceinline__ double of(int v, float xv, float qv) const {
        double w = weight_of(xv, m, inv_t, scale, c, (double)qv);
        for (int i = 0; i < n_gone; ++i) w = gone[i] == v ? 0.0 : w;
        return w;
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
    // of [i0, i1), in every thread
    __device__ __forceinline__ double sum(int i0, int i1) const {
        constexpr int kQuads = 2;
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
            for (int u = 0; u < kQuads; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) s += of(j + (u * THREADS + threadIdx.x) * 4 + e, xv[u][e], qv[u][e]);
        }
        return block_sum(s);
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
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = of(v + e, xv[e], qv[e]);
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
        double run = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const double y = shfl_up(run, o);
            if (lane >= o) run += y;
        }
        __syncthreads();
        if (lane == 63) lds[wave] = run;
        __syncthreads();
        for (int w = 0; w < wave; ++w) run += lds[w];
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
        if (first != kNone) atomicMin(&found[0], first);
        if (last >= 0) atomicMax(&found[1], last);
        __syncthreads();
        return found[0] != kNone ? found[0] : found[1];
    }
};

// The part that holds the point u W, from the parts' sums, one to a lane: the first whose running sum
// passes it; beyond the end (a random number of 1 and more) the last of any weight; -1 without weights.
// left: what is still to go within it.
__device__ __forceinline__ int part_of_point(double s, double u, double& left) {
    const int lane = threadIdx.x & 63;
    double run = s;
    for (int o = 1; o < 64; o <<= 1) {
        const double y = shfl_up(run, o);
        if (lane >= o) run += y;
    }
    double W = run;                               // the last lane's
    for (int o = 1; o < 64; o <<= 1) W = fmax(W, shfl_xor(W, o));
    const double point = u * W;
    const uint64_t past = __ballot(run > point), some = __ballot(s > 0.0);
    const int at = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : -1;
    const double rest = point - (run - s);
    const unsigned long long bits = __double_as_longlong(rest);
    const int from = max(at, 0);
    left = __longlong_as_double(((unsigned long long)(unsigned)__shfl((int)(bits >> 32), from) << 32) | (unsigned)__shfl((int)bits, from));
    return at;
}

constexpr int kWalkThreads = 1024;

__global__ void __launch_bounds__(kWalkThreads)
verify_walk_kernel(VerifyArgs a) {
    __shared__ VerifyPart rows[kMaxDrafts + 1];
    __shared__ double sums[kWalkThreads / 64];
    __shared__ int gone[kMaxDrafts], found[2];
    const int b = blockIdx.x, nodes = nodes_of(a, b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // a node to a lane, in every wave
    int parent = -2, token = -1;                  // -2: nobody's child; a token below 0 weighs nothing
    float u = 0.f;
    if (lane < nodes) {
        const int p = a.parents[(size_t)b * a.N + lane], x = a.tokens[(size_t)b * a.N + lane];
        parent = p >= -1 && p < lane ? p : -2;
        token = (uint32_t)x < (uint32_t)a.V ? x : -1;
        if (a.inv_t != 0.0) u = a.u[(size_t)b * (a.N + 1) + lane];
    }
    float logit = -INFINITY, q_own = 1.f;
    if (parent >= -1 && token >= 0 && a.inv_t != 0.0) {
        logit = row_of(a, b, parent + 1)[token];
        if (a.probs) q_own = draft_row(a, b, parent + 1)[token];
    }
    for (int row = wave; row <= nodes; row += kWalkThreads / 64) {
        VerifyPart p{0.0, -INFINITY, kNone};
        if (lane < a.split) p = a.part[((size_t)b * (a.N + 1) + row) * a.split + lane];
        float m = p.m;
        int at = p.at;
        for (int o = 1; o < 64; o <<= 1) {
            const float y = __shfl_xor(m, o);
            const int z = __shfl_xor(at, o);
            // a part without distribution (-1) takes all
            at = min(at, z) < 0 ? -1 : y > m ? z : y == m ? min(at, z) : at;
            m = fmaxf(m, y);
        }
        double S = 0.0;
        if (a.inv_t != 0.0) S = wave_sum(p.m == -INFINITY || at < 0 ? 0.0 : p.S * exp2_64(((double)p.m - m) * a.inv_t));
        if (lane == 0) rows[row] = VerifyPart{S, m, m == -INFINITY ? -1 : at};
    }
    __syncthreads();
    double mass = 0.0;                            // p(x) behind the parent
    if (parent >= -1 && token >= 0 && a.inv_t != 0.0) {
        const VerifyPart p = rows[parent + 1];
        if (p.at >= 0) mass = weight_of(logit, p.m, a.inv_t, 1.0 / p.S, 0.0, 0.0);
    }
    const double q = q_own;

    auto of_lane = [&](double x, int i) __attribute__((always_inline)) {
        const unsigned long long bits = __double_as_longlong(x);
        return __longlong_as_double(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(bits >> 32), i) << 32) |
                                    (unsigned)__builtin_amdgcn_readlane((int)bits, i));
    };
    int last = -1, n_path = 0;
    double W = 1.0, c = 0.0, c_before = -1.0;     // w = max(p - c q, 0), W its sum
    uint64_t rejected = 0;                        // since the last one kept
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
                if (!yes && !a.probs) W -= w;
            }
        }
        if (yes) {
            if (threadIdx.x == 0) a.path[(size_t)b * a.N + n_path] = i;
            ++n_path;
            last = i;
            W = 1.0;
            c = 0.0;
            rejected = 0;
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
            const Weights<kWalkThreads> w{row_of(a, b, last + 1), draft_row(a, b, last + 1), p.m, a.inv_t, 1.0 / p.S, c2, gone, 0, sums, found};
            const double sum = w.sum(0, a.V);
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
    const int n_gone = a.probs ? 0 : __popcll(rejected);
    if (n_gone && wave == 0 && (rejected >> lane & 1)) gone[__popcll(rejected & ((1ull << lane) - 1ull))] = token;
    __syncthreads();
    const Weights<kWalkThreads> w{row_of(a, b, last + 1), nullptr, p.m, a.inv_t, 1.0 / p.S, 0.0, gone, n_gone, sums, found};
    double s = 0.0;
    if (lane < a.split) {
        const VerifyPart mine = a.part[((size_t)b * (a.N + 1) + last + 1) * a.split + lane];
        if (mine.m > -INFINITY) s = mine.S * exp2_64(((double)mine.m - p.m) * a.inv_t) * w.scale;
    }
    uint64_t again = 0;                           // parts that hold a rejected token: summed without it
    for (int i = 0; i < n_gone; ++i) again |= 1ull << (gone[i] / a.part_len);
    for (; again; again &= again - 1) {
        const int sp = __builtin_ctzll(again);
        const double sum = w.sum(sp * a.part_len, min(a.V, (sp + 1) * a.part_len));
        if (lane == sp) s = sum;
    }
    double left;
    const int sp = part_of_point(s, (double)a.u[(size_t)b * (a.N + 1) + a.N], left);
    const int tok = sp < 0 ? -1 : w.find(sp * a.part_len, min(a.V, (sp + 1) * a.part_len), left);
    if (threadIdx.x == 0) a.next[b] = tok;
}

// ---- the draw from what a rejection has left ----

__global__ void __launch_bounds__(kThreads)
verify_rest_kernel(VerifyArgs a) {
    __shared__ double lds[kThreads / 64];
    __shared__ int last_arrival, found[2];
    const int sp = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63;
    const VerifyEnd e = a.end[b];
    if (e.row < 0) return;
    Weights<kThreads> w{row_of(a, b, e.row), draft_row(a, b, e.row), e.m, a.inv_t, e.scale, e.c, nullptr, 0, lds, found};
    {
        const double sum = w.sum(sp * a.part_len, min(a.V, (sp + 1) * a.part_len));
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
    const double u = a.u[(size_t)b * (a.N + 1) + a.N];
    const double s = lane < a.split ? __hip_atomic_load(a.sums + (size_t)b * a.split + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
    double left;
    const int part = part_of_point(s, u, left);
    int i0 = part * a.part_len, i1 = min(a.V, (part + 1) * a.part_len);
    if (part < 0) {
        // nothing is left by the last rejection, which then changes nothing: the whole row with
        // the weights before it
        w.c = e.c_before;
        left = u * w.sum(0, a.V);
        i0 = 0;
        i1 = a.V;
    }
    const int tok = w.find(i0, i1, left);
    if (threadIdx.x == 0) a.next[b] = tok;
}

}  // namespace

// Parts of 4096 logits, as many as a workgroup's threads hold in registers; longer ones for
// vocabularies of more than 64 such parts.
int verify_part_len(int V) {
    const int most = kVerifySplitMax * 4096;
    return 4096 * ((V + most - 1) / most);
}

hipError_t launch_verify(const VerifyArgs& args, hipStream_t s) {
    VerifyArgs a = args;
    a.part_len = verify_part_len(a.V);
    a.split = (a.V + a.part_len - 1) / a.part_len;
    hipLaunchKernelGGL(verify_sums_kernel, dim3(a.split, a.N + 1, a.B), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_walk_kernel, dim3(a.B), dim3(kWalkThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess || !a.probs) return e;
    hipLaunchKernelGGL(verify_rest_kernel, dim3(a.split, a.B), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
