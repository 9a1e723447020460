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
// Three launches: the sums of every row of logits in parts (bound by the bytes, or by the
// exponentials); the walk, a workgroup to a sequence; the draw, parts of the last row's weights,
// the part that holds the drawn point searched by the workgroup that arrives last.
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

// Two parts of a row as one.  A part without a logit has m = -inf, S = 0, at = kNone.
constexpr int kNone = 0x7FFFFFFF;
__device__ __forceinline__ VerifyPart merge(const VerifyPart& a, const VerifyPart& b, double inv_t) {
    VerifyPart r;
    if (a.at < 0 || b.at < 0) return VerifyPart{0.0, 0.f, -1};
    r.m = fmaxf(a.m, b.m);
    r.at = a.m > b.m ? a.at : b.m > a.m ? b.at : min(a.at, b.at);
    // (a part at the maximum keeps its sum; -inf - -inf is not formed)
    r.S = (a.m == r.m ? a.S : a.S * exp2_64(((double)a.m - r.m) * inv_t)) +
          (b.m == r.m ? b.S : b.S * exp2_64(((double)b.m - r.m) * inv_t));
    return r;
}
__device__ __forceinline__ VerifyPart from_lane(const VerifyPart& a, int o) {
    return VerifyPart{shfl_xor(a.S, o), __shfl_xor(a.m, o), __shfl_xor(a.at, o)};
}

__device__ __forceinline__ int nodes_of(const VerifyArgs& a, int b) {
    return a.count ? min(max(a.count[b], 0), a.N) : a.N;
}
// row 0: the root's, 1 + i: node i's
__device__ __forceinline__ const float* row_of(const VerifyArgs& a, int b, int row) {
    return row == 0 ? a.root + (size_t)b * a.V : a.logits + ((size_t)b * a.N + row - 1) * a.V;
}

// The logits [i0, i1) of a row that part sp of a.split takes; parts start 16-byte aligned but for the first.
struct Range { int head, i0, i1; };
__device__ __forceinline__ Range part_range(const float* x, int V, int sp, int split) {
    const int head = min(V, (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / 4);
    const int per = ((V - head) / 4 + split - 1) / split * 4;
    Range r;
    r.i0 = sp == 0 ? 0 : min(V, head + sp * per);
    r.i1 = sp == split - 1 ? V : min(V, head + (sp + 1) * per);
    r.head = sp == 0 ? head : 0;
    return r;
}

// ---- the sums of every row ----

__global__ void __launch_bounds__(kThreads)
verify_sums_kernel(VerifyArgs a) {
    __shared__ VerifyPart waves[kThreads / 64];
    const int sp = blockIdx.x, row = blockIdx.y, b = blockIdx.z;
    if (row > nodes_of(a, b)) return;
    const float* x = row_of(a, b, row);
    const Range r = part_range(x, a.V, sp, a.split);
    VerifyPart acc{0.0, -INFINITY, kNone};
    auto take = [&](const float (&v)[16], int n, auto at) __attribute__((always_inline)) {
        float top = -INFINITY;
        int where = kNone;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (i >= n) continue;
            bad |= !(v[i] < INFINITY);
            if (v[i] > top) {                     // the first of equals
                top = v[i];
                where = at(i);
            }
        }
        if (bad || acc.at < 0) {
            acc.at = -1;
            return;
        }
        if (top == -INFINITY) return;             // nothing of weight
        double S = 0.0;
        if (a.inv_t != 0.0) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < n) S += v[i] == -INFINITY ? 0.0 : exp2_64(((double)v[i] - top) * a.inv_t);
        }
        acc = merge(acc, VerifyPart{S, top, where}, a.inv_t);
    };
    const int body0 = r.i0 + r.head, n4 = (r.i1 - body0) / 4;
    typedef float f4 __attribute__((ext_vector_type(4)));
    const f4* body = reinterpret_cast<const f4*>(x + body0);
    for (int i0 = 0; i0 < n4; i0 += 4 * kThreads) {
        float v[16];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * kThreads + threadIdx.x;
            const f4 f = i < n4 ? __builtin_nontemporal_load(body + i) : f4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            v[4 * u] = f.x; v[4 * u + 1] = f.y; v[4 * u + 2] = f.z; v[4 * u + 3] = f.w;
        }
        take(v, 16, [&](int i) { return body0 + (i0 + i / 4 * kThreads + (int)threadIdx.x) * 4 + i % 4; });
    }
    {   // the few before the first 16-byte boundary and behind the last
        const int tail0 = body0 + 4 * n4, loose = r.head + r.i1 - tail0;
        if ((int)threadIdx.x < loose) {
            const int at = (int)threadIdx.x < r.head ? (int)threadIdx.x : tail0 + (int)threadIdx.x - r.head;
            float v[16] = {x[at]};
            take(v, 1, [&](int) { return at; });
        }
    }
    for (int o = 1; o < 64; o <<= 1) acc = merge(acc, from_lane(acc, o), a.inv_t);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 64; ++w) acc = merge(acc, waves[w], a.inv_t);
        a.part[((size_t)b * (a.N + 1) + row) * a.split + sp] = acc;
    }
}

// ---- the walk ----

// e^((x - m) / T) scale - c q of a token, not below 0
__device__ __forceinline__ double weight_of(float x, float m, double inv_t, double scale, double c, double q) {
    return fmax(x == -INFINITY ? -c * q : exp2_64(((double)x - m) * inv_t) * scale - c * q, 0.0);
}

constexpr int kWalkThreads = 1024;

__global__ void __launch_bounds__(kWalkThreads)
verify_walk_kernel(VerifyArgs a) {
    __shared__ VerifyPart rows[kMaxDrafts + 1];
    __shared__ double waves[kWalkThreads / 64];
    __shared__ double mass_lds[kMaxDrafts], q_lds[kMaxDrafts];
    __shared__ int parent_lds[kMaxDrafts], token_lds[kMaxDrafts];
    const int b = blockIdx.x, nodes = nodes_of(a, b);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int row = wave; row <= nodes; row += blockDim.x / 64) {
        VerifyPart p{0.0, -INFINITY, kNone};
        if (lane < a.split) p = a.part[((size_t)b * (a.N + 1) + row) * a.split + lane];
        for (int o = 1; o < 64; o <<= 1) p = merge(p, from_lane(p, o), a.inv_t);
        if (lane == 0) rows[row] = VerifyPart{p.S, p.m, p.at == kNone ? -1 : p.at};
    }
    __syncthreads();
    // of every node: p(x) and q(x) behind its parent
    if ((int)threadIdx.x < nodes) {
        const int i = threadIdx.x, parent = a.parents[(size_t)b * a.N + i], x = a.tokens[(size_t)b * a.N + i];
        const bool fits = parent >= -1 && parent < i && (uint32_t)x < (uint32_t)a.V;
        parent_lds[i] = parent >= -1 && parent < i ? parent : -2;           // -2: nobody's child
        token_lds[i] = fits ? x : -1 - i;                                   // no token: weighs nothing
        double mass = 0.0, q = 1.0;
        if (fits && rows[parent + 1].at >= 0) {
            const VerifyPart p = rows[parent + 1];
            if (a.inv_t != 0.0) mass = weight_of(row_of(a, b, parent + 1)[x], p.m, a.inv_t, 1.0 / p.S, 0.0, 0.0);
            if (a.probs) q = a.probs[((size_t)b * a.N + parent + 1) * a.V + x];
        }
        mass_lds[i] = mass;
        q_lds[i] = q;
    }
    __syncthreads();

    int last = -1, n_path = 0;
    double W = 1.0, c = 0.0, c_before = -1.0;     // w = max(p - c q, 0), W its sum
    uint64_t rejected = 0;                        // since the last accepted one
    for (int i = 0; i < nodes; ++i) {             // (the same in every thread)
        if (parent_lds[i] != last) continue;
        const VerifyPart p = rows[last + 1];
        bool yes = false;
        if (p.at >= 0 && token_lds[i] >= 0) {
            if (a.inv_t == 0.0) {
                yes = token_lds[i] == p.at;
            } else {
                double mass = mass_lds[i];
                if (a.probs) {
                    mass = fmax(mass - c * q_lds[i], 0.0);
                } else {
                    // a rejected sibling's token weighs nothing
                    const bool same = lane < i && (rejected >> lane & 1) && token_lds[lane] == token_lds[i];
                    if (__any(same)) mass = 0.0;
                }
                yes = (double)a.u[(size_t)b * (a.N + 1) + i] * q_lds[i] * W < mass;
                if (!yes && !a.probs) W -= mass;
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
        rejected |= 1ull << i;
        if (a.probs && a.inv_t != 0.0 && p.at >= 0) {
            const double c2 = c + W, scale = 1.0 / p.S;
            if (!__any(lane > i && lane < nodes && parent_lds[lane] == last)) {
                c_before = c;                     // nobody asks for the sum: the draw finds it
                c = c2;
                continue;
            }
            // the sum of what remains, over the vocabulary
            const float* x = row_of(a, b, last + 1);
            const float* q = a.probs + ((size_t)b * a.N + last + 1) * a.V;
            double sum = 0.0;
            for (int v = threadIdx.x; v < a.V; v += blockDim.x) sum += weight_of(x[v], p.m, a.inv_t, scale, c2, (double)q[v]);
            for (int o = 1; o < 64; o <<= 1) sum += shfl_xor(sum, o);
            __syncthreads();
            if (lane == 0) waves[wave] = sum;
            __syncthreads();
            sum = 0.0;
            for (int w = 0; w < (int)blockDim.x / 64; ++w) sum += waves[w];
            if (sum > 0.0) {
                c = c2;
                W = sum;
            }
        }
    }
    for (int i = n_path + threadIdx.x; i < a.N; i += blockDim.x) a.path[(size_t)b * a.N + i] = -1;
    if (threadIdx.x == 0) {
        const VerifyPart p = rows[last + 1];
        a.n_path[b] = n_path;
        if (a.inv_t == 0.0 || p.at < 0) a.next[b] = p.at;
        VerifyEnd e{};
        e.row = p.at < 0 ? -1 : last + 1;
        e.m = p.m;
        e.scale = 1.0 / p.S;
        e.c = c;
        e.c_before = c_before;
        e.rejected = a.probs ? 0 : rejected;
        a.end[b] = e;
    }
}

// ---- the draw ----

__global__ void __launch_bounds__(kThreads)
verify_draw_kernel(VerifyArgs a) {
    __shared__ double waves[kThreads / 64];
    __shared__ double base_lds;
    __shared__ int last_arrival, part_lds, found, last_of_weight;
    __shared__ int gone[kMaxDrafts];
    const int sp = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    VerifyEnd e = a.end[b];
    if (e.row < 0) return;
    const float* x = row_of(a, b, e.row);
    const float* q = a.probs && e.c != 0.0 ? a.probs + ((size_t)b * a.N + e.row) * a.V : nullptr;
    const int n_gone = __popcll(e.rejected);
    if (threadIdx.x < 64 && (e.rejected >> lane & 1))
        gone[__popcll(e.rejected & ((1ull << lane) - 1ull))] = a.tokens[(size_t)b * a.N + lane];
    __syncthreads();
    auto weight = [&](int v) __attribute__((always_inline)) {
        double w = weight_of(x[v], e.m, a.inv_t, e.scale, e.c, q ? (double)q[v] : 0.0);
        for (int i = 0; i < n_gone; ++i) w = gone[i] == v ? 0.0 : w;
        return w;
    };
    {
        const Range r = part_range(x, a.V, sp, a.split);
        double sum = 0.0;
        for (int v = r.i0 + threadIdx.x; v < r.i1; v += kThreads) sum += weight(v);
        for (int o = 1; o < 64; o <<= 1) sum += shfl_xor(sum, o);
        if (lane == 0) waves[wave] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.0;
            for (int w = 0; w < kThreads / 64; ++w) sum += waves[w];
            __hip_atomic_store(a.sums + (size_t)b * a.split + sp, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            // the store has completed before the ticket is taken
            __builtin_amdgcn_s_waitcnt(0);
            last_arrival = __hip_atomic_fetch_add(a.ticket + b, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.split - 1;
        }
        __syncthreads();
        if (!last_arrival) return;
    }
    if (wave == 0) {
        // the part that holds the drawn point: the first whose running sum passes it
        const double s = lane < a.split ? __hip_atomic_load(a.sums + (size_t)b * a.split + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
        double run = s;
        for (int o = 1; o < 64; o <<= 1) {
            const double y = shfl_up(run, o);
            if (lane >= o) run += y;
        }
        double W = run;                           // of the last lane
        for (int o = 1; o < 64; o <<= 1) W = fmax(W, shfl_xor(W, o));
        const double point = (double)a.u[(size_t)b * (a.N + 1) + a.N] * W;
        const uint64_t past = __ballot(run > point), some = __ballot(s > 0.0);
        // beyond the end (a random number of 1 and more): the last part of any weight
        const int at = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : -1;
        if (lane == max(at, 0)) base_lds = point - (run - s);     // still to go within the part
        if (lane == 0) {
            part_lds = at;
            found = kNone;
            last_of_weight = -1;
            a.ticket[b] = 0;                      // ready for the next launch
        }
    }
    __syncthreads();
    if (part_lds < 0 && e.c_before < 0.0) {       // nothing has any weight
        if (threadIdx.x == 0) a.next[b] = -1;
        return;
    }
    Range r = part_range(x, a.V, max(part_lds, 0), a.split);
    if (part_lds < 0) {
        // nothing is left by the last rejection, which then changes nothing: the whole row with
        // the weights before it
        e.c = e.c_before;
        r = Range{0, 0, a.V};
        double sum = 0.0;
        for (int v = threadIdx.x; v < a.V; v += kThreads) sum += weight(v);
        for (int o = 1; o < 64; o <<= 1) sum += shfl_xor(sum, o);
        if (lane == 0) waves[wave] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            sum = 0.0;
            for (int w = 0; w < kThreads / 64; ++w) sum += waves[w];
            base_lds = (double)a.u[(size_t)b * (a.N + 1) + a.N] * sum;
        }
        __syncthreads();
    }
    // the same within the part, a run of neighbouring tokens per thread
    const int per = (r.i1 - r.i0 + kThreads - 1) / kThreads;
    const int v0 = min(r.i1, r.i0 + (int)threadIdx.x * per), v1 = min(r.i1, v0 + per);
    double mine = 0.0;
    for (int v = v0; v < v1; ++v) mine += weight(v);
    double run = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const double y = shfl_up(run, o);
        if (lane >= o) run += y;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = run;
    __syncthreads();
    for (int w = 0; w < wave; ++w) run += waves[w];
    double before = run - mine;
    int first = kNone, last = -1;
    for (int v = v0; v < v1; ++v) {
        const double w = weight(v);
        before += w;
        if (w > 0.0) last = v;
        if (before > base_lds && w > 0.0 && first == kNone) first = v;
    }
    if (first != kNone) atomicMin(&found, first);
    if (last >= 0) atomicMax(&last_of_weight, last);
    __syncthreads();
    // the parts' sums and these round differently: then it is the part's last token of any weight
    if (threadIdx.x == 0) a.next[b] = found != kNone ? found : last_of_weight;
}

}  // namespace

int verify_split(int rows, int V) {
    int split = kVerifySplitMax;
    while (split > 1 && ((int64_t)split * rows > 4096 || split * 1024 > V)) split >>= 1;
    return split;
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(verify_sums_kernel, dim3(a.split, a.N + 1, a.B), dim3(kThreads), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(verify_walk_kernel, dim3(a.B), dim3(a.probs ? kWalkThreads : 256), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess || a.inv_t == 0.0) return e;
    hipLaunchKernelGGL(verify_draw_kernel, dim3(a.split, a.B), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
