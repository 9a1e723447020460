// Rotary positions: rows of queries and keys turned by their tokens' positions, in place or
// from slices of a fused projection into dense rows.
//
// A pair (a, b) of a head's values becomes (a cos - b sin, b cos + a sin) at the angle
// position x frequency.  Far positions have angles of 10^5 and more, of which 32 bits keep two
// decimals: turns, their fraction and the two polynomials are computed in 64 bits, and sine and
// cosine are rounded once.  The products and the sum are 32-bit operations of their own, so that
// a row's values do not depend on whether a compiler fuses them.
//
// Bound by the bytes: a workgroup first computes the sines and cosines of its rows' pairs, one to a
// thread, into LDS, where every head of those rows takes them.  32768 rows of 32 + 8 heads of 128 in bf16 take
// 127 us, 5.3 TB/s in both directions together; a step's 8 rows 4.3 us, the launch and two round trips.
#include <algorithm>

#include "kernels.h"
#include "tiles.h"

namespace asrkf {
namespace {

constexpr int kRotateThreads = 256;
constexpr int kRotateRows = 8;                // rows of a workgroup, at most

// cos and sin of 2 pi x, |x| any: the fraction's quarter turn, then the series on |z| <= pi / 4
// (the first terms left out are 2e-14 and 1e-15).
__device__ __forceinline__ void turn(double x, double& co, double& si) {
    const double r = x - rint(x);
    const double k = rint(4.0 * r);
    const double z = (r - 0.25 * k) * 6.283185307179586476925;
    const double w = z * z;
    const double s = z * fma(w, fma(w, fma(w, fma(w, fma(w, fma(w, 1.0 / 6227020800.0, -1.0 / 39916800.0), 1.0 / 362880.0),
                                            -1.0 / 5040.0), 1.0 / 120.0), -1.0 / 6.0), 1.0);
    const double c = fma(w, fma(w, fma(w, fma(w, fma(w, fma(w, fma(w, -1.0 / 87178291200.0, 1.0 / 479001600.0), -1.0 / 3628800.0),
                                               1.0 / 40320.0), -1.0 / 720.0), 1.0 / 24.0), -0.5), 1.0);
    const int quarter = (int)k & 3;
    co = quarter == 0 ? c : quarter == 1 ? -s : quarter == 2 ? -c : s;
    si = quarter == 0 ? s : quarter == 1 ? c : quarter == 2 ? -s : -c;
}

__device__ __forceinline__ void turn_pair(float& a, float& b, float2 cs) {
#pragma clang fp contract(off)
    const float x = a * cs.x, y = b * cs.y, z = b * cs.x, w = a * cs.y;
    a = x - y;
    b = z + w;
}

template <bool BF16>
struct Piece16 {
    static constexpr int kValues = BF16 ? 8 : 4;
    float v[kValues];
    __device__ __forceinline__ void from(uintx4 x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (BF16) {
                v[2 * i] = __uint_as_float(x[i] << 16);
                v[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
            } else {
                v[i] = __uint_as_float(x[i]);
            }
        }
    }
    __device__ __forceinline__ uintx4 bits() const {
        if constexpr (BF16) {
            bf16x8 r;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = (__bf16)v[i];
            return __builtin_bit_cast(uintx4, r);
        } else {
            return uintx4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        }
    }
};

// A thread takes two 16-byte pieces of a head at a time, whose values are each other's
// partners (or that are left as they are), several pairs of pieces in flight.
template <bool BF16, bool IN_PAIRS>
__global__ void __launch_bounds__(kRotateThreads)
rotate_kernel(RotateArgs a) {
    using P = Piece16<BF16>;
    constexpr int V = P::kValues;
    __shared__ float2 cs[kRotateRows * kMaxPairs];
    const int r0 = blockIdx.x * a.rows_per_block;
    const int rows = min(a.rows_per_block, a.n - r0);
    const int heads = a.heads[0] + a.heads[1];
    const int unit_shift = __ffs(a.D / (2 * V)) - 1;      // units of two pieces in a head: a power of two
    const int turned = a.pairs / V;                       // those that are turned
    const int total = (rows * heads) << unit_shift;

    struct Where { const uintx4* from[2]; uintx4* to[2]; int unit, row; };
    auto where = [&](int item) __attribute__((always_inline)) {
        Where w;
        w.unit = item & ((1 << unit_shift) - 1);
        const int rest = item >> unit_shift;
        w.row = heads == 1 ? rest : (int)__umulhi((uint32_t)rest, a.head_magic);
        int h = rest - w.row * heads;
        const int which = h >= a.heads[0] ? 1 : 0;
        h -= which ? a.heads[0] : 0;
        const bool apart = !IN_PAIRS && w.unit < turned;
        const int p0 = apart ? w.unit : 2 * w.unit, p1 = apart ? w.unit + turned : 2 * w.unit + 1;
        const size_t head = (size_t)h * a.D * (BF16 ? 2 : 4);
        const char* x = (which ? a.x[1] : a.x[0]) + (size_t)(r0 + w.row) * (which ? a.x_stride[1] : a.x_stride[0]) + head;
        char* y = (which ? a.y[1] : a.y[0]) + (size_t)(r0 + w.row) * (which ? a.y_stride[1] : a.y_stride[0]) + head;
        w.from[0] = reinterpret_cast<const uintx4*>(x) + p0;
        w.from[1] = reinterpret_cast<const uintx4*>(x) + p1;
        w.to[0] = reinterpret_cast<uintx4*>(y) + p0;
        w.to[1] = reinterpret_cast<uintx4*>(y) + p1;
        return w;
    };
    for (int i = threadIdx.x; i < rows * a.pairs; i += kRotateThreads) {
        const int row = i / a.pairs, pair = i - row * a.pairs;
        int64_t pos = a.pos ? a.pos[r0 + row] : 0;
        if (a.rows_per_seq) pos += (int64_t)a.plen[(r0 + row) / a.rows_per_seq] + *a.t_dev + a.t_offset;
        double co, si;
        turn((double)pos * a.turns[pair], co, si);
        cs[row * kMaxPairs + pair] = make_float2((float)(co * a.magnitude), (float)(si * a.magnitude));
    }
    __syncthreads();
    constexpr int kFlight = 4;
    for (int i0 = threadIdx.x; i0 < total; i0 += kFlight * kRotateThreads) {
        uintx4 x[kFlight][2];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            if (i0 + f * kRotateThreads >= total) continue;
            const Where w = where(i0 + f * kRotateThreads);
            x[f][0] = *w.from[0];
            x[f][1] = *w.from[1];
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            if (i0 + f * kRotateThreads >= total) continue;
            const Where w = where(i0 + f * kRotateThreads);
            P p0, p1;
            p0.from(x[f][0]);
            p1.from(x[f][1]);
            if (w.unit < turned) {
                const float2* c = cs + w.row * kMaxPairs + w.unit * V;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    if constexpr (IN_PAIRS) {
                        P& p = e < V / 2 ? p0 : p1;
                        turn_pair(p.v[e % (V / 2) * 2], p.v[e % (V / 2) * 2 + 1], c[e]);
                    } else {
                        turn_pair(p0.v[e], p1.v[e], c[e]);
                    }
                }
                x[f][0] = p0.bits();
                x[f][1] = p1.bits();
            }
            *w.to[0] = x[f][0];
            *w.to[1] = x[f][1];
        }
    }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& args, int bf16, hipStream_t s) {
    RotateArgs a = args;
    // as many rows as give every thread two pieces (rows of 10 heads of 64 in bf16, 65536 of them: 47 us, one to a
    // workgroup 104; of 40 heads of 128, 16384: 80 us, four to a workgroup 86); more where the grid would pass 2^31 threads
    const int items = (a.heads[0] + a.heads[1]) * a.D / (bf16 ? 16 : 8);
    constexpr int kMostBlocks = (1 << 30) / kRotateThreads * 2;
    static_assert(kMaxRotateRows / kMostBlocks <= kRotateRows, "the largest call's grid");
    a.rows_per_block = std::max(std::min(kRotateRows, std::max(1, kRotateThreads / items)), (a.n + kMostBlocks - 1) / kMostBlocks);
    a.head_magic = (uint32_t)(((uint64_t)1 << 32) / (a.heads[0] + a.heads[1])) + 1;
    const dim3 grid((a.n + a.rows_per_block - 1) / a.rows_per_block), block(kRotateThreads);
    if (bf16) {
        if (a.in_pairs) hipLaunchKernelGGL((rotate_kernel<true, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rotate_kernel<true, false>), grid, block, 0, s, a);
    } else {
        if (a.in_pairs) hipLaunchKernelGGL((rotate_kernel<false, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rotate_kernel<false, false>), grid, block, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace asrkf
