// Prompts: causal attention over packed prompts, and their rows into the cache.
//
// Attention, for every sequence of a batch and token i of it,
//   o[i,h] = sum_{j <= i} softmax_j(q[i,h] . k[j, h / G] / sqrt(D)) v[j, h / G].
//
// A (sequence, KV head) pair's queries, token by token and head by head, are the
// rows of one problem: row r is head r % G of token r / G, so that a K and V tile
// serves the G query heads and a block of rows spans only rows / G tokens.  A
// workgroup takes a block of rows and walks the tiles of keys up to its last
// token.  K and V tiles travel through registers into LDS, the next tile's while
// this one is computed; each of the two buffers is written behind the one barrier
// of a tile.
//
// Scores are formed transposed, S^T = K Q^T, with the query in the lane: the
// softmax statistics of a row are then a lane's own values (and those of lane
// +-32), the rescaling of O^T = V^T P^T is one factor per lane, and the weights
// are in place as the second product's operand: a C tile holds, of every 16 keys,
// 4 h .. 4 h + 3 and 8 + 4 h .. in lane half h, and V's transposed LDS reads take
// the same keys in the same order (a sum over keys has no order to keep).
#include <type_traits>

#include "kernels.h"
#include "rows.h"

namespace asrkf {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4* lds_shortx4;

constexpr int kBufferFlags = 0x00020000;      // raw buffer, 32-bit data

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, bytes, kBufferFlags);
}
__device__ __forceinline__ intx4 load16(__amdgpu_buffer_rsrc_t r, int off) {
    return __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}

template <int N, typename F>
__device__ __forceinline__ void unroll(F f) {
    if constexpr (N > 0) {
        unroll<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// The sequence of the batch whose units (blocks, given by their first ones) hold unit x.
__device__ __forceinline__ int find_sequence(const PromptBatch& b, int x) {
    int lo = 0, hi = b.n - 1;                 // the last with first <= x
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (b.first[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// ---- the rows into the cache ----

constexpr int kStoreThreads = 256;

// Packed rows [T][Hkv][D] into the head-major cache, a workgroup per kPromptStoreTokens
// tokens of a sequence.  A thread moves 16 bytes of a K and of a V row, or rounds a
// group of 32 values of each to 4 bits.
template <bool FOUR>
__global__ void __launch_bounds__(kStoreThreads)
prompt_store_kernel(PromptArgs a, PromptBatch batch) {
    const int i = find_sequence(batch, blockIdx.x);
    const int n = batch.len[i], seq = batch.seq[i];
    const int t0 = ((int)blockIdx.x - batch.first[i]) * kPromptStoreTokens;
    const int nt = min(kPromptStoreTokens, n - t0);
    if (t0 == 0 && threadIdx.x == 0) a.plen[seq] = n;
    constexpr int kUnit = FOUR ? 64 : 16;     // bytes of a source row that a thread takes
    const int per_head = a.head_bytes / kUnit, per_token = per_head * a.Hkv;      // powers of two
    const int head_shift = __ffs(per_head) - 1, token_shift = __ffs(per_token) - 1;
    const char* k = a.k + (size_t)(batch.start[i] + t0) * a.k_stride;
    const char* v = a.v + (size_t)(batch.start[i] + t0) * a.v_stride;
    const size_t row0 = (size_t)seq * a.Hkv * a.pool_rows + t0;
    for (int u = threadIdx.x; u < nt * per_token; u += kStoreThreads) {
        const int t = u >> token_shift, e = u & (per_token - 1);
        const int g = e >> head_shift, p = e & (per_head - 1);
        const size_t row = row0 + (size_t)g * a.pool_rows + t;
        const uintx4* ks = reinterpret_cast<const uintx4*>(k + (size_t)t * a.k_stride + e * kUnit);
        const uintx4* vs = reinterpret_cast<const uintx4*>(v + (size_t)t * a.v_stride + e * kUnit);
        if constexpr (FOUR) {
            auto round = [&](const uintx4* s, char* pool, uint8_t* scales) __attribute__((always_inline)) {
                uintx4 x[4], c;
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = s[j];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    top = max_magnitude(top, max_magnitude(max_magnitude(x[j][0], x[j][1]), max_magnitude(x[j][2], x[j][3])));
                const uint32_t byte = scale_byte(max(top & 0xFFFFu, top >> 16));
                const float f = scale_value(byte);
#pragma unroll
                for (int j = 0; j < 4; ++j) c[j] = encode8(x[j][0], x[j][1], x[j][2], x[j][3], f);
                *reinterpret_cast<uintx4*>(pool + (row * per_head + p) * 16) = c;
                scales[row * per_head + p] = (uint8_t)byte;
            };
            round(ks, a.kpool, a.kscale);
            round(vs, a.vpool, a.vscale);
        } else {
            const uintx4 x = *ks, y = *vs;
            *reinterpret_cast<uintx4*>(a.kpool + (row * per_head + p) * 16) = x;
            *reinterpret_cast<uintx4*>(a.vpool + (row * per_head + p) * 16) = y;
        }
    }
}

// Rows first .. first + n - 1 of a sequence's cache as [n][Hkv][D].
template <bool FOUR>
__global__ void __launch_bounds__(kStoreThreads)
rows_kernel(RowsArgs a) {
    constexpr int kUnit = FOUR ? 64 : 16;     // bytes of an output row that a thread writes
    const int per_head = a.head_bytes / kUnit, per_token = per_head * a.Hkv;
    const int head_shift = __ffs(per_head) - 1, token_shift = __ffs(per_token) - 1;
    const int64_t total = (int64_t)a.n << token_shift;
    for (int64_t u = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x; u < total; u += (int64_t)gridDim.x * kStoreThreads) {
        const int t = (int)(u >> token_shift), e = (int)u & (per_token - 1);
        const int g = e >> head_shift, p = e & (per_head - 1);
        const size_t unit = ((size_t)g * a.pool_rows + a.first + t) * per_head + p;
        if constexpr (FOUR) {
            auto read = [&](const char* pool, const uint8_t* scales, char* to) __attribute__((always_inline)) {
                const uintx4 c = *reinterpret_cast<const uintx4*>(pool + unit * 16);
                const float f = scale_value(scales[unit]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    reinterpret_cast<uintx4*>(to + u * 64)[j] =
                        uintx4{decode2<0>(c[j], f), decode2<1>(c[j], f), decode2<2>(c[j], f), decode2<3>(c[j], f)};
            };
            read(a.kpool, a.kscale, a.k);
            read(a.vpool, a.vscale, a.v);
        } else {
            *reinterpret_cast<uintx4*>(a.k + u * 16) = *reinterpret_cast<const uintx4*>(a.kpool + unit * 16);
            *reinterpret_cast<uintx4*>(a.v + u * 16) = *reinterpret_cast<const uintx4*>(a.vpool + unit * 16);
        }
    }
}

// ---- attention ----

template <bool BF16, int D, int WAVES>
struct Tile {
    static constexpr int kElem = BF16 ? 2 : 4;
    static constexpr int kRow = D * kElem;                // bytes of a row of one head
    static constexpr int kKeys = kRow <= 256 ? 64 : 32;   // keys of a tile
    static constexpr int kKB = kKeys / 32;                // score blocks of 32 keys
    static constexpr int kRows = WAVES * 32;              // query rows of a workgroup
    static constexpr int kThreads = WAVES * 64;
    // LDS row strides: 16 rows of a 16-byte piece (K), and 4 rows of 64 bytes (V, bf16) or
    // rows 4 apart of 128 bytes (V, fp32), meet no bank twice
    static constexpr int kKStride = kRow + 16;
    static constexpr int kVStride = kRow + (BF16 ? 64 : 32);
    static constexpr int kKBuffer = kKeys * kKStride, kVBuffer = kKeys * kVStride;     // two of each
    static constexpr int kLoads = kKeys * kRow / 16 / kThreads;   // 16-byte pieces of K (or V) per thread
    static constexpr int kQRegs = BF16 ? D / 16 : D / 8;  // 16-byte pieces of q per lane
    static_assert(kLoads * kThreads * 16 == kKeys * kRow, "whole pieces per thread");
};

// x with 0 in the place of infinities and NaNs; bad says whether there were any
template <bool BF16>
__device__ __forceinline__ intx4 finite_part(intx4 x, bool& bad) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
            const bool lo = (x[i] & 0x7F80) == 0x7F80, hi = (x[i] & 0x7F800000) == 0x7F800000;
            bad |= lo || hi;
            x[i] &= (lo ? 0 : 0xFFFF) | (hi ? 0 : (int)0xFFFF0000);
        } else {
            const bool is = (x[i] & 0x7F800000) == 0x7F800000;
            bad |= is;
            x[i] = is ? 0 : x[i];
        }
    }
    return x;
}

// The rescaling of O waits until a row's maximum has grown by 2^kLazy; weights are
// 2^(x - m - kLazy), so that none passes 1 and no sum the largest value times the
// number of tokens.
constexpr float kLazy = 8.f;

template <bool BF16, int D, int G, int WAVES>
__global__ void __launch_bounds__(WAVES * 64, (D * (BF16 ? 1 : 2) > 128 ? 1 : 2))
prompt_attention_kernel(PromptArgs a, PromptBatch batch) {
    using T = Tile<BF16, D, WAVES>;
    constexpr int NL = T::kLoads, KB = T::kKB, NQ = T::kQRegs, DB = D / 32;
    constexpr int kPieces = T::kRow / 16;                 // pieces of a row
    __shared__ __align__(16) char lds[2 * (T::kKBuffer + T::kVBuffer)];
    __shared__ int holds_infinite[2];                     // the tile whose V values are not all finite

    const int kvh = blockIdx.x % a.Hkv;
    const int unit = blockIdx.x / a.Hkv;
    const int si = find_sequence(batch, unit);
    const int n = batch.len[si];
    const int blocks = (n * G + T::kRows - 1) / T::kRows;
    const int block = blocks - 1 - (unit - batch.first[si]);      // the longest ones first
    const int r0 = block * T::kRows;
    const int first_token = r0 / G;
    const int last_token = min(n - 1, (r0 + T::kRows - 1) / G);
    const int tiles = last_token / T::kKeys + 1;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int row = r0 + wave * 32 + col;                 // the lane's query row
    const int token = min(row / G, n - 1);                // rows past the end repeat the last token's
    const int wave_first = (r0 + wave * 32) / G;
    const int wave_last = min(n - 1, (r0 + wave * 32 + 31) / G);

    intx4 q[NQ];
    {
        const char* p = a.q + (size_t)(batch.start[si] + token) * a.q_stride + (kvh * G + row % G) * T::kRow;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
            q[i] = *reinterpret_cast<const intx4*>(p + (BF16 ? i * 32 + half * 16 : half * (T::kRow / 2) + i * 16));
    }

    const char* k0 = a.k + (size_t)batch.start[si] * a.k_stride + kvh * T::kRow;
    const char* v0 = a.v + (size_t)batch.start[si] * a.v_stride + kvh * T::kRow;
    intx4 kx[NL], vx[NL];
    // rows past the sequence's end read as zeros
    auto request = [&](const char* base, int64_t stride, int j, intx4 (&x)[NL]) __attribute__((always_inline)) {
        const int left = min(T::kKeys, n - j * T::kKeys);
        const auto r = buffer(base + (size_t)j * T::kKeys * stride, left > 0 ? (int)((left - 1) * stride + T::kRow) : 0);
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = threadIdx.x + u * T::kThreads;
            x[u] = load16(r, (i / kPieces) * (int)stride + i % kPieces * 16);
        }
    };
    auto request_k = [&](int j) __attribute__((always_inline)) { request(k0, a.k_stride, j, kx); };
    auto request_v = [&](int j) __attribute__((always_inline)) { request(v0, a.v_stride, j, vx); };
    auto keep_k = [&](int j) __attribute__((always_inline)) {
        char* to = lds + (j & 1) * T::kKBuffer;
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = threadIdx.x + u * T::kThreads;
            *reinterpret_cast<intx4*>(to + i / kPieces * T::kKStride + i % kPieces * 16) = kx[u];
        }
    };
    auto keep_v = [&](int j) __attribute__((always_inline)) {
        char* to = lds + 2 * T::kKBuffer + (j & 1) * T::kVBuffer;
        // Where a tile holds keys behind some query of the block, a weight of zero must not
        // meet an infinity or a NaN: those values are added on their own.
        if (j * T::kKeys + T::kKeys - 1 > first_token) {
            bool bad = false;
#pragma unroll
            for (int u = 0; u < NL; ++u) vx[u] = finite_part<BF16>(vx[u], bad);
            if (bad) holds_infinite[j & 1] = j;
        }
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = threadIdx.x + u * T::kThreads;
            *reinterpret_cast<intx4*>(to + i / kPieces * T::kVStride + i % kPieces * 16) = vx[u];
        }
    };

    float m = -INFINITY, l = 0.f;                         // of the lane's row (l: the lane's own keys)
    floatx16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

    auto scores = [&](int j, floatx16 (&s)[KB]) __attribute__((always_inline)) {
        const char* kt = lds + (j & 1) * T::kKBuffer;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                const intx4 kr = *reinterpret_cast<const intx4*>(
                    kt + (b * 32 + col) * T::kKStride + (BF16 ? i * 32 + half * 16 : half * (T::kRow / 2) + i * 16));
                if (i == 0)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
                if constexpr (BF16) {
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr),
                                                                   __builtin_bit_cast(bf16x8, q[i]), s[b], 0, 0, 0);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(kr[e]), __int_as_float(q[i][e]), s[b], 0, 0, 0);
                }
            }
    };
    auto tile = [&](int j) __attribute__((always_inline)) {
        floatx16 s[KB];
        scores(j, s);
        const char* vt = lds + 2 * T::kKBuffer + (j & 1) * T::kVBuffer;
        // key of value i in block b: 32 b + 8 (i / 4) + 4 half + i % 4
        if (j * T::kKeys + T::kKeys - 1 > wave_first) {
            const int left = token - j * T::kKeys - half * 4;     // keys up to the lane's token, from its first
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[b][i] = b * 32 + i / 4 * 8 + i % 4 <= left ? s[b][i] : -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        if (__any(top > m + a.lazy)) {
            const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            const float mn = fmaxf(m, fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1])));
            const float sc = m < mn ? __builtin_amdgcn_exp2f((m - mn) * a.scale_log2) : 1.f;
            m = mn;
            l *= sc;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= sc;
        }
        const float bias = -(m == -INFINITY ? 0.f : m * a.scale_log2) - kLazy;
        // V's transposed reads (bf16): 4 keys of 16 dims per 16 lanes
        const char* vb = vt + (half * 4 + (lane & 15) / 4) * T::kVStride + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        constexpr int kGroups = KB * 2;                   // of 16 keys
        unroll<kGroups>([&](auto B) __attribute__((always_inline)) {
            constexpr int b = decltype(B)::value;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(s[b / 2][b % 2 * 8 + e], a.scale_log2, bias));
                l += p[e];
            }
            if constexpr (BF16) {
                bf16x8 w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (__bf16)p[e];
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    const char* at = vb + b * 16 * T::kVStride + d * 64;
                    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)at);
                    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(at + 8 * T::kVStride));
                    const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, w, acc[d], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const char* at = vt + (b * 16 + e / 4 * 8 + half * 4 + e % 4) * T::kVStride + col * 4;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(at + d * 128),
                                                                      p[e], acc[d], 0, 0, 0);
                }
            }
        });
        if (holds_infinite[j & 1] == j) {
            // the values that are not finite, from memory, to the queries that see their key
            // (whatever their weight)
            for (int key = j * T::kKeys; key <= min(wave_last, j * T::kKeys + T::kKeys - 1); ++key) {
                const char* at = v0 + (size_t)key * a.v_stride + half * 4 * T::kElem;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const char* e = at + (d * 32 + i / 4 * 8 + i % 4) * T::kElem;
                        float v;
                        if constexpr (BF16) v = (float)*reinterpret_cast<const __bf16*>(e);
                        else v = *reinterpret_cast<const float*>(e);
                        if (key <= token && !(fabsf(v) < INFINITY)) acc[d][i] += v;
                    }
            }
        }
    };
    if (threadIdx.x < 2) holds_infinite[threadIdx.x] = -1;
    request_k(0);
    request_v(0);
    __syncthreads();
    keep_k(0);
    keep_v(0);
    request_k(1);
    request_v(1);
    for (int j = 0; j < tiles; ++j) {
        __syncthreads();                                  // tile j is in place, tile j - 1 has been read
        if (j + 1 < tiles) {
            keep_k(j + 1);
            keep_v(j + 1);
            request_k(j + 2);
            request_v(j + 2);
        }
        if (j * T::kKeys <= wave_last) tile(j);           // else all of it lies behind the wave's queries
    }

    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float inv = 1.f / (__uint_as_float(x[0]) + __uint_as_float(x[1]));
    if (row < n * G) {
        char* o = a.out + ((size_t)(batch.start[si] + token) * a.Hq + kvh * G + row % G) * T::kRow;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                 // dims 32 d + 8 i + 4 half ..
                const int dim = d * 32 + i * 8 + half * 4;
                floatx4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = acc[d][i * 4 + e] * inv;
                if constexpr (BF16) {
                    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<bf16x4*>(o + dim * 2) = __builtin_convertvector(r, bf16x4);
                } else {
                    *reinterpret_cast<floatx4*>(o + dim * 4) = r;
                }
            }
    }
}

template <bool BF16, int D, int G>
hipError_t launch_rows(const PromptArgs& a, PromptBatch& b, hipStream_t s) {
    constexpr int kWaves = 4;
    int blocks = 0;
    for (int i = 0; i < b.n; ++i) {
        b.first[i] = blocks;
        blocks += (b.len[i] * G + kWaves * 32 - 1) / (kWaves * 32);
    }
    hipLaunchKernelGGL((prompt_attention_kernel<BF16, D, G, kWaves>), dim3(blocks * a.Hkv), dim3(kWaves * 64), 0, s, a, b);
    return hipGetLastError();
}

template <bool BF16, int D>
hipError_t launch_group(const PromptArgs& a, PromptBatch& b, int group, hipStream_t s) {
    switch (group) {
        case 1: return launch_rows<BF16, D, 1>(a, b, s);
        case 2: return launch_rows<BF16, D, 2>(a, b, s);
        case 4: return launch_rows<BF16, D, 4>(a, b, s);
        case 8: return launch_rows<BF16, D, 8>(a, b, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_prompt_attention(const PromptArgs& a, const PromptBatch& batch, int bf16, int head_dim, hipStream_t s) {
    PromptBatch b = batch;
    PromptArgs p = a;
    p.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)head_dim));
    p.lazy = kLazy / p.scale_log2;
    const int group = a.Hq / a.Hkv;
    if (bf16) {
        if (head_dim == 64) return launch_group<true, 64>(p, b, group, s);
        if (head_dim == 128) return launch_group<true, 128>(p, b, group, s);
        if (head_dim == 256) return launch_group<true, 256>(p, b, group, s);
    } else {
        if (head_dim == 64) return launch_group<false, 64>(p, b, group, s);
        if (head_dim == 128) return launch_group<false, 128>(p, b, group, s);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_prompt_store(const PromptArgs& a, const PromptBatch& batch, bool four, hipStream_t s) {
    PromptBatch b = batch;
    int blocks = 0;
    for (int i = 0; i < b.n; ++i) {
        b.first[i] = blocks;
        blocks += (b.len[i] + kPromptStoreTokens - 1) / kPromptStoreTokens;
    }
    if (four) hipLaunchKernelGGL(prompt_store_kernel<true>, dim3(blocks), dim3(kStoreThreads), 0, s, a, b);
    else hipLaunchKernelGGL(prompt_store_kernel<false>, dim3(blocks), dim3(kStoreThreads), 0, s, a, b);
    return hipGetLastError();
}

hipError_t launch_get_rows(const RowsArgs& a, bool four, hipStream_t s) {
    const int64_t units = (int64_t)a.n * a.Hkv * a.head_bytes / (four ? 64 : 16);
    const int64_t blocks = (units + kStoreThreads - 1) / kStoreThreads;
    const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
    if (four) hipLaunchKernelGGL(rows_kernel<true>, grid, dim3(kStoreThreads), 0, s, a);
    else hipLaunchKernelGGL(rows_kernel<false>, grid, dim3(kStoreThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
