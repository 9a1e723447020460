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

// The sequence of the batch whose units (given by their first ones) hold unit x: one
// round trip to the table, a sequence per lane.
__device__ __forceinline__ int find_sequence(const int32_t* first, int n, int x) {
    const int lane = threadIdx.x & 63;
    int before = 0;
#pragma unroll
    for (int i = 0; i < kPromptSeqs; i += 64)
        before += __popcll(__ballot(i + lane < n && first[i + lane] <= x));
    return before - 1;
}

// ---- the rows into the cache ----

constexpr int kStoreThreads = 256;

// Eight values of a row, whose group's others the lane's three neighbours hold, as
// codes, and (lanes at the start of a row's 16, or of rows of 64 values at the start of
// its 8) the scale bytes of those lanes' groups.
__device__ __forceinline__ uint32_t round8(uintx4 x, bool rows_of_64, uint32_t& scales) {
    uint32_t top = max_magnitude(max_magnitude(x[0], x[1]), max_magnitude(x[2], x[3]));
    top = max(top & 0xFFFFu, top >> 16);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, false));   // quad_perm [1,0,3,2]
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, false));   // quad_perm [2,3,0,1]
    const uint32_t byte = scale_byte(top);
    scales = byte << (threadIdx.x / 4 & (rows_of_64 ? 1 : 3)) * 8;
    if (rows_of_64) {
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x141, 0xF, 0xF, false);     // row_half_mirror
    } else {
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x124, 0xF, 0xF, false);     // row_ror 4
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x128, 0xF, 0xF, false);     // row_ror 8
    }
    return encode8(x[0], x[1], x[2], x[3], scale_value(byte));
}

// Packed rows [T][Hkv][D] into the head-major cache, a workgroup per kPromptStoreTokens
// tokens of a sequence.  A thread takes 16 bytes of K and of V at a time, several in
// flight; four neighbouring threads have a group of 32 values (a thread with a whole
// group took 148 us where this takes 127, for 8 x 16k tokens of 8 heads of 128, 0.68 GB).
template <bool FOUR>
__device__ __forceinline__ void store_rows(const PromptArgs& a, const PromptBatch& batch, int unit) {
    const int i = find_sequence(batch.first_store, batch.n, unit);
    const int n = batch.len[i], seq = batch.seq[i];
    const int t0 = (unit - batch.first_store[i]) * kPromptStoreTokens;
    const int nt = min(kPromptStoreTokens, n - t0);
    if (t0 == 0 && threadIdx.x == 0) a.plen[seq] = n;
    const int per_head = a.head_bytes / 16, per_token = per_head * a.Hkv;     // powers of two
    const int head_shift = __ffs(per_head) - 1, token_shift = __ffs(per_token) - 1;
    const int pool_bytes = FOUR ? a.head_bytes / 4 : a.head_bytes;
    const char* k = a.k + (size_t)(batch.start[i] + t0) * a.k_stride;
    const char* v = a.v + (size_t)(batch.start[i] + t0) * a.v_stride;
    const size_t row0 = (size_t)seq * a.Hkv * a.pool_rows + t0;
    const int total = nt * per_token;
    constexpr int kFlight = 4;
    for (int u0 = threadIdx.x; u0 < total; u0 += kFlight * blockDim.x) {
        uintx4 x[kFlight], y[kFlight];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            const int u = u0 + f * blockDim.x, t = u >> token_shift, e = u & (per_token - 1);
            if (u < total) {
                x[f] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(k + (size_t)t * a.k_stride + e * 16));
                y[f] = __builtin_nontemporal_load(reinterpret_cast<const uintx4*>(v + (size_t)t * a.v_stride + e * 16));
            }
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            const int u = u0 + f * blockDim.x, t = u >> token_shift, e = u & (per_token - 1);
            if (u >= total) continue;
            const int g = e >> head_shift, p = e & (per_head - 1);
            const size_t row = row0 + (size_t)g * a.pool_rows + t, at = row * pool_bytes;
            if constexpr (FOUR) {
                const bool of_64 = per_head == 8;
                uint32_t ks, vs;
                *reinterpret_cast<uint32_t*>(a.kpool + at + p * 4) = round8(x[f], of_64, ks);
                *reinterpret_cast<uint32_t*>(a.vpool + at + p * 4) = round8(y[f], of_64, vs);
                const size_t to = (row * per_head + p) / 4;           // the first of the lanes' groups
                if (of_64 && p == 0) {
                    *reinterpret_cast<uint16_t*>(a.kscale + to) = (uint16_t)ks;
                    *reinterpret_cast<uint16_t*>(a.vscale + to) = (uint16_t)vs;
                } else if (!of_64 && p % 16 == 0) {
                    *reinterpret_cast<uint32_t*>(a.kscale + to) = ks;
                    *reinterpret_cast<uint32_t*>(a.vscale + to) = vs;
                }
            } else {
                *reinterpret_cast<uintx4*>(a.kpool + at + p * 16) = x[f];
                *reinterpret_cast<uintx4*>(a.vpool + at + p * 16) = y[f];
            }
        }
    }
}

template <bool FOUR>
__global__ void __launch_bounds__(kStoreThreads)
prompt_store_kernel(PromptArgs a, PromptBatch batch) {
    store_rows<FOUR>(a, batch, blockIdx.x);
}

// Rows first .. first + n - 1 of a sequence's cache as [n][Hkv][D], 16 bytes of K and
// of V to a thread at a time, several in flight.
template <bool FOUR>
__global__ void __launch_bounds__(kStoreThreads)
rows_kernel(RowsArgs a) {
    const int per_head = a.head_bytes / 16, per_token = per_head * a.Hkv;
    const int head_shift = __ffs(per_head) - 1, token_shift = __ffs(per_token) - 1;
    const int pool_bytes = FOUR ? a.head_bytes / 4 : a.head_bytes;
    const int64_t total = (int64_t)a.n << token_shift, step = (int64_t)gridDim.x * kStoreThreads;
    constexpr int kFlight = 4;
    typedef std::conditional_t<FOUR, uint32_t, uintx4> Piece;
    for (int64_t u0 = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x; u0 < total; u0 += kFlight * step) {
        Piece x[kFlight], y[kFlight];
        uint8_t xs[kFlight], ys[kFlight];
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            const int64_t u = u0 + f * step;
            if (u >= total) continue;
            const int t = (int)(u >> token_shift), e = (int)u & (per_token - 1);
            const int g = e >> head_shift, p = e & (per_head - 1);
            const size_t row = (size_t)g * a.pool_rows + a.first + t, at = row * pool_bytes;
            x[f] = *reinterpret_cast<const Piece*>(a.kpool + at + p * sizeof(Piece));
            y[f] = *reinterpret_cast<const Piece*>(a.vpool + at + p * sizeof(Piece));
            if constexpr (FOUR) {
                xs[f] = a.kscale[(row * per_head + p) / 4];
                ys[f] = a.vscale[(row * per_head + p) / 4];
            }
        }
#pragma unroll
        for (int f = 0; f < kFlight; ++f) {
            const int64_t u = u0 + f * step;
            if (u >= total) continue;
            uintx4 k, v;
            if constexpr (FOUR) {
                const float kf = scale_value(xs[f]), vf = scale_value(ys[f]);
                k = uintx4{decode2<0>(x[f], kf), decode2<1>(x[f], kf), decode2<2>(x[f], kf), decode2<3>(x[f], kf)};
                v = uintx4{decode2<0>(y[f], vf), decode2<1>(y[f], vf), decode2<2>(y[f], vf), decode2<3>(y[f], vf)};
            } else {
                k = x[f];
                v = y[f];
            }
            __builtin_nontemporal_store(k, reinterpret_cast<uintx4*>(a.k + u * 16));
            __builtin_nontemporal_store(v, reinterpret_cast<uintx4*>(a.v + u * 16));
        }
    }
}

// ---- attention ----

template <bool BF16, int D, int WAVES, Walk WALK>
struct Tile {
    static constexpr bool kSplits = WALK == kSplit, kHalved = WALK == kHalves;
    static constexpr int kElem = BF16 ? 2 : 4;
    static constexpr int kRow = D * kElem;                // bytes of a row of one head
    static constexpr int kKeys = kRow <= 256 && !kSplits ? 64 : 32;   // keys of a wave's tile
    static constexpr int kTileKeys = kHalved ? 2 * kKeys : kKeys;     // keys of a tile in LDS
    static constexpr int kKB = kKeys / 32;                // score blocks of 32 keys
    static constexpr int kRowWaves = kSplits ? 1 : kHalved ? WAVES / 2 : WAVES;
    static constexpr int kRows = kRowWaves * 32;          // query rows of a workgroup
    static constexpr int kThreads = kSplits ? 64 : WAVES * 64;        // that load a tile
    // LDS row strides: 16 rows of a 16-byte piece (K), and 4 rows of 64 bytes (V, bf16) or
    // rows 4 apart of 128 bytes (V, fp32), meet no bank twice
    static constexpr int kKStride = kRow + 16;
    static constexpr int kVStride = kRow + (BF16 ? 64 : 32);
    static constexpr int kKBuffer = kTileKeys * kKStride, kVBuffer = kTileKeys * kVStride;
    static constexpr int kBuffers = kSplits ? 1 : 2;
    static constexpr int kTiles = kBuffers * (kKBuffer + kVBuffer);   // of the workgroup, or of a wave
    static constexpr int kLds = kTiles * (kSplits ? WAVES : 1);
    static constexpr int kLoads = kTileKeys * kRow / 16 / kThreads;   // 16-byte pieces of K (or V) per thread
    static constexpr int kQRegs = BF16 ? D / 16 : D / 8;  // 16-byte pieces of q per lane
    static constexpr int kState = D + 4;                  // floats of a row of a wave's state
    static_assert(kTileKeys <= kPromptTileKeys, "offsets within a tile");
    static_assert(kLoads * kThreads * 16 == kTileKeys * kRow, "whole pieces per thread");
    static_assert(!kHalved || kRowWaves * 64 * (D / 2 + 2) * 4 <= kLds, "the states of half the waves fit the tiles");
    static_assert(!kSplits || 32 * kState * 4 <= kTiles, "a wave's state fits its tile");
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
// 2^(x - m - kLazy - b) with 2^b >= twice the keys that a workgroup's rows see, so that no
// weight passes 2^-b and no sum half of the largest value: outputs are finite wherever the
// values are.  b costs what lies below 2^(b - 118) of a row's largest weight, which becomes 0.
// fp32 weights are scaled behind the exponential: b in its argument is rounded with it (512
// tokens: 4.9e-7 off in the 2-norm, 4.0e-7 so; 2000 tokens of 32/8 heads of 128: 290 us, 296 so).
constexpr float kLazy = 8.f;

template <bool BF16, int D, int G, int WAVES, Walk WALK>
__global__ void __launch_bounds__(WAVES * 64, (prompt_waves(BF16, D, WAVES, WALK)))
prompt_attention_kernel(PromptArgs a, PromptBatch batch) {
    using T = Tile<BF16, D, WAVES, WALK>;
    constexpr int NL = T::kLoads, KB = T::kKB, NQ = T::kQRegs, DB = D / 32;
    constexpr int kPieces = T::kRow / 16;                 // pieces of a row
    __shared__ __align__(16) char lds[T::kLds];
    __shared__ int holds_infinite[2];                     // the tile whose V values are not all finite
    __shared__ float ml_lds[T::kSplits ? WAVES * 2 * 32 : 1];

    if ((int)blockIdx.x >= a.attention_blocks) {          // the rest of the grid fills the cache
        if (a.four) store_rows<true>(a, batch, blockIdx.x - a.attention_blocks);
        else store_rows<false>(a, batch, blockIdx.x - a.attention_blocks);
        return;
    }
    const int kvh = blockIdx.x % a.Hkv;
    const int unit = prompt_unit(blockIdx.x / a.Hkv, a.fold, a.attention_blocks / a.Hkv);
    const int si = find_sequence(batch.first, batch.n, unit);
    const int n = batch.len[si];
    const int blocks = (n * G + T::kRows - 1) / T::kRows;
    const int block = blocks - 1 - (unit - batch.first[si]);      // the longest ones first
    const int r0 = block * T::kRows;
    const int first_token = r0 / G;
    const int last_token = min(n - 1, (r0 + T::kRows - 1) / G);
    const int tiles = last_token / T::kTileKeys + 1;
    const int headroom = 33 - __builtin_clz(last_token + 1);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int loader = T::kSplits ? lane : threadIdx.x;   // among those that load a tile
    const int wr0 = r0 + wave % T::kRowWaves * 32;
    const int key0 = T::kHalved ? wave / T::kRowWaves * T::kKeys : 0;    // the wave's keys within a tile
    const int row = wr0 + col;                            // the lane's query row
    const int token = min(row / G, n - 1);                // rows past the end repeat the last token's
    const int wave_first = wr0 / G;
    const int wave_last = min(n - 1, (wr0 + 31) / G);
    char* tiles_lds = T::kSplits ? lds + wave * T::kTiles : lds;

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
        const int left = min(T::kTileKeys, n - j * T::kTileKeys);
        const auto r = buffer(base + (size_t)j * T::kTileKeys * stride, left > 0 ? (int)((left - 1) * stride + T::kRow) : 0);
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = loader + u * T::kThreads;
            x[u] = load16(r, (i / kPieces) * (int)stride + i % kPieces * 16);
        }
    };
    auto request_k = [&](int j) __attribute__((always_inline)) { request(k0, a.k_stride, j, kx); };
    auto request_v = [&](int j) __attribute__((always_inline)) { request(v0, a.v_stride, j, vx); };
    auto keep_k = [&](int j) __attribute__((always_inline)) {
        char* to = tiles_lds + j % T::kBuffers * T::kKBuffer;
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = loader + u * T::kThreads;
            *reinterpret_cast<intx4*>(to + i / kPieces * T::kKStride + i % kPieces * 16) = kx[u];
        }
    };
    // whether some value of the caller's pieces was not finite
    auto keep_v = [&](int j) __attribute__((always_inline)) {
        char* to = tiles_lds + T::kBuffers * T::kKBuffer + j % T::kBuffers * T::kVBuffer;
        bool bad = false;
        // Where a tile holds keys behind some query of the block, a weight of zero must not
        // meet an infinity or a NaN: those values are added on their own.
        if (j * T::kTileKeys + T::kTileKeys - 1 > first_token) {
#pragma unroll
            for (int u = 0; u < NL; ++u) vx[u] = finite_part<BF16>(vx[u], bad);
        }
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int i = loader + u * T::kThreads;
            *reinterpret_cast<intx4*>(to + i / kPieces * T::kVStride + i % kPieces * 16) = vx[u];
        }
        return bad;
    };

    float m = -INFINITY, l = 0.f;                         // of the lane's row (l: the lane's own keys)
    floatx16 acc[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

    auto scores = [&](int j, floatx16 (&s)[KB]) __attribute__((always_inline)) {
        const char* kt = tiles_lds + j % T::kBuffers * T::kKBuffer + key0 * T::kKStride;
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
    auto tile = [&](int j, bool infinite) __attribute__((always_inline)) {
        floatx16 s[KB];
        scores(j, s);
        const char* vt = tiles_lds + T::kBuffers * T::kKBuffer + j % T::kBuffers * T::kVBuffer + key0 * T::kVStride;
        const int from = j * T::kTileKeys + key0;
        // key of value i in block b: 32 b + 8 (i / 4) + 4 half + i % 4
        if (from + T::kKeys - 1 > wave_first) {
            const int left = token - from - half * 4;     // keys up to the lane's token, from its first
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
        const float bias = -(m == -INFINITY ? 0.f : m * a.scale_log2) - (BF16 ? kLazy + headroom : kLazy);
        // V's transposed reads (bf16): 4 keys of 16 dims per 16 lanes
        const char* vb = vt + (half * 4 + (lane & 15) / 4) * T::kVStride + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
        constexpr int kGroups = KB * 2;                   // of 16 keys
        unroll<kGroups>([&](auto B) __attribute__((always_inline)) {
            constexpr int b = decltype(B)::value;
            float p[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(fmaf(s[b / 2][b % 2 * 8 + e], a.scale_log2, bias));
                if constexpr (!BF16) {
                    p[e] *= __uint_as_float((127 - headroom) << 23);
                    l += p[e];
                }
            }
            if constexpr (BF16) {
                // The weights as the product takes them, rounded to bf16; their sums too, so that an
                // output is an average under the weights it was formed with.  Against 64 bits the
                // outputs are 2.0e-3 to 2.1e-3 off in the 2-norm, 1.6e-3 of it their own rounding to
                // bf16; a second bf16 part of each weight brings 1.6e-3 and takes 8k tokens of 32/8
                // heads of 128 from 554 to 747 us, 2500 of 16/2 of 64 from 30 to 39.
                bf16x8 w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (__bf16)p[e];
#pragma unroll
                for (int e = 0; e < 8; e += 2)
                    l = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[e], w[e + 1]}, bf16x2{(__bf16)1.f, (__bf16)1.f}, l, false);
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
        if (infinite) {
            // the values that are not finite, from memory, to the queries that see their key
            // (whatever their weight)
            for (int key = from; key <= min(wave_last, from + T::kKeys - 1); ++key) {
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
    if constexpr (T::kSplits) {
        request_k(wave);
        request_v(wave);
        for (int j = wave; j < tiles; j += WAVES) {
            keep_k(j);
            const bool infinite = __any(keep_v(j));
            __builtin_amdgcn_wave_barrier();
            request_k(j + WAVES);
            request_v(j + WAVES);
            tile(j, infinite);
            __builtin_amdgcn_wave_barrier();
        }
    } else {
        if (threadIdx.x < 2) holds_infinite[threadIdx.x] = -1;
        request_k(0);
        request_v(0);
        __syncthreads();
        keep_k(0);
        if (keep_v(0)) holds_infinite[0] = 0;
        request_k(1);
        request_v(1);
        for (int j = 0; j < tiles; ++j) {
            __syncthreads();                              // tile j is in place, tile j - 1 has been read
            if (j + 1 < tiles) {
                keep_k(j + 1);
                if (keep_v(j + 1)) holds_infinite[(j + 1) & 1] = j + 1;
                request_k(j + 2);
                request_v(j + 2);
            }
            // else all of it lies behind the wave's queries
            if (j * T::kTileKeys + key0 <= wave_last) tile(j, holds_infinite[j & 1] == j);
        }
    }

    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    const auto write = [&](int r, int dim, floatx4 o) __attribute__((always_inline)) {
        if (r >= n * G) return;
        char* to = a.out + ((size_t)(batch.start[si] + r / G) * a.Hq + kvh * G + r % G) * T::kRow + dim * T::kElem;
        if constexpr (BF16) {
            typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
            *reinterpret_cast<bf16x4*>(to) = __builtin_convertvector(o, bf16x4);
        } else {
            *reinterpret_cast<floatx4*>(to) = o;
        }
    };
    if constexpr (T::kHalved) {
        // the second halves' states, value by value in the same lanes
        float* state = reinterpret_cast<float*>(lds) + wave % T::kRowWaves * 64 * (D / 2 + 2) + lane;
        __syncthreads();
        if (key0) {
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) state[(d * 16 + i) * 64] = acc[d][i];
            state[D / 2 * 64] = m;
            state[(D / 2 + 1) * 64] = l;
        }
        __syncthreads();
        if (key0) return;
        const float m2 = state[D / 2 * 64];
        const float M = fmaxf(m, m2), Mr = M == -INFINITY ? 0.f : M;     // waves without a key weigh 0
        const float f = m == M ? 1.f : __builtin_amdgcn_exp2f((m - Mr) * a.scale_log2);
        const float f2 = m2 == M ? 1.f : __builtin_amdgcn_exp2f((m2 - Mr) * a.scale_log2);
        l = l * f + state[(D / 2 + 1) * 64] * f2;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = fmaf(state[(d * 16 + i) * 64], f2, acc[d][i] * f);
    }
    if constexpr (!T::kSplits) {
        const float inv = 1.f / l;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                 // dims 32 d + 8 i + 4 half ..
                floatx4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = acc[d][i * 4 + e] * inv;
                write(row, d * 32 + i * 8 + half * 4, r);
            }
    } else {
        float* state = reinterpret_cast<float*>(tiles_lds);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<floatx4*>(state + col * T::kState + d * 32 + i * 8 + half * 4) =
                    floatx4{acc[d][i * 4], acc[d][i * 4 + 1], acc[d][i * 4 + 2], acc[d][i * 4 + 3]};
        if (half == 0) {
            ml_lds[wave * 64 + col] = m;
            ml_lds[wave * 64 + 32 + col] = l;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 32 * (D / 4); e += WAVES * 64) {
            const int r = e / (D / 4), dim = e % (D / 4) * 4;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) M = fmaxf(M, ml_lds[w * 64 + r]);
            const float Mr = M == -INFINITY ? 0.f : M;    // waves without a tile weigh 0
            float L = 0.f;
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float mw = ml_lds[w * 64 + r];
                const float f = mw == M ? 1.f : __builtin_amdgcn_exp2f((mw - Mr) * a.scale_log2);
                const floatx4 v = *reinterpret_cast<const floatx4*>(lds + w * T::kTiles + (r * T::kState + dim) * 4);
                L = fmaf(f, ml_lds[w * 64 + 32 + r], L);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = fmaf(f, v[i], o[i]);
            }
            const float inv = 1.f / L;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] *= inv;
            write(r0 + r, dim, o);
        }
    }
}

int store_blocks(PromptBatch& b) {
    int blocks = 0;
    for (int i = 0; i < b.n; ++i) {
        b.first_store[i] = blocks;
        blocks += (b.len[i] + kPromptStoreTokens - 1) / kPromptStoreTokens;
    }
    return blocks;
}

template <bool BF16, int D, int G, int WAVES, Walk WALK>
hipError_t launch_walk(PromptArgs& a, PromptBatch& b, hipStream_t s) {
    using T = Tile<BF16, D, WAVES, WALK>;
    constexpr PromptWalk w{WALK, WAVES};
    int blocks = 0;
    for (int i = 0; i < b.n; ++i) {
        b.first[i] = blocks;
        blocks += (b.len[i] * G + T::kRows - 1) / T::kRows;
    }
    a.attention_blocks = blocks * a.Hkv;
    a.fold = prompt_fold(w, BF16, D, blocks, a.Hkv);
    const int grid = a.attention_blocks + store_blocks(b);
    hipLaunchKernelGGL((prompt_attention_kernel<BF16, D, G, WAVES, WALK>), dim3(grid), dim3(WAVES * 64), 0, s, a, b);
    return hipGetLastError();
}

template <bool BF16, int D, int G>
hipError_t launch_rows(PromptArgs& a, PromptBatch& b, hipStream_t s) {
    const PromptWalk w = prompt_walk(BF16, D, G, a.Hkv, b.len, b.n);
    if (w.walk == kTeam && w.waves == 8) return launch_walk<BF16, D, G, 8, kTeam>(a, b, s);
    if constexpr (BF16)
        if (w.walk == kTeam) return launch_walk<BF16, D, G, 4, kTeam>(a, b, s);
    if constexpr (!BF16 || D < 256) {
        if (w.walk == kSplit) return launch_walk<BF16, D, G, 4, kSplit>(a, b, s);
        if (w.walk == kHalves) return launch_walk<BF16, D, G, 8, kHalves>(a, b, s);
    }
    return hipErrorInvalidValue;
}

template <bool BF16, int D>
hipError_t launch_group(PromptArgs& a, PromptBatch& b, int group, hipStream_t s) {
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

hipError_t launch_prompt_store(const PromptArgs& a, const PromptBatch& batch, hipStream_t s) {
    PromptBatch b = batch;
    const int blocks = store_blocks(b);
    if (a.four) hipLaunchKernelGGL(prompt_store_kernel<true>, dim3(blocks), dim3(kStoreThreads), 0, s, a, b);
    else hipLaunchKernelGGL(prompt_store_kernel<false>, dim3(blocks), dim3(kStoreThreads), 0, s, a, b);
    return hipGetLastError();
}

hipError_t launch_get_rows(const RowsArgs& a, bool four, hipStream_t s) {
    const int64_t units = (int64_t)a.n * a.Hkv * a.head_bytes / 16;
    const int64_t blocks = (units + 4 * kStoreThreads - 1) / (4 * kStoreThreads);
    const dim3 grid((unsigned)(blocks < 2048 ? blocks : 2048));
    if (four) hipLaunchKernelGGL(rows_kernel<true>, grid, dim3(kStoreThreads), 0, s, a);
    else hipLaunchKernelGGL(rows_kernel<false>, grid, dim3(kStoreThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
