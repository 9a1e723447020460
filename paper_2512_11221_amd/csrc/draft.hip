// Drafted tokens: their attention over the active cache, and accepted ones' rows into it.
//
// Attention, for node i of sequence b's drafts and query head h,
//   o[i,h] = sum_j softmax_j(q[i,h] . k_j / sqrt(D)) v_j,
// j over the sequence's active list (Eq. 1's set) and over the nodes that sees[i] names.  Every
// row sees the whole list, so a (sequence, KV head) pair's query rows, node by node and head
// by head, are one matrix that the list's K and V rows pass by once: row r is head r % G of
// node r / G.
//
// A tile holds 32 or 64 keys.  The pair's nodes are its first tiles, with a bit per key and
// row; the list's tiles follow, rows gathered by their positions and, of a cache held in 4 bits,
// turned into bf16 on the way to LDS.  Products and softmax are as for prompts: scores
// transposed, S^T = K Q^T with the query row in the lane, O^T = V^T P^T, whose operands are
// the scores' registers and V's transposed LDS reads.
//
// The tiles of all pairs are dealt to a fixed number of workgroups from the counts on the
// device (attention_split.h).  A pair that several workgroups share leaves one partial each, which a
// second launch folds in order.
//
// Bound, by the query rows that a list's bytes meet: to 32 rows by the stream of K and V (8 sequences of 32768 tokens, a
// third of them active, 8 KV heads of 128 in bf16, 20 query rows: 73 us, 5.2 TB/s of rows; 5% more is fetched, of tiles
// behind a part's end, which are asked for ahead); with 256 by matrix cores, LDS and exponentials, a third each (4 of
// 12000 to 16384: 86 us, 0.6 PFLOP/s; the slope of long lists is 0.96); short lists by five round trips, one after the other: 10 us for 512 tokens.  (Folded by the workgroup that
// arrives last, a megabyte of partials went through one compute unit: 64 rows of one sequence of 8000 tokens, 8 KV
// heads, took 77 us, with a launch of its own 40.)
#include <algorithm>
#include <type_traits>

#include "attention_split.h"
#include "kernels.h"
#include "rows.h"
#include "tiles.h"

namespace asrkf {
namespace {

constexpr int kStreamPolicy = 2;              // non-temporal: rows that one workgroup reads
constexpr int kNowhere = (int)0x80000000;     // past every buffer's range: reads as zeros
// What a piece costs a workgroup beside its rows, in tiles: about 5.5 us against 1.7 a tile of 128 keys in 4 bits (32
// sequences of 350 to 2800 tokens, 8 KV heads, 64 rows each: 62.7 us, with 2 64.6, with 5 63.0).
constexpr int kDraftPieceCost = 3;
// The tiles of a part up to which half of the workgroups do (32 rows of 8 sequences of 2000 tokens, 8 KV heads: 28.6 us, with
// 4 32.8), and the parts of a pair at most (one sequence of 8000: 25.2 us with 16 parts, 28.2 with 32; 64 rows 29.2, with 8 32.5).
constexpr int kDraftShort = 8, kDraftParts = 16;
// Tiles of a part at least: a tile of nodes and one of the list stay together (100 tokens: 12.2 us, apart 13.6), but for fp32,
// whose products take sixteen times as long.
constexpr int kDraftLeast = 2;
// As for prompts: the rescaling of O waits until a row's maximum has grown by 2^kLazy.
constexpr float kLazy = 8.f;

__device__ __forceinline__ int wave_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A workgroup's waves: RW take 32 query rows each, KW a share of a tile's keys, DW a share of the
// outputs' dims (rows of 256 values: their sums would take half of the registers).
template <int ROWS, int D, int RW, int KW, int DW>
struct Tile {
    static constexpr bool kFour = ROWS == kRowsFour, kBF16 = ROWS != kRowsF32;
    static constexpr bool kSplit = RW == 1 && DW == 1;    // every wave has a tile of its own
    // The list's K goes from memory into the matrix operands' registers, and not through LDS: 4-bit rows of which a lane
    // takes half a row, that no other wave needs.
    static constexpr bool kDirect = kFour && kSplit;
    static constexpr int kWaves = RW * KW * DW, kThreads = kWaves * 64;
    static constexpr int kRows = 32 * RW;                 // query rows of a workgroup
    static constexpr int kElem = kBF16 ? 2 : 4;
    static constexpr int kRow = D * kElem;                // bytes of a row of one head, in LDS
    static constexpr int kKeys = KW > 1 || kRow > 256 ? 32 : 64;      // keys of a wave's tile
    static constexpr int kStep = KW * kKeys;              // ... of the workgroup's
    static constexpr int kTileKeys = kSplit ? kKeys : kStep;          // ... of a tile in LDS
    static constexpr int kKB = kKeys / 32;                // score blocks of 32 keys
    static constexpr int kDims = D / DW, kDB = kDims / 32;            // of a wave's sums
    static constexpr int kLoaders = kSplit ? 64 : kThreads;
    // LDS row strides: 16 rows of a 16-byte piece (K), and 4 rows of 64 bytes (V, bf16) or
    // rows 4 apart of 128 bytes (V, fp32), meet no bank twice
    static constexpr int kKStride = kRow + 16;
    static constexpr int kVStride = kRow + (kBF16 ? 64 : 32);
    static constexpr int kKBuffer = kTileKeys * kKStride, kVBuffer = kTileKeys * kVStride;
    // one buffer where two of them would leave a compute unit one workgroup of four waves
    static constexpr int kBuffers = kSplit || (kWaves == 4 && 2 * (kKBuffer + kVBuffer) > 80 * 1024) ? 1 : 2;
    static constexpr int kTiles = kBuffers * (kKBuffer + kVBuffer);   // of the workgroup, or of a wave
    static constexpr int kLds = kTiles * (kSplit ? kWaves : 1);
    static constexpr int kPieces = kRow / 16;             // 16-byte pieces of a row in LDS
    static constexpr int kNodeLoads = kTileKeys * kPieces / kLoaders; // of a tile of nodes, per thread
    // pieces of a row in the cache: 16 bytes each, 32 codes of 4 bits with one scale
    static constexpr int kPoolRow = kFour ? D / 2 : kRow;
    static constexpr int kPoolPieces = kPoolRow / 16;
    static constexpr int kPoolTotal = kTileKeys * kPoolPieces;
    static constexpr int kLoads = (kPoolTotal + kLoaders - 1) / kLoaders;
    // Tiles of the list on their way in registers: a launch is bound by what is in flight, and a tile of 4-bit
    // rows, or one that eight waves share, is small.
    static constexpr int kStageRegs = kLoads * (kFour ? 10 : 8);
    static constexpr int kStages = kStageRegs <= 10 ? 4 : kStageRegs <= 16 || DW == 4 ? 2 : 1;
    static constexpr int kQRegs = kBF16 ? D / 16 : D / 8; // 16-byte pieces of q per lane
    static constexpr int kState = D + 4;                  // floats of a row of a wave's state
    static constexpr int kPerSimd = kRow <= 256 || kWaves == 8 || DW > 1 ? 2 : 1;
    static_assert(kNodeLoads * kLoaders == kTileKeys * kPieces, "whole pieces per thread");
    static_assert(kTileKeys <= 64, "a lane per key's list entry");
    static_assert(kSplit || KW == 1 || RW * DW * 64 * (kDims / 2 + 2) * 4 <= kLds, "the states of half the waves fit the tiles");
    static_assert(!kSplit || 32 * kState * 4 <= kTiles, "a wave's state fits its tile");
};

// The tiles dealt to the workgroups.  Batches of up to 64 sequences are planned by every wave
// for itself, one sequence per lane; larger ones by wave 0 into LDS: [B + 1] offsets, then [B]
// tiles.
struct Deal : Split {
    int tiles, units, off;          // of the lane's sequence (up to 64 sequences)
    int n, nodes;                   // its list and its nodes
    int least;                      // tiles of a part
    const int32_t* lds;
    int B;

    // As Split has it, with fewer tiles to a part: a tile costs a round trip to memory.  Half of the workgroups
    // where that leaves short parts, all of them else.
    __device__ __forceinline__ void choose(int total, int longest, int filled) {
        const int average = (total * groups + limit - 1) / limit;
        auto share_of = [&](int most) { return most > 0 ? (longest + most - 1) / most : 1 << 30; };      // most: parts to a pair
        const int pairs = greater(1, filled * groups), half = share_of(limit / 2 / pairs);
        const int all = share_of(limit / pairs);
        share = greater(half <= kDraftShort ? half : all, (longest + kDraftParts - 1) / kDraftParts);
        share = greater(share, least);
        aligned = limit >= pairs && share <= greater(average + cost, kDraftShort);
    }
    __device__ __forceinline__ void ranges(int sum) {
        if (aligned) {
            live = sum;
            return;
        }
        live = greater(1, lesser(limit, sum / (cost + 1)));
        share = sum / live;
        extra = sum - share * live;
        if (sum == 0) live = 0;
    }

    // the sequence that owns unit x
    __device__ __forceinline__ int find(int x) const {
        if (B <= 64) return __popcll(__ballot((int)(threadIdx.x & 63) < B && off + units <= x));
        int lo = 0, hi = B;                       // the first b with lds[b + 1] > x
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (wave_uniform(lds[mid + 1]) <= x) lo = mid + 1; else hi = mid;
        }
        return lo;
    }
    __device__ __forceinline__ int offset(int b) const {
        return B <= 64 ? __builtin_amdgcn_readlane(off, b) : wave_uniform(lds[b]);
    }
    __device__ __forceinline__ int count(int b) const {
        return B <= 64 ? __builtin_amdgcn_readlane(tiles, b) : wave_uniform(lds[B + 1 + b]);
    }
};

__device__ __forceinline__ int nodes_of(const DraftArgs& a, int b) {
    return a.count ? min(max(a.count[b], 0), a.N) : a.N;
}
__device__ __forceinline__ int listed(const DraftArgs& a, int b) { return max(a.n_active[b] - a.list_tail, 0); }

// x of the lane that CTRL names, `old` where there is none (DPP)
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved_in(int old, int x) { return __builtin_amdgcn_update_dpp(old, x, CTRL, ROWS, 0xF, false); }

template <int STEP, int LEAST>
__device__ __forceinline__ Deal make_deal(const DraftArgs& a, int32_t* lds) {
    Deal p;
    p.init(1, a.Hkv * a.row_blocks, 1, a.grid);
    p.cost = kDraftPieceCost;
    p.least = LEAST;
    p.B = a.B;
    p.lds = lds;
    const int lane = threadIdx.x & 63;
    auto tiles = [&](int n, int c) __attribute__((always_inline)) { return c == 0 ? 0 : (n + STEP - 1) / STEP + (c + STEP - 1) / STEP; };
    auto before = [&](int x) __attribute__((always_inline)) {     // inclusive sum over the lanes
        x += moved_in<0x111, 0xF>(0, x);                          // row_shr 1, 2, 4, 8
        x += moved_in<0x112, 0xF>(0, x);
        x += moved_in<0x114, 0xF>(0, x);
        x += moved_in<0x118, 0xF>(0, x);
        x += moved_in<0x142, 0xA>(0, x);                          // row_bcast 15 into rows 1 and 3
        x += moved_in<0x143, 0xC>(0, x);                          // row_bcast 31 into rows 2 and 3
        return x;
    };
    auto total_of = [&](int& sum, int& top, int& filled) __attribute__((always_inline)) {
        sum = __builtin_amdgcn_readlane(before(sum), 63);
        filled = __builtin_amdgcn_readlane(before(filled), 63);
        top = max(top, moved_in<0x111, 0xF>(top, top));
        top = max(top, moved_in<0x112, 0xF>(top, top));
        top = max(top, moved_in<0x114, 0xF>(top, top));
        top = max(top, moved_in<0x118, 0xF>(top, top));
        top = max(top, moved_in<0x142, 0xA>(top, top));
        top = max(top, moved_in<0x143, 0xC>(top, top));
        top = __builtin_amdgcn_readlane(top, 63);
    };
    if (a.B <= 64) {
        p.n = listed(a, min(lane, a.B - 1));
        p.nodes = nodes_of(a, min(lane, a.B - 1));
        p.tiles = lane < a.B ? tiles(p.n, p.nodes) : 0;
        int sum = p.tiles, top = p.tiles, filled = p.tiles > 0;
        total_of(sum, top, filled);
        p.choose(sum, top, filled);
        p.units = p.units_of(p.tiles);
        const int incl = before(p.units);
        p.off = incl - p.units;
        p.ranges(__builtin_amdgcn_readlane(incl, 63));
        return p;
    }
    __shared__ int summary[2];
    if (threadIdx.x < 64) {
        const int per = (a.B + 63) / 64, b0 = min(a.B, lane * per), b1 = min(a.B, b0 + per);
        int sum = 0, top = 0, filled = 0;
        for (int b = b0; b < b1; ++b) {
            const int t = tiles(listed(a, b), nodes_of(a, b));
            lds[a.B + 1 + b] = t;
            sum += t;
            top = max(top, t);
            filled += t > 0;
        }
        total_of(sum, top, filled);
        p.choose(sum, top, filled);
        int mine = 0;
        for (int b = b0; b < b1; ++b) mine += p.units_of(lds[a.B + 1 + b]);
        const int incl = before(mine);
        int run = incl - mine;
        for (int b = b0; b < b1; ++b) {
            lds[b] = run;
            run += p.units_of(lds[a.B + 1 + b]);
        }
        if (lane == 63) {
            lds[a.B] = incl;
            summary[0] = p.share;
            summary[1] = p.aligned ? 1 : 0;
        }
    }
    __syncthreads();
    p.share = wave_uniform(summary[0]);
    p.aligned = wave_uniform(summary[1]) != 0;
    p.ranges(wave_uniform(lds[a.B]));
    return p;
}

// x[from], x[from + 1], ... around, from 0 .. 3
__device__ __forceinline__ intx4 quarters_from(intx4 x, int from) {
    const intx4 y = from & 1 ? intx4{x[1], x[2], x[3], x[0]} : x;
    return from & 2 ? intx4{y[2], y[3], y[0], y[1]} : y;
}

// The weight of a state whose reference is m, in one whose reference is M.
__device__ __forceinline__ float weight(float m, float M, float scale_log2) {
    return m == M ? 1.f : __builtin_amdgcn_exp2f((m - (M == -INFINITY ? 0.f : M)) * scale_log2);
}

// Where part k of a pair lies: a workgroup has a slot in the aligned form, and else two, one for the pair
// that it ends (or holds the middle of) and one for the pair that it begins.
__device__ __forceinline__ int draft_slot(int first, bool aligned, int k) { return aligned ? first + k : first + (k ? 2 * k : 1); }

// Where four dims of a row stand in a partial, as the walk's threads write them: rows one after the other, or a
// row to a lane.
template <bool SPLIT, int D>
__device__ __forceinline__ int partial_at(int rows, int row, int quad) { return SPLIT ? row * D + quad * 4 : (quad * rows + row) * 4; }

// Four dims of a query row of (sequence, KV head), from its sums: zeros where nothing was seen.
template <bool BF16, int D>
__device__ __forceinline__ void write_row(const DraftArgs& a, int b, int kvh, int row, int quad, floatx4 o, float sum) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] *= inv;
    const int G = a.Hq / a.Hkv, shift = __ffs(G) - 1;
    const size_t at = (((size_t)b * a.N + (row >> shift)) * a.Hq + kvh * G + (row & (G - 1))) * D + quad * 4;
    if constexpr (BF16) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<bf16x4*>(reinterpret_cast<__bf16*>(a.out) + at) = __builtin_convertvector(o, bf16x4);
    } else {
        *reinterpret_cast<floatx4*>(reinterpret_cast<float*>(a.out) + at) = o;
    }
}

template <int ROWS, int D, int RW, int KW, int DW>
__global__ void __launch_bounds__((Tile<ROWS, D, RW, KW, DW>::kThreads), (Tile<ROWS, D, RW, KW, DW>::kPerSimd))
draft_kernel(DraftArgs a) {
    using T = Tile<ROWS, D, RW, KW, DW>;
    constexpr bool BF16 = T::kBF16, FOUR = T::kFour;
    constexpr int KB = T::kKB, NQ = T::kQRegs, NL = T::kLoads, DB = T::kDB;
    __shared__ __align__(16) char lds[T::kLds];
    __shared__ float ml_lds[T::kSplit ? T::kWaves * 2 * 32 : 1];
    __shared__ int infinite_lds;
    extern __shared__ __align__(16) int32_t deal_lds[];           // more than 64 sequences

    const int wave = wave_uniform(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int loader = T::kSplit ? lane : threadIdx.x;    // among those that load a tile
    const int row_wave = wave % RW;
    const int key0 = T::kSplit ? 0 : wave / RW % KW * T::kKeys;   // the wave's keys within a tile in LDS
    const int dim0 = wave / (RW * KW) % DW * T::kDims;            // ... dims of the outputs
    char* tiles_lds = T::kSplit ? lds + wave * T::kTiles : lds;
    const int G = a.Hq / a.Hkv, group_shift = __ffs(G) - 1;

    const Deal deal = make_deal<T::kStep, BF16 ? kDraftLeast : 1>(a, deal_lds);
    for (int wi = blockIdx.x; wi < deal.live; wi += gridDim.x) {
    const int w = deal.range_of(wi);
    int x, x_end;
    deal.range(w, x, x_end);
    x = wave_uniform(x);
    x_end = wave_uniform(x_end);
    Piece pc;
    while (next_piece(deal, deal, w, x, x_end, pc)) {
        const int b = wave_uniform(pc.b), gi = wave_uniform(pc.group);
        const int t0 = wave_uniform(pc.t0), t1 = wave_uniform(pc.t1);
        const int n_parts = wave_uniform(pc.n_parts), part = wave_uniform(pc.part);
        const int kvh = gi / a.row_blocks, r0 = gi % a.row_blocks * T::kRows;
        const int n = a.B <= 64 ? __builtin_amdgcn_readlane(deal.n, b) : wave_uniform(listed(a, b));
        const int nodes = a.B <= 64 ? __builtin_amdgcn_readlane(deal.nodes, b) : wave_uniform(nodes_of(a, b));
        const int live_rows = (nodes << group_shift) - r0;        // of the block, at least
        if (live_rows <= 0) continue;             // (every workgroup of the pair does)
        const int node_tiles = (nodes + T::kStep - 1) / T::kStep;
        const int headroom = 33 - __builtin_clz(n + nodes);

        const size_t pair = (size_t)b * a.Hkv + kvh;
        const auto rk = buffer(a.kpool + pair * a.pool_rows * T::kPoolRow, a.pool_rows * T::kPoolRow);
        const auto rv = buffer(a.vpool + pair * a.pool_rows * T::kPoolRow, a.pool_rows * T::kPoolRow);
        const auto rks = buffer(FOUR ? a.kscale + pair * a.pool_rows * (D / kScaleGroup) : nullptr, FOUR ? a.pool_rows * (D / kScaleGroup) : 0);
        const auto rvs = buffer(FOUR ? a.vscale + pair * a.pool_rows * (D / kScaleGroup) : nullptr, FOUR ? a.pool_rows * (D / kScaleGroup) : 0);
        const auto rl = buffer(a.list + (size_t)b * a.cap, n * 4);
        const char* kn = a.k + (size_t)b * a.N * a.k_stride + kvh * T::kRow;
        const char* vn = a.v + (size_t)b * a.N * a.v_stride + kvh * T::kRow;

        const int wr0 = r0 + row_wave * 32;
        const bool idle = row_wave * 32 >= live_rows;     // no row of the wave is written
        const int row = wr0 + col;                        // the lane's query row
        const int node = min(row >> group_shift, nodes - 1);      // rows past the end repeat the last node's
        // where the lane's i-th piece of K and q lies in a row: the two halves of a wave's lanes take eight dims each
        // of a product of 16, or 32 in turn, or a half row
        const auto piece_at = [&](int i) __attribute__((always_inline)) {
            if constexpr (T::kDirect) return (i / 4 * 2 + half) * 64 + i % 4 * 16;
            else return BF16 ? i * 32 + half * 16 : half * (T::kRow / 2) + i * 16;
        };
        // ---- the list's tiles: an entry per lane, then the rows ----
        constexpr int kStages = T::kStages;
        intx4 kx[kStages][NL], vx[kStages][NL];
        uint32_t ks[kStages][FOUR ? NL : 1], vs[kStages][FOUR ? NL : 1];
        // tile j of the wave (split) or of the workgroup
        auto entries = [&](int j) __attribute__((always_inline)) {
            const int at = j * T::kTileKeys + (lane & (T::kTileKeys - 1));
            const int p = __builtin_amdgcn_raw_buffer_load_b32(rl, at < n ? at * 4 : kNowhere, 0, 0);
            return at < n ? p : -1;
        };
        auto request = [&](auto STAGE, int entry) __attribute__((always_inline)) {
            constexpr int g = decltype(STAGE)::value;
#pragma unroll
            for (int u = 0; u < NL; ++u) {
                const int i = loader + u * T::kLoaders;
                const int p = __shfl(entry, i / T::kPoolPieces & (T::kTileKeys - 1));
                const bool in = p >= 0 && (T::kPoolTotal % T::kLoaders == 0 || i < T::kPoolTotal);
                const int off = in ? p * T::kPoolRow + i % T::kPoolPieces * 16 : kNowhere;
                const int so = in ? p * (D / kScaleGroup) + i % T::kPoolPieces : kNowhere;
                int k_off = off;
                if constexpr (T::kDirect) {               // the lane's key, every other piece of its row
                    const int kp = __shfl(entry, col);
                    k_off = kp >= 0 ? kp * T::kPoolRow + (2 * u + half) * 16 : kNowhere;
                    if (u == 0) {                         // all scales of the row
                        const int k_so = kp >= 0 ? kp * (D / kScaleGroup) : kNowhere;
                        ks[g][0] = NL == 2 ? __builtin_amdgcn_raw_buffer_load_b32(rks, k_so, 0, 0) : __builtin_amdgcn_raw_buffer_load_b16(rks, k_so, 0, 0);
                    }
                }
                kx[g][u] = __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(rk, k_off, 0, kStreamPolicy));
                vx[g][u] = __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, kStreamPolicy));
                if constexpr (FOUR) {
                    if constexpr (!T::kDirect) ks[g][u] = __builtin_amdgcn_raw_buffer_load_b8(rks, so, 0, 0);
                    vs[g][u] = __builtin_amdgcn_raw_buffer_load_b8(rvs, so, 0, 0);
                }
            }
        };
        auto keep = [&](auto STAGE, int from, int buf) __attribute__((always_inline)) {
            constexpr int g = decltype(STAGE)::value;
            if (T::kSplit && from >= n) return;           // (nothing of it is the wave's)
            char* kt = tiles_lds + buf * T::kKBuffer;
            char* vt = tiles_lds + T::kBuffers * T::kKBuffer + buf * T::kVBuffer;
#pragma unroll
            for (int u = 0; u < NL; ++u) {
                const int i = loader + u * T::kLoaders;
                if (T::kPoolTotal % T::kLoaders != 0 && i >= T::kPoolTotal) continue;
                const int key = i / T::kPoolPieces, piece = i % T::kPoolPieces;
                if constexpr (FOUR) {
                    // neighbouring lanes stand 64 bytes apart: each writes its four quarters from another one on, so
                    // that they meet no bank twice
                    const float kf = T::kDirect ? 0.f : scale_value(ks[g][u]), vf = scale_value(vs[g][u]);
                    const int turned = lane & 3;
                    const intx4 kq = quarters_from(kx[g][u], turned), vq = quarters_from(vx[g][u], turned);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t kc = (uint32_t)kq[c], vc = (uint32_t)vq[c];
                        const int at = piece * 64 + ((c + turned) & 3) * 16;
                        if constexpr (!T::kDirect)
                            *reinterpret_cast<uintx4*>(kt + key * T::kKStride + at) =
                                uintx4{decode2<0>(kc, kf), decode2<1>(kc, kf), decode2<2>(kc, kf), decode2<3>(kc, kf)};
                        *reinterpret_cast<uintx4*>(vt + key * T::kVStride + at) =
                            uintx4{decode2<0>(vc, vf), decode2<1>(vc, vf), decode2<2>(vc, vf), decode2<3>(vc, vf)};
                    }
                } else {
                    *reinterpret_cast<intx4*>(kt + key * T::kKStride + piece * 16) = kx[g][u];
                    *reinterpret_cast<intx4*>(vt + key * T::kVStride + piece * 16) = vx[g][u];
                }
            }
        };
        // Nodes from .. of a tile into LDS, zeros past the last; whether some value of V was not finite (it is
        // left out there: a weight of zero must not meet it).  Asked for behind the list's rows, they arrive
        // with them; asked for before, their registers were spilled.
        auto keep_nodes = [&](int from) __attribute__((always_inline)) {
            bool bad = false;
            if (T::kSplit && from >= nodes) return bad;
#pragma unroll 4
            for (int u = 0; u < T::kNodeLoads; ++u) {
                const int i = loader + u * T::kLoaders, key = i / T::kPieces, piece = i % T::kPieces;
                intx4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
                if (from + key < nodes) {
                    k = *reinterpret_cast<const intx4*>(kn + (size_t)(from + key) * a.k_stride + piece * 16);
                    v = *reinterpret_cast<const intx4*>(vn + (size_t)(from + key) * a.v_stride + piece * 16);
                }
                v = finite_part<BF16>(v, bad);
                *reinterpret_cast<intx4*>(tiles_lds + key * T::kKStride + piece * 16) = k;
                *reinterpret_cast<intx4*>(tiles_lds + T::kBuffers * T::kKBuffer + key * T::kVStride + piece * 16) = v;
            }
            return bad;
        };

        // List tiles [l0, l1) of the workgroup's steps; those of nodes come first.  Loads come back in the order
        // in which they were asked for, so that waiting for a tile's entries means waiting for all rows asked
        // for before them: they are asked for as many tiles earlier as rows are on their way.
        const int l0 = max(t0, node_tiles) - node_tiles, l1 = t1 - node_tiles;
        const auto tile_of = [&](int j) __attribute__((always_inline)) { return T::kSplit ? j * KW + wave : j; };
        int ahead[kStages + 1];                           // entries of the next tiles to ask for
        int first[kStages];
#pragma unroll
        for (int g = 0; g < kStages; ++g) first[g] = entries(tile_of(l0 + g));
#pragma unroll
        for (int g = 0; g <= kStages; ++g) ahead[g] = entries(tile_of(l0 + kStages + g));
        intx4 q[NQ];
        {
            const char* p = a.q + ((size_t)b * a.N + node) * a.q_stride + (kvh * G + (row & (G - 1))) * T::kRow;
#pragma unroll
            for (int i = 0; i < NQ; ++i) q[i] = *reinterpret_cast<const intx4*>(p + piece_at(i));
        }
        const uint64_t sees = a.sees[(size_t)b * a.N + node] & (nodes >= 64 ? ~0ull : (1ull << nodes) - 1ull);

        unroll<kStages>([&](auto STAGE) __attribute__((always_inline)) { request(STAGE, first[decltype(STAGE)::value]); });

        float m = -INFINITY, l = 0.f;                     // of the lane's row (l: the lane's own keys)
        floatx16 acc[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;

        // the wave's tile in buffer buf; visible: bit j where the lane's row sees key j; piece_of: the i-th of K
        auto tile = [&](int buf, bool masked, uint64_t visible, auto piece_of) __attribute__((always_inline)) {
            const char* vt = tiles_lds + T::kBuffers * T::kKBuffer + buf * T::kVBuffer + key0 * T::kVStride + dim0 * T::kElem;
            floatx16 s[KB];
#pragma unroll
            for (int i = 0; i < NQ; ++i)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const intx4 kr = piece_of(i, kb);
                    if (i == 0)
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
                    if constexpr (BF16) {
                        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr),
                                                                        __builtin_bit_cast(bf16x8, q[i]), s[kb], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__int_as_float(kr[e]), __int_as_float(q[i][e]), s[kb], 0, 0, 0);
                    }
                }
            __builtin_amdgcn_sched_barrier(0);
            // key of value i in block kb: 32 kb + 8 (i / 4) + 4 half + i % 4
            if (masked) {
                const uint64_t mine = visible >> (half * 4);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const uint32_t word = (uint32_t)(mine >> (kb * 32));
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = word >> (i / 4 * 8 + i % 4) & 1 ? s[kb][i] : -INFINITY;
                }
            }
            float top = s[0][0];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
            if (__any(top > m + a.lazy)) {
                const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                const float mn = fmaxf(m, fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
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
            unroll<KB * 2>([&](auto GROUP) __attribute__((always_inline)) {      // of 16 keys
                constexpr int g = decltype(GROUP)::value;
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(fmaf(s[g / 2][g % 2 * 8 + e], a.scale_log2, bias));
                    if constexpr (!BF16) {
                        p[e] *= __uint_as_float((127 - headroom) << 23);
                        l += p[e];
                    }
                }
                if constexpr (BF16) {
                    // weights rounded to bf16 as the product takes them, and their sums of the rounded
                    // ones: an output is an average under the weights it was formed with
                    bf16x8 pw;
#pragma unroll
                    for (int e = 0; e < 8; ++e) pw[e] = (__bf16)p[e];
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        l = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pw[e], pw[e + 1]}, bf16x2{(__bf16)1.f, (__bf16)1.f}, l, false);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        const char* at = vb + g * 16 * T::kVStride + d * 64;
                        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)at);
                        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(at + 8 * T::kVStride));
                        const bf16x8 v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pw, acc[d], 0, 0, 0);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const char* at = vt + (g * 16 + e / 4 * 8 + half * 4 + e % 4) * T::kVStride + col * 4;
#pragma unroll
                        for (int d = 0; d < DB; ++d)
                            acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(at + d * 128),
                                                                          p[e], acc[d], 0, 0, 0);
                    }
                }
            });
        };
        auto in_lds = [&](int buf) __attribute__((always_inline)) {
            const char* kt = tiles_lds + buf * T::kKBuffer + (key0 + col) * T::kKStride;
            return [=](int i, int kb) __attribute__((always_inline)) {
                return *reinterpret_cast<const intx4*>(kt + kb * 32 * T::kKStride + piece_at(i));
            };
        };
        auto list_tile = [&](int buf, int from, auto piece_of) __attribute__((always_inline)) {
            const int left = n - from;
            if (left > 0 && !idle) tile(buf, left < T::kKeys, left >= 64 ? ~0ull : (1ull << left) - 1ull, piece_of);
        };
        auto node_tile = [&](int from, bool infinite) __attribute__((always_inline)) {
            if (from >= nodes || idle) return;
            tile(0, true, sees >> from, in_lds(0));
            if (infinite) {
                // values that are not finite, from memory, to the rows that see their node
                for (int key = from; key < min(nodes, from + T::kKeys); ++key) {
                    const char* at = vn + (size_t)key * a.v_stride + (dim0 + half * 4) * T::kElem;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const char* e = at + (d * 32 + i / 4 * 8 + i % 4) * T::kElem;
                            float v;
                            if constexpr (BF16) v = (float)*reinterpret_cast<const __bf16*>(e);
                            else v = *reinterpret_cast<const float*>(e);
                            if ((sees >> key & 1) && !(fabsf(v) < INFINITY)) acc[d][i] += v;
                        }
                }
            }
        };

        // tile j out of its stage into LDS, and tile j + kStages on its way
        auto turn = [&](auto STAGE, int j, int buf) __attribute__((always_inline)) {
            keep(STAGE, tile_of(j) * T::kTileKeys, buf);
            const int entry = ahead[0];
#pragma unroll
            for (int g = 0; g < kStages; ++g) ahead[g] = ahead[g + 1];
            ahead[kStages] = entries(tile_of(j + 2 * kStages + 1));
            request(STAGE, entry);
        };
        for (int j = t0; j < min(t1, node_tiles); ++j) {
            if constexpr (T::kSplit) {
                const bool infinite = __any(keep_nodes(j * T::kStep + wave * T::kKeys));
                __builtin_amdgcn_wave_barrier();
                node_tile(j * T::kStep + wave * T::kKeys, infinite);
                __builtin_amdgcn_wave_barrier();
            } else {
                if (threadIdx.x == 0) infinite_lds = 0;
                __syncthreads();
                if (keep_nodes(j * T::kStep)) infinite_lds = 1;
                __syncthreads();
                node_tile(j * T::kStep + key0, infinite_lds != 0);
                __syncthreads();
            }
        }
        if constexpr (T::kSplit) {
            for (int j0 = l0; j0 < l1; j0 += kStages)
                unroll<kStages>([&](auto STAGE) __attribute__((always_inline)) {
                    const int j = j0 + decltype(STAGE)::value;
                    if (j >= l1) return;
                    if constexpr (T::kDirect) {
                        constexpr int g = decltype(STAGE)::value;
                        intx4 x[NL];
                        float f[NL];
#pragma unroll
                        for (int u = 0; u < NL; ++u) {
                            x[u] = kx[g][u];
                            f[u] = scale_value(ks[g][0] >> (2 * u + half) * 8 & 0xFF);
                        }
                        turn(STAGE, j, 0);
                        __builtin_amdgcn_wave_barrier();
                        list_tile(0, tile_of(j) * T::kKeys, [&](int i, int) __attribute__((always_inline)) {
                            const uint32_t c = (uint32_t)x[i / 4][i % 4];
                            return __builtin_bit_cast(intx4, uintx4{decode2<0>(c, f[i / 4]), decode2<1>(c, f[i / 4]), decode2<2>(c, f[i / 4]),
                                                                    decode2<3>(c, f[i / 4])});
                        });
                    } else {
                        turn(STAGE, j, 0);
                        __builtin_amdgcn_wave_barrier();
                        list_tile(0, tile_of(j) * T::kKeys, in_lds(0));
                    }
                    __builtin_amdgcn_wave_barrier();
                });
        } else if constexpr (T::kBuffers == 1) {
            for (int j0 = l0; j0 < l1; j0 += kStages)
                unroll<kStages>([&](auto STAGE) __attribute__((always_inline)) {
                    const int j = j0 + decltype(STAGE)::value;
                    if (j >= l1) return;
                    turn(STAGE, j, 0);
                    __syncthreads();
                    list_tile(0, j * T::kStep + key0, in_lds(0));
                    __syncthreads();
                });
        } else {
            if (l0 < l1) turn(std::integral_constant<int, 0>{}, l0, 0);
            for (int j0 = l0; j0 < l1; j0 += kStages)
                unroll<kStages>([&](auto STAGE) __attribute__((always_inline)) {
                    constexpr int g = decltype(STAGE)::value;
                    const int j = j0 + g, buf = kStages % 2 == 0 ? g & 1 : (j - l0) & 1;
                    if (j >= l1) return;
                    __syncthreads();                      // tile j is in place, tile j - 1 has been read
                    if (j + 1 < l1) turn(std::integral_constant<int, (g + 1) % kStages>{}, j + 1, buf ^ 1);
                    list_tile(buf, j * T::kStep + key0, in_lds(buf));
                });
        }

        // ---- the waves' states together, and the outputs or the partial ----
        {
            const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
            l = __uint_as_float(y[0]) + __uint_as_float(y[1]);
        }
        const int first_slot = deal.aligned ? wave_uniform(pc.slot) - part : 2 * (w - part);
        const int slot = draft_slot(first_slot, deal.aligned, part);
        if (part == 0 && threadIdx.x == 0)
            a.fold[(size_t)b * a.Hkv * a.row_blocks + gi] = make_int2(deal.aligned ? n_parts : -n_parts, first_slot);
        float* my_acc = a.part_acc + (size_t)slot * T::kRows * D;
        float* my_ml = a.part_ml + (size_t)slot * 2 * T::kRows;
        auto finish = [&](int r, int quad, floatx4 o, float mx, float sum) __attribute__((always_inline)) {
            if (r >= live_rows) return;
            if (n_parts == 1) {
                write_row<BF16, D>(a, b, kvh, r0 + r, quad, o, sum);
                return;
            }
            *reinterpret_cast<floatx4*>(my_acc + partial_at<T::kSplit, D>(T::kRows, r, quad)) = o;
            if (quad == 0) {
                my_ml[r] = mx;
                my_ml[T::kRows + r] = sum;
            }
        };
        __syncthreads();                                  // every wave has read its tiles
        if constexpr (T::kSplit) {
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
            // rows one after the other, so that only those that are written take time (12 rows of 8 sequences of 8000
            // tokens: 65 us, a row to a lane of all 32 71; 32 rows in 4 bits 43 and 42)
#pragma unroll 2
            for (int e = threadIdx.x; e < min(live_rows, 32) * (D / 4); e += T::kThreads) {
                const int r = e / (D / 4), quad = e % (D / 4);
                float M = -INFINITY, L = 0.f;
#pragma unroll
                for (int k = 0; k < KW; ++k) M = fmaxf(M, ml_lds[k * 64 + r]);
                floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KW; ++k) {
                    const float f = weight(ml_lds[k * 64 + r], M, a.scale_log2);
                    const floatx4 v = *reinterpret_cast<const floatx4*>(lds + k * T::kTiles + (r * T::kState + quad * 4) * 4);
                    L = fmaf(f, ml_lds[k * 64 + 32 + r], L);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = fmaf(f, v[i], o[i]);
                }
                finish(r, quad, o, M, L);
            }
        } else {
            if constexpr (KW == 2) {
                // the second halves' states, value by value in the same lanes
                constexpr int kSums = T::kDims / 2;       // a lane's
                float* state = reinterpret_cast<float*>(lds) + (row_wave + RW * (dim0 / T::kDims)) * 64 * (kSums + 2) + lane;
                if (key0) {
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) state[(d * 16 + i) * 64] = acc[d][i];
                    state[kSums * 64] = m;
                    state[(kSums + 1) * 64] = l;
                }
                __syncthreads();
                if (!key0) {
                    const float m2 = state[kSums * 64], M = fmaxf(m, m2);
                    const float f = weight(m, M, a.scale_log2), f2 = weight(m2, M, a.scale_log2);
                    l = l * f + state[(kSums + 1) * 64] * f2;
                    m = M;
#pragma unroll
                    for (int d = 0; d < DB; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[d][i] = fmaf(state[(d * 16 + i) * 64], f2, acc[d][i] * f);
                }
            }
            if (!key0) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)           // dims 32 d + 8 i + 4 half ..
                        finish(row_wave * 32 + col, dim0 / 4 + d * 8 + i * 2 + half,
                               floatx4{acc[d][i * 4], acc[d][i * 4 + 1], acc[d][i * 4 + 2], acc[d][i * 4 + 3]}, m, l);
            }
        }
        __syncthreads();                                  // the states have been read: tiles may be rewritten
    }
    }
}

// The partials of a pair folded in their order, four dims of a row to a thread, several partials in
// flight: 4 to 8 us, its launch and two round trips.
constexpr int kFoldThreads = 256;
template <bool BF16, int D, bool SPLIT>
__global__ void __launch_bounds__(kFoldThreads)
fold_kernel(DraftArgs a, int rows) {
    constexpr int kQuads = D / 4, kRowsHere = kFoldThreads / kQuads, kPass = 8;
    const int gi = blockIdx.y, b = blockIdx.z;
    const int2 f = a.fold[(size_t)b * a.Hkv * a.row_blocks + gi];
    const int kvh = gi / a.row_blocks, r0 = gi % a.row_blocks * rows;
    const int r = blockIdx.x * kRowsHere + (SPLIT ? threadIdx.x / kQuads : threadIdx.x % kRowsHere);
    const int quad = SPLIT ? threadIdx.x % kQuads : threadIdx.x / kRowsHere;
    // (pairs without nodes were not dealt: what stands there is of an earlier launch)
    if (r >= rows || r0 + r >= nodes_of(a, b) * (a.Hq / a.Hkv)) return;
    const bool aligned = f.x > 0;
    const int n_parts = aligned ? f.x : -f.x;
    if (n_parts == 1) return;
    float M = -INFINITY, L = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < n_parts; k0 += kPass) {
        float pm[kPass], pl[kPass];
        floatx4 po[kPass];
#pragma unroll
        for (int u = 0; u < kPass; ++u) {
            const size_t slot = draft_slot(f.y, aligned, min(k0 + u, n_parts - 1));
            pm[u] = a.part_ml[slot * 2 * rows + r];
            pl[u] = a.part_ml[(slot * 2 + 1) * rows + r];
            po[u] = *reinterpret_cast<const floatx4*>(a.part_acc + slot * rows * D + partial_at<SPLIT, D>(rows, r, quad));
        }
        float Mn = M;
#pragma unroll
        for (int u = 0; u < kPass; ++u)
            if (k0 + u < n_parts) Mn = fmaxf(Mn, pm[u]);
        const float f0 = weight(M, Mn, a.scale_log2);
        L *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= f0;
#pragma unroll
        for (int u = 0; u < kPass; ++u) {
            if (k0 + u >= n_parts) continue;
            const float fu = weight(pm[u], Mn, a.scale_log2);
            L = fmaf(fu, pl[u], L);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fmaf(fu, po[u][i], o[i]);
        }
        M = Mn;
    }
    write_row<BF16, D>(a, b, kvh, r0 + r, quad, o, L);
}

struct DraftLaunch {
    int blocks;
    hipStream_t stream;
    int* occupancy;                 // non-null: report it instead
};

template <int ROWS, int D, int RW, int KW, int DW>
hipError_t launch_walk(const DraftArgs& args, const DraftLaunch& l) {
    using T = Tile<ROWS, D, RW, KW, DW>;
    auto kernel = draft_kernel<ROWS, D, RW, KW, DW>;
    if (l.occupancy) return hipOccupancyMaxActiveBlocksPerMultiprocessor(l.occupancy, kernel, T::kThreads, 0);
    DraftArgs a = args;
    a.row_blocks = (a.N * (a.Hq / a.Hkv) + T::kRows - 1) / T::kRows;
    const size_t lds = a.B > 64 ? (size_t)(2 * a.B + 1) * 4 : 0;
    hipLaunchKernelGGL(kernel, dim3(l.blocks), dim3(T::kThreads), lds, l.stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = std::min(T::kRows, a.N * (a.Hq / a.Hkv)), per = kFoldThreads / (D / 4);
    hipLaunchKernelGGL((fold_kernel<T::kBF16, D, T::kSplit>), dim3((rows + per - 1) / per, a.Hkv * a.row_blocks, a.B), dim3(kFoldThreads), 0, l.stream, a,
                       T::kRows);
    return hipGetLastError();
}

template <int ROWS, int D>
hipError_t launch_rows(const DraftArgs& a, int rows, const DraftLaunch& l) {
    if constexpr (D == 256) {
        switch (rows) {
            case 32: return launch_walk<ROWS, D, 1, 2, 4>(a, l);
            case 64: return launch_walk<ROWS, D, 2, 1, 2>(a, l);
            case 128: return launch_walk<ROWS, D, 4, 1, 2>(a, l);
        }
    } else {
        switch (rows) {
            case 32: return launch_walk<ROWS, D, 1, 4, 1>(a, l);
            case 64:
                if constexpr (ROWS != kRowsFour) return launch_walk<ROWS, D, 2, 2, 1>(a, l);
                break;
            case 128: return launch_walk<ROWS, D, 4, 1, 1>(a, l);
            case 256: return launch_walk<ROWS, D, 8, 1, 1>(a, l);
        }
    }
    return hipErrorInvalidValue;
}

hipError_t dispatch(const DraftArgs& a, int rows_kind, int head_dim, int rows, const DraftLaunch& l) {
    if (rows_kind == kRowsBF16) {
        if (head_dim == 64) return launch_rows<kRowsBF16, 64>(a, rows, l);
        if (head_dim == 128) return launch_rows<kRowsBF16, 128>(a, rows, l);
        if (head_dim == 256) return launch_rows<kRowsBF16, 256>(a, rows, l);
    } else if (rows_kind == kRowsFour) {
        if (head_dim == 64) return launch_rows<kRowsFour, 64>(a, rows, l);
        if (head_dim == 128) return launch_rows<kRowsFour, 128>(a, rows, l);
        if (head_dim == 256) return launch_rows<kRowsFour, 256>(a, rows, l);
    } else {
        if (head_dim == 64) return launch_rows<kRowsF32, 64>(a, rows, l);
        if (head_dim == 128) return launch_rows<kRowsF32, 128>(a, rows, l);
    }
    return hipErrorInvalidValue;
}

// ---- accepted nodes ----

constexpr int kAcceptThreads = 256;

// A workgroup copies the rows of one (layer, sequence); the last to finish extends every
// sequence's lists and lengths, which all of them have read by then.  Bound by round trips: 2.3 us for one sequence,
// 7.1 for 4 layers of 8 with 8 nodes.
template <bool FOUR>
__global__ void __launch_bounds__(kAcceptThreads)
accept_kernel(AcceptArgs a) {
    __shared__ int path[kMaxDrafts];
    __shared__ int last;
    const int b = blockIdx.x, layer = blockIdx.y;
    const int t = *a.t_dev;
    // nodes taken: up to the first entry that names none, and none where the room is short
    auto taken = [&](int seq, int n) __attribute__((always_inline)) {
        int take = min(max(a.n_path[seq], 0), a.N);
        for (int i = 0; i < take; ++i)
            if ((uint32_t)a.path[(size_t)seq * a.N + i] >= (uint32_t)a.N) take = i;
        return n + take > a.max_ctx ? -1 : take;
    };
    const int n = a.plen[b] + t;
    const int take = max(taken(b, n), 0);
    if ((int)threadIdx.x < take) path[threadIdx.x] = a.path[(size_t)b * a.N + threadIdx.x];
    __syncthreads();
    const int per_head = a.head_bytes / 16, per_token = per_head * a.Hkv;     // powers of two
    const int head_shift = __ffs(per_head) - 1, token_shift = __ffs(per_token) - 1;
    const int pool_bytes = FOUR ? a.head_bytes / 4 : a.head_bytes;
    const char* k = a.k + (size_t)layer * a.k_layer + (size_t)b * a.N * a.k_stride;
    const char* v = a.v + (size_t)layer * a.v_layer + (size_t)b * a.N * a.v_stride;
    const size_t row0 = ((size_t)layer * a.B + b) * a.Hkv * a.pool_rows + n;
    for (int u = threadIdx.x; u < take << token_shift; u += kAcceptThreads) {
        const int i = u >> token_shift, e = u & (per_token - 1);
        const int g = e >> head_shift, p = e & (per_head - 1);
        const uintx4 x = *reinterpret_cast<const uintx4*>(k + (size_t)path[i] * a.k_stride + e * 16);
        const uintx4 y = *reinterpret_cast<const uintx4*>(v + (size_t)path[i] * a.v_stride + e * 16);
        const size_t row = row0 + (size_t)g * a.pool_rows + i, at = row * pool_bytes;
        if constexpr (FOUR) {
            const bool of_64 = per_head == 8;
            uint32_t ks, vs;
            *reinterpret_cast<uint32_t*>(a.kpool + at + p * 4) = round8(x, of_64, ks);
            *reinterpret_cast<uint32_t*>(a.vpool + at + p * 4) = round8(y, of_64, vs);
            const size_t to = (row * per_head + p) / 4;           // the first of the lanes' groups
            if (of_64 && p == 0) {
                *reinterpret_cast<uint16_t*>(a.kscale + to) = (uint16_t)ks;
                *reinterpret_cast<uint16_t*>(a.vscale + to) = (uint16_t)vs;
            } else if (!of_64 && p % 16 == 0) {
                *reinterpret_cast<uint32_t*>(a.kscale + to) = ks;
                *reinterpret_cast<uint32_t*>(a.vscale + to) = vs;
            }
        } else {
            *reinterpret_cast<uintx4*>(a.kpool + at + p * 16) = x;
            *reinterpret_cast<uintx4*>(a.vpool + at + p * 16) = y;
        }
    }
    __syncthreads();                              // n and take have been read by every thread
    if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(a.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)(gridDim.x * gridDim.y) - 1;
    __syncthreads();
    if (!last) return;
    unsigned long long more = 0;
    for (int i = threadIdx.x; i < a.states * a.B; i += kAcceptThreads) {
        const int seq = i % a.B, len = a.plen[seq] + t, grow = taken(seq, len);
        if (grow < 0) *a.no_room = 1;
        if (grow <= 0) continue;
        const int na = a.n_active[i];             // the last entry is the next token's position, len
        for (int j = 1; j <= grow; ++j) a.list[(size_t)i * a.cap + na - 1 + j] = len + j;
        a.n_active[i] = na + grow;
        more += grow;
    }
    if (more) atomicAdd(a.listed_total, more);
    __syncthreads();                              // every list has been extended from the old lengths
    for (int seq = threadIdx.x; seq < a.B; seq += kAcceptThreads) {
        const int grow = taken(seq, a.plen[seq] + t);
        if (grow > 0) a.plen[seq] += grow;
    }
    if (threadIdx.x == 0) *a.ticket = 0;          // ready for the next launch
}

}  // namespace

// Rows of a pair by the least workgroup that has room for all of them, so that the list is read once; but twice 32 for 64
// rows over a cache in 4 bits, which waits for its products and not for memory, and needs no barrier there (64 rows, 8 KV
// heads of 128 values: 32 sequences of 2000 tokens 44 us against 56, 8 of 32000 134 against 143, one of 8000 22 against 29;
// 128 rows in fours 80, 221 and 26 against 79, 192 and 37).  In bf16: 64 rows of 8 sequences of 8000 tokens 99 us in two
// blocks, 70 in one; 256 rows 191 by 32, 160 by 64, 122 by 128, 104 in one.
int draft_rows(int rows_kind, int n, int group, int head_dim) {
    const int rows = n * group;
    if (rows <= 32 || (rows <= 64 && rows_kind == kRowsFour && head_dim <= 128)) return 32;
    return rows <= 64 ? 64 : rows <= 128 || head_dim == 256 ? 128 : 256;
}

hipError_t draft_occupancy(int rows_kind, int head_dim, int rows, int* blocks_per_cu) {
    return dispatch(DraftArgs{}, rows_kind, head_dim, rows, DraftLaunch{0, nullptr, blocks_per_cu});
}

hipError_t launch_drafts(const DraftArgs& args, int rows_kind, int head_dim, int blocks, hipStream_t s) {
    DraftArgs a = args;
    a.scale_log2 = (float)(1.4426950408889634 / __builtin_sqrt((double)head_dim));
    a.lazy = kLazy / a.scale_log2;
    return dispatch(a, rows_kind, head_dim, draft_rows(rows_kind, a.N, a.Hq / a.Hkv, head_dim), DraftLaunch{blocks, s, nullptr});
}

hipError_t launch_accept(const AcceptArgs& a, hipStream_t s) {
    const dim3 grid(a.B, a.L);
    if (a.four) hipLaunchKernelGGL(accept_kernel<true>, grid, dim3(kAcceptThreads), 0, s, a);
    else hipLaunchKernelGGL(accept_kernel<false>, grid, dim3(kAcceptThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace asrkf
