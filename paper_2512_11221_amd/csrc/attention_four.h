// The walk of a wave over a cache's 4-bit rows; included by attention.hip, whose
// kernel it is a part of.
//
// The bytes of a 4-bit row are so few that the arithmetic counts, and the score
// products of the 16-bit rows, whose query heads fill the matrix instruction's 16
// columns by repetition, do every exponential 16 / G times.  Here the columns
// hold several tokens' scores instead: the instruction's contraction runs over
// four slices, slice q4 of A holds dims of one of the tokens c16 + 16 p, and
// column (p, h) of B holds query head h in the slices of part p and zeros in the
// others, so that C has token c16 + 16 p's score under head h in row c16, column
// (p, h).  With up to four query heads there are four parts (64 tokens in one C
// tile, a whole row of K per lane), with eight two (32 tokens, half a row).  One
// or two query heads repeat to fill four.
//
// The weights, exact sums of three bf16 parts each, are rows of the second
// product: block p's leading parts stand in rows (p, h), where C left them, the
// middle and trailing ones in the rows of the next parts (a rotation within 16
// lanes), the rest are zeros, and the rows of one head are summed when the waves
// are merged.  With eight heads the second product takes two passes.  A zero
// weight meets no infinity: 4-bit rows hold none, and a NaN is meant to show.
//
// Loads take whole rows in neighbouring lanes (1 KiB of a dense list in one
// instruction); K's codes pass through LDS into the rows that the lanes hold, V's
// values as bf16, 32 tokens at a time, into transposed reads.
//
// Dense launches over 8 sequences of 32k, 8 KV heads of 128, four query heads each (285 MB),
// random scores: 79.4 us with repeated columns and the 16-bit rows' layouts, 71.8 with several
// tokens a tile, 62 to 69 with non-temporal loads of the scales too (60 with scores that bring
// few new maxima; one query head 60, eight 71); the arithmetic alone takes 58, the loads alone
// 53 to 62, and two waves a SIMD overlap them that far.  Rows of 64 (143 MB, four query heads)
// 43 us, rows of 256 (8 x 16k, 285 MB) 80.

// A group of 32 values as codes, with its scale byte.
__device__ __forceinline__ void encode_group(const intx4 (&x)[4], intx4& codes, uint32_t& byte) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        top = max_magnitude(top, max_magnitude(max_magnitude(x[j][0], x[j][1]), max_magnitude(x[j][2], x[j][3])));
    byte = scale_byte(max(top & 0xFFFFu, top >> 16));
    const float f = scale_value(byte);
#pragma unroll
    for (int j = 0; j < 4; ++j) codes[j] = (int)encode8(x[j][0], x[j][1], x[j][2], x[j][3], f);
}

// Eight codes as bf16.
__device__ __forceinline__ intx4 decode8(uint32_t c, float f) {
    return intx4{(int)decode2<0>(c, f), (int)decode2<1>(c, f), (int)decode2<2>(c, f), (int)decode2<3>(c, f)};
}

// Columns of a part of the score products: a tile of four parts holds 64 tokens, of
// two parts 32 (rows of 256, whose loads and sums take the registers).
constexpr int four_columns(int head_dim, int group) { return group == 8 || head_dim == 256 ? 8 : 4; }

// the value of the lane N places along the lane's row of 16 (which way is the same
// for every use)
template <int N>
__device__ __forceinline__ int row_rotate(int v) {
    return __builtin_amdgcn_update_dpp(0, v, 0x120 + N, 0xF, 0xF, false);
}

// A wave's accumulators as [G][D + 4] sums in LDS: row (p, h) of the weights is one
// part of head h's sums.
template <int D, int G, typename Acc>
__device__ __forceinline__ void store_state_four(const Acc& acc, float* st, int lane) {
    constexpr int S = D + 4;
    const int c16 = lane & 15, q4 = lane >> 4;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        float* col = st + k * 16 + c16;
        const floatx4 v = acc[k];
        if constexpr (four_columns(D, G) == 8) {
            const int h = (q4 & 1) * 4 + (q4 >> 1);
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float x = add_halves(v[i], v[i + 1]);
                if (h + i < G) col[(h + i) * S] = x;
            }
        } else if constexpr (G == 1) {
            const float x = add_halves(add_rows16(v[0], v[0]), 0.f);
            if (q4 == 0) col[0] = x;
        } else if constexpr (G == 2) {
            const float x = add_halves(add_rows16(v[0], v[1]), 0.f);
            if (q4 < 2) col[q4 * S] = x;
        } else {
            col[q4 * S] = add_halves(add_rows16(v[0], v[1]), add_rows16(v[2], v[3]));
        }
    }
}

template <int D, int G>
struct FourStream {
    using R = Row<kRowsFour, D>;
    static constexpr int GC = four_columns(D, G);         // columns of a part
    static constexpr int kParts = 16 / GC;
    static constexpr int kTile = R::kTile;
    static constexpr int kC = kTile / (16 * kParts);      // C tiles of a tile
    static constexpr int kPieces = kParts == 4 ? D / 32 : D / 64;     // 16-byte pieces of K per lane
    static_assert(kPieces == 1 || kPieces == 2 || kPieces == 4, "a lane's scales are one word");
    static constexpr int NL = R::kFourLoads, NB = D / 16;

    int lane, t, t1, n, step, rel_abs;
    char* lds;
    float* rel_kept;
    float scale_log2;
    __amdgpu_buffer_rsrc_t list, k, v, ks, vs;

    int next_rows, next_scale_rows, t_new;
    bool owns_new;
    FourTile<D> kx, vx;
    intx4 k_new, v_new;
    uint32_t k_byte, v_byte;
    const char* q;                                        // the lane's operand of the score products

    __device__ __forceinline__ char* k_scales() const { return lds + R::kTileLds + R::kRelLds; }
    __device__ __forceinline__ char* v_scales() const { return k_scales() + kTile * R::kScales; }
    __device__ __forceinline__ char* queries() const { return v_scales() + kTile * R::kScales; }

    // The list entry that a lane holds, among a tile's: row lane / kScales of load
    // lane % NL, so that the lanes of a row have what they need in every load; and
    // entry `lane`, for the scales, which a load takes in the list's order.
    __device__ __forceinline__ int entry() const { return R::kFourRows * (lane % NL) + lane / R::kScales; }
    template <int J>
    __device__ __forceinline__ int from_entry(int x) const {
        return __builtin_amdgcn_update_dpp(0, x, D == 64 ? J | J << 2 | (2 + J) << 4 | (2 + J) << 6 : J * 0x55, 0xF, 0xF, false);
    }
    __device__ __forceinline__ int rows(int t) const {
        return __builtin_amdgcn_raw_buffer_load_b32(list, t < t1 ? (t * kTile + entry()) * 4 : kNowhere, 0, 0);
    }
    __device__ __forceinline__ int scale_rows(int t) const {
        return __builtin_amdgcn_raw_buffer_load_b32(list, t < t1 ? (t * kTile + lane) * 4 : kNowhere, 0, 0);
    }
    // the list's last entry is the new token: its row comes from the arguments
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, __amdgpu_buffer_rsrc_t rs, int t, int row, int scale_row, FourTile<D>& x) const {
        const int lim = t < t1 ? n - 1 - t * kTile : 0;
        __builtin_amdgcn_sched_barrier(0);
        unroll<NL>([&](auto J) __attribute__((always_inline)) {
            constexpr int j = decltype(J)::value;
            const int o = from_entry<j>(row) * R::kPoolBytes + lane % R::kScales * 16;
            x.codes[j] = load16<kStreamPolicy>(r, j * R::kFourRows + lane / R::kScales < lim ? o : kNowhere);
        });
        const int so = lane < lim && lane < kTile ? scale_row * R::kScales : kNowhere;
        if constexpr (D == 64) x.scale[0] = __builtin_amdgcn_raw_buffer_load_b16(rs, so, 0, kStreamPolicy);
        else if constexpr (D == 128) x.scale[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, so, 0, kStreamPolicy);
        else {
            const uintx2 w = __builtin_bit_cast(uintx2, __builtin_amdgcn_raw_buffer_load_b64(rs, so, 0, kStreamPolicy));
            x.scale[0] = w[0];
            x.scale[1] = w[1];
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void keep_scales(char* to, const FourTile<D>& x) const {
        if (lane >= kTile) return;
        to += lane * R::kScales;
        if constexpr (D == 64) *reinterpret_cast<uint16_t*>(to) = (uint16_t)x.scale[0];
        else if constexpr (D == 128) *reinterpret_cast<uint32_t*>(to) = x.scale[0];
        else *reinterpret_cast<uintx2*>(to) = uintx2{x.scale[0], x.scale[1]};
    }
    // Where LDS holds 16-byte piece p of a row of codes: pieces change places so that 16
    // rows' p-th pieces meet no bank twice.
    __device__ static __forceinline__ int code_at(int row, int p) {
        constexpr int kShift = D == 64 ? 3 : D == 128 ? 2 : 1;
        return row * (D / 2) + (p ^ (row >> kShift & (R::kScales - 1))) * 16;
    }

    // The first tile's loads, the queries into LDS, and the new token's codes where
    // the wave's tiles hold it.  row: of the arguments.
    __device__ __forceinline__ void begin(const AttnArgs& a, int first, int t0, int row, size_t pool_row0) {
        t = first;
        t_new = (n - 1) / kTile;
        owns_new = t_new >= first && t_new < t1 && (t_new - first) % step == 0;
        const int now = rows(t), scales_now = scale_rows(t);
        constexpr int kQ = G * D / 8;                     // 16-byte pieces of the queries
        const auto rq = buffer((const char*)a.q + (size_t)row * G * R::kBytes, G * R::kBytes);
        intx4 qx[(kQ + 63) / 64];
#pragma unroll
        for (int i = 0; i < (kQ + 63) / 64; ++i) qx[i] = load16<0>(rq, (i * 64 + lane) * 16);
        intx4 kn[4], vn[4];
        const int no = owns_new && lane < R::kScales ? lane * 64 : kNowhere;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            kn[e] = load16<0>(buffer((const char*)a.knew + (size_t)row * R::kBytes, R::kBytes), no + e * 16);
            vn[e] = load16<0>(buffer((const char*)a.vnew + (size_t)row * R::kBytes, R::kBytes), no + e * 16);
        }
        const int new_row = __builtin_amdgcn_raw_buffer_load_b32(list, owns_new ? (n - 1) * 4 : kNowhere, 0, 0);
        next_rows = rows(t + step);
        next_scale_rows = scale_rows(t + step);
        load(k, ks, t, now, scales_now, kx);
        load(v, vs, t, now, scales_now, vx);
#pragma unroll
        for (int i = 0; i < (kQ + 63) / 64; ++i) {
            const int e = i * 64 + lane;
            if (e < kQ) *reinterpret_cast<intx4*>(queries() + e / (D / 8) * R::kQStride + e % (D / 8) * 16) = qx[i];
        }
        if (lane < D / 8) *reinterpret_cast<intx4*>(queries() + G * R::kQStride + lane * 16) = intx4{0, 0, 0, 0};
        {
            const int c16 = lane & 15, q4 = lane >> 4;
            const bool mine = q4 / (4 / kParts) == c16 / GC;
            q = queries() + (mine ? c16 % G : G) * R::kQStride + (kParts == 2 ? (q4 & 1) * D : 0);
        }
        if (owns_new) {
            encode_group(kn, k_new, k_byte);
            encode_group(vn, v_new, v_byte);
            if (lane < R::kScales) {                      // the append
                const size_t at = (pool_row0 + new_row) * R::kScales + lane;
                *reinterpret_cast<intx4*>((char*)a.kpool_w + at * 16) = k_new;
                *reinterpret_cast<intx4*>((char*)a.vpool_w + at * 16) = v_new;
                a.kscale_w[at] = (uint8_t)k_byte;
                a.vscale_w[at] = (uint8_t)v_byte;
            }
        }
    }

    // C tile c of the scores: value i is token 32 c + 16 p + 4 q4 + i under the lane's column.
    // A row of A holds a token of every part, so that a NaN would reach the others' scores
    // through their zeros in B: a token with one is computed without and set to NaN behind.
    __device__ __forceinline__ floatx4 scores(int c) const {
        const int c16 = lane & 15, q4 = lane >> 4;
        const int token = kParts == 4 ? lane : c * 32 + (q4 >> 1) * 16 + c16;
        const int piece0 = kParts == 4 ? 0 : (q4 & 1) * kPieces;
        uint32_t sc;
        const char* s = k_scales() + token * R::kScales + piece0;
        if constexpr (kPieces == 1) sc = *reinterpret_cast<const uint8_t*>(s);
        else if constexpr (kPieces == 2) sc = *reinterpret_cast<const uint16_t*>(s);
        else sc = *reinterpret_cast<const uint32_t*>(s);
        const uint32_t none = (~sc - 0x01010101u) & sc & 0x80808080u;     // nonzero: some scale byte is 255
        const uint64_t nans = __ballot(none != 0);        // (lanes of the tokens)
        if (nans && none) sc = 0x7F7F7F7Fu;
        floatx4 sum[2] = {};
#pragma unroll
        for (int e = 0; e < kPieces; ++e) {
            const intx4 x = *reinterpret_cast<const intx4*>(lds + code_at(token, piece0 + e));
            const float f = scale_value(sc >> e * 8 & 255u);
            if constexpr (D == 256) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const intx4 b = *reinterpret_cast<const intx4*>(q + (e * 4 + w) * 16);
                sum[w % 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                    __builtin_bit_cast(bf16x8, decode8(x[w], f)), __builtin_bit_cast(bf16x8, b), sum[w % 2], 0, 0, 0);
            }
        }
        floatx4 r = sum[0] + sum[1];
        if (nans) {
            // four parts: a lane to a token; two: lanes c16 and 16 + c16 of each half have halves of one
            const int first = c16 / GC * (kParts == 4 ? 16 : 32) + q4 * 4;
            const uint64_t of = (kParts == 4 ? nans : nans | nans >> 16) >> first;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = of >> i & 1 ? __builtin_nanf("") : r[i];
        }
        return r;
    }

    // V's rows kSpan J .. of the tile, codes -> LDS as bf16
    template <int J>
    __device__ __forceinline__ void keep_values() {
        constexpr int kFrom = J * R::kSpan / R::kFourRows;
        unroll<R::kSpan / R::kFourRows>([&](auto I) __attribute__((always_inline)) {
            constexpr int i = decltype(I)::value;
            const float f = scale_value((uint8_t)v_scales()[(kFrom + i) * 64 + lane]);
            char* row = lds + (i * R::kFourRows + lane / R::kScales) * R::kVStride + lane % R::kScales * 64;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<intx4*>(row + e * 16) = decode8(vx.codes[kFrom + i][e], f);
        });
        if (t == t_new && (n - 1) % kTile / R::kSpan == J && lane < R::kScales) {
            char* row = lds + (n - 1) % R::kSpan * R::kVStride + lane * 64;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<intx4*>(row + e * 16) = decode8(v_new[e], scale_value(v_byte));
        }
    }

    __device__ __forceinline__ void tile(int kept, float& m, float& l, floatx4 (&acc)[NB]) {
        const int c16 = lane & 15, q4 = lane >> 4;
        const int part = c16 / GC;
        // K's codes and the scales -> LDS
#pragma unroll
        for (int j = 0; j < NL; ++j)
            *reinterpret_cast<intx4*>(lds + code_at(j * R::kFourRows + lane / R::kScales, lane % R::kScales)) = kx.codes[j];
        keep_scales(k_scales(), kx);
        if (t == t_new && lane < R::kScales) {
            const int e = (n - 1) % kTile;
            *reinterpret_cast<intx4*>(lds + code_at(e, lane)) = k_new;
            k_scales()[e * R::kScales + lane] = (char)k_byte;
        }
        __builtin_amdgcn_wave_barrier();
        const int row = next_rows;
        const int scale_row = next_scale_rows;
        next_rows = rows(t + 2 * step);
        next_scale_rows = scale_rows(t + 2 * step);
        load(k, ks, t + step, row, scale_row, kx);

        floatx4 s[kC];
#pragma unroll
        for (int c = 0; c < kC; ++c) s[c] = scores(c);
        __builtin_amdgcn_wave_barrier();

        float y[kC][4];
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[c][i] = s[c][i] * scale_log2;
        if (t * kTile + kTile > n) {                            // entries past the list's end
            const int left = n - t * kTile - part * 16 - q4 * 4;
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[c][i] = c * 32 + i < left ? y[c][i] : -INFINITY;
        }
        // relevance: the sum of |q.k| over the KV head's query heads (neighbouring
        // columns), or the logits themselves
        float* keep = rel_kept + (size_t)(kept * (rel_abs ? 1 : G) + (rel_abs ? 0 : c16 % GC)) * kTile + part * 16 + q4 * 4;
        if (rel_abs) {
#pragma unroll
            for (int c = 0; c < kC; ++c) {
                floatx4 r;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    r[i] = fabsf(s[c][i]);
                    if constexpr (G >= 2) r[i] += dpp_mov<0xB1>(r[i]);     // quad_perm [1,0,3,2]
                    if constexpr (G >= 4) r[i] += dpp_mov<0x4E>(r[i]);     // quad_perm [2,3,0,1]
                    if constexpr (G >= 8) r[i] += dpp_mov<0x141>(r[i]);    // row_half_mirror
                }
                if (c16 % GC == 0) *reinterpret_cast<floatx4*>(keep + c * 32) = r;
            }
        } else if (c16 % GC < G) {
#pragma unroll
            for (int c = 0; c < kC; ++c) *reinterpret_cast<floatx4*>(keep + c * 32) = floatx4{y[c][0], y[c][1], y[c][2], y[c][3]};
        }

        // online softmax; any new maximum rescales the sums
        float top = y[0][0];
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, y[c][i]);
        if (__any(top > m)) {
            top = fmaxf(top, __int_as_float(row_rotate<8>(__float_as_int(top))));
            if constexpr (kParts == 4) top = fmaxf(top, __int_as_float(row_rotate<4>(__float_as_int(top))));
            const float mn = fmaxf(m, column_max(top));
            const float sc = m < mn ? __builtin_amdgcn_exp2f(m - mn) : 1.f;
            l *= sc;
            m = mn;
            float row_sc[4];                              // the scale of row 4 q4 + i: column (4 q4 + i) % GC
            unroll<4>([&](auto I) __attribute__((always_inline)) {
                constexpr int i = decltype(I)::value;
                const int x = row_bcast<i>(__float_as_int(sc));
                if constexpr (G == 8) {
                    const int z = row_bcast<4 + i>(__float_as_int(sc));
                    row_sc[i] = __int_as_float(q4 & 1 ? z : x);
                } else {
                    row_sc[i] = __int_as_float(x);
                }
            });
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[d][i] *= row_sc[i];
        }
        // weights: three bf16 parts of every one, two tokens a word
        const float mr = reference(m);
        int hi[kC][2], mid[kC][2], lo[kC][2];
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                uint32_t u[2], r1[2], r2[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = __builtin_amdgcn_exp2f(y[c][i + e] - mr);
                    l += p;
                    u[e] = __float_as_uint(p);
                    const float rest = p - __uint_as_float(u[e] & 0xFFFF0000u);
                    r1[e] = __float_as_uint(rest);
                    r2[e] = __float_as_uint(rest - __uint_as_float(r1[e] & 0xFFFF0000u));
                }
                hi[c][i / 2] = (int)__builtin_amdgcn_perm(u[1], u[0], 0x07060302u);
                mid[c][i / 2] = (int)__builtin_amdgcn_perm(r1[1], r1[0], 0x07060302u);
                lo[c][i / 2] = (int)__builtin_amdgcn_perm(r2[1], r2[0], 0x07060302u);
            }
        // the parts of the blocks that a lane's rows carry after the rotations
        const int part_mid = kParts == 4 ? row_rotate<4>(part) : row_rotate<8>(part);
        const int part_lo = row_rotate<8>(part);
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mid[c][i] = kParts == 4 ? row_rotate<4>(mid[c][i]) : row_rotate<8>(mid[c][i]);
                if constexpr (kParts == 4) lo[c][i] = row_rotate<8>(lo[c][i]);
            }
        // rows of block b (16 tokens): first pass, second pass (eight heads); masks, because
        // the compiler made branches of selects
        auto weights = [&](int b, int i) __attribute__((always_inline)) {
            const int c = b / kParts, p = b % kParts;
            const int w = (hi[c][i] & -(int)(p == part)) | (mid[c][i] & -(int)(p == part_mid));
            return kParts == 2 ? w : w | (lo[c][i] & -(int)(p == part_lo));
        };
        auto weights_lo = [&](int b, int i) __attribute__((always_inline)) {
            return lo[b / kParts][i] & -(int)(b % kParts == part);
        };

        // V, and O += P V
        keep_scales(v_scales(), vx);
        const char* vb = lds + (q4 * 4 + c16 / 4) * R::kVStride + (c16 % 4) * 8;
        unroll<kTile / R::kSpan>([&](auto J) __attribute__((always_inline)) {
            constexpr int j = decltype(J)::value;
            __builtin_amdgcn_wave_barrier();
            keep_values<j>();
            if constexpr (j == kTile / R::kSpan - 1) load(v, vs, t + step, row, scale_row, vx);
            __builtin_amdgcn_wave_barrier();
            if constexpr (R::kSpan == 16) {
                const shortx4 w = __builtin_bit_cast(shortx4, intx2{weights(j, 0), weights(j, 1)});
                const shortx4 w2 = __builtin_bit_cast(shortx4, intx2{weights_lo(j, 0), weights_lo(j, 1)});
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const shortx4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(vb + d * 32));
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(w, x, acc[d], 0, 0, 0);
                    if constexpr (kParts == 2) acc[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(w2, x, acc[d], 0, 0, 0);
                }
            } else {
                const bf16x8 w = __builtin_bit_cast(bf16x8, intx4{weights(2 * j, 0), weights(2 * j, 1),
                                                                  weights(2 * j + 1, 0), weights(2 * j + 1, 1)});
                const bf16x8 w2 = __builtin_bit_cast(bf16x8, intx4{weights_lo(2 * j, 0), weights_lo(2 * j, 1),
                                                                   weights_lo(2 * j + 1, 0), weights_lo(2 * j + 1, 1)});
#pragma unroll
                for (int d = 0; d < NB; ++d) {
                    const shortx4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(vb + d * 32));
                    const shortx4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(vb + 16 * R::kVStride + d * 32));
                    const bf16x8 x = __builtin_bit_cast(bf16x8, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
                    acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc[d], 0, 0, 0);
                    if constexpr (kParts == 2) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w2, x, acc[d], 0, 0, 0);
                }
            }
        });
    }
};
