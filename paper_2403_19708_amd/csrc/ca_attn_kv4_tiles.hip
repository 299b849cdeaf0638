// Causal attention over the 4-bit cache (layout: ca_kv4.h; Sections 2.1, 3.1, 3.4) for tiles of 256 or 128 stacked query rows.
//
// Eight wavefronts share every key tile of 64: all threads convert it, from codes to fp16 keys, rotated in packed fp16, and to bf16 values
// in LDS, and every wavefront multiplies it in the transposed formulation of ca_attn_dma.hip (v_mfma_f32_32x32x16, S^T = K Q^T, O^T += V^T P^T;
// a lane owns a query row).  Tiles of 256 rows: 32 rows to a wavefront.  Of 128 (SPLIT): two wavefronts have the same rows and half of each
// tile's keys, and add up their sums at the end.  The codes of a tile are asked for a tile ahead, into registers (five or six a thread),
// and tile T + 1 is converted beside the products of tile T (two buffers, one barrier a tile); a workgroup has a compute unit to
// itself, but two of 128 rows with heads of 64 share one (128 registers a thread, none of them spilled: 221 -> 175 us for 16 first turns of
// 128-2048 tokens, 32/4 heads).
//
// Roundings: queries rotated in fp32 to fp16, eleven bits; keys rotated in packed fp16 with angles in fp16; values not at all (two significant
// bits); probabilities to bf16, of which the denominator sums what the product uses.  Relative error against 64 bits 0.0022, half of that
// from the output's own rounding, where operands rotated in fp32 and rounded to bf16 had 0.0033.  The range of fp16: a power of two for a
// query row (query_pieces) and one for a key (key_shift) where it leaves the middle.  Bits are lost (all of them 2^14 further down) where a
// block of 32 dimensions of a key has less than 2^-10 of 1, or of the key's largest block, and where dimensions of a query have less than
// 2^-14 of the row's largest.
//
// What bounds it: a tile of 256 rows is 2176 cycles of matrix instructions a SIMD, 2050 of reads from LDS a compute unit, and some 1900 of
// vector instructions a SIMD; it takes 2.2 us, some 4600 cycles, and one of 128 rows 1.5, where the kernel over expanded keys
// (ca_attn_prerot.hip) takes 1.65 for 256.  us of one layer for 16 turns of 512-2048 + 32-256 tokens, 32 heads: two workgroups of four
// wavefronts and tiles of 32 keys 155; eight wavefronts, keys in fp32 and bf16 103; in fp16 102; the second product at a raised
// priority 100.  These did not help: codes asked for two tiles ahead, the scores of the next tile formed under the softmax of this one, half
// the wavefronts half a tile behind, a fixed order of products and conversions (107-111).
//
// Keys past the end of the item get a scale of zero, whatever the page holds there; a key that is NaN gives NaN scores to the rows that see
// it; values that are NaN are left out of the product and put into the rows that see them afterwards.
#include "ca_kv4.h"

#include <algorithm>
#include <type_traits>

namespace ca {

namespace {

#define CA_INLINE __attribute__((always_inline))

// N words (1, 2 or 4) in one load
template <int N, int W>
__device__ CA_INLINE inline void words_from(const uint8_t *at, uint32_t (&to)[W], int first) {
    if (N == 4) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(at);
#pragma unroll
        for (int i = 0; i < N; ++i) to[first + i] = v[i];
    } else if (N == 2) {
        const u32x2 v = *reinterpret_cast<const u32x2 *>(at);
#pragma unroll
        for (int i = 0; i < N; ++i) to[first + i] = v[i % 2];
    } else {
        to[first] = *reinterpret_cast<const uint32_t *>(at);
    }
}

template <int D, int STYLE, bool SPLIT>
__device__ CA_INLINE inline void attn_kv4_tiles(const AttnArgs &a, const WorkItem &item) {
    constexpr int NW = 8, BN = 64, KSTEPS = D / 16, DBLKS = D / 32;
    constexpr int GROUPS = SPLIT ? NW / 2 : NW;      // of 32 rows
    constexpr int MB = SPLIT ? 1 : 2;                // blocks of 32 keys of a tile that a wavefront multiplies
    constexpr int PPR = D / 8;
    constexpr int E = D / 16;                  // values of each half of a key that a thread converts (eight threads a key)
    constexpr int VW = D / 64;                 // words of codes of a value row that a thread converts
    constexpr int KSTR = 2 * D + 16, VSTR = 2 * D + 64;      // row strides in LDS (bytes)
    constexpr int QSTR = 2 * D + 16;
    constexpr int KBUF = BN * KSTR, VBUF = BN * VSTR;
    static_assert(32 * GROUPS * QSTR <= 2 * (KBUF + VBUF) && GROUPS * QueryRows<D, STYLE>::kQueryBytes <= 2 * (KBUF + VBUF), "queries and outputs pass through the tiles' place");
    static_assert(!SPLIT || GROUPS * 64 * (D / 2 + 2) * 4 <= 2 * (KBUF + VBUF), "and the sums of half the wavefronts");

    __shared__ __attribute__((aligned(16))) uint8_t smem[2 * (KBUF + VBUF)];
    __shared__ uint64_t v_bad[2][NW];
    enum : uint8_t { kBad = 1, kShifted = 2 };
    struct Flags {
        uint8_t marks[NW];                           // of a wavefront: some of its values are NaN, some of its keys were divided
        int8_t up[BN];                               // ... by this power of two
    };
    __shared__ __attribute__((aligned(16))) Flags flags[2];
    __shared__ float q_up[32 * GROUPS];              // factors of the rows of the queries

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int lq = lane & 31, half = lane >> 5;
    const int c = item.seq, g = item.kv_head;
    const int G = a.n_q_heads / a.n_kv_heads, Hkv = a.n_kv_heads;
    const int n = a.n_keep[c], q0 = a.cu_q[c];
    const int32_t *table = a.block_table + (int64_t)c * a.max_pages;
    const int row_last = item.row0 + item.n_rows - 1;
    const int kmax = min(n + row_last / G + 1, item.key_end);       // exclusive end of the keys this item reads
    const int t_begin = item.key_begin / BN, n_tiles = (kmax + BN - 1) / BN, last_page = (kmax - 1) / kPageSize;

    // ---- this lane's query row
    const int group = SPLIT ? wave % GROUPS : wave, mb0 = SPLIT ? wave / GROUPS : 0;
    const int r_raw = item.row0 + group * 32 + lq, r = min(r_raw, row_last);
    const bool row_valid = r_raw <= row_last, wave_live = item.row0 + group * 32 <= row_last;
    const int qpos = n + r / G;                                      // keys 0..qpos are visible
    const int wq_min = n + min(item.row0 + group * 32, row_last) / G, wq_max = n + min(item.row0 + group * 32 + 31, row_last) / G;

    // ---- codes of a tile: a thread has an eighth of both halves of a key and of a value row; a wavefront has eight keys
    const int row = 8 * wave + (lane >> 3), slot = row % kPageSize, sub = lane & 7;
    constexpr int KW = E / 2;                  // words of two values of each half
    struct RawKey {
        uint32_t lo, hi, e;
        uint32_t c[KW], s[KW];                 // rotary pairs of the key's position
    };
    struct RawValue {
        uint32_t w[VW], e;
    };
    const uint8_t *const k_pool = reinterpret_cast<const uint8_t *>(a.k_pool), *const v_pool = reinterpret_cast<const uint8_t *>(a.v_pool);
    // (page ids come by vector loads, one iteration ahead of the loads that need them: what a scalar load brings is waited for together
    // with the reads of LDS around it)
    const auto page_of = [&](int tile) CA_INLINE { return table[min(tile * (BN / kPageSize) + wave / 2, last_page)]; };
    const uint32_t k_at = slot * Kv4<D>::kCodes + sub * (E / 2), v_at = slot * Kv4<D>::kCodes + sub * (VW * 4);
    const uint32_t k_e_at = Kv4<D>::kScaleAt + slot * Kv4<D>::kScales, v_e_at = k_e_at + sub * Kv4<D>::kScales / 8;
    const uint32_t cs_at = row * (2 * D) + sub / 2 * (D / 2) + sub % 2 * (STYLE == 0 ? 2 * E : E);
    auto issue_keys = [&](RawKey &s, int page_v, int tile) CA_INLINE {
        const int page = __builtin_amdgcn_readfirstlane(page_v);
        const uint8_t *kb = k_pool + ((int64_t)page * Hkv + g) * Kv4<D>::kBlock;
        if (D == 128) {
            s.lo = *reinterpret_cast<const uint32_t *>(kb + k_at);
            s.hi = *reinterpret_cast<const uint32_t *>(kb + (k_at + D / 4));
            s.e = *reinterpret_cast<const uint32_t *>(kb + k_e_at);
        } else {
            s.lo = *reinterpret_cast<const uint16_t *>(kb + k_at);
            s.hi = *reinterpret_cast<const uint16_t *>(kb + (k_at + D / 4));
            s.e = *reinterpret_cast<const uint16_t *>(kb + k_e_at);
        }
        // (a tile starts inside the window, and the table ends kRopeSpareRows rows behind it)
        static_assert(BN <= kRopeSpareRows, "rows of a tile that starts at the window's last position");
        const uint8_t *const cs = reinterpret_cast<const uint8_t *>(a.rope16) + (int64_t)min(tile, (a.max_positions - 1) / BN) * (BN * 2 * D) + cs_at;
        if (STYLE == 0) {
            words_from<KW>(cs, s.c, 0);
            words_from<KW>(cs + D / 4, s.s, 0);
        } else {
            words_from<KW / 2>(cs, s.c, 0);
            words_from<KW / 2>(cs + D / 8, s.c, KW / 2);
            words_from<KW / 2>(cs + D / 4, s.s, 0);
            words_from<KW / 2>(cs + (D / 4 + D / 8), s.s, KW / 2);
        }
    };
    auto issue_values = [&](RawValue &s, int page_v) CA_INLINE {
        const int page = __builtin_amdgcn_readfirstlane(page_v);
        const uint8_t *vb = v_pool + ((int64_t)page * Hkv + g) * Kv4<D>::kBlock;
        if (VW == 2) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(vb + v_at);
            s.w[0] = v[0]; s.w[VW - 1] = v[1];
        } else {
            s.w[0] = *reinterpret_cast<const uint32_t *>(vb + v_at);
        }
        s.e = vb[v_e_at];
    };
    RawKey raw_k;
    RawValue raw_v;
    int page0 = page_of(t_begin), page1 = page_of(t_begin + 1), page2 = page_of(t_begin + 2);
    issue_keys(raw_k, page0, t_begin);
    issue_values(raw_v, page0);

    // ---- queries, normalised, rotated, scaled: through LDS to the lanes that multiply them
    const float cscale = a.softmax_scale * 1.4426950408889634f;
    for (int i = tid; i < item.n_rows * (PPR / 2); i += 64 * NW) {
        const int at = i / (PPR / 2), piece = i % (PPR / 2), j = (item.row0 + at) / G;
        const uint16_t *q_row = a.q + ((int64_t)(q0 + j) * a.n_q_heads + g * G + (item.row0 + at - j * G)) * D;
        uint4 x, y;
        const float up = query_pieces<D, STYLE>(a, q_row, n + j, piece, cscale, x, y);
        if (piece == 0) q_up[at] = up;
        *reinterpret_cast<uint4 *>(smem + at * QSTR + 16 * piece) = x;
        *reinterpret_cast<uint4 *>(smem + at * QSTR + D + 16 * piece) = y;
    }
    __syncthreads();
    half8v Qf[KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) Qf[ks] = *reinterpret_cast<const half8v *>(smem + (r - item.row0) * QSTR + 16 * (2 * ks + half));
    const float row_up = q_up[r - item.row0];
    const bool rows_scaled = __builtin_amdgcn_ballot_w64(row_up != 1.f) != 0;
    __syncthreads();

    // ---- codes -> fp16 keys and bf16 values in LDS
    // Where a scale byte leaves the middle of fp16's range (no value past 6 * 2^12 before its rotation; 2^-10 keeps its bits), every key of the
    // wavefront is divided by the power of two returned, its own largest scale: what other keys hold takes no bits from it.  Asked for in front
    // of the products, whose block a branch would end.
    auto key_shift = [&](uint32_t e, int tile) CA_INLINE {
        const bool valid = tile * BN + row < kmax;
        const int block = sub * E / 32;
        const uint32_t e_lo = e >> 8 * block & 255u, e_hi = e >> (8 * block + D / 8) & 255u, most = max(e_lo, e_hi);
        int up = 0;
        if (__builtin_amdgcn_ballot_w64(valid && (most > 127 + 12 || most < 127 - 10)) != 0 && valid) up = (int)kv4_most_scale<D>(e) - 127;
        return up;
    };
    auto convert_keys = [&](const RawKey &s, int up, int tile) CA_INLINE {
        const int buf = tile & 1;
        const bool valid = tile * BN + row < kmax;
        const int block = sub * E / 32;
        uint32_t e_lo = s.e >> 8 * block & 255u, e_hi = s.e >> (8 * block + D / 8) & 255u;
        e_lo = !valid ? 0u : kv4_is_nan(e_lo) ? 255u : (uint32_t)max((int)e_lo - up, 0);
        e_hi = !valid ? 0u : kv4_is_nan(e_hi) ? 255u : (uint32_t)max((int)e_hi - up, 0);
        flags[buf].up[row] = (int8_t)up;
        const float s_lo = kv4_scale(e_lo), s_hi = kv4_scale(e_hi);
        uint32_t lo[KW], hi[KW];
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            half2v l = pair_f16(s.lo, s_lo, w), h = pair_f16(s.hi, s_hi, w);
            rotate_pair<STYLE, KW>(l, h, s.c, s.s, w);
            lo[w] = __builtin_bit_cast(uint32_t, l);
            hi[w] = __builtin_bit_cast(uint32_t, h);
        }
        uint8_t *const to = smem + buf * KBUF + row * KSTR + 2 * sub * E;
        if (E == 8) {
            *reinterpret_cast<uint4 *>(to) = make_uint4(lo[0], lo[1], lo[E / 2 - 2], lo[E / 2 - 1]);
            *reinterpret_cast<uint4 *>(to + D) = make_uint4(hi[0], hi[1], hi[E / 2 - 2], hi[E / 2 - 1]);
        } else {
            *reinterpret_cast<uint2 *>(to) = make_uint2(lo[0], lo[1]);
            *reinterpret_cast<uint2 *>(to + D) = make_uint2(hi[0], hi[1]);
        }
    };
    auto convert_values = [&](const RawValue &s, int up, int tile) CA_INLINE {
        const int buf = tile & 1;
        const bool valid = tile * BN + row < kmax, bad = valid && kv4_is_nan(s.e);
        const uint64_t bads = __builtin_amdgcn_ballot_w64(bad);
        v_bad[buf][wave] = bads;               // by all lanes: a branch would end the block that the conversion shares with the products
        flags[buf].marks[wave] = (bads != 0 ? kBad : 0) | (__builtin_amdgcn_ballot_w64(up != 0) != 0 ? kShifted : 0);
        const float scale = kv4_scale(valid && !bad ? s.e : 0u);
        uint8_t *const v_to = smem + 2 * KBUF + buf * VBUF + row * VSTR + 16 * VW * sub;
#pragma unroll
        for (int w = 0; w < VW; ++w)
            *reinterpret_cast<uint4 *>(v_to + 16 * w) = make_uint4(pair_bf16(s.w[w], scale, 0), pair_bf16(s.w[w], scale, 1), pair_bf16(s.w[w], scale, 2), pair_bf16(s.w[w], scale, 3));
    };

    f32x16 O[DBLKS];
#pragma unroll
    for (int db = 0; db < DBLKS; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;      // reference maximum (exponent units; -inf: no key seen yet), this lane's part of the denominator
    f32x16 neg_ref = {};                       // -m_run (0 while there is none), the accumulator that scores start from
    const bf16x2 ones2 = {(__bf16)1.0f, (__bf16)1.0f};

    f32x16 S[MB];                              // scores of a tile, relative to the reference
    auto scores = [&](int tile) CA_INLINE {
        const uint8_t *const kb = smem + (tile & 1) * KBUF + (32 * mb0 + lq) * KSTR + 16 * half;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                S[mb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8v *>(kb + 32 * mb * KSTR + 32 * ks), Qf[ks], ks == 0 ? neg_ref : S[mb], 0, 0, 0);
    };
    // softmax and second product of `tile`
    auto multiply = [&](int tile, const u32x2 &flag, bool scaled) CA_INLINE {
        const int buf = tile & 1, kt0 = tile * BN + 32 * mb0;
        if (scaled) {                              // from units of the row and of the key
            const float neg = m_run == -INFINITY ? 0.f : -m_run;
            const int up = (int)(__float_as_uint(row_up) >> 23) - 127;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const uint32_t ups = *reinterpret_cast<const uint32_t *>(&flags[buf].up[32 * (mb0 + mb) + 8 * i4 + 4 * half]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) S[mb][4 * i4 + i] = __builtin_ldexpf(S[mb][4 * i4 + i], up + (int8_t)(ups >> 8 * i)) + neg;
                }
#pragma unroll
            for (int i = 0; i < 16; ++i) neg_ref[i] = neg;
        }
        if (kt0 + 32 * MB - 1 > min(wq_min, kmax - 1)) {             // some key may be hidden from some row
            const int last = min(qpos, kmax - 1) - kt0 - 4 * half;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (32 * mb + 8 * (i / 4) + i % 4 > last) S[mb][i] = -INFINITY;
        }
        float mx = S[0][0];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, S[mb][i]);
        constexpr float kHeadroom = 8.0f;
        const bool unseen = m_run == -INFINITY;
        if (__builtin_amdgcn_ballot_w64(mx > (unseen ? -INFINITY : kHeadroom)) != 0) {
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            const float all = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
            const bool raise = all > (unseen ? -INFINITY : kHeadroom);
            const float delta = raise ? all : 0.f;
            const float alpha = raise && !unseen ? __builtin_amdgcn_exp2f(-delta) : 1.0f;
            if (raise) m_run = (unseen ? 0.f : m_run) + all;
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DBLKS; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[db][i] *= alpha;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i) S[mb][i] -= delta;
            const float neg = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
            for (int i = 0; i < 16; ++i) neg_ref[i] = neg;
        }
        // V^T operand (transposing reads): lane s of a 16-lane group points at key k0 + s / 4, dims d0 + 4 (s % 4) .. and receives dim d0 + s of
        // keys k0 .. + 3; an operand has keys 16 ks2 + 4 half + 0..3 and those 8 further, the order of the C registers of S^T
        __builtin_amdgcn_s_setprio(1);
        const uint8_t *const vb = smem + 2 * KBUF + buf * VBUF + (32 * mb0 + 4 * half + (lane >> 2 & 3)) * VSTR + 32 * (lane >> 4 & 1) + 8 * (lane & 3);
#pragma unroll
        for (int ks2 = 0; ks2 < 2 * MB; ++ks2) {
            uint32_t pk[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int i = 8 * (ks2 % 2) + 2 * w;
                pk[w] = pack_bf16(__builtin_amdgcn_exp2f(S[ks2 / 2][i]), __builtin_amdgcn_exp2f(S[ks2 / 2][i + 1]));
                // the denominator sums the rounded probabilities, the very values the second product uses
                l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[w]), ones2, l_run, false);
            }
            const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pk[0], pk[1], pk[2], pk[3]));
#pragma unroll
            for (int db = 0; db < DBLKS; ++db) {
                const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(vb + 16 * ks2 * VSTR + 64 * db));
                const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(vb + (16 * ks2 + 8) * VSTR + 64 * db));
                O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7)), pb, O[db], 0, 0, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if ((__builtin_amdgcn_readfirstlane(flag[0] | flag[1]) & kBad * 0x01010101u) != 0) {       // values that are NaN: the rows that see them
            uint32_t seen = 0;                                       // bit: this lane's row sees one in that block of dimensions
            for (int w = 0; w < NW; ++w)
                for (uint64_t left = v_bad[buf][w]; left; left &= left - 1) {
                    const int at = __builtin_ctzll(left), key = tile * BN + 8 * w + (at >> 3);
                    if (key <= qpos) seen |= 1u << (at & 7) * Kv4<D>::kScales / 8;
                }
#pragma unroll
            for (int db = 0; db < DBLKS; ++db) {
                const float add = seen >> db & 1 ? NAN : 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) O[db][i] += add;
            }
        }
    };

    // Iteration T converts tile T + 1 beside the scores of T, then takes the softmax and the second product of T.  (Past the last tile the
    // last page is asked for and converted once more, for nobody.)
    auto ahead = [&](int tile, int up) CA_INLINE {
        convert_keys(raw_k, up, tile + 1);
        convert_values(raw_v, up, tile + 1);
        issue_keys(raw_k, page2, tile + 2);
        issue_values(raw_v, page2);
        page2 = page_of(tile + 3);
    };
    const int up0 = key_shift(raw_k.e, t_begin);
    convert_keys(raw_k, up0, t_begin);
    convert_values(raw_v, up0, t_begin);
    issue_keys(raw_k, page1, t_begin + 1);
    issue_values(raw_v, page1);
    __syncthreads();
    const int n_mine = wave_live ? min(n_tiles, wq_max / BN + 1) : t_begin;      // tiles that some row of the wavefront sees
    int tile = t_begin;
    for (; tile < n_mine; ++tile) {
        const int up = key_shift(raw_k.e, tile + 1);
        const u32x2 flag = *reinterpret_cast<const u32x2 *>(flags[tile & 1].marks);
        const bool scaled = rows_scaled || (__builtin_amdgcn_readfirstlane(flag[0] | flag[1]) & kShifted * 0x01010101u) != 0;
        if (scaled) neg_ref = f32x16{};            // (the reference would be of other units)
        scores(tile);
        ahead(tile, up);
        multiply(tile, flag, scaled);
        __syncthreads();
    }
    for (; tile < n_tiles; ++tile) {
        ahead(tile, key_shift(raw_k.e, tile + 1));
        __syncthreads();
    }

    float l_all = l_run + __shfl_xor(l_run, 32);
    if (SPLIT) {
        // the other half of the keys: its sums come through LDS, register by register
        float *const other = reinterpret_cast<float *>(smem) + group * 64 * (D / 2 + 2) + lane;
        if (mb0 == 1 && wave_live) {
#pragma unroll
            for (int db = 0; db < DBLKS; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) other[64 * (16 * db + i)] = O[db][i];
            other[64 * (D / 2)] = m_run;
            other[64 * (D / 2 + 1)] = l_all;
        }
        __syncthreads();
        if (mb0 == 1) return;
        if (wave_live) {
            const float m_other = other[64 * (D / 2)], m = fmaxf(m_run, m_other);
            // (a half that saw no key of the row has sums of zero or, of a NaN, NaN)
            const float f = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m), f_other = m_other == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_other - m);
            l_all = f * l_all + f_other * other[64 * (D / 2 + 1)];
#pragma unroll
            for (int db = 0; db < DBLKS; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[db][i] = f * O[db][i] + f_other * other[64 * (16 * db + i)];
            m_run = m;
        }
        lds_handover();                            // the reads are in front of the outputs that pass through the same bytes
    }
    // ---- normalise and store, or leave a share (as the tile kernels over a bf16 cache do)
    if (item.part >= 0) {
        if (row_valid) {
            const int rt = r - item.row0;
            float *base = a.partial + (int64_t)item.part * a.tile_rows * (D + 2);
#pragma unroll
            for (int db = 0; db < DBLKS; ++db)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
                    reinterpret_cast<float4 *>(base)[(8 * db + 2 * i4 + half) * a.tile_rows + rt] = make_float4(O[db][4 * i4], O[db][4 * i4 + 1], O[db][4 * i4 + 2], O[db][4 * i4 + 3]);
            if (half == 0) {
                base[(int64_t)a.tile_rows * D + rt] = m_run / cscale;      // in score units
                base[(int64_t)a.tile_rows * (D + 1) + rt] = l_all;
            }
        }
        return;
    }
    if (wave_live) {
        // (in SPLIT a wavefront's place is that of its own group's sums, which other lanes have read)
        store_rows<D>(a, q0, g, G, item.row0 + group * 32, row_last, smem + group * (SPLIT ? 64 * (D / 2 + 2) * 4 : QueryRows<D, STYLE>::kQueryBytes), O, 1.f / l_all);
    }
}

template <int D, int STYLE, bool SPLIT>
__global__ __launch_bounds__(512, SPLIT && D == 64 ? 4 : 2) void attn_kv4_tiles_kernel(AttnArgs a) {
    const WorkItem item = a.items[blockIdx.x];
    if (item.seq >= 0) attn_kv4_tiles<D, STYLE, SPLIT>(a, item);
}

// ---- behind the attention over the expanded cache (ca_attn_prerot.hip) -------------------------------------------------------------
// NaN into the blocks of the output rows that see a value marked by kv4_expand_kernel: a workgroup looks through the marks of a
// (conversation, kv head) for the first key of each block.
template <int D>
__device__ inline void mark_nan(const AttnArgs &a, int unit, int (&first)[D / 32]) {
    constexpr int BLOCKS = D / 32;
    const int c = unit / a.n_kv_heads, g = unit % a.n_kv_heads, G = a.n_q_heads / a.n_kv_heads, n_threads = blockDim.x;
    const int n = a.n_keep[c], q0 = a.cu_q[c], len = a.cu_q[c + 1] - q0;
    __syncthreads();                                             // (of the unit before)
    if (threadIdx.x < BLOCKS) first[threadIdx.x] = INT_MAX;
    __syncthreads();
    const uint4 *const marks = reinterpret_cast<const uint4 *>(a.v_nan) + (int64_t)g * a.n_dense_pages + a.dense_page0[c];
    const int pages = (n + len + kPageSize - 1) / kPageSize;
#pragma unroll 4
    for (int p = threadIdx.x; p < pages; p += n_threads) {
        const uint4 m = marks[p];
        if ((m.x | m.y | m.z | m.w) == 0) continue;
        const uint32_t word[4] = {m.x, m.y, m.z, m.w};
        for (int t = 0; t < kPageSize; ++t)
            for (int b = 0; b < BLOCKS; ++b)
                if (word[t / 4] >> (8 * (t % 4) + b) & 1u) atomicMin(&first[b], p * kPageSize + t);
    }
    __syncthreads();
    for (int b = 0; b < BLOCKS; ++b) {
        const int from = max(first[b] - n, 0);                   // first new token that sees it
        if (first[b] == INT_MAX) continue;
        for (int64_t i = (int64_t)from * G * 4 + threadIdx.x; i < (int64_t)len * G * 4; i += n_threads) {
            uint16_t *const row = a.out + ((q0 + i / (4 * G)) * a.n_q_heads + g * G + i / 4 % G) * D;
            *reinterpret_cast<uint4 *>(row + 32 * b + 8 * (i % 4)) = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        }
    }
}

template <int D>
__global__ __launch_bounds__(256) void kv4_mark_kernel(AttnArgs a) {
    __shared__ int first[D / 32];
    mark_nan<D>(a, blockIdx.x, first);
}

// The items that it has left, because of a key or a query outside the middle of fp16's range: a workgroup looks at 64 of them at a time and
// there is none, as a rule.  Where no shares are merged in between, also the marks of n_units (conversation, kv head); a row that both
// write gets NaN from either.  With nothing left and no marks 4 us of a launch, 7 behind 4776 items and 512 units.
template <int D, int STYLE, bool SPLIT>
__global__ __launch_bounds__(512, 2) void attn_kv4_rest_kernel(AttnArgs a, int n_units) {
    __shared__ int first[D / 32];
    for (int unit = blockIdx.x; unit < n_units; unit += gridDim.x) mark_nan<D>(a, unit, first);
    for (int from = blockIdx.x; from < a.n_items; from += 64 * gridDim.x) {
        const int at = from + (int)(threadIdx.x & 63) * (int)gridDim.x;
        const bool mine = at < a.n_items && a.items[at].seq >= 0 && a.rest[at] != 0;
        for (uint64_t left = __builtin_amdgcn_ballot_w64(mine); left; left &= left - 1) {
            const WorkItem item = a.items[from + __builtin_ctzll(left) * (int)gridDim.x];
            __syncthreads();                                     // (the wavefronts are through with the item before)
            attn_kv4_tiles<D, STYLE, SPLIT>(a, item);
        }
    }
}

}  // namespace

hipError_t launch_attn_kv4_tiles(const AttnArgs &a, hipStream_t stream) {
    if (a.n_items <= 0) return hipSuccess;
    if (!a.rope16 || (a.tile_rows != 128 && a.tile_rows != 256) || (a.n_combine > 0 && (!a.partial || !a.combine))) return hipErrorInvalidValue;
    if (a.head_dim != 128 && a.head_dim != 64) return hipErrorInvalidValue;
    const auto pick = [&](auto split) {
        constexpr bool S = decltype(split)::value;
        return a.head_dim == 128 ? (a.rope_style == 0 ? attn_kv4_tiles_kernel<128, 0, S> : attn_kv4_tiles_kernel<128, 1, S>)
                                 : (a.rope_style == 0 ? attn_kv4_tiles_kernel<64, 0, S> : attn_kv4_tiles_kernel<64, 1, S>);
    };
    hipLaunchKernelGGL(a.tile_rows == 128 ? pick(std::true_type{}) : pick(std::false_type{}), dim3(a.n_items), dim3(512), 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.n_combine <= 0 ? e : launch_combine_tiles(a, stream);
}

hipError_t launch_attn_kv4_rest(const AttnArgs &a, int n_seqs, int n_cus, hipStream_t stream) {
    if (a.n_items <= 0 || n_seqs <= 0) return hipSuccess;
    if (!a.rope16 || (a.tile_rows != 128 && a.tile_rows != 256) || !a.rest || !a.v_nan || !a.dense_page0 || (a.n_combine > 0 && (!a.partial || !a.combine)))
        return hipErrorInvalidValue;
    if (a.head_dim != 128 && a.head_dim != 64) return hipErrorInvalidValue;
    const auto pick = [&](auto split) {
        constexpr bool S = decltype(split)::value;
        return a.head_dim == 128 ? (a.rope_style == 0 ? attn_kv4_rest_kernel<128, 0, S> : attn_kv4_rest_kernel<128, 1, S>)
                                 : (a.rope_style == 0 ? attn_kv4_rest_kernel<64, 0, S> : attn_kv4_rest_kernel<64, 1, S>);
    };
    const int n_units = n_seqs * a.n_kv_heads, marked = a.n_combine > 0 ? 0 : n_units;
    hipLaunchKernelGGL(a.tile_rows == 128 ? pick(std::true_type{}) : pick(std::false_type{}), dim3(std::min(std::max(a.n_items, marked), n_cus)), dim3(512), 0, stream, a, marked);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_combine <= 0) return e;
    e = launch_combine_tiles(a, stream);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(a.head_dim == 128 ? kv4_mark_kernel<128> : kv4_mark_kernel<64>, dim3(n_units), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ca
