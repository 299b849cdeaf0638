// Causal attention over the 4-bit cache (layout: ca_kv4.h; Sections 2.1, 3.1, 3.4): codes and scales are read, and become operands of the
// matrix cores, fp16 keys rotated to their rebased positions on the way, bf16 values.  The heads of the queries are normalised first where
// the layer has a weight for them (x / sqrt(mean(x^2) + eps) * weight), in fp32.  Here: the kernel for few rows, which rounds queries to fp16
// and rotates them and the keys in packed fp16; the expansion of the cache; the scalar check kernel.
#include "ca_kv4.h"

namespace ca {

namespace {

#define CA_INLINE __attribute__((always_inline))

// f over the four lanes l, l ^ 16, l ^ 32, l ^ 48, which have the keys of one row
template <typename F>
__device__ inline float over_row(float v, F f) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// ---- up to 16 stacked rows to a workgroup, codes straight to the matrix operands -----------------------------------------------
//
// Four wavefronts; each walks a quarter of the item's keys by itself, two pages (32 keys) a step, for all rows:
//   * S^T = K Q^T with v_mfma_f32_16x16x32_f16.  A lane (key m16 of a page, group q4) reads D / 4 codes of its key: dims of the lower half
//     from q4 * D / 8 on and the same of the upper half, so that both members of every rotary pair are its own.
//   * Positions: R(p) q . R(t) k = R(p - t0) q . R(t - t0) k.  Keys are rotated by their place in a block of 64 keys, with (cos, sin) from a
//     table of 64 positions in LDS, and the queries once for every such block by what is left.  Both in packed fp16, eleven bits where
//     bf16 operands have eight: 48 vector instructions a page for the conversion and the rotation of its keys, where advancing
//     the angles in fp32 and rotating in fp32 take 160.
//   * The range of fp16: queries are scaled by a power of two to at most 1, and where a key of a step leaves the range's middle every key of it
//     by one of its own to at most 6; the scores are multiplied by both in fp32.  Bits are lost (all of them 2^14 further down) where a
//     block of a key has less than 2^-10 of 1, or of the key's largest block, and where dimensions of a query have less than 2^-14 of its largest.
//   * O^T += V^T P^T, 32 keys an instruction, in bf16, which holds codes times scales exactly.  A lane reads 32 codes, the block of one
//     scale byte, and writes them to LDS as bf16; the transposing reads bring them back as operands.
//   * The codes and scales of the next step are asked for as soon as this one's are converted, into the same registers.
// Keys past the end of the item get a scale of zero, whatever the page holds there; keys that a row may not see have the score -inf.
// A key that is NaN gives NaN scores to the rows that see it; values that are NaN are left out of the product and put into the rows
// that see them afterwards.
template <int D, int STYLE>
__global__ __launch_bounds__(256, 3) void attn_kv4_kernel(AttnArgs a) {
    constexpr int NWV = 4;
    constexpr int PPR = D / 8, KK = D / 32, DB = D / 16, ROWS = kKv4Rows;
    constexpr int KW = D / 64;                 // words of codes of each half of a key that a lane has (2 or 1)
    constexpr int QSTR = 2 * D + 16;           // row stride of queries, values and angles in LDS (bytes); 5.5 of 11.4 million LDS cycles of a decode of
                                               // 64 conversations are bank conflicts (which accesses they are of was not measured)
    constexpr int OSTR = D + 4;                // of the merge buffer (floats)
    constexpr int VBUF = 32 * QSTR;            // a wavefront's values of one step
    constexpr int SPAN = 64;                   // keys that one rotation of the queries serves
    static_assert(ROWS == 16 && 16 * OSTR * 4 <= VBUF, "sixteen rows of sums fit where the values were");
    static_assert(ROWS * QSTR <= VBUF, "and the queries");

    __shared__ __attribute__((aligned(16))) uint8_t angles[SPAN * QSTR];
    __shared__ __attribute__((aligned(16))) uint8_t v_buf[NWV * VBUF];
    __shared__ float q_scale[ROWS];
    __shared__ float red_m[NWV][ROWS], red_l[NWV][ROWS];
    __shared__ int32_t is_last;

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int q4 = lane >> 4, m16 = lane & 15;
    const int G = a.n_q_heads / a.n_kv_heads, Hkv = a.n_kv_heads;
    // ---- angles of the first SPAN positions -> LDS ---------------------------------------------------------------------------
    // a row of the table: for each q4 the cosines of its D / 8 pairs, then their sines
    const uint8_t *const rope = reinterpret_cast<const uint8_t *>(a.rope16);
    constexpr int APR = 2 * D / 16;            // 16-byte pieces of a row
#pragma unroll
    for (int i = 0; i < SPAN * APR / (64 * NWV); ++i) {
        const int at = i * 64 * NWV + tid;
        *reinterpret_cast<u32x4 *>(angles + at / APR * QSTR + at % APR * 16) = *reinterpret_cast<const u32x4 *>(rope + at * 16);
    }

    const int32_t *iw = reinterpret_cast<const int32_t *>(a.kv4_items + blockIdx.x);
    const int c = load_uniform(iw), g = load_uniform(iw + 1), n_rows = load_uniform(iw + 2);
    const int key_begin = load_uniform(iw + 3), key_end = load_uniform(iw + 4), part = load_uniform(iw + 5);
    const int n = load_uniform(iw + 6), q0 = load_uniform(iw + 7);
    const int32_t *table = a.block_table + (int64_t)c * a.max_pages;
    const int kmax = min(n + (n_rows - 1) / G + 1, key_end);       // exclusive end of the keys this item reads
    const int last_page = (kmax - 1) / kPageSize;
    // pairs of pages of this wavefront (cuts of an item's keys are multiples of 32)
    const int first_pair = key_begin / (2 * kPageSize), n_pairs = last_page / 2 + 1 - first_pair;
    const int per_wave = (n_pairs + NWV - 1) / NWV;
    const int pair_begin = first_pair + wave * per_wave, pair_end = min(first_pair + n_pairs, pair_begin + per_wave);

    // ---- codes and scales of a step ------------------------------------------------------------------------------------
    struct Step {
        uint32_t k_lo[2][KW], k_hi[2][KW];     // [page]
        uint32_t k_e[2];                       // the key's scale bytes
        u32x4 v[KW];                           // D = 128: [page]; 64: lanes 0 to 31 have page 0
        uint32_t v_e[KW];
    };
    const uint8_t *const k_pool = reinterpret_cast<const uint8_t *>(a.k_pool), *const v_pool = reinterpret_cast<const uint8_t *>(a.v_pool);
    const uint32_t k_at = m16 * Kv4<D>::kCodes + q4 * (D / 16), k_e_at = Kv4<D>::kScaleAt + m16 * Kv4<D>::kScales;
    const uint32_t v_lane = KW == 2 ? lane : lane & 31;
    auto issue = [&](Step &s, const int (&page)[2]) CA_INLINE {
        const uint8_t *vb[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int64_t at = ((int64_t)page[x] * Hkv + g) * Kv4<D>::kBlock;
            const uint8_t *kb = k_pool + at;
            vb[x] = v_pool + at;
            if (KW == 2) {
                const u32x2 lo = *reinterpret_cast<const u32x2 *>(kb + k_at), hi = *reinterpret_cast<const u32x2 *>(kb + (k_at + D / 4));
                s.k_lo[x][0] = lo[0]; s.k_lo[x][KW - 1] = lo[1];
                s.k_hi[x][0] = hi[0]; s.k_hi[x][KW - 1] = hi[1];
                s.k_e[x] = *reinterpret_cast<const uint32_t *>(kb + k_e_at);
            } else {
                s.k_lo[x][0] = *reinterpret_cast<const uint32_t *>(kb + k_at);
                s.k_hi[x][0] = *reinterpret_cast<const uint32_t *>(kb + (k_at + D / 4));
                s.k_e[x] = *reinterpret_cast<const uint16_t *>(kb + k_e_at);
            }
        }
        if (KW == 2) {
#pragma unroll
            for (int x = 0; x < KW; ++x) {
                s.v[x] = *reinterpret_cast<const u32x4 *>(vb[x] + 16 * v_lane);
                s.v_e[x] = vb[x][Kv4<D>::kScaleAt + v_lane];
            }
        } else {
            const uint8_t *b = lane < 32 ? vb[0] : vb[1];
            s.v[0] = *reinterpret_cast<const u32x4 *>(b + 16 * v_lane);
            s.v_e[0] = b[Kv4<D>::kScaleAt + v_lane];
        }
    };
    auto page_ids = [&](int pair, int (&page)[2]) CA_INLINE {
#pragma unroll
        for (int x = 0; x < 2; ++x) page[x] = load_uniform(table + min(2 * pair + x, last_page));
    };

    Step s;
    int ids[2];
    page_ids(pair_begin, ids);
    if (pair_begin < pair_end) issue(s, ids);
    page_ids(pair_begin + 1, ids);

    // ---- queries, normalised and scaled, handed on through LDS ------------------------------------------------------------------
    const float cscale = a.softmax_scale * 1.4426950408889634f;
    if (tid < n_rows * PPR) {                  // eight values of a row to a thread
        const int r = tid / PPR, piece = tid % PPR, j = r / G;
        const uint4 raw = *reinterpret_cast<const uint4 *>(a.q + ((int64_t)(q0 + j) * a.n_q_heads + g * G + (r - j * G)) * D + 8 * piece);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        float u[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u[2 * i] = bf_lo(w[i]);
            u[2 * i + 1] = bf_hi(w[i]);
        }
        if (a.q_weight) {
            const float inv = head_norm<D, PPR>(u, a.norm_eps);
            const uint4 gain = *reinterpret_cast<const uint4 *>(a.q_weight + 8 * piece);
            const uint32_t gw[4] = {gain.x, gain.y, gain.z, gain.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u[2 * i] *= inv * bf_lo(gw[i]);
                u[2 * i + 1] *= inv * bf_hi(gw[i]);
            }
        }
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] *= cscale;
            most = fmaxf(most, fabsf(u[i]));
        }
#pragma unroll
        for (int m = 1; m < PPR; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
        const int up = min(max((int)(__float_as_uint(most) >> 23) - 126, -100), 127);     // most <= 2^up
        half2v h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = half2v{(_Float16)__builtin_ldexpf(u[2 * i], -up), (_Float16)__builtin_ldexpf(u[2 * i + 1], -up)};
        *reinterpret_cast<uint4 *>(v_buf + r * QSTR + 16 * piece) =
            make_uint4(__builtin_bit_cast(uint32_t, h[0]), __builtin_bit_cast(uint32_t, h[1]), __builtin_bit_cast(uint32_t, h[2]), __builtin_bit_cast(uint32_t, h[3]));
        if (piece == 0) q_scale[r] = __builtin_ldexpf(1.0f, up);
    }
    __syncthreads();
    const int my_row = min(m16, n_rows - 1);
    const int qpos = n + my_row / G;
    const float q_up = q_scale[my_row];
    half2v q_lo[4 * KW], q_hi[4 * KW];         // this lane's part of its row, without positions
#pragma unroll
    for (int p = 0; p < KW; ++p) {
        const uint4 lo = *reinterpret_cast<const uint4 *>(v_buf + my_row * QSTR + 16 * (KW * q4 + p)), hi = *reinterpret_cast<const uint4 *>(v_buf + my_row * QSTR + D + 16 * (KW * q4 + p));
        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            q_lo[4 * p + w] = __builtin_bit_cast(half2v, wl[w]);
            q_hi[4 * p + w] = __builtin_bit_cast(half2v, wh[w]);
        }
    }
    __syncthreads();

    // operands of the queries for the block of SPAN keys that starts at t0
    half8v Qf[KK];
    auto turn_queries = [&](int t0) CA_INLINE {
        const uint8_t *row = rope + (int64_t)max(qpos - t0, 0) * (2 * D) + q4 * (D / 2);       // (a row that sees none of the keys: any)
        uint32_t cw[4 * KW], sw[4 * KW];
#pragma unroll
        for (int p = 0; p < KW; ++p) {
            const u32x4 cv = *reinterpret_cast<const u32x4 *>(row + 16 * p), sv = *reinterpret_cast<const u32x4 *>(row + D / 4 + 16 * p);
#pragma unroll
            for (int w = 0; w < 4; ++w) { cw[4 * p + w] = cv[w]; sw[4 * p + w] = sv[w]; }
        }
#pragma unroll
        for (int p = 0; p < KW; ++p) {
            u32x4 lo, hi;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                half2v l = q_lo[4 * p + w], h = q_hi[4 * p + w];
                rotate_pair<STYLE, 4 * KW>(l, h, cw, sw, 4 * p + w);
                lo[w] = __builtin_bit_cast(uint32_t, l);
                hi[w] = __builtin_bit_cast(uint32_t, h);
            }
            Qf[p] = __builtin_bit_cast(half8v, lo);
            Qf[p + KW] = __builtin_bit_cast(half8v, hi);
        }
    };

    f32x4 O[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) O[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;      // reference maximum of this lane's row (exponent units), its part of the denominator
    const bf16x2 ones2 = {(__bf16)1.0f, (__bf16)1.0f};

    uint8_t *const my_v = v_buf + wave * VBUF;
    // V^T operand (transposing read): lane s of a 16-lane group points at key 4 q4 + s / 4, dims 4 (s % 4) .. and receives dim s of
    // keys 4 q4 .. + 3
    const uint8_t *const v_rd = my_v + (4 * q4 + (m16 >> 2)) * QSTR + 8 * (m16 & 3);

    for (int pair = pair_begin; pair < pair_end; ++pair) {
        const int key0 = pair * 2 * kPageSize;
        if (pair % 2 == 0 || pair == pair_begin) turn_queries(key0 / SPAN * SPAN);
        // ---- values -> LDS ----
        uint64_t v_bad[KW];
#pragma unroll
        for (int x = 0; x < KW; ++x) {
            const int row = KW == 2 ? 16 * x + lane / 4 : lane / 2, block = KW == 2 ? lane % 4 : lane % 2;
            const uint32_t e = key0 + row < kmax ? s.v_e[x] : 0u;
            v_bad[x] = __builtin_amdgcn_ballot_w64(kv4_is_nan(e));
            const float scale = kv4_scale(kv4_is_nan(e) ? 0u : e);
            uint8_t *to = my_v + row * QSTR + 64 * block;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t word = s.v[x][w];
                *reinterpret_cast<uint4 *>(to + 16 * w) = make_uint4(pair_bf16(word, scale, 0), pair_bf16(word, scale, 1), pair_bf16(word, scale, 2), pair_bf16(word, scale, 3));
            }
        }
        // ---- keys: rotated operands, one page after the other ----
        // Where some key's largest scale byte leaves the middle of fp16's range (no value past 6 * 2^12 before its rotation; 2^-10 keeps its bits),
        // every key of the step is divided by its own: what other keys hold takes no bits from it.
        uint32_t e_all[2], e_key[2];
        bool far = false;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool valid = key0 + x * kPageSize + m16 < kmax;
            e_all[x] = valid ? s.k_e[x] : 0u;
            e_key[x] = kv4_most_scale<D>(e_all[x]);
            far = far || (valid && (e_key[x] < 127 - 10 || e_key[x] > 127 + 12));
        }
        const bool apart = __builtin_amdgcn_ballot_w64(far) != 0;
        f32x4 S[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int shift = apart ? 127 - (int)e_key[x] : 0;
            const auto scale_of = [&](int block) CA_INLINE {               // (zero past the range of a float)
                const uint32_t e = e_all[x] >> 8 * block & 255u;
                return kv4_scale(kv4_is_nan(e) ? 255u : (uint32_t)max((int)e + shift, 0));
            };
            const float s_lo = scale_of(KW == 2 ? q4 >> 1 : 0), s_hi = scale_of(KW == 2 ? 2 + (q4 >> 1) : 1);
            const uint8_t *row = angles + (pair % 2 * 2 * kPageSize + x * kPageSize + m16) * QSTR + q4 * (D / 2);
            uint32_t cw[4 * KW], sw[4 * KW];
#pragma unroll
            for (int p = 0; p < KW; ++p) {
                const u32x4 cv = *reinterpret_cast<const u32x4 *>(row + 16 * p), sv = *reinterpret_cast<const u32x4 *>(row + D / 4 + 16 * p);
#pragma unroll
                for (int w = 0; w < 4; ++w) { cw[4 * p + w] = cv[w]; sw[4 * p + w] = sv[w]; }
            }
            S[x] = f32x4{0.f, 0.f, 0.f, 0.f};
            half8v k[KK];
#pragma unroll
            for (int p = 0; p < KW; ++p) {
                u32x4 lo, hi;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    half2v l = pair_f16(s.k_lo[x][p], s_lo, w), h = pair_f16(s.k_hi[x][p], s_hi, w);
                    rotate_pair<STYLE, 4 * KW>(l, h, cw, sw, 4 * p + w);
                    lo[w] = __builtin_bit_cast(uint32_t, l);
                    hi[w] = __builtin_bit_cast(uint32_t, h);
                }
                k[p] = __builtin_bit_cast(half8v, lo);
                k[p + KW] = __builtin_bit_cast(half8v, hi);
            }
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) S[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[kk], Qf[kk], S[x], 0, 0, 0);
        }
        lds_handover();                        // the values are in LDS
        if (pair + 1 < pair_end) {
            issue(s, ids);
            page_ids(pair + 2, ids);
        }
        // ---- softmax ----
        const float nm = m_run == -INFINITY ? 0.f : -m_run;
        if (apart) {
            const int q_exponent = (int)(__float_as_uint(q_up) >> 23) - 127;
#pragma unroll
            for (int i = 0; i < 8; ++i) {      // (key 4 q4 + i of a page is that of lane 4 q4 + i in each group)
                const int k_exponent = __shfl((int)e_key[i / 4], 16 * q4 + 4 * q4 + i % 4) - 127;
                S[i / 4][i % 4] = __builtin_ldexpf(S[i / 4][i % 4], q_exponent + k_exponent) + nm;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) S[i / 4][i % 4] = S[i / 4][i % 4] * q_up + nm;
        }
        if (key0 + 2 * kPageSize - 1 > min(n, kmax - 1)) {               // some key of the step may be hidden from some row
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (key0 + i / 4 * kPageSize + 4 * q4 + i % 4 > min(qpos, kmax - 1)) S[i / 4][i % 4] = -INFINITY;
        }
        float mx = S[0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, S[i / 4][i % 4]);
        constexpr float kHeadroom = 8.0f;
        const bool unseen = m_run == -INFINITY;
        if (__builtin_amdgcn_ballot_w64(mx > (unseen ? -INFINITY : kHeadroom)) != 0) {
            const float all = over_row(mx, [](float u, float v) { return fmaxf(u, v); });
            const bool raise = all > (unseen ? -INFINITY : kHeadroom);
            const float delta = raise ? all : 0.f;
            const float alpha = raise && !unseen ? __builtin_amdgcn_exp2f(-delta) : 1.0f;
            if (raise) m_run = (unseen ? 0.f : m_run) + all;
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < 8; ++i) S[i / 4][i % 4] -= delta;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) O[db][i] *= alpha;
        }
        uint32_t pw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            pw[i] = pack_bf16(__builtin_amdgcn_exp2f(S[i / 2][2 * (i % 2)]), __builtin_amdgcn_exp2f(S[i / 2][2 * (i % 2) + 1]));
            // the denominator sums the rounded probabilities, the very values the second product uses
            l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pw[i]), ones2, l_run, false);
        }
        const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
        // ---- second product ----
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(v_rd + 32 * db));
            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3))) *)(v_rd + 16 * QSTR + 32 * db));
            O[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7)), pb, O[db], 0, 0, 0);
        }
        if ((v_bad[0] | v_bad[KW - 1]) != 0) {                          // values that are NaN: the rows that see them
            uint32_t seen = 0;                 // bit: this lane's row sees one in that block of dimensions
#pragma unroll
            for (int x = 0; x < KW; ++x)
                for (uint64_t left = v_bad[x]; left; left &= left - 1) {
                    const int at = __builtin_ctzll(left), key = key0 + (KW == 2 ? 16 * x + at / 4 : at / 2);
                    if (key <= qpos) seen |= 1u << (KW == 2 ? at % 4 : at % 2);
                }
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const float add = seen >> (db / 2) & 1 ? NAN : 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) O[db][i] += add;
            }
        }
        lds_handover();                        // the reads are in front of the next step's writes
    }

    // ---- merge the wavefronts ------------------------------------------------------------------------------------------------
    // a share: [ROWS][D] sums, [ROWS] (maximum, denominator)
    constexpr int VPR = D / 4, PART = ROWS * (D + 2) * 4;
    const auto shares = buffer_at(a.partial);
    {
        float *mo = reinterpret_cast<float *>(my_v);
        const float l = over_row(l_run, [](float u, float v) { return u + v; });
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(mo + m16 * OSTR + db * 16 + 4 * q4) = O[db];
        if (q4 == 0) {
            red_m[wave][m16] = m_run;
            red_l[wave][m16] = l;
        }
    }
    __syncthreads();
    for (int i = tid; i < n_rows * VPR; i += 64 * NWV) {
        const int row = i / VPR, d = 4 * (i % VPR);
        float M = red_m[0][row];
#pragma unroll
        for (int w = 1; w < NWV; ++w) M = fmaxf(M, red_m[w][row]);
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < NWV; ++w) {
            // a wavefront that saw no key of the row has sums of zero (or, of a NaN, NaN)
            const float f = red_m[w][row] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(red_m[w][row] - M);
            acc += f * *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(v_buf + w * VBUF) + row * OSTR + d);
            l += f * red_l[w][row];
        }
        if (part < 0) {
            store_out_row4<D>(a, q0, g, G, row, d, acc, 1.f / l);
        } else {
            store_agent4(shares, part * PART + (row * D + d) * 4, acc);
            if (d == 0) store_agent2(shares, part * PART + (ROWS * D + 2 * row) * 4, make_float2(M, l));
        }
    }
    if (part < 0) return;
    // the workgroup that brings a unit's last share merges them all
    const int merge = load_uniform(iw + 8), first = load_uniform(iw + 9), n_parts = load_uniform(iw + 10);
    if (!arrive_last(a.arrived + merge, n_parts, &is_last)) return;
    for (int i = tid; i < n_rows * VPR; i += 64 * NWV) {
        const int row = i / VPR, d = 4 * (i % VPR);
        float M = -INFINITY, l = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        constexpr int U = 4, BATCHES = 4;       // shares of a batch, batches in flight (as many as there are shares for)
        for (int s0 = 0; s0 < n_parts; s0 += BATCHES * U) {
            float2 ml[BATCHES][U];
            f32x4 os[BATCHES][U];
#pragma unroll
            for (int b = 0; b < BATCHES; ++b)
                if (s0 + b * U < n_parts)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int at = (first + min(s0 + b * U + u, n_parts - 1)) * PART;
                        ml[b][u] = load_agent2(shares, at + (ROWS * D + 2 * row) * 4);
                        os[b][u] = load_agent4(shares, at + (row * D + d) * 4);
                    }
#pragma unroll
            for (int b = 0; b < BATCHES; ++b)
                if (s0 + b * U < n_parts) {
                    float M2 = M;
#pragma unroll
                    for (int u = 0; u < U; ++u) M2 = fmaxf(M2, ml[b][u].x);        // (past the last share: that one again)
                    const float fa = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - M2);
                    acc *= fa;
                    l *= fa;
                    M = M2;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const float fb = s0 + b * U + u >= n_parts ? 0.f : ml[b][u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[b][u].x - M2);
                        acc += fb * os[b][u];
                        l += fb * ml[b][u].y;
                    }
                }
        }
        store_out_row4<D>(a, q0, g, G, row, d, acc, 1.f / l);
    }
}

// ---- the batch's context as pages of 16-bit values ------------------------------------------------------------------------------
// Keys rotated at their positions in fp32, rounded to fp16, values as they are in bf16, into the scratch copies that the kernels over keys
// rotated beforehand (ca_attn_prerot.hip) read: dense page dp = pool page rot_src_page[dp].  For plans in which many row tiles share the keys of a
// (conversation, kv head).  Slots past the end of a context become zero (rot_nvalid[dp] of a page are its context's).  Bound by HBM:
// 17/32 of a byte a value in, two out.  A workgroup has a dense page, a thread one (token, pair of 16-byte pieces) of HEADS heads:
// the table row is fetched once for all of them and their loads are all in flight.  Measured with 8 kv heads of 128 dims, a grid of
// 11716 pages: a thread per head 280 us, HEADS 4 196 us (4.9 TB/s, what a copy reaches here); with 4 kv heads of 64 dims only one
// head is left to a thread.
// A product of matrix instructions adds 0 x NaN for the keys that a row does not see, so values that are NaN become 0 here and are
// marked: bit b of v_nan[head][dense page][token] for dims 32 b .. 32 b + 31.  mark_nan gives them to the rows that see them.
// Keys that leave the middle of fp16's range (key_shift in ca_attn_kv4_tiles.hip; zeros do not) are marked too, eight together, and the items
// that load one are left to the kernel that knows a power of two for every key.
template <int D, int STYLE, int HEADS>
__global__ __launch_bounds__(256) void kv4_expand_kernel(AttnArgs a) {
    constexpr int HALF = D / 2, PAIRS = D / 16, SIDE = 256 / (kPageSize * PAIRS);        // heads side by side
    const int H = a.n_kv_heads, slices = (H + SIDE * HEADS - 1) / (SIDE * HEADS);
    const int dp = blockIdx.x / slices, g0 = blockIdx.x % slices * (SIDE * HEADS) + (int)threadIdx.x / (kPageSize * PAIRS);
    const int key = threadIdx.x / PAIRS % kPageSize, pr = threadIdx.x % PAIRS;
    const bool valid = key < a.rot_nvalid[dp];
    const int pos = min(a.rot_pos0[dp] + key, a.max_positions - 1);
    const uint8_t *const from_k = reinterpret_cast<const uint8_t *>(a.k_pool) + (int64_t)a.rot_src_page[dp] * H * Kv4<D>::kBlock;
    const uint8_t *const from_v = reinterpret_cast<const uint8_t *>(a.v_pool) + (int64_t)a.rot_src_page[dp] * H * Kv4<D>::kBlock;
    const int64_t to = ((int64_t)dp * H * kPageSize + key) * D + 8 * pr;
    uint32_t k[HEADS][2], v[HEADS][2], ke[HEADS], ve[HEADS];      // [head][half]
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const uint32_t at = (uint32_t)min(g0 + i * SIDE, H - 1) * Kv4<D>::kBlock;
        const uint32_t codes = at + key * Kv4<D>::kCodes + 4 * pr, scales = at + Kv4<D>::kScaleAt + key * Kv4<D>::kScales;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            k[i][h] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(from_k + (codes + h * (HALF / 2))));
            v[i][h] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t *>(from_v + (codes + h * (HALF / 2))));
        }
        ke[i] = D == 128 ? *reinterpret_cast<const uint32_t *>(from_k + scales) : *reinterpret_cast<const uint16_t *>(from_k + scales);
        ve[i] = D == 128 ? *reinterpret_cast<const uint32_t *>(from_v + scales) : *reinterpret_cast<const uint16_t *>(from_v + scales);
    }
    float2 cs[8];
    load_cs<D, STYLE>(a.rope, pos, pr, cs);
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int g = g0 + i * SIDE;
        if (g >= H) return;
        uint32_t bad = 0;                                        // blocks of the token's values that are NaN
        if (valid)
#pragma unroll
            for (int b = 0; b < D / 32; ++b) bad |= kv4_is_nan(ve[i] >> 8 * b & 255u) ? 1u << b : 0u;
        if (pr == 0) a.v_nan[((int64_t)g * a.n_dense_pages + dp) * kPageSize + key] = (uint8_t)bad;
        const uint32_t most = kv4_most_scale<D>(ke[i]);
        const uint64_t far = __builtin_amdgcn_ballot_w64(valid && most != 0 && (most < 127 - 10 || most > 127 + 12));
        static_assert(64 / PAIRS == 8 || 64 / PAIRS == 16, "a wavefront has eight keys of a head, or all sixteen");
        if (threadIdx.x % 64 == 0) {
            uint8_t *const to = a.k_far + ((int64_t)g * a.n_dense_pages + dp) * 2;
            if (PAIRS == 8) to[key / 8] = far != 0;
            else *reinterpret_cast<uint16_t *>(to) = far != 0;
        }
        const auto scale_of = [&](uint32_t e, int h) CA_INLINE {
            e = e >> 8 * (pr / 4 + h * (D / 64)) & 255u;
            return kv4_scale(!valid ? 0u : kv4_is_nan(e) ? 255u : e);
        };
        const float s0 = scale_of(ke[i], 0), s1 = scale_of(ke[i], 1);
        const uint32_t w0 = valid ? k[i][0] : 0u, w1 = valid ? k[i][1] : 0u;
        uint4 lo, hi;
        uint32_t *pl = reinterpret_cast<uint32_t *>(&lo), *ph = reinterpret_cast<uint32_t *>(&hi);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 x = pair_f32(w0, s0, w), y = pair_f32(w1, s1, w);
            if (STYLE == 0) {
                const float2 c0 = cs[2 * w], c1 = cs[2 * w + 1];
                pl[w] = pack_f16(x.x * c0.x - y.x * c0.y, x.y * c1.x - y.y * c1.y);
                ph[w] = pack_f16(y.x * c0.x + x.x * c0.y, y.y * c1.x + x.y * c1.y);
            } else {
                const float2 c0 = cs[w], c1 = cs[4 + w];
                pl[w] = pack_f16(x.x * c0.x - x.y * c0.y, x.y * c0.x + x.x * c0.y);
                ph[w] = pack_f16(y.x * c1.x - y.y * c1.y, y.y * c1.x + y.x * c1.y);
            }
        }
        const int64_t at = to + (int64_t)g * kPageSize * D;
        *reinterpret_cast<uint4 *>(a.k_rot + at) = lo;
        *reinterpret_cast<uint4 *>(a.k_rot + at + HALF) = hi;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int b = pr / 4 + h * (D / 64);
            const bool is = valid && !(bad >> b & 1u);
            const float scale = kv4_scale(is ? ve[i] >> 8 * b & 255u : 0u);
            const uint32_t word = is ? v[i][h] : 0u;
            *reinterpret_cast<uint4 *>(a.v_t + at + h * HALF) = make_uint4(pair_bf16(word, scale, 0), pair_bf16(word, scale, 1), pair_bf16(word, scale, 2), pair_bf16(word, scale, 3));
        }
    }
}

// ---- scalar check kernel ----------------------------------------------------------------------------------------------------------
// The same operation the slow way, in fp32 (the norm in 64 bits) and without matrix cores, one wavefront per (new token, query head), a lane per key.
template <int D>
__global__ __launch_bounds__(64) void attn_kv4_ref_kernel(AttnArgs a) {
    constexpr int HALF = D / 2;
    const int i = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int c = a.q_seq[i], pos = a.q_pos[i];
    const int g = h / (a.n_q_heads / a.n_kv_heads);
    const int32_t *table = a.block_table + (int64_t)c * a.max_pages;
    const auto first = [&](int p) { return a.rope_style == 0 ? p : 2 * p; };
    const auto second = [&](int p) { return a.rope_style == 0 ? p + HALF : 2 * p + 1; };
    const auto value = [](const uint8_t *block, int slot, int d) {
        uint32_t e = block[Kv4<D>::kScaleAt + slot * Kv4<D>::kScales + d / 32];
        if (kv4_is_nan(e)) e = 255;
        const float2 v = pair_f32(block[slot * Kv4<D>::kCodes + d / 2], kv4_scale(e), 0);
        return d % 2 ? v.y : v.x;
    };
    __shared__ float qr[D];
    {
        const uint16_t *q = a.q + ((int64_t)i * a.n_q_heads + h) * D;
        double inv = 1.0;
        if (a.q_weight) {
            double sum = 0.0;
            for (int d = lane; d < D; d += 64) sum += (double)bf_lo(q[d]) * (double)bf_lo(q[d]);
            for (int w = 32; w >= 1; w >>= 1) sum += __shfl_xor(sum, w);
            inv = 1.0 / sqrt(sum / D + (double)a.norm_eps);
        }
        for (int p = lane; p < HALF; p += 64) {
            const int ia = first(p), ib = second(p);
            const float2 cs = a.rope[(int64_t)pos * HALF + p];
            float x = bf_lo(q[ia]), y = bf_lo(q[ib]);
            if (a.q_weight) { x = (float)(x * inv * bf_lo(a.q_weight[ia])); y = (float)(y * inv * bf_lo(a.q_weight[ib])); }
            qr[ia] = x * cs.x - y * cs.y;
            qr[ib] = y * cs.x + x * cs.y;
        }
    }
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[D];
#pragma unroll
    for (int d = 0; d < D; ++d) o[d] = 0.f;
    for (int t = lane; t <= pos; t += 64) {
        const int64_t off = ((int64_t)table[t / kPageSize] * a.n_kv_heads + g) * Kv4<D>::kBlock;
        const uint8_t *k = reinterpret_cast<const uint8_t *>(a.k_pool) + off, *v = reinterpret_cast<const uint8_t *>(a.v_pool) + off;
        float s = 0.f;
        for (int p = 0; p < HALF; ++p) {
            const int ia = first(p), ib = second(p);
            const float2 cs = a.rope[(int64_t)t * HALF + p];
            const float x = value(k, t % kPageSize, ia), y = value(k, t % kPageSize, ib);
            s += qr[ia] * (x * cs.x - y * cs.y) + qr[ib] * (y * cs.x + x * cs.y);
        }
        s *= a.softmax_scale;
        const float m_new = fmaxf(m, s), alpha = expf(m - m_new), p = expf(s - m_new);
        l = l * alpha + p;
#pragma unroll
        for (int d = 0; d < D; ++d) o[d] = o[d] * alpha + p * value(v, t % kPageSize, d);
        m = m_new;
    }
    float m_all = m;
    for (int w = 32; w >= 1; w >>= 1) m_all = fmaxf(m_all, __shfl_xor(m_all, w));
    const float f = m == -INFINITY ? (l == 0.f ? 0.f : 1.f) : expf(m - m_all);       // (no key, or one that is NaN)
    l *= f;
    for (int w = 32; w >= 1; w >>= 1) l += __shfl_xor(l, w);
    uint16_t *out = a.out + ((int64_t)i * a.n_q_heads + h) * D;
#pragma unroll
    for (int d = 0; d < D; ++d) {
        float x = o[d] * f;
        for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
        if (lane == (d & 63)) out[d] = (uint16_t)pack_bf16(x / l, 0.f);
    }
}

template <int D, int STYLE>
hipError_t launch_rows(const AttnArgs &a, hipStream_t stream) {
    const dim3 grid(a.n_wgs), block(256);
    hipLaunchKernelGGL((attn_kv4_kernel<D, STYLE>), grid, block, 0, stream, a);
    return hipGetLastError();
}

template <int D, int STYLE, int HEADS>
hipError_t launch_expand_heads(const AttnArgs &a, hipStream_t stream) {
    const int per = 256 / D * HEADS;
    const dim3 grid((uint32_t)a.n_dense_pages * (uint32_t)((a.n_kv_heads + per - 1) / per));
    hipLaunchKernelGGL((kv4_expand_kernel<D, STYLE, HEADS>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}
template <int D, int STYLE>
hipError_t launch_expand(const AttnArgs &a, hipStream_t stream) {
    const int heads = (a.n_kv_heads + 256 / D - 1) / (256 / D);   // a thread's, with one workgroup to a page
    return heads >= 3 ? launch_expand_heads<D, STYLE, 4>(a, stream) : heads == 2 ? launch_expand_heads<D, STYLE, 2>(a, stream) : launch_expand_heads<D, STYLE, 1>(a, stream);
}

}  // namespace

hipError_t launch_attn_kv4(const AttnArgs &a, hipStream_t stream) {
    if (a.n_wgs <= 0) return hipSuccess;
    if (!a.rope16 || !a.kv4_items || (a.n_combine > 0 && (!a.partial || !a.arrived))) return hipErrorInvalidValue;
    if (a.head_dim == 128) return a.rope_style == 0 ? launch_rows<128, 0>(a, stream) : launch_rows<128, 1>(a, stream);
    if (a.head_dim == 64) return a.rope_style == 0 ? launch_rows<64, 0>(a, stream) : launch_rows<64, 1>(a, stream);
    return hipErrorInvalidValue;
}

hipError_t launch_kv4_expand(const AttnArgs &a, hipStream_t stream) {
    if (a.n_dense_pages <= 0) return hipSuccess;
    if (!a.k_rot || !a.v_t || !a.v_nan || !a.k_far || !a.rot_src_page || !a.rot_pos0 || !a.rot_nvalid) return hipErrorInvalidValue;
    return a.head_dim == 128 ? (a.rope_style == 0 ? launch_expand<128, 0>(a, stream) : launch_expand<128, 1>(a, stream))
           : a.head_dim == 64 ? (a.rope_style == 0 ? launch_expand<64, 0>(a, stream) : launch_expand<64, 1>(a, stream))
                              : hipErrorInvalidValue;
}

hipError_t launch_attn_kv4_ref(const AttnArgs &a, hipStream_t stream) {
    if (a.total_q <= 0) return hipSuccess;
    const dim3 grid(a.total_q, a.n_q_heads);
    if (a.head_dim == 128) hipLaunchKernelGGL(attn_kv4_ref_kernel<128>, grid, dim3(64), 0, stream, a);
    else if (a.head_dim == 64) hipLaunchKernelGGL(attn_kv4_ref_kernel<64>, grid, dim3(64), 0, stream, a);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace ca
