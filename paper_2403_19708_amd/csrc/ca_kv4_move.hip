// The 4-bit cache (layout: ca_kv4.h): a turn's keys and values quantised into it, moves between the pool and the tier, and reading it back.
//
// All of it is bound by HBM, or by the host link where the tier is pinned host memory.
#include "ca_kv4.h"

#include <algorithm>

namespace ca {

namespace {

constexpr int kThreads = 256;

// ---- quantising append -----------------------------------------------------------------------------------------------
// x -> the e2m1 number nearest to x / 2^p (ties to the even code), p the smallest with M <= 6 * 2^p, M the largest magnitude of the
// block, from -127 to 125: no value is cut off but for magnitudes above 6 * 2^125, which become that, and every step is exact
// (6 = 1.5 * 2^2: p follows from M's exponent and whether its mantissa passes 1.5).  A block that holds an infinity or a NaN becomes NaN as a whole.  Eight values a lane, four lanes a block, D / 8 a row.
// With `weight`, rows are normalised first: x / sqrt(mean(x^2) + eps) * weight, rounded to fp32 and then to bf16.  In 64 bits: a value
// next to a border of its rounding falls on the side that the definition gives it, and the products and the root are few beside the bytes.
template <int D>
__device__ inline void quantise(const uint4 raw, const uint16_t *weight, double eps, int lane, uint32_t &codes, uint32_t &byte) {
    constexpr int LPR = D / 8;
    uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    if (weight) {
        double x[8], sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf_lo(w[i]);
            x[2 * i + 1] = bf_hi(w[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += x[i] * x[i];
#pragma unroll
        for (int m = 1; m < LPR; m *= 2) sum += __shfl_xor(sum, m);
        const double inv = 1.0 / sqrt(sum / D + eps);
        const uint4 wt = *reinterpret_cast<const uint4 *>(weight + 8 * (lane % LPR));
        const uint32_t g[4] = {wt.x, wt.y, wt.z, wt.w};
        // (to 32 bits, then to 16, where left alone the compiler takes one step)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo = (float)(x[2 * i] * inv * (double)bf_lo(g[i])), hi = (float)(x[2 * i + 1] * inv * (double)bf_hi(g[i]));
            asm("" : "+v"(lo), "+v"(hi));
            w[i] = pack_bf16(lo, hi);
        }
    }
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, max(w[i] & 0x7fffu, w[i] >> 16 & 0x7fffu));
    most = max(most, (uint32_t)__shfl_xor((int)most, 1));
    most = max(most, (uint32_t)__shfl_xor((int)most, 2));
    const bool bad = most >= 0x7f80u;
    const int e = (int)(most >> 7) - 2 + ((most & 0x7f) > 0x40);
    const uint32_t at = min((uint32_t)max(e, 0), kKv4MostScale);
    byte = bad ? 255u : at;
    const float up = kv4_scale(254u - at);                         // 2^(127 - at)
    codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, bf_lo(w[0]) * up, bf_hi(w[0]) * up, 1.0f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, bf_lo(w[1]) * up, bf_hi(w[1]) * up, 1.0f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, bf_lo(w[2]) * up, bf_hi(w[2]) * up, 1.0f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, bf_lo(w[3]) * up, bf_hi(w[3]) * up, 1.0f, 3);
    if (bad) codes = 0;
}

// 256 / (D / 8) new tokens to a workgroup, eight values of HEADS heads side by side to a thread, all of them asked for at once: grid (token
// groups x groups of heads, {K, V}).
template <int D, bool kSave, int HEADS>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(Kv4Append a) {
    constexpr int LPR = D / 8, TOKENS = kThreads / LPR;
    const int H = a.n_kv_heads, slices = (H + HEADS - 1) / HEADS;
    const bool values = blockIdx.y != 0;
    const int h0 = blockIdx.x % slices * HEADS;
    const int t = a.first_token + (int)(blockIdx.x / slices) * TOKENS + (int)threadIdx.x / LPR;
    if (t >= a.end_token) return;
    const int part = threadIdx.x % LPR;
    const uint8_t *const from = (values ? a.new_v : a.new_k) + (((int64_t)t * H + h0) * D + 8 * part) * 2;
    uint4 raw[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i)
        raw[i] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(from + min(i, H - 1 - h0) * (2 * D))));
    const int seq = a.q_seq[t], pos = a.q_pos[t];
    const int page = a.block_table[(int64_t)seq * a.max_pages + pos / kPageSize], slot = pos % kPageSize;
    uint8_t *block = (values ? a.v_pool : a.k_pool) + ((int64_t)page * H + h0) * Kv4<D>::kBlock;
    uint8_t *row = nullptr;
    if (kSave) row = (values ? a.second.dst_v : a.second.dst_k)[seq - a.first_seq] + (int64_t)(pos - a.n_keep[seq]) * a.row_bytes;
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
        const int head = h0 + i;
        if (head >= H) return;
        uint32_t codes, byte;
        quantise<D>(raw[i], values ? nullptr : a.k_weight, a.eps, (int)threadIdx.x, codes, byte);
        *reinterpret_cast<uint32_t *>(block + slot * Kv4<D>::kCodes + 4 * part) = codes;
        if (part % 4 == 0) block[Kv4<D>::kScaleAt + slot * Kv4<D>::kScales + part / 4] = (uint8_t)byte;
        block += Kv4<D>::kBlock;
        if (kSave) {
            *reinterpret_cast<uint32_t *>(row + head * Kv4<D>::kCodes + 4 * part) = codes;
            const int scales = H * Kv4<D>::kCodes;
            if (part % 4 == 0) row[scales + head * Kv4<D>::kScales + part / 4] = (uint8_t)byte;
            // the bytes that fill the row up (fewer than 16)
            const int pad = scales + H * Kv4<D>::kScales + part;
            if (head == H - 1) {
                if (pad < a.row_bytes) row[pad] = 0;
                if (pad + LPR < a.row_bytes) row[pad + LPR] = 0;
            }
        }
    }
}

// ---- pool <-> rows -------------------------------------------------------------------------------------------------------
// A unit is kUnitVecs 16-byte vectors of one entry's rows, which lie back to back on the contiguous side; a workgroup takes unit after
// unit, all its loads in flight before the first store.  first[e] = units of the entries before e.  To pinned memory few workgroups go
// (as in link_kernel of ca_move.hip, where the numbers are), else one for every unit.
constexpr int kUnroll = 8, kUnitVecs = kThreads * kUnroll;
struct Units {
    int32_t first[kMaxSeqsPerLaunch + 1];
};

template <int D, bool kToPool>
__global__ __launch_bounds__(kThreads) void kv4_move_kernel(MoveArgs a, Units units, MoveShape s, int row_bytes, uint8_t *__restrict__ k_pool,
                                                            uint8_t *__restrict__ v_pool) {
    constexpr int CV = D / 32;                         // vectors of codes per head and token
    constexpr int HPV = 16 / Kv4<D>::kScales;          // heads whose scale bytes a vector holds
    const int H = s.n_kv_heads, row_vecs = row_bytes / 16, code_vecs = H * CV;
    const bool values = blockIdx.x & 1;
    uint8_t *const pool = values ? v_pool : k_pool;
    const int n_units = units.first[s.n_in_launch];
    int e = 0;
    for (int unit = blockIdx.x >> 1; unit < n_units; unit += gridDim.x >> 1) {
        while (unit >= units.first[e + 1]) ++e;
        const int64_t total = (int64_t)a.count[e] * row_vecs;
        const int64_t v0 = (int64_t)(unit - units.first[e]) * kUnitVecs + threadIdx.x;
        uint8_t *const rows = (values ? a.contig_v[e] : a.contig_k[e]) + a.contig_tok0[e] * row_bytes;
        const int32_t *table = s.block_table + (int64_t)a.seq[e] * s.max_pages;
        u32x4 r[kUnroll];
        uint8_t *block[kUnroll];                       // (page, head 0) of the vector's token
        int rem[kUnroll], slot[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t v = min(v0 + u * kThreads, total - 1);       // past the end: the last one again, not stored
            const int token = (int)(v / row_vecs);
            rem[u] = (int)(v - (int64_t)token * row_vecs);
            const int t = a.ctx_tok0[e] + token;
            slot[u] = t % kPageSize;
            block[u] = pool + (int64_t)table[t / kPageSize] * H * Kv4<D>::kBlock;
            if (kToPool) r[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(rows + v * 16));
        }
        if (!kToPool) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (rem[u] < code_vecs) {
                    r[u] = *reinterpret_cast<const u32x4 *>(block[u] + (rem[u] / CV) * Kv4<D>::kBlock + slot[u] * Kv4<D>::kCodes + rem[u] % CV * 16);
                } else {
                    const int h0 = (rem[u] - code_vecs) * HPV;
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < HPV; ++i) {
                        if (h0 + i >= H) break;
                        const uint8_t *at = block[u] + (h0 + i) * Kv4<D>::kBlock + Kv4<D>::kScaleAt + slot[u] * Kv4<D>::kScales;
                        if (D == 128) w[i % 4] = *reinterpret_cast<const uint32_t *>(at);
                        else w[i / 2] |= (uint32_t) * reinterpret_cast<const uint16_t *>(at) << 16 * (i % 2);
                    }
                    r[u] = u32x4{w[0], w[1], w[2], w[3]};
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);            // all loads before the first store
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t v = v0 + u * kThreads;
            if (v >= total) break;
            if (!kToPool) {
                __builtin_nontemporal_store(r[u], reinterpret_cast<u32x4 *>(rows + v * 16));
            } else if (rem[u] < code_vecs) {
                *reinterpret_cast<u32x4 *>(block[u] + (rem[u] / CV) * Kv4<D>::kBlock + slot[u] * Kv4<D>::kCodes + rem[u] % CV * 16) = r[u];
            } else {
                const int h0 = (rem[u] - code_vecs) * HPV;
#pragma unroll
                for (int i = 0; i < HPV; ++i) {
                    if (h0 + i >= H) break;
                    uint8_t *at = block[u] + (h0 + i) * Kv4<D>::kBlock + Kv4<D>::kScaleAt + slot[u] * Kv4<D>::kScales;
                    if (D == 128) *reinterpret_cast<uint32_t *>(at) = r[u][i % 4];
                    else *reinterpret_cast<uint16_t *>(at) = (uint16_t)(r[u][i / 2] >> 16 * (i % 2));
                }
            }
        }
    }
}

// ---- reading back ----------------------------------------------------------------------------------------------------------
// Context tokens of an entry -> bf16 rows [token][head][D] (exact: a value has two significant bits).  grid (16-token groups x kv heads
// of the longest entry, {K, V}, entry); eight values a lane.
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(MoveArgs a, MoveShape s, int groups, const uint8_t *__restrict__ k_pool,
                                                            const uint8_t *__restrict__ v_pool) {
    constexpr int LPR = D / 8, TOKENS = kThreads / LPR;
    const int H = s.n_kv_heads, e = blockIdx.z;
    const bool values = blockIdx.y != 0;
    const int part = threadIdx.x % LPR;
    const uint8_t *const pool = values ? v_pool : k_pool;
    for (int64_t at = blockIdx.x; at < (int64_t)groups * H; at += gridDim.x) {
        const int head = (int)(at % H), i = (int)(at / H) * TOKENS + (int)threadIdx.x / LPR;
        if (i >= a.count[e]) return;
        const int t = a.ctx_tok0[e] + i;
        const uint8_t *block = pool + ((int64_t)s.block_table[(int64_t)a.seq[e] * s.max_pages + t / kPageSize] * H + head) * Kv4<D>::kBlock;
        const uint32_t codes = *reinterpret_cast<const uint32_t *>(block + t % kPageSize * Kv4<D>::kCodes + 4 * part);
        uint32_t byte = block[Kv4<D>::kScaleAt + t % kPageSize * Kv4<D>::kScales + part / 4];
        if (kv4_is_nan(byte)) byte = 255;
        const float scale = kv4_scale(byte);
        u32x4 o;
        o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
        o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
        o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
        o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
        uint8_t *to = (values ? a.contig_v[e] : a.contig_k[e]) + (((a.contig_tok0[e] + i) * H + head) * D + 8 * part) * 2;
        __builtin_nontemporal_store(o, reinterpret_cast<u32x4 *>(to));
    }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Append &a, int head_dim, bool save, int n_cus, hipStream_t stream) {
    const int n = a.end_token - a.first_token;
    if (n <= 0) return hipSuccess;
    const int tokens = kThreads / (head_dim / 8);
    // a head per thread until every compute unit has 16 workgroups of that: the loads of more need fewer wavefronts, and a token's table
    // entries are looked up once
    const int64_t groups = (n + tokens - 1) / tokens;
    const int heads = 2 * groups * a.n_kv_heads > (int64_t)16 * n_cus ? 4 : 1;
    const dim3 grid((uint32_t)groups * (uint32_t)((a.n_kv_heads + heads - 1) / heads), 2);
    if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
    const auto kernel = head_dim == 128 ? (save ? (heads == 4 ? kv4_append_kernel<128, true, 4> : kv4_append_kernel<128, true, 1>)
                                                : (heads == 4 ? kv4_append_kernel<128, false, 4> : kv4_append_kernel<128, false, 1>))
                                        : (save ? (heads == 4 ? kv4_append_kernel<64, true, 4> : kv4_append_kernel<64, true, 1>)
                                                : (heads == 4 ? kv4_append_kernel<64, false, 4> : kv4_append_kernel<64, false, 1>));
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_kv4_move(bool to_pool, const MoveArgs &args, const MoveShape &shape, int head_dim, int row_bytes, int workgroups, uint8_t *k_pool,
                           uint8_t *v_pool, hipStream_t stream) {
    Units units;
    units.first[0] = 0;
    int64_t n = 0;
    for (int i = 0; i < shape.n_in_launch; ++i) {
        n += ((int64_t)std::max(0, args.count[i]) * (row_bytes / 16) + kUnitVecs - 1) / kUnitVecs;
        if (n > INT32_MAX / 4) return hipErrorInvalidValue;
        units.first[i + 1] = (int32_t)n;
    }
    if (n <= 0) return hipSuccess;
    const dim3 grid(2 * (uint32_t)(workgroups > 0 ? std::min<int64_t>(n, std::max(1, workgroups / 2)) : n));
    if (head_dim != 128 && head_dim != 64) return hipErrorInvalidValue;
    const auto kernel = head_dim == 128 ? (to_pool ? kv4_move_kernel<128, true> : kv4_move_kernel<128, false>)
                                        : (to_pool ? kv4_move_kernel<64, true> : kv4_move_kernel<64, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, args, units, shape, row_bytes, k_pool, v_pool);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const MoveArgs &args, const MoveShape &shape, int head_dim, const uint8_t *k_pool, const uint8_t *v_pool, hipStream_t stream) {
    int most = 0;
    for (int i = 0; i < shape.n_in_launch; ++i) most = std::max(most, args.count[i]);
    if (most <= 0) return hipSuccess;
    const int tokens = kThreads / (head_dim / 8), groups = (most + tokens - 1) / tokens;
    const dim3 grid((uint32_t)std::min<int64_t>((int64_t)groups * shape.n_kv_heads, 1 << 20), 2, shape.n_in_launch);
    if (head_dim == 128) hipLaunchKernelGGL(kv4_read_kernel<128>, grid, dim3(kThreads), 0, stream, args, shape, groups, k_pool, v_pool);
    else if (head_dim == 64) hipLaunchKernelGGL(kv4_read_kernel<64>, grid, dim3(kThreads), 0, stream, args, shape, groups, k_pool, v_pool);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace ca
