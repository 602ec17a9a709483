// Attention of up to eight query rows per KV head over a cache held in 8 or 4 bits: the form for single tokens.
//
// As k_attend_quant, but a product's eight columns are four query rows times the two halves of a 32-bit word of codes: column 2 r + e has
// row r's numbers in the places of halves e and zeros in the others.  A word of a key then goes into both products as it is, whatever
// groups its halves belong to, where the other kernel first brings halves of one group, and of two keys, together; and four rows, the group
// that most models have, take half the exponentials, transposes and registers.
// Bound by arithmetic in 4 bits: taking codes apart is 124 of the 290 instructions for sixteen keys of 128 channels, on the integer pipe at two cycles each, and
// products and fp32 arithmetic partly wait for the same ports.  32 sequences of 8192 keys: issue slots 70 % busy, the integer pipe 59 %, DRAM 59 %, and what warps
// wait for most is a pipe.  4 tokens over 100001 to 131072 keys 104 us from a graph, 5.1 TB/s; one of 8192 keys for 16 and for 32 sequences 36 and
// 62 us.  Bound by HBM in 8 bits: DRAM 77 % busy, 16 tokens over 4096 of 8192 keys 27 us.  fp32 takes twice the matrix products for logits and
// three times those for outputs: 60 us against 36.
#pragma once

#include "attend_quant.cuh"

namespace obf {

// Blocks of a multiprocessor.
template <typename TIN, int NT>
constexpr int AQF_BLOCKS = sizeof(TIN) == 4 ? (NT == 2 ? 3 : 4) : NT == 2 ? 4 : 5;

template <typename TIN, int BITS, int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(AF_NT, (AQF_BLOCKS<TIN, NT>)) k_attend_quant_few(const __grid_constant__ AttendDev p, const __grid_constant__ QuantDev c)
{
    extern __shared__ __align__(128) unsigned char aq_sm[];
    typedef QuantStage<BITS, D> Stage;
    typedef QuantRow<BITS, D> Row;
    constexpr int ROWS = 4 * NT, ST = Stage::STAGES, KEYS = Stage::KEYS, RB = Row::BYTES, SB = Row::SCALE_BYTES, SUB = KEYS / 16;
    constexpr int PAIRS = BITS == 4 ? D / 64 : 1;         // pairs of groups that share a word (8 bits: the one scale)
    constexpr int KM = D / 16, KW = RB / 16, MW = KM / KW;            // products of K, words of a lane, products of a word
    constexpr int W = RB / 32, OT = D / 32, HT = OT / W;  // words of V, tiles of O, tiles of a word
    constexpr int PARTS = sizeof(TIN) == 4 ? 2 : 1;       // of a query
    constexpr int WPARTS = sizeof(TIN) == 4 ? 3 : 1;      // of a weight
    constexpr bool EXACT = sizeof(TIN) == 4;              // codes at their full size
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) attend_status(p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
    const bool upper = g8 & 1;                            // this lane's column is one of upper halves
    const int rows_seq = p.n_q * p.G, tiles = (rows_seq + ROWS - 1) / ROWS, parts = p.slots;
    unsigned x = blockIdx.x;
    const int part = x % parts;
    x /= parts;
    const int tile = x % tiles;
    x /= tiles;
    const int h = x % p.kv_heads, b = x / p.kv_heads;
    const int len = attend_len(p, b), ql = attend_q_len(p, b);
    const int i0 = tile * ROWS / p.G, i1 = min((min((tile + 1) * ROWS, rows_seq) - 1) / p.G, ql - 1);
    QuantWalk<BITS, D> walk(p, c, aq_sm, b, h, len, ql, i0, i1, part, parts);
    const uint32_t ring = walk.ring;

    // Queries as B fragments: row 4 nt + lane / 8, a quarter of the channels, of those the ones that stand in this column's halves.
    uint32_t qf[PARTS][NT][KM][2];
    float q_off[NT][PAIRS][2], row_c[NT];                 // of row 4 nt + lane mod 4: what offsets add up to, what makes logits (log2)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = tile * ROWS + nt * 4 + (g8 >> 1), i = r / p.G, g = r - i * p.G;
        const bool real = r < rows_seq && i < ql;
        const TIN *src = static_cast<const TIN *>(p.q) + b * p.qs[0] + (long long)(h * p.G + g) * p.qs[1] + (long long)i * p.qs[2];
        float q[D / 4];
        uint32_t top = 0;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {                // eight channels at a time
            const int ch = BITS == 8 && D == 128 ? 16 * t4 + 8 * (w & 1) + 64 * (w >> 1) : t4 * (D / 4) + 8 * w;
            float y[8];
            if (real) {
                Eight<TIN> e;
                e.load(src + ch);
                e.get(y);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                q[8 * w + k] = real ? y[k] : 0.f;
                top = max(top, __float_as_uint(q[8 * w + k]) & 0x7fffffffu);
            }
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max((int)(top >> 23), 27), 254);             // exponent of the largest, at least that of 2^-100
        const float up = __uint_as_float((uint32_t)(267 - e) << 23), down = __uint_as_float((uint32_t)(e - 13) << 23);
        float sum[PAIRS];
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) sum[j] = 0.f;
#pragma unroll
        for (int k = 0; k < KM; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                // (4 bits: the second register meets codes sixteen times as large)
                const int a = BITS == 4 ? 8 * (k >> 1) + 2 * (k & 1) + u : 4 * k + 2 * u, a2 = BITS == 4 ? a + 4 : a + 1;
                float y = (upper ? q[a2] : q[a]) * (BITS == 4 && u == 1 ? up * 0.0625f : up);
#pragma unroll
                for (int part_q = 0; part_q < PARTS; ++part_q) {
                    const __half v = __float2half_rn(y);
                    const uint32_t bits = __half_as_ushort(v);
                    qf[part_q][nt][k][u] = upper ? bits << 16 : bits;
                    y -= __half2float(v);
                    sum[BITS == 4 && PAIRS == 2 ? k >> 1 & 1 : 0] += __half2float(v) * (BITS == 4 && u == 1 ? 16.f : 1.f);
                }
            }
#pragma unroll
        for (int j = 0; j < PAIRS; ++j) {
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
            sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
#pragma unroll
            for (int u = 0; u < 2; ++u) q_off[nt][j][u] = __shfl_sync(0xffffffffu, sum[j], 4 * (2 * t4 + u)) * (BITS == 4 ? -0x1p-21f : -0x1p-17f);
        }
        row_c[nt] = p.c * (EXACT ? 1.f : 0x1p24f) * __shfl_sync(0xffffffffu, down, 8 * t4);
    }

    float o[NT][OT][4], m[NT], l[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt] = AQ_NONE;
        l[nt] = 0.f;
#pragma unroll
        for (int k = 0; k < OT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[nt][k][e] = 0.f;
    }
    // the halves of a transposed pair of weights (of keys lane mod 4 and + 4) to this column's half of a word, the other one zero
    const uint32_t sel_x = upper ? 0x1044 : 0x4410, sel_y = upper ? 0x3244 : 0x4432;
    const int key_s = (g8 >> 1) + 4 * (g8 & 1);           // keys as in k_attend_quant
    const uint32_t k_at = ring + (RB == 32 ? chunk_at<RB>(key_s, t4 >> 1) + (t4 & 1) * 8 : chunk_at<RB>(key_s, t4));
    uint32_t v_at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v_at[i] = ring + Stage::CODES + (W == 4 ? chunk_at<RB>(t4 + 4 * i, g8) : W == 2 ? chunk_at<RB>(t4 + 4 * i, g8 >> 1) + (g8 & 1) * 8 : chunk_at<RB>(t4 + 4 * i, g8 >> 2) + (g8 & 3) * 4);
    const uint32_t s_at = ring + 2 * Stage::CODES + key_s * SB;
    int slot = 0;
    for (int va = walk.first(); va < walk.v1; va += AF_WARPS * KEYS) {
        walk.next(va, slot);
        const uint32_t off = slot * Stage::BYTES, kd = k_at + off, vd0 = v_at[0] + off, vd1 = v_at[1] + off, sd = s_at + off;
        // ---- logits: s[sub][nt][u] of key 8 u + key_s of sixteen, row 4 nt + lane mod 4 ----
        float s[SUB][NT][2];
        {
            float acc[SUB][NT][PAIRS][4];
            constexpr int KV = KW < 4 ? KW : 4;           // words read at once
#pragma unroll
            for (int part_k = 0; part_k < KW / KV; ++part_k) {
                uint32_t w0[SUB][KV], w1[SUB][KV];
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub) {
                    lds(w0[sub], (part_k ? kd ^ 64u : kd) + sub * 16 * RB);     // (rows of 128 bytes: chunks t and t + 4)
                    lds(w1[sub], (part_k ? kd ^ 64u : kd) + (sub * 16 + 8) * RB);
                }
#pragma unroll
                for (int i = 0; i < KV; ++i)
#pragma unroll
                    for (int hh = 0; hh < MW; ++hh)
#pragma unroll
                        for (int sub = 0; sub < SUB; ++sub) {
                            const int k = (part_k * KV + i) * MW + hh, j = BITS == 4 && PAIRS == 2 ? i & 1 : 0;
                            const uint32_t y = w0[sub][i], z = w1[sub][i];
                            uint32_t a[4];
                            if constexpr (BITS == 4) {
                                a[0] = (hh ? y >> 8 : y) & 0x000f000fu;
                                a[1] = (hh ? z >> 8 : z) & 0x000f000fu;
                                a[2] = (hh ? y >> 8 : y) & 0x00f000f0u;
                                a[3] = (hh ? z >> 8 : z) & 0x00f000f0u;
                                if constexpr (EXACT) {
#pragma unroll
                                    for (int e = 0; e < 4; ++e) a[e] = add_f16(a[e] | 0x64006400u, e < 2 ? AQ_F16_8 : AQ_F16_128);
                                }
                            } else if constexpr (EXACT) {
                                a[0] = bytes_f16(y, 0x4140);
                                a[1] = bytes_f16(z, 0x4140);
                                a[2] = bytes_f16(y, 0x4342);
                                a[3] = bytes_f16(z, 0x4342);
                            } else {
                                a[0] = __byte_perm(y ^ 0x80808080u, 0u, 0x4140);
                                a[1] = __byte_perm(z ^ 0x80808080u, 0u, 0x4140);
                                a[2] = __byte_perm(y ^ 0x80808080u, 0u, 0x4342);
                                a[3] = __byte_perm(z ^ 0x80808080u, 0u, 0x4342);
                            }
#pragma unroll
                            for (int part_q = PARTS - 1; part_q >= 0; --part_q)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    if (part_q == PARTS - 1 && hh == 0 && part_k == 0 && i == j) mma_f16_first(acc[sub][nt][j], a, qf[part_q][nt][k][0], qf[part_q][nt][k][1]);
                                    else mma_f16(acc[sub][nt][j], a, qf[part_q][nt][k][0], qf[part_q][nt][k][1]);
                                }
                        }
            }
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t f[PAIRS];
                    lds(f, sd + (sub * 16 + 8 * u) * SB);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int j = 0; j < PAIRS; ++j) {
                            const float y = EXACT ? acc[sub][nt][j][2 * u] : acc[sub][nt][j][2 * u] + q_off[nt][j][0];
                            const float z = EXACT ? acc[sub][nt][j][2 * u + 1] : acc[sub][nt][j][2 * u + 1] + q_off[nt][j][1];
                            if constexpr (BITS == 4) {
                                s[sub][nt][u] = j == 0 ? y * bf16_lo(f[0]) : fmaf(y, bf16_lo(f[j]), s[sub][nt][u]);
                                s[sub][nt][u] = fmaf(z, bf16_hi(f[j]), s[sub][nt][u]);
                            } else {
                                s[sub][nt][u] = (y + z) * __uint_as_float(f[0]);
                            }
                        }
                        s[sub][nt][u] *= row_c[nt];
                    }
                }
        }
        // ---- weights ----
        if (!walk.whole(va)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int t = len - ql + (tile * ROWS + nt * 4 + t4) / p.G;     // (of rows that are none: anything)
#pragma unroll
                for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int v = va + 16 * sub + key_s + 8 * u;
                        if (v >= walk.v1 || !attend_sees(p, t, walk.kr.key(v))) s[sub][nt][u] = -INFINITY;
                    }
            }
        }
        float top[NT], over = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            top[nt] = fmaxf(s[0][nt][0], s[0][nt][1]);
#pragma unroll
            for (int sub = 1; sub < SUB; ++sub) top[nt] = fmaxf(top[nt], fmaxf(s[sub][nt][0], s[sub][nt][1]));
            over = fmaxf(over, top[nt] - m[nt]);
        }
        if (__any_sync(0xffffffffu, over > AF_RAISE)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float mx = top[nt];
#pragma unroll
                for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
                mx = fmaxf(mx, m[nt]);
                const float f = ex2(m[nt] - mx);
                m[nt] = mx;
                l[nt] *= f;
#pragma unroll
                for (int k = 0; k < OT; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[nt][k][e] *= f;
            }
        }
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    s[sub][nt][u] = aq_weight<TIN>(s[sub][nt][u], m[nt]);
                    l[nt] += s[sub][nt][u];
                }
        // ---- values: columns 2 r + e of O are row r's channels in halves e of the words ----
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t w[2][W], f[PAIRS];               // of keys 8 u + lane mod 4, + 4
                lds(w[0], vd0 + (sub * 16 + 8 * u) * RB);
                lds(w[1], vd1 + (sub * 16 + 8 * u) * RB);
                lds(f, sd + Stage::SCALES + (sub * 16 + 8 * u) * SB);
                uint32_t pf[NT][PAIRS][WPARTS][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < PAIRS; ++j) {
                        const float y = s[sub][nt][u];
                        uint32_t pw[WPARTS];
                        if constexpr (BITS == 4) split_weights<WPARTS>(pw, y * bf16_lo(f[j]), y * bf16_hi(f[j]));
                        else split_weights<WPARTS>(pw, y * __uint_as_float(f[0]), y * __uint_as_float(f[0]));
#pragma unroll
                        for (int q = 0; q < WPARTS; ++q) {
                            const uint32_t both = transpose8x8(pw[q]);
                            pf[nt][j][q][0] = __byte_perm(both, 0u, sel_x);
                            pf[nt][j][q][1] = __byte_perm(both, 0u, sel_y);
                        }
                    }
#pragma unroll
                for (int q = 0; q < W; ++q) {
                    uint32_t a[HT][4];                    // per tile: two kinds of codes of either key
#pragma unroll
                    for (int key = 0; key < 2; ++key) {
                        const uint32_t y = w[key][q];
                        if constexpr (BITS == 4 && EXACT) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) a[i / 2][2 * key + i % 2] = nibble_bf16(y, i);
                        } else if constexpr (EXACT) {
                            a[0][2 * key] = byte_pair_bf16(y ^ 0x80808080u, (y ^ 0x80808080u) >> 8, 0);
                            a[0][2 * key + 1] = byte_pair_bf16(y ^ 0x80808080u, (y ^ 0x80808080u) >> 8, 2);
                        } else if constexpr (BITS == 4) {
                            // codes 0 and 2 of the halves alone, with 1 and 3 sixteenfold on top
                            const uint32_t z = __byte_perm(y, 0u, 0x4341);
                            a[0][2 * key] = add_bf16(y & 0x000f000fu, AQ_MINUS_8);
                            a[0][2 * key + 1] = add_bf16(y & 0x00ff00ffu, AQ_MINUS_136);
                            a[HT - 1][2 * key] = add_bf16(z & 0x000f000fu, AQ_MINUS_8);
                            a[HT - 1][2 * key + 1] = add_bf16(z, AQ_MINUS_136);
                        } else {
                            a[0][2 * key] = add_bf16(__byte_perm(y ^ 0x80808080u, 0u, 0x4140), AQ_MINUS_128);
                            a[0][2 * key + 1] = add_bf16(__byte_perm(y ^ 0x80808080u, 0u, 0x4342), AQ_MINUS_128);
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < HT; ++i) mma_weights<EXACT, WPARTS>(o[nt][q * HT + i], a[i], pf[nt][BITS == 4 ? q : 0]);
                }
            }
        slot = slot + 1 == ST ? 0 : slot + 1;
    }
    cp_wait<0>();
    __syncthreads();

    // the warps' results: O as [warp][row][D + 4], then references and sums
    constexpr int LD = D + 4;
    float *osm = reinterpret_cast<float *>(aq_sm), *ml = osm + AF_WARPS * ROWS * LD;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float z = l[nt];
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) z += __shfl_xor_sync(0xffffffffu, z, w);
        const int row = 4 * nt + t4;
        if (lane < 4) { ml[(warp * ROWS + row) * 2] = m[nt]; ml[(warp * ROWS + row) * 2 + 1] = z * AQ_SUM<TIN>; }
        float *dst = &osm[(warp * ROWS + row) * LD + g8 * (D / 8)];
        constexpr float U = AQ_VALUE<TIN>, U2 = BITS == 4 && !EXACT ? U * 0.0625f : U;
        if constexpr (BITS == 4) {
#pragma unroll
            for (int q = 0; q < W; ++q)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float (&lo)[4] = o[nt][2 * q], (&hi)[4] = o[nt][2 * q + 1];
                    *reinterpret_cast<float4 *>(dst + 8 * q + 4 * e) = make_float4(lo[e] * U, (EXACT ? lo[2 + e] : lo[2 + e] - lo[e]) * U2, hi[e] * U, (EXACT ? hi[2 + e] : hi[2 + e] - hi[e]) * U2);
                }
        } else {
#pragma unroll
            for (int q = 0; q < W; ++q)
                *reinterpret_cast<float4 *>(dst + 4 * q) = make_float4(o[nt][q][0] * U, o[nt][q][1] * U, o[nt][q][2] * U, o[nt][q][3] * U);
        }
    }
    __syncthreads();
    few_finish<TIN, D, ROWS, false, CLUSTER>(p, osm, ml, tile, part, parts, rows_seq, rows_seq, h, b, len, ql, walk.kr, walk.v0, walk.v1, AQ_LSE<TIN>);
}

}  // namespace obf
