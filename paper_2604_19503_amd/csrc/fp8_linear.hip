// Products of E4M3 operands with a scale per 128 elements along K (activation rows) and per 128 x 128 block (weights), and the
// gated feed-forward block on them:
//   y[m,n] = sum_b xs[b,m] ws[n/128,b] sum_{k in block b} xq[m,k] wq[n,k]  (+ bias[n]) (+ add[m,n])
//
// One v_mfma_f32_16x16x128_f8f6f4 is a whole block of K: it starts from zero, and its result goes into the FP32 accumulator with
// one multiply-add per element, the factor being the product of the two scales.  The weights are its A operand, so a lane ends up
// with one activation row and four weight rows, i.e. output columns; the rows of a group of 32 weights sit in LDS in such an order
// that the two MFMA tiles of the group leave a lane 8 consecutive columns.
//
// The 8-bit instruction aligns the products of 8 consecutive codes of a row to the largest of them and cuts off what lies 13 bits below
// it (found with single products, whatever the tile); the sums of 8 add up in FP32.  On blocks of normal values its sums are 1.5e-5
// of their rms off, with one channel in 64 twenty times as large 5e-5.  Against the rounding of a BF16 output (1.7e-3) that is
// nothing; h of the feed-forward block gets codes on the other side of a rounding boundary about once in 1000, and its output is 0.0018 to 0.0026
// off the formula (small calls up to 0.0039) where FP32 sums leave 0.0017.  Callers who want FP32 sums ask for them, by FP32 outputs or
// by REALB_SUMS_F32: there the codes are widened to BF16, which holds every E4M3 number, and multiplied by v_mfma_f32_16x16x32_bf16 (1e-8), at half
// the rate and in the smaller tiles.  The feed-forward block, 8-bit instruction / FP32 sums: 65 rows, H 2048, I 1408 21.6 / 33.0 us; 3001 rows, I 768 30.9 / 54.5;
// 65 536 rows, I 1408 529 / 1177.  Up to 64 rows that costs nothing, the weights' bytes being what takes the time, so all calls of so few rows do it.
#include "fp8_device.h"
#include "ffn_device.h"
#include <climits>

namespace realb {

__device__ __align__(16) uint8_t g_zeros[16];              // what stands behind the last element of a row whose length is no multiple of 128

struct Fp8Gemm {
    const uint8_t* x;          // codes [M, K], pitch ld_x
    const float* xs;           // [KB, ld_xs]
    const uint8_t* w;          // codes [w_rows, K]
    const float* ws;           // [ceil(w_rows/128), KB]
    uint8_t* out;              // bf16 / f32 [M, N]; gate/up: codes of h [M, I]
    float* out_s;              // gate/up: scales of h [I/128, ld_s]
    const uint8_t* bias;       // bf16 [N] or NULL
    const uint8_t* add;        // [M, N] of out's type or NULL
    long long ld_x, ld_xs, ld_out, ld_add, ld_s;
    int M, N, K, KB;           // N: output columns (gate/up: I)
    int tiles;                 // large tiles: all of them; in panels of 8 columns, panel_tiles each, and rest_cols columns behind full_panels of them
    int panel_tiles, full_panels, rest_cols;               // (small tiles: panel_tiles = tiles of a row or, if rows_first, of a column of them)
    int rows_first;
    uint32_t panel_magic, rest_magic;      // t / panel_tiles == (t * panel_magic) >> panel_shift, and for rest_cols
    int panel_shift, rest_shift;
};

template <bool GATEUP>
__device__ __forceinline__ int fp8_w_row(int pos, int n0, int N) {
    const int in_group = w_row_of_slot16(pos & 31);
    if constexpr (GATEUP) return ((pos >> 5) & 1 ? N : 0) + n0 + (pos >> 6) * 32 + in_group;      // groups alternate: gate rows, up rows
    else return min(n0 + (pos & ~31) + in_group, N - 1);
}

// Eight codes -> eight BF16, exactly.
__device__ __forceinline__ v8bf_t fp8_widen(uint32_t a, uint32_t b) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf2;
    const bf2 v0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.0f, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, 1.0f, true);
    const bf2 v2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.0f, false), v3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, 1.0f, true);
    return v8bf_t{v0.x, v0.y, v1.x, v1.y, v2.x, v2.y, v3.x, v3.y};
}

// acc += f * (16 weight rows x 16 activation rows over a block of 128): lane l feeds bytes 16*(l/16) .. and 64 + 16*(l/16) .. of row l%16 of
// either operand (the order along K is the same in both, so it does not matter which), and gets weight rows 4*(l/16) + r of
// activation row l%16.
template <bool WIDE>
__device__ __forceinline__ void fp8_mma(v4f_t& acc, const u32x4 (&w)[2], const u32x4 (&x)[2], float f) {
    v4f_t d = {0.f, 0.f, 0.f, 0.f};
    if constexpr (WIDE) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_widen(w[h].x, w[h].y), fp8_widen(x[h].x, x[h].y), d, 0, 0, 0);
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp8_widen(w[h].z, w[h].w), fp8_widen(x[h].z, x[h].w), d, 0, 0, 0);
        }
    } else {
        const v8i_t a = {(int)w[0].x, (int)w[0].y, (int)w[0].z, (int)w[0].w, (int)w[1].x, (int)w[1].y, (int)w[1].z, (int)w[1].w};
        const v8i_t b = {(int)x[0].x, (int)x[0].y, (int)x[0].z, (int)x[0].w, (int)x[1].x, (int)x[1].y, (int)x[1].z, (int)x[1].w};
        d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, d, 0, 0, 0, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(d[r], f, acc[r]);
}

// Epilogue of a wave: RT row tiles of 16, whose first row is `first` within the block's tile at (m0, n0), and 64 weight rows, the wn-th
// such group of the tile.  acc[i][t][r]: row 16 i + l%16, weight row 8*(l/16) + 4*(t&1) + r of the group of 32 number t/2.
// Gate/up: the first 32 weight rows are gate rows, the others the up rows of the same 32 columns of h; four waves side by side hold the
// 128 columns of one E4M3 block, whose maximum they find through `amax` (4 x tile_rows floats of LDS) and one barrier.
template <bool GATEUP, int RT, bool NT, bool F32OUT = false, int CT = 4, typename Barrier>
__device__ __forceinline__ void fp8_store_tile(const Fp8Gemm& p, v4f_t (&acc)[RT][CT], uint8_t* amax_lds, int tile_rows, int m0, int n0, int first, int wn, int lane,
                                               Barrier barrier) {
    asm volatile("" : "+v"(lane));                          // (what follows from it is worked out here, not kept in registers through the K-loop)
    const int l16 = lane & 15, g = lane >> 4;
    if constexpr (GATEUP) {
        static_assert(CT == 4, "32 gate and 32 up rows");
        float* amax = reinterpret_cast<float*>(amax_lds);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float m = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {                   // h takes the gate's place
                const float gate = acc[i][e >> 2][e & 3], up = acc[i][2 + (e >> 2)][e & 3];
                // (reciprocal and exponential to a few ulp, some 1e-7 of h, where half a code's step is 1/16 of it; a division is ten instructions)
                const float h = gate * __builtin_amdgcn_rcpf(1.0f + __expf(-gate)) * up;
                acc[i][e >> 2][e & 3] = h;
                m = fmaxf(m, fabsf(h));
            }
            m = groups_max(m);
            if (g == 0) amax[wn * tile_rows + first + i * 16 + l16] = m;
            __builtin_amdgcn_sched_barrier(0);              // (row tiles one after the other: side by side they take too many registers)
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = first + i * 16 + l16;
            const Fp8Scale sc = fp8_scale(fmaxf(fmaxf(amax[r], amax[tile_rows + r]), fmaxf(amax[2 * tile_rows + r], amax[3 * tile_rows + r])));
            float h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] = acc[i][e >> 2][e & 3];
            const u32x2 codes = fp8_encode8(h, sc.inv);
            if (m0 + r < p.M) {
                *reinterpret_cast<u32x2*>(p.out + (long long)(m0 + r) * p.ld_out + n0 + wn * 32 + g * 8) = codes;
                if (wn == 0 && g == 0) p.out_s[(n0 >> 7) * p.ld_s + m0 + r] = sc.scale;
            }
        }
    } else if (!F32OUT && RT % 2 == 0 && CT == 4 && n0 + wn * 64 + 64 <= p.N && m0 + first + 16 * RT <= p.M) {
        // All there (at any alignment: the memory takes wide stores anywhere): two row tiles at a time, exchanged between lanes so that an instruction writes 64 bytes or more of every row
        const int col = n0 + wn * 64 + g * 8;
        auto store_all = [&](auto plain) __attribute__((always_inline)) {
            float b[2][8];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) b[c][e] = !plain && p.bias ? bf16_lo(reinterpret_cast<const uint16_t*>(p.bias)[col + c * 32 + e]) : 0.f;
#pragma unroll
            for (int i = 0; i < RT; i += 2) {
                u32x4_t q[2][2];                            // [column group][half of the exchanged rows]
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t d[2][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = plain ? acc[i + j][2 * c + (e >> 2)][e & 3] : acc[i + j][2 * c + (e >> 2)][e & 3] + b[c][e];
                        if (!plain && p.add) {
                            float a[8];
                            load8_any(p.add, (long long)(m0 + first + (i + j) * 16 + l16) * p.ld_add + col + c * 32, false, a);
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] += a[e];
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) d[j][k] = pack2(v[2 * k], v[2 * k + 1]);
                    }
                    uint32_t r0[4], r1[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const auto s = __builtin_amdgcn_permlane16_swap(d[0][k], d[1][k], false, false);
                        r0[k] = s[0];
                        r1[k] = s[1];
                    }
                    q[c][0] = u32x4_t{r0[0], r0[1], r0[2], r0[3]};
                    q[c][1] = u32x4_t{r1[0], r1[1], r1[2], r1[3]};
                }
                store_tile_pair<NT>(p.out + ((long long)(m0 + first + i * 16) * p.ld_out + n0 + wn * 64) * 2, (size_t)p.ld_out * 2, lane, 32, q[0][0], q[0][1], q[1][0], q[1][1]);
            }
        };
        if (p.bias || p.add) store_all(std::false_type{});
        else store_all(std::true_type{});
    } else {
#pragma unroll
        for (int c = 0; c < CT / 2; ++c) {
            const int col = n0 + wn * 16 * CT + c * 32 + g * 8;
            if (col >= p.N) continue;
            const bool whole = col + 8 <= p.N;
            float b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (p.bias) {
#pragma unroll
                for (int e = 0; e < 8; ++e) b[e] = bf16_lo(reinterpret_cast<const uint16_t*>(p.bias)[min(col + e, p.N - 1)]);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const long long m = m0 + first + i * 16 + l16;
                if (m >= p.M) continue;
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = acc[i][2 * c + (e >> 2)][e & 3] + b[e];
                if (whole) {
                    if (p.add) {
                        float a[8];
                        load8_any(p.add, m * p.ld_add + col, F32OUT, a);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += a[e];
                    }
                    store8_any(p.out, m * p.ld_out + col, F32OUT, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (col + e >= p.N) break;
                        if constexpr (F32OUT) {
                            if (p.add) v[e] += reinterpret_cast<const float*>(p.add)[m * p.ld_add + col + e];
                            reinterpret_cast<float*>(p.out)[m * p.ld_out + col + e] = v[e];
                        } else {
                            if (p.add) v[e] += bf16_lo(reinterpret_cast<const uint16_t*>(p.add)[m * p.ld_add + col + e]);
                            reinterpret_cast<__bf16*>(p.out)[m * p.ld_out + col + e] = (__bf16)v[e];
                        }
                    }
                }
            }
        }
    }
}

// Small tiles, for products that have too few large ones to fill the chip: 16*RT*WM activation rows x 16*CT*WN weight rows, WM x WN waves of
// 16*RT x 16*CT.  A K-step is 128 bytes of every row, brought to LDS without passing through registers (8 rows per instruction; the 16-byte
// parts of row R sit XOR-swizzled by (R >> 1) & 7, which keeps the fragment reads free of bank conflicts); NS stages filled NS - 1 steps
// ahead, one barrier per step.  K is summed in order, as in the large tiles, so the bits of a row do not depend on which tiles it is in.
// Bound by the transfers' latency, once a step: the wait at the step's barrier counts, but the loop may load weight scales (every 64th
// step), so the compiler waits for all vector memory in front of the lane reads of them in each step, and with it for the transfers that
// the step before sent.  That makes 0.35 to 0.4 us a step whatever NS is (two K blocks per step, six and eight stages changed nothing; they were
// measured with this wait and say nothing about a pipeline without it), and few tiles get more waves of fewer columns: 65 rows, N = K = 2048, 64 x 64
// tiles, 4 waves of 16 x 64 8.7 us, 8 waves of 16 x 32 7.4 us; 2000 rows x 1408 x 4096, 128 x 128 tiles, 8 waves 29.6, 16 waves 25 us;
// gate/up tiles of 128 x 256, 8 waves of 64 x 64 or 16 of 32 x 64: the feed-forward block of 3001 rows, H 2048, I 768 33.0 / 32.3 us.
template <int RT, int WM, int WN, int NS, int CT>
struct SmallGeo {
    static constexpr int TA = 16 * RT * WM, TW = 16 * CT * WN, WAVES = WM * WN;
    static constexpr int SC = (TA + TW) * 128;             // activation scales of a stage
    static constexpr int SCG = TA / 64;             // transfers of them
    static constexpr int STAGE = SC + SCG * 256;
    static constexpr int LDS = NS * STAGE;
    static constexpr int OPS = (TA + TW) / 8 / WAVES;      // 8-row transfers per wave and step; one more for the scales
    static_assert(TA % 64 == 0 && (TA + TW) % (8 * WAVES) == 0, "tile shapes");
};

// WIDE: FP32 sums, on the BF16 instruction.
template <bool GATEUP, bool WIDE, bool F32OUT, int RT, int WM, int WN, int NS, int CT>
__global__ void __launch_bounds__(64 * WM * WN) fp8_tile_kernel(const Fp8Gemm p) {
    using G = SmallGeo<RT, WM, WN, NS, CT>;
    constexpr int TA = G::TA, OPS = G::OPS, COLS = GATEUP ? G::TW / 2 : G::TW;
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;

    // blocks b, b + 8, .. share an XCD: each XCD takes a contiguous range of tiles
    const int per_xcd = (p.tiles + 7) >> 3;
    const int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || tile >= p.tiles) return;
    const int major = div_by_magic(tile, p.panel_magic, p.panel_shift), minor = tile - major * p.panel_tiles;
    const int m0 = (p.rows_first ? minor : major) * TA, n0 = (p.rows_first ? major : minor) * COLS;

    // source of this lane's part of the 8-row groups its wave moves (group j: LDS rows 8j .. 8j+7, activations first)
    const uint8_t* src[OPS];
    int part[OPS];
#pragma unroll
    for (int j = 0; j < OPS; ++j) {
        const int R = (wave * OPS + j) * 8 + (lane >> 3);
        part[j] = (((lane & 7) ^ ((R >> 1) & 7)) << 4);
        if (R < TA) src[j] = p.x + min(m0 + R, p.M - 1) * p.ld_x;
        else src[j] = p.w + (long long)fp8_w_row<GATEUP>(R - TA, n0, p.N) * p.K;
    }
    const int sc_group = wave % G::SCG;
    const float* sc_src = p.xs + min(m0 + sc_group * 64 + lane, p.M - 1);
    auto issue = [&](int from, int to, int kb, uint8_t* l) __attribute__((always_inline)) {      // transfers from .. to-1 of a K block; OPS: the scales
#pragma unroll
        for (int j = from; j < to; ++j) {
            if (j == OPS) {
                lds_dma4(reinterpret_cast<const uint32_t*>(sc_src + kb * p.ld_xs), l + G::SC + sc_group * 256);
            } else {
                const int k = kb * 128 + part[j];
                lds_dma16(k < p.K ? src[j] + k : g_zeros, l + (wave * OPS + j) * 1024);
            }
        }
    };

    v4f_t acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = v4f_t{0.f, 0.f, 0.f, 0.f};
    const int f_off = l16 * 128 + ((g ^ (l16 >> 1)) << 4);
    const int nb = GATEUP ? n0 >> 7 : min((n0 + wn * 16 * CT) >> 7, (p.N - 1) >> 7);
    const float* ws0 = p.ws + (long long)nb * p.KB;
    const float* ws1 = GATEUP ? ws0 + (long long)(p.N >> 7) * p.KB : ws0;
    // the weights' scales: lane l holds those of K block l, 64 + l, ..  (scalar loads in each step, waited for together with the fragments,
    // were slower: 65 rows 10.4 -> 8.4 us)
    float wsv[2] = {0.f, 0.f};
    auto load_scales = [&](int kb) __attribute__((always_inline)) {
        wsv[0] = ws0[min(kb + lane, p.KB - 1)];
        if constexpr (GATEUP) wsv[1] = ws1[min(kb + lane, p.KB - 1)];
    };
    auto readlane = [](float v, int l) __attribute__((always_inline)) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
    load_scales(0);
#pragma unroll
    for (int s = 0; s < NS - 1; ++s)
        if (s < p.KB) issue(0, OPS + 1, s, smem + s * G::STAGE);
    int stage = 0, fill = NS - 1;
    for (int kb = 0; kb < p.KB; ++kb) {
        // step kb has landed everywhere (NS - 2 steps behind it may be under way), and every wave has read the step before it
        if (kb + NS - 2 < p.KB) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NS - 2) * (OPS + 1)) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const uint8_t* st = smem + stage * G::STAGE;
        u32x4 fw[CT][2], fx[RT][2];
        float xs[RT];
#pragma unroll
        for (int t = 0; t < CT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) fw[t][h] = *reinterpret_cast<const u32x4*>(st + (TA + wn * 16 * CT + t * 16) * 128 + (f_off ^ (h << 6)));
#pragma unroll
        for (int i = 0; i < RT; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) fx[i][h] = *reinterpret_cast<const u32x4*>(st + ((wm * RT + i) * 16) * 128 + (f_off ^ (h << 6)));
            xs[i] = *reinterpret_cast<const float*>(st + G::SC + ((wm * RT + i) * 16 + l16) * 4);
        }
        if ((kb & 63) == 0 && kb > 0) load_scales(kb);
        const float s0 = readlane(wsv[0], kb & 63), s1 = GATEUP ? readlane(wsv[1], kb & 63) : s0;
        constexpr int EACH = (OPS + 1 + RT - 1) / RT;
#pragma unroll
        for (int i = 0; i < RT; ++i) {                     // the transfers go out between the MFMAs: a wave blocks while one is accepted
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < CT; ++t) fp8_mma<WIDE>(acc[i][t], fw[t], fx[i], xs[i] * (t < 2 ? s0 : s1));
            __builtin_amdgcn_sched_barrier(0);
            if (kb + NS - 1 < p.KB) issue(i * EACH, min((i + 1) * EACH, OPS + 1), kb + NS - 1, smem + fill * G::STAGE);
        }
        fill = stage;
        stage = stage + 1 == NS ? 0 : stage + 1;
    }
    __syncthreads();
    fp8_store_tile<GATEUP, RT, false, F32OUT, CT>(p, acc, smem, TA, m0, n0, wm * RT * 16, wn, lane, [] { __syncthreads(); });
}

// Large tiles: 256 activation rows x 256 weight rows, 8 waves of 128 x 64 (2 x 4), persistent blocks whose transfers run on across
// tiles.  A K-step is 64 KB brought in for 32 MFMAs of 32 cycles per wave.  The two waves of a SIMD take turns at the matrix cores, as in
// the BF16 tiles of the layer: waves 0..3 (upper 128 rows, one per SIMD) multiply while waves 4..7 read fragments and issue transfers,
// then the other way round, a barrier at each change, waves 4..7 one change behind.  A step is two turns of 16 MFMAs (4 row tiles x 4
// column tiles), whose multiply-adds onto the accumulators run beside the MFMAs behind them:
//   section 0: fragments of the weights and of rows 0..63; transfers of the next step's rows
//   section 1: of rows 64..127; transfers of the weights of the step after; the next step has landed
// Bound by power and by the change of turns: the matrix cores are busy in 52 % of the cycles, at 2.0 GHz; 8192^3 takes 428 to 450 us (2440 to 2570
// TFLOP/s; 366 without transfers, 360 with operands of zeros), 32768 x 4096 x 2048 236 to 260 (2110 to 2330; 270 when launched without a pause
// for milliseconds), where the epilogue's 3.6 us a tile count.  Four turns a step instead of two took 304 us there (two: 255 at that time).
struct BigGeo {
    static constexpr int TA = 256, TW = 256;
    static constexpr int STAGE = (TA + TW) * 128;
    static constexpr int XS = 2 * STAGE;                   // activation scales [2][256]
    static constexpr int WS = XS + 2 * TA * 4;             // weight scales [4 tiles][2 column blocks][64 K blocks]
    static constexpr int AMAX = WS + 4 * 2 * 64 * 4;       // gate/up: row maxima [4 waves][256]
    static constexpr int LDS = AMAX + 4 * TA * 4;
};
constexpr long long kBigMaxPitch = 1 << 23;               // 256 rows of this pitch are within 32-bit offsets
// K blocks whose weight scales one transfer of a wave holds.  Above, K > 8192, small tiles: 8192 x 8192 x 8192 465 us, 8192 x 8192 x 8208 823.
constexpr int kBigMaxBlocks = 64;

template <bool GATEUP, bool RAGGED, bool NT>
__global__ void __launch_bounds__(512, 1) fp8_big_kernel(const Fp8Gemm p) {
    using G = BigGeo;
    constexpr int COLS = GATEUP ? 128 : 256;
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
    const int nks = p.KB;

    const int per_xcd = (p.tiles + 7) >> 3, nslots = (int)(gridDim.x >> 3);
    const int tile_hi = min(p.tiles, ((int)(blockIdx.x & 7) + 1) * per_xcd);
    int tile = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (tile >= tile_hi) return;
    // Order: panels of 8 column tiles, row tiles within a panel, so that the 32 blocks of an XCD that work side by side share 4 row tiles
    // and 8 column tiles.
    auto decode = [&](int t, int& m0, int& n0) __attribute__((always_inline)) {
        const int panel = div_by_magic(t, p.panel_magic, p.panel_shift);
        int mi, nt;
        if (panel < p.full_panels) {
            const int r = t - panel * p.panel_tiles;
            mi = r >> 3;
            nt = panel * 8 + (r & 7);
        } else {
            const int r = t - p.full_panels * p.panel_tiles;
            mi = div_by_magic(r, p.rest_magic, p.rest_shift);
            nt = p.full_panels * 8 + r - mi * p.rest_cols;
        }
        m0 = mi * G::TA;
        n0 = nt * COLS;
    };

    // ---- producer
    auto part16 = [](int j, int lane) __attribute__((always_inline)) { return (uint32_t)(((lane & 7) ^ (((j & 1) * 4 + (lane >> 4)) & 7)) << 4); };   // LDS row 8j + lane/8 of 32
    const uint8_t *x_tile = nullptr, *w_tile = nullptr;    // scalar bases of the tile being fetched; per lane 32-bit offsets
    const float *xs_tile = nullptr;
    uint32_t x_off[4], w_off[GATEUP ? 2 : 4], xs_off = 0;  // (gate/up: 32 whole rows, so the rows of group j are w_below(j) under those of group 0)
    auto w_below = [](int j) { return 16 * (j & 1) + 4 * (j >> 1); };
    int seq = 0;                                           // tiles begun by the producer
    auto setup = [&](int t) __attribute__((always_inline)) {
        int m0, n0, lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                     // (what follows from it is worked out here, not kept in registers through the K-loop)
        const int prow = lane >> 3;
        decode(t, m0, n0);
        x_tile = p.x + (long long)m0 * p.ld_x;
        xs_tile = p.xs + m0;
        const int x_last = min(p.M - m0, G::TA) - 1;       // rows behind the last one: the last one again
        // this wave's 32 weight rows: gate/up, alternately 32 gate and 32 up rows
        const int w0 = GATEUP ? (wave & 1 ? p.N : 0) + n0 + (wave >> 1) * 32 : min(n0 + wave * 32, p.N - 1);
        w_tile = p.w + (long long)w0 * p.K;
        const int w_last = GATEUP ? 31 : min(p.N - 1 - w0, 31);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x_off[j] = (uint32_t)min(wave * 32 + j * 8 + prow, x_last) * (uint32_t)p.ld_x + part16(j, lane);
            if (!GATEUP || j < 2) w_off[j] = (uint32_t)min((GATEUP ? 0 : w_below(j)) + 8 * (prow >> 2) + (prow & 3), w_last) * (uint32_t)p.K + part16(j, lane);
        }
        xs_off = (uint32_t)min((wave & 3) * 64 + lane, x_last);
        const int nb = GATEUP ? ((wave & 1 ? p.N : 0) + n0) >> 7 : min((n0 >> 7) + (wave & 1), (p.N - 1) >> 7);
        lds_dma4(reinterpret_cast<const uint32_t*>(p.ws + (long long)nb * nks + min(lane, nks - 1)), smem + G::WS + (((seq & 3) * 2) + (wave & 1)) * 256);
        ++seq;
    };
    auto issue = [&](int op, int k, int stage) __attribute__((always_inline)) {
        if (op == 0) {
            lds_dma4(reinterpret_cast<const uint32_t*>(xs_tile + k * p.ld_xs) + xs_off, smem + G::XS + stage * (G::TA * 4) + (wave & 3) * 256);
            return;
        }
        const int j = (op - 1) & 3;
        uint8_t* l = smem + stage * G::STAGE + (op < 5 ? 0 : G::TA * 128) + (wave * 4 + j) * 1024;
        const uint8_t* src = (op < 5 ? x_tile + k * 128 + x_off[j] : w_tile + (GATEUP ? w_below(j) * p.K : 0) + k * 128 + w_off[GATEUP ? j & 1 : j]);
        if constexpr (RAGGED) {
            if (k * 128 + (int)part16(j, lane) >= p.K) src = g_zeros;
        }
        lds_dma16(src, l);
    };
    auto issue_some = [&](int from, int to, int k, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int op = from; op < to; ++op) issue(op, k, stage);
    };
    int ptile = tile, pk = 0;
    auto advance = [&]() __attribute__((always_inline)) {
        pk = pk + 1 == nks ? 0 : pk + 1;
        if (pk == 0 && ptile + nslots < tile_hi) {
            ptile += nslots;
            setup(ptile);
        }
    };

    // ---- consumer
    const int f_off = l16 * 128 + ((g ^ (l16 >> 1)) << 4);
    int stg = 0;
    const int x_base = wm * 128 * 128 + f_off, w_base = G::TA * 128 + wn * 64 * 128 + f_off;
    u32x4 fw[4][2], fx[4][2];                              // weights; four row tiles
    float xs[4], ws[2];
    v4f_t acc[8][4];
    auto fence = [&]() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    auto barrier = [&]() __attribute__((always_inline)) { fence(); asm volatile("s_barrier" ::: "memory"); fence(); };
    auto lds_wait = [&]() __attribute__((always_inline)) { fence(); __builtin_amdgcn_s_waitcnt(0xC07F); fence(); };      // LDS counter alone
    auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[i][t] = v4f_t{0.f, 0.f, 0.f, 0.f};
    };
    auto read_rows = [&](int half) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) fx[i][h] = *reinterpret_cast<const u32x4*>(smem + stg * G::STAGE + (x_base ^ (h << 6)) + (4 * half + i) * 2048);
            xs[i] = *reinterpret_cast<const float*>(smem + G::XS + stg * (G::TA * 4) + (wm * 128 + (4 * half + i) * 16 + l16) * 4);
        }
    };
    // A turn: 16 MFMAs, each followed by the multiply-adds of the one LAG before it, whose result is there by then.  Those of the last LAG
    // are left to the section behind the turn, so that the other wave's MFMAs need not wait for them.
    constexpr int LAG = 3;
    v4f_t d[16];
    float f[4][2];
    auto add_up = [&](int half, int k) __attribute__((always_inline)) {
        v4f_t& a = acc[4 * half + (k >> 2)][k & 3];
#pragma unroll
        for (int r = 0; r < 4; ++r) a[r] = __builtin_fmaf(d[k][r], f[k >> 2][GATEUP ? (k >> 1) & 1 : 0], a[r]);
    };
    auto turn = [&](int half) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i][0] = xs[i] * ws[0];
            if constexpr (GATEUP) f[i][1] = xs[i] * ws[1];
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const u32x4 *w = fw[k & 3], *x = fx[k >> 2];
            const v8i_t a = {(int)w[0].x, (int)w[0].y, (int)w[0].z, (int)w[0].w, (int)w[1].x, (int)w[1].y, (int)w[1].z, (int)w[1].w};
            const v8i_t b = {(int)x[0].x, (int)x[0].y, (int)x[0].z, (int)x[0].w, (int)x[1].x, (int)x[1].y, (int)x[1].z, (int)x[1].w};
            d[k] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, v4f_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
            fence();
            if (k >= LAG) add_up(half, k - LAG);
            fence();
        }
#pragma unroll
        for (int k = 0; k < 16 - LAG; ++k) asm volatile("" : "+v"(acc[4 * half + (k >> 2)][k & 3]));      // (they stay in this turn instead of moving to where their results are used)
        __builtin_amdgcn_s_setprio(0);
    };
    auto rest = [&](int half) __attribute__((always_inline)) {
        fence();
#pragma unroll
        for (int k = 16 - LAG; k < 16; ++k) add_up(half, k);
#pragma unroll
        for (int k = 16 - LAG; k < 16; ++k) asm volatile("" : "+v"(acc[4 * half + (k >> 2)][k & 3]));
        fence();
    };

    setup(tile);
    issue_some(0, 9, pk, 0);
    advance();
    issue_some(5, 9, pk, 1);
    asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    int ks = 0, cseq = 0, m0, n0;
    decode(tile, m0, n0);
    clear();
    if (wm) barrier();
    while (true) {
        const bool last = ks == nks - 1;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) fw[t][h] = *reinterpret_cast<const u32x4*>(smem + stg * G::STAGE + (w_base ^ (h << 6)) + t * 2048);
        read_rows(0);
        {
            const float* w = reinterpret_cast<const float*>(smem + G::WS + (cseq & 3) * 512) + ks;
            ws[0] = w[GATEUP ? 0 : (wn >> 1) * 64];
            if constexpr (GATEUP) ws[1] = w[64];
        }
        fence();
        issue_some(0, 5, pk, stg ^ 1);
        lds_wait();
        barrier();
        turn(0);
        barrier();                                         // (waves 4..7 have read the weights too)
        read_rows(1);
        fence();
        rest(0);
        advance();
        fence();
        issue_some(5, 9, pk, stg);
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");   // the next step, this wave's part
        lds_wait();
        barrier();
        turn(1);
        stg ^= 1;
        ++ks;
        if (!(last && wm)) barrier();
        rest(1);
        if (!last) continue;
        fp8_store_tile<GATEUP, 8, NT>(p, acc, smem + G::AMAX, G::TA, m0, n0, wm * 128, wn, lane, barrier);
        if (wm) barrier();
        tile += nslots;
        if (tile >= tile_hi) break;
        decode(tile, m0, n0);
        clear();
        ks = 0;
        ++cseq;
    }
    if (!wm) barrier();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // no transfer may still be writing this block's LDS when it ends
}

// Few rows (decode steps): the weights' bytes are what takes the time, so they go from memory straight to registers, AHEAD K blocks of a
// wave's behind one another (between two of them the wave waits for the weights' scale, a scalar load; down: one K block at a time), and
// the waves of a block share the K blocks of 16 weight rows; their sums meet in LDS, in the order of the waves.  The
// rows come from the caches: a block reads all of them.  Sums are FP32 here (see above).  Gate/up: 8 gate and 8 up rows, so that I = 1408
// makes 176 blocks.  h of the feed-forward block: gate/up leaves it in FP32, and the down product's waves encode the blocks of it that
// they multiply: an E4M3 block spans 128 columns, which would leave a block per 128 columns of h, 11, to read the weights.
// One row: 8192 x 8192 13.1 to 13.8 us (5.1 TB/s), 2048 x 2048 3.1 us (launch, the scales' latencies and the weights'); 24 rows 4.8 us; the
// feed-forward block of 24 rows, H 2048, I 1408 10.7 us.  8 waves per block; 4 and 16 were slower, so were non-temporal loads.
enum FewKind { kFewLinear, kFewLinearF32, kFewGateUp, kFewDown };

// Where h of (row m, column k) of M rows is: column 64 a + 16 g + 4 q + r of a block of 128 sits with the other rows' and g's of the same
// a, q, so that each of the eight loads by which lane (row, g) gets its 32 columns is contiguous over the wave.
__device__ __forceinline__ long long few_h_at(int m, int k, int M) {
    const int e = (k >> 6 & 1) * 4 + (k >> 2 & 3);
    return ((long long)((k >> 7) * 8 + e) * M + m) * 16 + (k >> 4 & 3) * 4 + (k & 3);
}

template <int RT, FewKind KIND, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) fp8_few_kernel(const Fp8Gemm p) {
    constexpr int COLS = KIND == kFewGateUp ? 8 : 16;      // output columns of a block
    constexpr int AHEAD = KIND == kFewDown ? 1 : RT == 1 ? 4 : 2;              // K blocks in flight per wave
    extern __shared__ __align__(16) uint8_t smem[];
    float* part = reinterpret_cast<float*>(smem);          // [WAVES][RT][256]
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * COLS;
    const int n = KIND == kFewGateUp ? (l16 & 8 ? p.N : 0) + n0 + (l16 & 7) : min(n0 + l16, p.N - 1);
    const uint8_t* w_row = p.w + (long long)n * p.K + g * 16;
    const float* w_scale = p.ws + (long long)(n0 >> 7) * p.KB;
    const float* u_scale = KIND == kFewGateUp ? w_scale + (long long)(p.N >> 7) * p.KB : w_scale;     // (lane groups 2 and 3 end up with the up rows)
    const uint8_t* x_row[RT];                              // rows behind the last one: the last one again
    int row[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        row[i] = min(i * 16 + l16, p.M - 1);
        x_row[i] = p.x + (KIND == kFewDown ? row[i] * 64 + g * 16 : row[i] * p.ld_x + g * 16);
    }
    v4f_t acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = v4f_t{0.f, 0.f, 0.f, 0.f};

    for (int k0 = wave; k0 < p.KB; k0 += AHEAD * WAVES) {
        u32x4 w[AHEAD][2], x[AHEAD][RT][2];
        f32x4_t hv[KIND == kFewDown ? RT : 1][8];
        float ws[AHEAD], xs[AHEAD][RT];
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const int kb = k0 + a * WAVES;
            if (kb >= p.KB) break;
            const bool there[2] = {kb * 128 + g * 16 < p.K, kb * 128 + 64 + g * 16 < p.K};
#pragma unroll
            for (int h = 0; h < 2; ++h) w[a][h] = there[h] ? *reinterpret_cast<const u32x4*>(w_row + kb * 128 + h * 64) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                if constexpr (KIND == kFewDown) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) hv[i][e] = *reinterpret_cast<const f32x4_t*>(x_row[i] + (long long)(kb * 8 + e) * p.M * 64);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) x[a][i][h] = there[h] ? *reinterpret_cast<const u32x4*>(x_row[i] + kb * 128 + h * 64) : u32x4{0, 0, 0, 0};
                    xs[a][i] = p.xs[kb * p.ld_xs + row[i]];
                }
            }
            const float s0 = w_scale[kb], s1 = u_scale[kb];
            ws[a] = KIND == kFewGateUp && g >= 2 ? s1 : s0;
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if (k0 + a * WAVES >= p.KB) break;
            if constexpr (KIND == kFewDown) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    float m = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int r = 0; r < 4; ++r) m = fmaxf(m, fabsf(hv[i][e][r]));
                    m = groups_max(m);
                    const Fp8Scale sc = fp8_scale(m);
                    xs[a][i] = sc.scale;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t c[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const f32x4_t v = hv[i][4 * h + q];
                            const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * sc.inv, v[1] * sc.inv, 0, false);
                            c[q] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2] * sc.inv, v[3] * sc.inv, lo, true);
                        }
                        x[a][i][h] = u32x4{c[0], c[1], c[2], c[3]};
                    }
                }
            }
            v8bf_t wv[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                wv[2 * h] = fp8_widen(w[a][h].x, w[a][h].y);
                wv[2 * h + 1] = fp8_widen(w[a][h].z, w[a][h].w);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                v4f_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[2 * h], fp8_widen(x[a][i][h].x, x[a][i][h].y), d, 0, 0, 0);
                    d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv[2 * h + 1], fp8_widen(x[a][i][h].z, x[a][i][h].w), d, 0, 0, 0);
                }
                const float f = xs[a][i] * ws[a];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][r] = __builtin_fmaf(d[r], f, acc[i][r]);
            }
        }
    }
    // acc[i][r]: row 16 i + l16, weight row 4 g + r
#pragma unroll
    for (int i = 0; i < RT; ++i) *reinterpret_cast<v4f_t*>(&part[(wave * RT + i) * 256 + l16 * 16 + g * 4]) = acc[i];
    __syncthreads();
    auto sum = [&](int at) __attribute__((always_inline)) {
        float v = part[at];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += part[w * RT * 256 + at];
        return v;
    };
    for (int at = threadIdx.x; at < RT * 16 * COLS; at += 64 * WAVES) {
        const int m = at / COLS, c = at % COLS, col = n0 + c;
        if (m >= p.M || col >= p.N) continue;
        float y = sum(m * 16 + c);
        if constexpr (KIND == kFewGateUp) {
            reinterpret_cast<float*>(p.out)[few_h_at(m, col, p.M)] = y * __builtin_amdgcn_rcpf(1.0f + __expf(-y)) * sum(m * 16 + 8 + c);
        } else {
            if (p.bias) y += bf16_lo(reinterpret_cast<const uint16_t*>(p.bias)[col]);
            if constexpr (KIND == kFewLinearF32) {
                if (p.add) y += reinterpret_cast<const float*>(p.add)[m * p.ld_add + col];
                reinterpret_cast<float*>(p.out)[m * p.ld_out + col] = y;
            } else {
                if (p.add) y += bf16_lo(reinterpret_cast<const uint16_t*>(p.add)[m * p.ld_add + col]);
                reinterpret_cast<__bf16*>(p.out)[m * p.ld_out + col] = (__bf16)y;
            }
        }
    }
}

static int current_device(int* dev) { REALB_HIP(hipGetDevice(dev)); return REALB_OK; }

template <bool GATEUP, bool WIDE, bool F32OUT, int RT, int WM, int WN, int NS, int CT>
static int launch_fp8_small(Fp8Gemm p, hipStream_t s) {
    using G = SmallGeo<RT, WM, WN, NS, CT>;
    static_assert(G::LDS <= 160 * 1024, "LDS");
    static std::atomic<unsigned long long> seen{0};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != REALB_OK) return rc;
    if (first_use_on_device(seen, dev)) {
        REALB_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_tile_kernel<GATEUP, WIDE, F32OUT, RT, WM, WN, NS, CT>), hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS));
        mark_used_on_device(seen, dev);
    }
    const int rows = ceil_div(p.M, G::TA), cols = ceil_div(p.N, GATEUP ? G::TW / 2 : G::TW);
    const long long tiles = (long long)rows * cols;
    REALB_REQUIRE(tiles < (1ll << 22), REALB_ECAP, "M=%d N=%d: too many tiles for one launch", p.M, p.N);
    // What an XCD's blocks share they fetch once; of the two operands the larger should be fetched by one XCD only.
    p.tiles = (int)tiles;
    p.rows_first = p.M < (GATEUP ? 2 : 1) * p.N;
    p.panel_tiles = p.rows_first ? rows : cols;
    division_magic(p.panel_tiles, &p.panel_magic, &p.panel_shift);
    hipLaunchKernelGGL((fp8_tile_kernel<GATEUP, WIDE, F32OUT, RT, WM, WN, NS, CT>), dim3((unsigned)(8 * ((tiles + 7) / 8))), dim3(64 * G::WAVES), G::LDS, s, p);
    REALB_HIP(hipGetLastError());
    return REALB_OK;
}

// Outputs above this size are streamed past the caches, as those of the layer's GEMMs are.  Product alone, temporal / streamed, us: 268 MB
// 259.6 / 241.7; 134 MB 234.4 / 228.0; 92 MB 94.9 / 90.7.  Product and the norm that reads it: 64 MB 120.0 / 121.4, 96 MB 170.4 / 173.6, 128 MB
// 226.9 / 226.8, 192 MB 336.0 / 334.1, 256 MB 448.3 / 443.0.
constexpr long long kStreamBytes = 160ll << 20;

template <bool GATEUP, bool RAGGED, bool NT>
static int launch_fp8_big(Fp8Gemm p, hipStream_t s) {
    const int rows = ceil_div(p.M, BigGeo::TA), cols = ceil_div(p.N, GATEUP ? 128 : 256);
    const long long tiles = (long long)rows * cols;
    REALB_REQUIRE(tiles < (1ll << 26), REALB_ECAP, "M=%d N=%d: too many tiles for one launch", p.M, p.N);
    p.tiles = (int)tiles;
    p.panel_tiles = rows * 8;
    p.full_panels = cols / 8;
    p.rest_cols = cols % 8 > 0 ? cols % 8 : 1;
    division_magic(p.panel_tiles, &p.panel_magic, &p.panel_shift);
    division_magic(p.rest_cols, &p.rest_magic, &p.rest_shift);
    static std::atomic<unsigned long long> seen{0};
    int dev = 0, cus = 0;
    int rc = current_device(&dev);
    if (rc == REALB_OK) rc = static_scratch_lookup(nullptr, &cus);
    if (rc != REALB_OK) return rc;
    if (first_use_on_device(seen, dev)) {
        REALB_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_big_kernel<GATEUP, RAGGED, NT>), hipFuncAttributeMaxDynamicSharedMemorySize, BigGeo::LDS));
        mark_used_on_device(seen, dev);
    }
    const long long slots = 8ll * (cus / 8 > 0 ? cus / 8 : 1);                            // a block per CU, a multiple of 8 (XCDs)
    const unsigned grid = (unsigned)(tiles < slots ? 8 * ((tiles + 7) / 8) : slots);
    hipLaunchKernelGGL((fp8_big_kernel<GATEUP, RAGGED, NT>), dim3(grid), dim3(512), BigGeo::LDS, s, p);
    REALB_HIP(hipGetLastError());
    return REALB_OK;
}

// Up to here fp8_few_kernel, above tiles; products alone, us, few / tiles:   17 rows      32 rows      48 rows      64 rows
//   2048 x 2048                                                           4.6 / 7.4    5.2 / 7.5    6.4 / 7.5    7.4 / 7.6
//   2048 x 8192 (K)                                                      10.9 / 27.8  13.7 / 28.0  18.5 / 27.9  22.3 / 28.2
//   8192 x 8192                                                          20.8 / 28.9  25.3 / 29.2  33.4 / 29.0  43.9 / 29.4
// It is also where FP32 sums cost nothing, which the wide products of 33 to 64 rows pay for.
constexpr int kFewRows = 64;
template <int RT, FewKind KIND>
static int launch_fp8_few_rows(const Fp8Gemm& p, hipStream_t s) {
    constexpr int WAVES = 8;
    REALB_REQUIRE(p.N < (1 << 24), REALB_ECAP, "N=%d: too many columns for one launch", p.N);
    hipLaunchKernelGGL((fp8_few_kernel<RT, KIND, WAVES>), dim3((unsigned)ceil_div(p.N, KIND == kFewGateUp ? 8 : 16)), dim3(64 * WAVES), WAVES * RT * 1024, s, p);
    REALB_HIP(hipGetLastError());
    return REALB_OK;
}
template <FewKind KIND>
static int launch_fp8_few(const Fp8Gemm& p, hipStream_t s) {
    if (p.M <= 16) return launch_fp8_few_rows<1, KIND>(p, s);
    if (p.M <= 32) return launch_fp8_few_rows<2, KIND>(p, s);
    if (p.M <= 48) return launch_fp8_few_rows<3, KIND>(p, s);
    return launch_fp8_few_rows<4, KIND>(p, s);
}
// Which tiles: those with the least time by rounds of them on the chip.  A round's time at K = 2048, us, where a round is one tile on every
// slot, that is as many blocks as run at once:
//                              8-bit     FP32 sums (half the rate)
//   64 x 64                        9       12    a block per CU
//   128 x 64                      11       17    a block per CU
//   128 x 128, 16 waves           15       26    a block per CU, one round
//   128 x 128, 8 or 4 waves       21       40    two blocks per CU
//   256 x 256                     25
//   gate/up, h columns half the weight rows, a block per CU:
//   64 x 256                      15       24
//   128 x 256                     22       37
//   256 x 256                     31
// They are used for every K: between tiles the ratios hold roughly, but a launch weighs more where a round is short.
// Where the last round of 256-row tiles would be short, the rows behind the whole rounds go to a second launch with smaller tiles, if that is
// faster by more than a launch.  One launch / two, us: 10 000 rows, N = 2048, K = 2048 54.6 / 51.1, 512 22.2 / 23.7, 128 14.4 / 16.3; 17 000 rows 85.5 / 79.6, 32.1 / 31.0,
// 20.4 / 21.0; the feed-forward block of 6000 rows, I 1408, H = 2048 83.8 / 73.6, 1024 53.7 / 47.6, 128 25.5 / 23.4.
enum Fp8Tile { kTile64, kTile128x64, kTile128One, kTile128, kTile256, kTileSplit };      // (Split: whole rounds of 256 and a second launch)
struct Fp8Choice { Fp8Tile tile; int us; };

template <bool GATEUP, bool WIDE>
static Fp8Choice choose_tiles(const Fp8Gemm& p, int M, int cus, int* whole) {
    auto rounds = [&](int rows, int cols, int per_cu) {
        const long long slots = (long long)per_cu * cus;
        return (int)(((long long)ceil_div(M, rows) * ceil_div(p.N, cols) + slots - 1) / slots);
    };
    Fp8Choice best{kTile64, INT_MAX};
    auto offer = [&](Fp8Tile tile, int us) { if (us < best.us) best = Fp8Choice{tile, us}; };
    const int one = GATEUP ? 31 : 25;                      // a round of 256-row tiles
    const int cols = GATEUP ? 128 : 256;                   // their output columns
    if (!WIDE && p.KB <= kBigMaxBlocks && p.ld_x <= kBigMaxPitch) {
        offer(kTile256, one * rounds(256, cols, 1));
        const int wide = ceil_div(p.N, cols);
        const long long full = (long long)ceil_div(M, 256) * wide / cus, rows = full * cus / wide * 256;      // whole rounds, rows of them
        if (whole && full > 0 && rows > 0 && rows < M) {
            constexpr int kLaunch = 3;
            *whole = (int)rows;
            offer(kTileSplit, (int)full * one + kLaunch + choose_tiles<GATEUP, WIDE>(p, M - (int)rows, cus, nullptr).us);
        }
    }
    if (GATEUP) {
        offer(kTile128, (WIDE ? 37 : 22) * rounds(128, 128, 1));
        offer(kTile64, (WIDE ? 24 : 15) * rounds(64, 128, 1));
    } else {
        offer(kTile128, (WIDE ? 40 : 21) * rounds(128, 128, 2));
        if (rounds(128, 128, 1) == 1) offer(kTile128One, WIDE ? 26 : 15);
        offer(kTile128x64, (WIDE ? 17 : 11) * rounds(128, 64, 1));
        offer(kTile64, (WIDE ? 12 : 9) * rounds(64, 64, 1));
    }
    return best;
}

template <bool GATEUP, bool WIDE, bool F32OUT>
static int launch_fp8_tiles_of(const Fp8Gemm& p, Fp8Tile tile, bool stream, hipStream_t s) {
    if constexpr (GATEUP) {
        if constexpr (WIDE) {                               // (widened codes of 16 waves a block would not fit the registers)
            if (tile == kTile128) return launch_fp8_small<true, true, false, 4, 2, 4, 3, 4>(p, s);
        } else {
            if (tile == kTile256) return launch_fp8_big<true, false, false>(p, s);
            if (tile == kTile128) return launch_fp8_small<true, false, false, 2, 4, 4, 3, 4>(p, s);
        }
        return launch_fp8_small<true, WIDE, false, 2, 2, 4, 3, 4>(p, s);
    } else {
        if constexpr (WIDE) {
            if (tile == kTile128) return launch_fp8_small<false, true, F32OUT, 4, 2, 2, 2, 4>(p, s);
        } else {
            if (tile == kTile256 && p.K % 128 != 0) return stream ? launch_fp8_big<false, true, true>(p, s) : launch_fp8_big<false, true, false>(p, s);
            if (tile == kTile256) return stream ? launch_fp8_big<false, false, true>(p, s) : launch_fp8_big<false, false, false>(p, s);
            if (tile == kTile128) return launch_fp8_small<false, false, false, 2, 4, 2, 2, 4>(p, s);
        }
        if (tile == kTile128One) return launch_fp8_small<false, WIDE, F32OUT, 2, 4, 4, 4, 2>(p, s);
        return tile == kTile64 ? launch_fp8_small<false, WIDE, F32OUT, 1, 4, 2, 4, 2>(p, s) : launch_fp8_small<false, WIDE, F32OUT, 2, 4, 2, 4, 2>(p, s);
    }
}

template <bool GATEUP, bool WIDE, bool F32OUT>
static int launch_fp8_tile(const Fp8Gemm& p, hipStream_t s) {
    static_assert(WIDE || !F32OUT, "F32 outputs have FP32 sums");
    int cus = 0;
    int rc = static_scratch_lookup(nullptr, &cus);
    if (rc != REALB_OK) return rc;
    int whole = 0;
    const Fp8Choice c = choose_tiles<GATEUP, WIDE>(p, p.M, cus, &whole);
    const bool stream = !GATEUP && (long long)p.M * p.N * 2 > kStreamBytes;
    if (c.tile != kTileSplit) return launch_fp8_tiles_of<GATEUP, WIDE, F32OUT>(p, c.tile, stream, s);
    Fp8Gemm head = p, rest = p;
    head.M = whole;
    rest.M = p.M - whole;
    rest.x += whole * p.ld_x;
    rest.xs += whole;
    rest.out += whole * p.ld_out * (GATEUP ? 1 : F32OUT ? 4 : 2);
    if (GATEUP) rest.out_s += whole;
    if (p.add) rest.add += whole * p.ld_add * (F32OUT ? 4 : 2);
    rc = launch_fp8_tiles_of<GATEUP, WIDE, F32OUT>(head, kTile256, stream, s);
    if (rc != REALB_OK) return rc;
    return launch_fp8_tiles_of<GATEUP, WIDE, F32OUT>(rest, choose_tiles<GATEUP, WIDE>(rest, rest.M, cus, nullptr).tile, stream, s);
}

static int check_rows(const uint8_t* q, long long ld, const float* s, long long ld_s, long long rows, int K) {
    REALB_REQUIRE(ld >= K && ld % 16 == 0 && aligned_to(q, 16), REALB_EINVAL, "rows of codes must be K=%d apart or more and start at multiples of 16 bytes", K);
    REALB_REQUIRE(ld_s >= rows && aligned_to(s, 4), REALB_EINVAL, "rows of scales must be %lld apart or more", rows);
    return REALB_OK;
}

// What h of T rows takes.
static size_t ffn_h_bytes(int T, int I) {
    if (T <= kFewRows) return (size_t)T * I * 4;            // FP32
    const size_t pitch = ((size_t)T + 3) / 4 * 4;
    return (size_t)T * I + pitch * (I / 128) * 4;          // codes and scales
}

}  // namespace realb

using namespace realb;

extern "C" {

int realb_linear_fp8(const realb_linear_io* io, void* stream) {
    REALB_REQUIRE(io != nullptr, REALB_EINVAL, "io is NULL");
    REALB_REQUIRE(io->M >= 0 && io->N > 0 && io->K > 0 && io->K % 16 == 0 && io->K <= 65536, REALB_ESHAPE,
                  "M=%d N=%d K=%d: K must be a positive multiple of 16 up to 65536", io->M, io->N, io->K);
    REALB_REQUIRE(io->out_type == REALB_TYPE_BF16 || io->out_type == REALB_TYPE_F32, REALB_EINVAL, "bad type %d", io->out_type);
    if (io->M == 0) return REALB_OK;
    REALB_REQUIRE(io->x_q && io->x_s && io->w_q && io->w_s && io->out, REALB_EINVAL, "NULL argument");
    const int rc = check_rows(io->x_q, io->ld_x, io->x_s, io->ld_xs, io->M, io->K);
    if (rc != REALB_OK) return rc;
    const bool f32 = io->out_type == REALB_TYPE_F32;
    REALB_REQUIRE(aligned_to(io->w_q, 16) && aligned_to(io->w_s, 4), REALB_EINVAL, "w_q must start at a multiple of 16 bytes");
    REALB_REQUIRE(io->ld_out >= io->N && aligned_to(io->out, f32 ? 4 : 2), REALB_EINVAL, "rows of out must be N=%d apart or more", io->N);
    REALB_REQUIRE(!io->add || (io->ld_add >= io->N && aligned_to(io->add, f32 ? 4 : 2)), REALB_EINVAL, "rows of add must be N=%d apart or more", io->N);
    REALB_REQUIRE(aligned_to(io->bias, 2), REALB_EINVAL, "bias must be aligned to its type");
    Fp8Gemm p{};
    p.x = io->x_q; p.xs = io->x_s; p.w = io->w_q; p.ws = io->w_s; p.out = (uint8_t*)io->out; p.bias = (const uint8_t*)io->bias; p.add = (const uint8_t*)io->add;
    p.ld_x = io->ld_x; p.ld_xs = io->ld_xs; p.ld_out = io->ld_out; p.ld_add = io->ld_add;
    p.M = io->M; p.N = io->N; p.K = io->K; p.KB = ceil_div(io->K, 128);
    if (p.M <= kFewRows) return f32 ? launch_fp8_few<kFewLinearF32>(p, as_stream(stream)) : launch_fp8_few<kFewLinear>(p, as_stream(stream));
    return f32 ? launch_fp8_tile<false, true, true>(p, as_stream(stream)) : launch_fp8_tile<false, false, false>(p, as_stream(stream));
}

size_t realb_gated_ffn_workspace_bytes(int T, int I) {
    if (T < 0 || I <= 0 || I % 128 != 0) {
        set_error("T=%d I=%d: I must be a positive multiple of 128", T, I);
        return 0;
    }
    const size_t need = ffn_h_bytes(T, I), few = ffn_h_bytes(kFewRows, I);
    return T > kFewRows && need < few ? few : need;         // (a workspace for T rows holds any smaller batch)
}

int realb_gated_ffn_fp8(const realb_ffn_io* io, void* stream) {
    REALB_REQUIRE(io != nullptr, REALB_EINVAL, "io is NULL");
    REALB_REQUIRE(io->T >= 0 && io->H > 0 && io->I > 0 && io->H % 128 == 0 && io->I % 128 == 0 && io->H <= 65536 && io->I <= 65536, REALB_ESHAPE,
                  "T=%d H=%d I=%d: H and I must be positive multiples of 128 up to 65536", io->T, io->H, io->I);
    REALB_REQUIRE(io->sums == REALB_SUMS_MFMA8 || io->sums == REALB_SUMS_F32, REALB_EINVAL, "bad choice of sums %d", io->sums);
    if (io->T == 0) return REALB_OK;
    REALB_REQUIRE(io->x_q && io->x_s && io->w13_q && io->w13_s && io->w2_q && io->w2_s && io->out && io->workspace, REALB_EINVAL, "NULL argument");
    const int rc = check_rows(io->x_q, io->ld_x, io->x_s, io->ld_xs, io->T, io->H);
    if (rc != REALB_OK) return rc;
    REALB_REQUIRE(aligned_to(io->w13_q, 16) && aligned_to(io->w2_q, 16) && aligned_to(io->w13_s, 4) && aligned_to(io->w2_s, 4) && aligned_to(io->workspace, 16), REALB_EINVAL,
                  "codes and workspace must start at multiples of 16 bytes");
    REALB_REQUIRE(io->workspace_bytes >= ffn_h_bytes(io->T, io->I), REALB_EINVAL, "the workspace has %zu bytes, T=%d I=%d needs %zu",
                  io->workspace_bytes, io->T, io->I, ffn_h_bytes(io->T, io->I));
    REALB_REQUIRE(io->ld_out >= io->H && aligned_to(io->out, 2), REALB_EINVAL, "rows of out must be H=%d apart or more", io->H);
    REALB_REQUIRE(!io->add || (io->ld_add >= io->H && aligned_to(io->add, 2)), REALB_EINVAL, "rows of add must be H=%d apart or more", io->H);
    hipStream_t s = as_stream(stream);
    uint8_t* h_q = (uint8_t*)io->workspace;
    const long long pitch = ((long long)io->T + 3) / 4 * 4;
    float* h_s = reinterpret_cast<float*>(h_q + (size_t)io->T * io->I);
    Fp8Gemm a{};
    a.x = io->x_q; a.xs = io->x_s; a.w = io->w13_q; a.ws = io->w13_s; a.out = h_q; a.out_s = h_s;
    a.ld_x = io->ld_x; a.ld_xs = io->ld_xs; a.ld_out = io->I; a.ld_s = pitch;
    a.M = io->T; a.N = io->I; a.K = io->H; a.KB = io->H / 128;
    Fp8Gemm b{};
    b.x = h_q; b.xs = h_s; b.w = io->w2_q; b.ws = io->w2_s; b.out = (uint8_t*)io->out; b.add = (const uint8_t*)io->add;
    b.ld_x = io->I; b.ld_xs = pitch; b.ld_out = io->ld_out; b.ld_add = io->ld_add;
    b.M = io->T; b.N = io->H; b.K = io->I; b.KB = io->I / 128;
    if (io->T <= kFewRows) {                                // h in FP32
        const int rc1 = launch_fp8_few<kFewGateUp>(a, s);
        return rc1 != REALB_OK ? rc1 : launch_fp8_few<kFewDown>(b, s);
    }
    if (io->sums == REALB_SUMS_F32) {
        const int rc1 = launch_fp8_tile<true, true, false>(a, s);
        return rc1 != REALB_OK ? rc1 : launch_fp8_tile<false, true, false>(b, s);
    }
    const int rc1 = launch_fp8_tile<true, false, false>(a, s);
    return rc1 != REALB_OK ? rc1 : launch_fp8_tile<false, false, false>(b, s);
}

}  // extern "C"
