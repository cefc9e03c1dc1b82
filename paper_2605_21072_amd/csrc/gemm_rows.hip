// Few tokens, or few outputs: the dual-scale GEMM with its fused ending where the tiles of gemm_dma128.h leave most CUs without work (one token's 1536
// outputs are 24 of its smallest) and walk the whole of K one stage after another.
//
// A workgroup has CT times 16 output columns and MT times 16 rows; its eight waves share K: spans of 128 packed positions (one cache line of an INT8
// row), wave w every eighth.  Operands go from memory to the matrix instructions without LDS: in v_mfma_i32_16x16x64_i8 lane l supplies sixteen K
// bytes of row l & 15, and which sixteen is free as long as both operands agree, so lane quarter l >> 4 takes the positions 32 (l >> 4) .. + 31
// of a span, two instructions' worth, 32 bytes of INT8 or 16 of INT4 in one piece.  Four spans of a wave are in flight; what a span has
// delivered is multiplied and its registers are asked to hold the fourth next.  The outlier range ends at a multiple of 32: a quarter lies on one side of it.
//
// P = 2, eight rows: the sixteen rows of either operand are eight of one span and the same eight of the next.  Of the 16 x 16 products
// the two 8 x 8 blocks whose spans agree are sums of the result; the others are left.  A workgroup then has eight columns, there are twice as many,
// and still every lane fetches weights of its own.
//
// Sums are integers, so the waves add theirs in LDS in any order, and the epilogue is the tiles' own arithmetic: the same bits.
//
// Operands are read again by every workgroup that shares them, at 16 multiplications to a byte at most: once the workgroups no longer all run side by
// side, tiles that pass operands through LDS are faster (the choice and what it measured: pick_rows).
//
// Bound by the latency of the first loads (2 us of launch and epilogue, about 2 us until the weights are there) and beyond a few MB by how much 256 CUs
// keep in flight.  us against the best tile, INT8 weights: 1 x 1536 -> 1536 3.7 (6.4), 1 x 8960 -> 1536 5.8 (16), 16 x 8960 -> 1536 12.1 (16.9),
// 1 x 13824 -> 4608 17 (28.7); INT4: 1 x 8960 -> 1536 4.6 (21), 16 x 4096 -> 8960 10.7 (13), 32 x 8960 -> 1536 9.5 (22.6).
#include <type_traits>

#include "gemm_dma_common.h"

namespace qarvd_gemm {

namespace {

constexpr int NW = 8;                     // waves of a workgroup
constexpr int SPAN = 128, AHEAD = 4;      // AHEAD: spans whose loads are in flight
constexpr int ROWS_QUANT_MAX_K = 10240;   // channels that the workgroup of the quantizing build holds in registers

struct RowsX {                            // the row to quantize
    const void *X;
    const int32_t *perm;
};

// Quantizes the one row of X as quant_act does (the same codes and scale): its channels in registers, their absmax over the workgroup, codes
// in natural order in LDS, from where the packed row picks its bytes.  The row and the permutation's entries are requested before the first
// weights, which come from farther away.
template <typename T> struct RowQuantizer {
    static constexpr int NT = 64 * NW, CHUNKS = ROWS_QUANT_MAX_K / (4 * NT), PACKED = CHUNKS + 1;      // (packed: up to 31 + 127 pads)
    typedef T four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef int entries __attribute__((ext_vector_type(4), aligned(4)));
    four f[CHUNKS];
    entries ch[PACKED];                        // channels of the four positions of this thread's words, -1: padding

    __device__ __forceinline__ void request(const GemmArgs &g, const RowsX &in);
    __device__ __forceinline__ float quantize(const GemmArgs &g, const RowsX &in, unsigned char *image, float *red) const;      // returns the scale
};
template <> struct RowQuantizer<void> {};

template <typename T> __device__ __forceinline__ void RowQuantizer<T>::request(const GemmArgs &g, const RowsX &in)
{
    const T *const x = reinterpret_cast<const T *>(in.X);
    const int tid = threadIdx.x;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = 4 * (tid + c * NT);
        f[c] = four{0, 0, 0, 0};
        if (k + 4 <= g.K) {
            f[c] = *reinterpret_cast<const four *>(x + k);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (k + e < g.K) f[c][e] = x[k + e];
        }
    }
    if (!in.perm) return;
#pragma unroll
    for (int c = 0; c < PACKED; ++c) {
        const int p = 4 * (tid + c * NT);
        const int i = p < g.n_off ? p : g.K_o + (p - g.n_off), end = p < g.n_off ? g.K_o : g.K;     // (n_off is a multiple of 32)
        ch[c] = entries{-1, -1, -1, -1};
        if (i + 4 <= end) {
            ch[c] = *reinterpret_cast<const entries *>(in.perm + i);
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (i + e < end) ch[c][e] = in.perm[i + e];
        }
    }
}

template <typename T>
__device__ __forceinline__ float RowQuantizer<T>::quantize(const GemmArgs &g, const RowsX &in, unsigned char *image, float *red) const
{
    constexpr float MAGIC = 12582912.0f;       // 1.5 * 2^23: the sum rounds half-to-even, the code is its low byte
    const int tid = threadIdx.x;
    unsigned char *const natural = in.perm ? image + g.kp : image;      // without a permutation the packed row is the natural one and zeros
    auto widen = [](T v) {
        if constexpr (sizeof(T) == 2) return bf16_bits_to_f32(v);
        else return v;
    };
    float amax = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(widen(f[c][e])));
    amax = wave_max_all(amax);
    if ((tid & 63) == 0) red[tid >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NW; ++w) amax = fmaxf(amax, red[w]);
    const float s = amax / 127.0f;
    const ExactQuotient q(s, 127.0f);
    const int end = in.perm ? g.K : g.kp;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int k = 4 * (tid + c * NT);
        if (k >= end) continue;
        unsigned word = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float v = widen(f[c][e]);
            const unsigned code = q.exact() ? __float_as_uint(q.clamped(v) + MAGIC) : (unsigned)quantize_i8(v, s);
            word |= (code & 255u) << (8 * e);
        }
        *reinterpret_cast<unsigned *>(natural + k) = word;
    }
    __syncthreads();
    if (in.perm) {
#pragma unroll
        for (int c = 0; c < PACKED; ++c) {
            const int p = 4 * (tid + c * NT);
            if (p >= g.kp) continue;
            unsigned word = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ch[c][e] >= 0) word |= (unsigned)natural[min(ch[c][e], g.K - 1)] << (8 * e);
            *reinterpret_cast<unsigned *>(image + p) = word;
        }
        __syncthreads();
    }
    return s;
}

// XT: the type of the activations that the workgroup quantizes itself, or void: g.Xq and g.s_x hold them.
template <int MT, int CT, int P, bool W4, typename OutT, typename XT>
__global__ __launch_bounds__(64 * NW) void gemm_rows_kernel(GemmArgs g, RowsX in)
{
    constexpr bool QUANT = !std::is_void<XT>::value;
    static_assert(P == 1 || (MT == 1 && CT == 1), "parts of K take the place of rows and columns");
    constexpr int PER = 16 / P, COLS = PER * CT, ROWS = MT * PER;
    __shared__ int sums[2][ROWS][COLS];              // outlier, normal
    __shared__ float red[NW];                        // (QUANT)
    extern __shared__ __align__(16) unsigned char image[];      // (QUANT) the packed row, then the row in natural order
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & (PER - 1), part = (lane & 15) / PER, q = lane >> 4;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * ROWS, rows = min(ROWS, g.M - m0);
    const int spans = g.kp / SPAN;
    const int8_t *pw[CT], *px[MT];
#pragma unroll
    for (int c = 0; c < CT; ++c)      // (a column past the matrix: the last one again, what comes of it is not stored)
        pw[c] = g.Wq + (size_t)min(n0 + 16 * c + r, g.N - 1) * g.ldwq + q * (W4 ? 16 : 32);
#pragma unroll
    for (int t = 0; t < MT; ++t)
        px[t] = QUANT ? reinterpret_cast<const int8_t *>(image) + q * 32
                      : g.Xq + (size_t)(m0 + min(t * 16 + r, rows - 1)) * g.ldxq + q * 32;

    v4i acc[2][MT][CT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[0][t][c] = acc[1][t][c] = v4i{0, 0, 0, 0};
    for (int i = tid; i < 2 * ROWS * COLS; i += 64 * NW) (&sums[0][0][0])[i] = 0;

    v4i w[AHEAD][CT][W4 ? 1 : 2], x[AHEAD][MT][2];
    auto load_x = [&](int u, int s) {                // s: this lane's span
#pragma unroll
        for (int t = 0; t < MT; ++t)
            if (s < spans && t * 16 + r < rows) {     // lanes of rows that do not exist fetch nothing
                const v4i *b = reinterpret_cast<const v4i *>(px[t] + (size_t)s * SPAN);
                x[u][t][0] = b[0];
                x[u][t][1] = b[1];
            }
    };
    auto load = [&](int u, int s) {
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int h = 0; h < (W4 ? 1 : 2); ++h) {
                if (P > 1) w[u][c][h] = v4i{0, 0, 0, 0};        // a part may have a span less than the others
                if (s < spans) w[u][c][h] = reinterpret_cast<const v4i *>(pw[c] + (size_t)s * (W4 ? SPAN / 2 : SPAN))[h];
            }
        if constexpr (!QUANT) load_x(u, s);
    };
    RowQuantizer<XT> row;
    if constexpr (QUANT) row.request(g, in);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
#pragma unroll
        for (int t = 0; t < MT; ++t) x[u][t][0] = x[u][t][1] = v4i{0, 0, 0, 0};
        load(u, (wave + u * NW) * P + part);
    }
    float own_scale = 0.0f;
    if constexpr (QUANT) own_scale = row.quantize(g, in, image, red);
    for (int s0 = wave * P; s0 < spans; s0 += NW * AHEAD * P) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * NW * P;           // of part 0
            if (s >= spans) break;
            const int outlier = (s + part) * SPAN + 32 * q < g.n_off ? -1 : 0;
            if constexpr (QUANT) load_x(u, s + part);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                v4i wf[2];
                if constexpr (W4) {
                    wf[0] = unpack_w4(v2i{w[u][c][0].x, w[u][c][0].y});
                    wf[1] = unpack_w4(v2i{w[u][c][0].z, w[u][c][0].w});
                } else {
                    wf[0] = w[u][c][0];
                    wf[1] = w[u][c][1];
                }
                auto add = [&](int to, int keep) {
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            acc[to][t][c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[h] & keep, x[u][t][h], acc[to][t][c], 0, 0, 0);
                };
                if (s * SPAN < g.n_off) {
                    add(0, outlier);
                    add(1, ~outlier);
                } else {
                    add(1, -1);
                }
            }
            load(u, s + NW * AHEAD * P + part);
        }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // this lane: token row r of its part, column 4 q + e, which is of another part where the two K ranges differ
                const int col = (4 * q + e) & (PER - 1);
                if (t * 16 + r >= rows || (4 * q + e) / PER != part) continue;
                if (wave * P * SPAN < g.n_off) atomicAdd(&sums[0][t * PER + r][PER * c + col], acc[0][t][c][e]);      // (the waves that saw outliers)
                atomicAdd(&sums[1][t * PER + r][PER * c + col], acc[1][t][c][e]);
            }
    __syncthreads();

    OutT *const Y = reinterpret_cast<OutT *>(g.Y);
    const OutT *const R = reinterpret_cast<const OutT *>(g.R);
    for (int i = tid; i < ROWS * COLS; i += 64 * NW) {
        const int row = i / COLS, m = m0 + row, c = i % COLS, n = n0 + c;
        if (row >= rows || n >= g.N) continue;
        constexpr float ws = W4 ? 0.0625f : 1.0f;     // INT4 codes enter the matrix instructions times 16
        float v = (float)sums[0][row][c] * (g.n_off > 0 ? g.s_o[n] * ws : 0.0f);
        v = fmaf((float)sums[1][row][c], g.s_n[n] * ws, v);
        v = fmaf(v, QUANT ? own_scale : g.s_x[m], g.bias ? g.bias[n] : 0.0f);
        if (g.act == QARVD_ACT_GELU_TANH) v = gelu_tanh(v);
        if (g.gate || g.R) {
            float res = 0.0f;
            if (g.R) {
                if constexpr (sizeof(OutT) == 2) res = bf16_bits_to_f32(R[(size_t)m * g.ldr + n]);
                else res = R[(size_t)m * g.ldr + n];
            }
            v = fmaf(g.gate ? g.gate[(size_t)(m / g.gate_rows) * g.ldg + n] : 1.0f, v, res);
        }
        if constexpr (sizeof(OutT) == 2) Y[(size_t)m * g.ldy + n] = (OutT)cvt_pk_bf16(v, 0.0f);
        else Y[(size_t)m * g.ldy + n] = v;
    }
}

}  // namespace

template <int MT, int CT, int P, bool W4> qarvd_status launch_rows_gemm(const GemmArgs &g, qarvd_dtype ydt, hipStream_t st)
{
    constexpr int COLS = 16 / P * CT, ROWS = 16 / P * MT;
    const dim3 grid((g.N + COLS - 1) / COLS, (g.M + ROWS - 1) / ROWS), block(64 * NW);
    if (ydt == QARVD_BF16) hipLaunchKernelGGL((gemm_rows_kernel<MT, CT, P, W4, uint16_t, void>), grid, block, 0, st, g, RowsX{});
    else hipLaunchKernelGGL((gemm_rows_kernel<MT, CT, P, W4, float, void>), grid, block, 0, st, g, RowsX{});
    return qarvd_launch_status();
}

// One row of activations straight into the GEMM: a launch less.  Every workgroup quantizes the row for itself, so only as many
// as run side by side.  us with one launch and with two (quant_act and the kernel above), the host's part included: 1 x 1536 -> 1536 5.4 and 7.6, 1 x 8960 -> 1536 INT4
// 6.9 and 8.4; 1 x 1536 -> 4608 would be 9.1 and 8.1.
bool rows_quant_fits(const GemmArgs &g, int cus) { return g.M == 1 && g.N <= 8 * cus && g.K <= ROWS_QUANT_MAX_K; }

template <bool W4> qarvd_status launch_rows_quant(const GemmArgs &g, const void *X, qarvd_dtype xdt, const int32_t *perm, qarvd_dtype ydt,
                                                  hipStream_t st)
{
    constexpr int P = 2, COLS = 16 / P;
    const RowsX in = {X, g.K_o > 0 ? perm : nullptr};
    const dim3 grid((g.N + COLS - 1) / COLS), block(64 * NW);
    const size_t lds = 2 * (size_t)g.kp;
    auto go = [&](auto out, auto x) {
        hipLaunchKernelGGL((gemm_rows_kernel<1, 1, P, W4, decltype(out), decltype(x)>), grid, block, lds, st, g, in);
        return qarvd_launch_status();
    };
    if (ydt == QARVD_BF16) return xdt == QARVD_F32 ? go(uint16_t{}, float{}) : go(uint16_t{}, uint16_t{});
    return xdt == QARVD_F32 ? go(float{}, float{}) : go(float{}, uint16_t{});
}
template qarvd_status launch_rows_quant<false>(const GemmArgs &, const void *, qarvd_dtype, const int32_t *, qarvd_dtype, hipStream_t);
template qarvd_status launch_rows_quant<true>(const GemmArgs &, const void *, qarvd_dtype, const int32_t *, qarvd_dtype, hipStream_t);

#define QARVD_INST_ROWS(MT, CT, P, W4) template qarvd_status launch_rows_gemm<MT, CT, P, W4>(const GemmArgs &, qarvd_dtype, hipStream_t);
QARVD_INST_ROWS(1, 1, 2, false)
QARVD_INST_ROWS(1, 1, 1, false)
QARVD_INST_ROWS(2, 1, 1, false)
QARVD_INST_ROWS(1, 1, 2, true)
QARVD_INST_ROWS(1, 1, 1, true)
QARVD_INST_ROWS(1, 2, 1, true)

}  // namespace qarvd_gemm
