// Norm of queries and keys and their rotation by position (time, height, width), one pass over both.
//
//     r = 1 / sqrt(mean(x^2) + eps);   x <- x r w;   (a, b) <- (a cos t - b sin t, a sin t + b cos t),   t = pos[axis(i)] freq[i]
#include <algorithm>
#include <type_traits>

#include "qarvd_common.h"

namespace {

constexpr int TPB = 256;
constexpr int MAX_D = 512;

struct Tensor {                // qarvd_heads, strides in elements
    const void *x;
    void *out;
    const float *w;
    int64_t ld, hs, ld_out, hs_out;
    int32_t heads;
};
struct HeadArgs {
    Tensor t[2];               // queries, keys
    const int32_t *pos;
    const double *freq;
    int64_t ldpos;
    float eps;
    int32_t M, D, norm, pairs;             // pairs = R / 2
    int32_t end0, end1;                    // pairs before end0 turn with axis 0, before end1 with axis 1, the rest with axis 2
    int32_t interleaved;
};

template <typename T> __device__ __forceinline__ float widen1(T v);
template <> __device__ __forceinline__ float widen1<float>(float v) { return v; }
template <> __device__ __forceinline__ float widen1<uint16_t>(uint16_t v) { return bf16_bits_to_f32(v); }
template <typename T> __device__ __forceinline__ T narrow1(float v);
template <> __device__ __forceinline__ float narrow1<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow1<uint16_t>(float v)       // one v_cvt_pk_bf16_f32, NaN kept
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef float v2f __attribute__((ext_vector_type(2)));
    const v2f f = {v, 0.0f};
    return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2bf));
}

// Cosine and sine of pos * freq.  The angle in quarter turns and its reduction to [-1/2, 1/2] are fp64: a position of 2^31 leaves an angle that is off by
// 5e-7.  1.5 2^52 added puts the nearest whole number into the low bits.  The rest, at most an eighth of a turn, is fp32 (off by 5e-8); its sine and
// cosine are their Taylor series to z^9 and z^10, whose next terms are below 2e-9 there.  Where a wave has little else to do it is most of the instructions: with
// the library's function of any argument and a reduction to a turn before that to a quarter, us: 32760 x (1 + 1) heads of 128 14.6 instead of 11.7,
// 1560 x (12 + 12) rotated alone 4.6 instead of 4.1.
__device__ __forceinline__ float2 cos_sin(int pos, double freq)
{
    constexpr double MAGIC = 6755399441055744.0;
    const double quarters = (double)pos * freq * 0.63661977236758134;
    const double rounded = quarters + MAGIC;
    const float z = (float)(quarters - (rounded - MAGIC)) * 1.57079632679f, z2 = z * z;
    const unsigned k = (unsigned)__double_as_longlong(rounded);
    float s = fmaf(z2, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(z2, s, 8.3333333e-3f);
    s = fmaf(z2, s, -0.16666667f);
    s = fmaf(z * z2, s, z);
    float c = fmaf(z2, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(z2, c, -1.3888889e-3f);
    c = fmaf(z2, c, 4.1666667e-2f);
    c = fmaf(z2, c, -0.5f);
    c = fmaf(z2, c, 1.0f);
    const float x = k & 1 ? s : c, y = k & 1 ? c : s;
    return make_float2(__uint_as_float(__float_as_uint(x) ^ (((k + 1) << 30) & 0x80000000u)), __uint_as_float(__float_as_uint(y) ^ ((k << 30) & 0x80000000u)));
}
__device__ __forceinline__ int axis_of(const HeadArgs &a, int pair) { return pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2; }

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// What the kernel below has no room for: rows of more than 64 vectors under one norm, heads of more than 64 lanes (512 channels of which a part turns
// in halves).  A workgroup has a token's queries or its keys, a wave every fourth head, and the elements are loaded one by one, a second time after
// the norm is known (the caches hold them).
template <typename T>
__global__ __launch_bounds__(TPB) void heads_any_kernel(HeadArgs a)
{
    __shared__ float2 turn[MAX_D / 2];
    __shared__ float red[TPB / 64];
    const int m = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Tensor t = a.t[blockIdx.y];
    const T *x = reinterpret_cast<const T *>(t.x) + (size_t)m * t.ld;
    T *out = reinterpret_cast<T *>(t.out) + (size_t)m * t.ld_out;
    for (int i = threadIdx.x; i < a.pairs; i += TPB) turn[i] = cos_sin(a.pos[(size_t)m * a.ldpos + axis_of(a, i)], a.freq[i]);
    float scale = 1.0f;
    if (a.norm == QARVD_NORM_ROW) {
        float sum = 0.0f;
        for (int h = wave; h < t.heads; h += TPB / 64)
            for (int d = lane; d < a.D; d += 64) {
                const float v = widen1<T>(x[(size_t)h * t.hs + d]);
                sum = fmaf(v, v, sum);
            }
        sum = wave_sum(sum);
        if (lane == 0) red[wave] = sum;
    }
    __syncthreads();
    if (a.norm == QARVD_NORM_ROW) scale = rsqrtf((red[0] + red[1] + red[2] + red[3]) / (float)((int64_t)t.heads * a.D) + a.eps);
    for (int h = wave; h < t.heads; h += TPB / 64) {
        const T *xh = x + (size_t)h * t.hs;
        T *oh = out + (size_t)h * t.hs_out;
        const float *w = t.w ? t.w + (a.norm == QARVD_NORM_ROW ? (size_t)h * a.D : 0) : nullptr;
        if (a.norm == QARVD_NORM_HEAD) {
            float sum = 0.0f;
            for (int d = lane; d < a.D; d += 64) {
                const float v = widen1<T>(xh[d]);
                sum = fmaf(v, v, sum);
            }
            scale = rsqrtf(wave_sum(sum) / (float)a.D + a.eps);
        }
        auto normed = [&](int d) {
            const float v = widen1<T>(xh[d]);
            return a.norm == QARVD_NORM_NONE ? v : v * scale * (w ? w[d] : 1.0f);
        };
        for (int i = lane; i < a.pairs; i += 64) {           // a lane reads both elements of a pair before it writes either
            const int da = a.interleaved ? 2 * i : i, db = a.interleaved ? 2 * i + 1 : i + a.pairs;
            const float u = normed(da), v = normed(db);
            const float2 cs = turn[i];
            oh[da] = narrow1<T>(fmaf(u, cs.x, -(v * cs.y)));
            oh[db] = narrow1<T>(fmaf(u, cs.y, v * cs.x));
        }
        for (int d = 2 * a.pairs + lane; d < a.D; d += 64) oh[d] = narrow1<T>(normed(d));
    }
}

// Rows in registers.  A wave has a token and CH vectors of its queries or keys; a vector is 64 lanes of 8 channels, lph (a power of two)
// to a head, whole heads side by side.  All loads go out first, then lane i works out the angle of pair i, once for the
// token instead of once in every lane that needs it, and the wave reads them back from LDS in the order of its channels: a lane's four pairs
// are the same in every vector, so they stay in registers, like a head's weights.
//   interleaved  bf16: the lane's channels are 8 j .. 8 j + 7, its pairs 4 j .. 4 j + 3
//                fp32: channels 4 j .. and D/2 + 4 j .., so that neighbouring lanes' 16-byte pieces are neighbours in memory: 24 heads of 128
//                with a row's norm, 1560 tokens 12.9 -> 8.3 us, 4680 37.5 -> 22.7
//   HALF         channels 4 j .. and R/2 + 4 j .., the same pairs; lanes behind the rotary channels have 8 neighbours again
// WHOLE: every lane's pieces are whole and 16-byte aligned (HALF bf16: 8).  Otherwise they are loaded from any address, and the last lane of a
// head (HALF: also of its rotary channels) takes what there is one by one.
struct FastArgs {
    HeadArgs h;
    int32_t lph_log, hpv_log;      // lanes to a head, heads to a vector (log2)
    int32_t rotary_lanes;          // (HALF) lanes of a head that hold pairs
    int32_t lanes;                 // lanes of a head that hold channels
    int32_t nv[2], parts_q;        // vectors of a token's queries and keys; how many waves share the queries
    int32_t tokens_log[2];         // (TOKENS) tokens to a wave (log2)
    int32_t pairs_log;             // (TOKENS) room for a token's angles (log2)
    int32_t write_through;         // how the outputs leave (see stores_through)
    float inv_n[2];                // 1 / (channels under a norm)
};
typedef float v4 __attribute__((ext_vector_type(4)));
typedef float v4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));

// Four neighbouring channels as they lie in memory, and the same at any element's address (one instruction whatever the alignment).
template <typename T> struct Four;
template <> struct Four<float> {
    typedef v4 raw;
    typedef v4_any raw_any;
    static __device__ __forceinline__ raw of(const float (&e)[4]) { return v4{e[0], e[1], e[2], e[3]}; }
    static __device__ __forceinline__ float get(raw r, int k) { return r[k]; }
    static __device__ __forceinline__ raw pack(const float *f) { return v4{f[0], f[1], f[2], f[3]}; }
};
template <> struct Four<uint16_t> {
    typedef u2 raw;
    typedef uint32_t raw_any __attribute__((ext_vector_type(2), aligned(2)));
    static __device__ __forceinline__ raw of(const uint16_t (&e)[4]) { return u2{e[0] | ((uint32_t)e[1] << 16), e[2] | ((uint32_t)e[3] << 16)}; }
    static __device__ __forceinline__ float get(raw r, int k) { return __uint_as_float(k & 1 ? r[k >> 1] & 0xFFFF0000u : r[k >> 1] << 16); }
    static __device__ __forceinline__ uint32_t pack2(float x, float y)
    {
        typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
        typedef float v2f __attribute__((ext_vector_type(2)));
        const v2f f = {x, y};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2bf));
    }
    static __device__ __forceinline__ raw pack(const float *f) { return u2{pack2(f[0], f[1]), pack2(f[2], f[3])}; }
};
// The first n of four elements at p, zeros behind.
template <typename T> __device__ __forceinline__ typename Four<T>::raw load_some(const T *p, int n)
{
    if (n == 4) return *reinterpret_cast<const typename Four<T>::raw_any *>(p);
    T e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = k < n ? p[k] : (T)0;
    return Four<T>::of(e);
}
template <typename T> __device__ __forceinline__ void store_some(T *p, int n, typename Four<T>::raw r)
{
    if (n == 4) {
        *reinterpret_cast<typename Four<T>::raw_any *>(p) = r;
        return;
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
        if (k < n) {
            if constexpr (sizeof(T) == 4) p[k] = r[k];
            else p[k] = (T)(r[k >> 1] >> (16 * (k & 1)));
        }
}

// A piece to out + off (bytes), written through the L2 (sc0 sc1); out is the same in all lanes.
template <typename P> __device__ __forceinline__ void store_through(void *out, int off, P piece)
{
#if defined(__HIP_DEVICE_COMPILE__)
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(out, 0, 0x7fffffff, 0x00020000);
    if constexpr (sizeof(P) == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, piece), r, off, 0, 17);
    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, piece), r, off, 0, 17);
#else
    (void)out; (void)off; (void)piece;
#endif
}

// Sums over groups of 2^log neighbouring lanes, in every lane of the group, of several values at once (`log` is uniform).
template <int CH> __device__ __forceinline__ void group_sum(float (&v)[CH], int log)
{
    auto all = [&](auto move) {
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] += __int_as_float(move(__float_as_int(v[c])));
    };
    if (log > 0) all([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false); });       // quad_perm 1,0,3,2
    if (log > 1) all([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, false); });       // quad_perm 2,3,0,1
    if (log > 2) all([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, false); });      // mirrored in 8: the other four
    if (log > 3) all([](int x) { return __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, false); });      // mirrored in 16: the other eight
    if (log > 4) all([](int x) { return __shfl_xor(x, 16, 64); });
    if (log > 5) all([](int x) { return __shfl_xor(x, 32, 64); });
}

// SPLIT (the norm of a row of several waves): a workgroup has one token's queries or its keys; its waves share the angles and add up their sums.
// Against one wave that holds the whole row, us for 80 heads of 128 bf16: one token 7.2 -> 3.4, 1560 18.0 -> 13.4, 4680 53.5 -> 44.7.
// TOKENS (few heads, many tokens): the wave's one vector has 2^tokens_log tokens side by side, each with its heads.
constexpr int MOST_WAVES = 16, MOST_VECTORS = 64;
enum Mode { PLAIN, SPLIT_ROW, SEVERAL_TOKENS };
template <typename T, int CH, bool HALF, int NORM, bool WHOLE, Mode MODE>
__global__ __launch_bounds__(MODE == SPLIT_ROW ? 64 * MOST_WAVES : TPB) void heads_kernel(FastArgs f)
{
    constexpr bool SPLIT = MODE == SPLIT_ROW, TOKENS = MODE == SEVERAL_TOKENS;
    typedef typename Four<T>::raw raw;
    constexpr bool WIDE = WHOLE && !HALF && sizeof(T) == 2;         // the eight channels are one 16-byte piece
    constexpr bool APART = !HALF && sizeof(T) == 4;
    __shared__ __align__(16) float turns[SPLIT ? 1 : TPB / 64][MAX_D];
    __shared__ float red[SPLIT ? MOST_VECTORS : 1];
    const HeadArgs &a = f.h;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool keys = (int)blockIdx.y >= f.parts_q;
    const Tensor &t = a.t[keys];
    const int tokens_log = TOKENS ? f.tokens_log[keys] : 0;
    if (SPLIT ? false : ((int64_t)(blockIdx.x * (TPB / 64) + wave) << tokens_log) >= a.M) return;
    const int m = SPLIT ? blockIdx.x : (blockIdx.x * (TPB / 64) + wave) << tokens_log;       // (the wave's first token)
    const int first = (SPLIT ? wave : (int)blockIdx.y - (keys ? f.parts_q : 0)) * CH;     // vector
    const int heads_log = f.hpv_log - tokens_log;
    const int j = lane & ((1 << f.lph_log) - 1), sub = (lane >> f.lph_log) & ((1 << heads_log) - 1);
    const int token = TOKENS ? lane >> (f.lph_log + heads_log) : 0;
    const bool rotary = 4 * j < a.pairs;
    const int rest = HALF ? 2 * a.pairs + 8 * (j - f.rotary_lanes) : 8 * j;       // first channel of a lane with eight neighbours
    const int c0 = APART || (HALF && rotary) ? 4 * j : rest, apart = APART ? 4 * f.lanes : HALF && rotary ? a.pairs : 4;
    auto some = [](int left) { return min(max(left, 0), 4); };
    int n0 = some(a.D - rest), n1 = some(a.D - rest - 4);
    if (HALF && rotary) n0 = n1 = some(a.pairs - 4 * j);
    if (APART) {
        n0 = some(min(a.D, apart) - c0);
        n1 = some(a.D - apart - c0);
    }
    const bool inside = n0 > 0 && (!TOKENS || (unsigned)(m + token) < (unsigned)a.M);
    auto pair = [&](int k) { return APART ? 2 * j + (k & 1) + (k & 2) * f.lanes : 4 * j + k; };       // of the lane's four

    const T *x = reinterpret_cast<const T *>(t.x) + (size_t)m * t.ld + c0;
    if (TOKENS) x += token * t.ld;
    raw v[CH][2];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        v[c][0] = v[c][1] = raw{};
        const int head = ((first + c) << f.hpv_log) + sub;
        if (inside && head < t.heads) {
            const T *p = x + (size_t)head * t.hs;
            if constexpr (WIDE) {
                const u4 r = *reinterpret_cast<const u4 *>(p);
                v[c][0] = raw{r.x, r.y};
                v[c][1] = raw{r.z, r.w};
            } else if constexpr (WHOLE) {
                v[c][0] = *reinterpret_cast<const raw *>(p);
                v[c][1] = *reinterpret_cast<const raw *>(p + apart);
            } else {
                v[c][0] = load_some<T>(p, n0);
                v[c][1] = load_some<T>(p + apart, n1);
            }
        }
    }

    float w[8];
    auto load_weights = [&](const float *p) {
        const v4 w0 = WHOLE ? (v4) * reinterpret_cast<const v4_any *>(p) : load_some<float>(p, n0);
        const v4 w1 = WHOLE ? (v4) * reinterpret_cast<const v4_any *>(p + apart) : load_some<float>(p + apart, n1);
#pragma unroll
        for (int k = 0; k < 4; ++k) { w[k] = w0[k]; w[4 + k] = w1[k]; }
    };
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = 1.0f;
    if (NORM == QARVD_NORM_HEAD && t.w && inside) load_weights(t.w + c0);

    float *const mine = turns[SPLIT ? 0 : wave];
    if (TOKENS && a.pairs) {
        for (int i = lane; i < 1 << (tokens_log + f.pairs_log); i += 64) {
            const int p = i & ((1 << f.pairs_log) - 1), at = (int)min((unsigned)(m + (i >> f.pairs_log)), (unsigned)a.M - 1);
            if (p >= a.pairs) continue;
            const float2 cs = cos_sin(a.pos[(size_t)at * a.ldpos + axis_of(a, p)], a.freq[p]);
            mine[i] = cs.x;
            mine[MAX_D / 2 + i] = cs.y;
        }
    } else if (a.pairs) {
        const int32_t *pos = a.pos + (size_t)m * a.ldpos;
        for (int i = SPLIT ? threadIdx.x : lane; i < a.pairs; i += SPLIT ? blockDim.x : 64) {
            const float2 cs = cos_sin(pos[axis_of(a, i)], a.freq[i]);
            mine[i] = cs.x;
            mine[MAX_D / 2 + i] = cs.y;
        }
    }

    float scale[CH];
    if constexpr (NORM != QARVD_NORM_NONE) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            scale[c] = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float e = Four<T>::get(v[c][k >> 2], k & 3);
                scale[c] = fmaf(e, e, scale[c]);
            }
        }
        if constexpr (NORM == QARVD_NORM_ROW) {
            // a sum for each vector, and those in an order of their numbers: the same bits however many tokens there are and waves share the row
            group_sum<CH>(scale, 6 - tokens_log);
            float sum[1] = {scale[0]};
            if constexpr (SPLIT) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    if (lane == 0) red[first + c] = scale[c];
                __syncthreads();
                sum[0] = lane < CH * ((int)blockDim.x >> 6) ? red[lane] : 0.0f;
                group_sum<1>(sum, 6);
            } else if constexpr (CH > 1) {
                sum[0] += scale[1];
                if constexpr (CH == 3) sum[0] += scale[2];
                if constexpr (CH == 4) sum[0] += scale[2] + scale[3];
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) scale[c] = sum[0];
        } else {
            group_sum<CH>(scale, f.lph_log);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) scale[c] = rsqrtf(fmaf(scale[c], f.inv_n[keys], a.eps));
    }

    float co[4], si[4];
    if (a.pairs) {
        if (!SPLIT) __builtin_amdgcn_wave_barrier();       // (one wave's LDS accesses complete in order)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = TOKENS ? (token << f.pairs_log) + (pair(k) & ((1 << f.pairs_log) - 1)) : pair(k);
            co[k] = mine[p];
            si[k] = mine[MAX_D / 2 + p];
        }
    }

    T *const out = reinterpret_cast<T *>(t.out) + (size_t)m * t.ld_out;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int head = ((first + c) << f.hpv_log) + sub;
        if (!inside || head >= t.heads) continue;
        float e[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) e[k] = Four<T>::get(v[c][k >> 2], k & 3);
        if constexpr (NORM != QARVD_NORM_NONE) {
            if (NORM == QARVD_NORM_ROW && t.w) load_weights(t.w + (size_t)head * a.D + c0);
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = e[k] * scale[c] * w[k];
        }
        if (a.pairs) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int p = HALF ? k : 2 * k, q = HALF ? 4 + k : 2 * k + 1;
                const float u = e[p], z = e[q];
                const float up = fmaf(u, co[k], -(z * si[k])), zp = fmaf(u, si[k], z * co[k]);
                const bool turn = pair(k) < a.pairs;     // (selected, not multiplied by 1 and 0: the rest may be infinite)
                e[p] = turn ? up : u;
                e[q] = turn ? zp : z;
            }
        }
        const int64_t at = (TOKENS ? token * t.ld_out : 0) + (int64_t)head * t.hs_out + c0;      // from the (first) token's first element
        const raw lo = Four<T>::pack(e), hi = Four<T>::pack(e + 4);
        if constexpr (!WHOLE) {
            store_some<T>(out + at, n0, lo);
            store_some<T>(out + at + apart, n1, hi);
        } else {
            auto put = [&](int k, auto piece) {
                if (f.write_through) store_through(out, (int)(at + k) * (int)sizeof(T), piece);
                else __builtin_nontemporal_store(piece, reinterpret_cast<decltype(piece) *>(out + at + k));
            };
            if constexpr (WIDE) {
                put(0, u4{lo.x, lo.y, hi.x, hi.y});
            } else {
                put(0, lo);
                put(apart, hi);
            }
        }
    }
}

int ceil_log2(int n)
{
    int l = 0;
    while ((1 << l) < n) ++l;
    return l;
}

template <typename T, bool HALF, int NORM, bool WHOLE> void launch_fast(const FastArgs &f, int ch, int waves, hipStream_t st)
{
    auto go = [&](auto n) {
        constexpr int CH = decltype(n)::value;
        if constexpr (NORM == QARVD_NORM_ROW)
            if (waves > 1) {
                hipLaunchKernelGGL((heads_kernel<T, CH, HALF, NORM, WHOLE, SPLIT_ROW>), dim3(f.h.M, f.nv[1] ? 2 : 1), dim3(64 * waves), 0, st, f);
                return;
            }
        const int per = (TPB / 64) << (f.nv[1] ? std::min(f.tokens_log[0], f.tokens_log[1]) : f.tokens_log[0]);
        const dim3 grid((unsigned)(((int64_t)f.h.M + per - 1) / per), f.parts_q + (f.nv[1] + ch - 1) / ch);
        if constexpr (CH == 1 || sizeof(T) == 2)
            if (f.tokens_log[0] + f.tokens_log[1] > 0) {
                hipLaunchKernelGGL((heads_kernel<T, CH, HALF, NORM, WHOLE, SEVERAL_TOKENS>), grid, dim3(TPB), 0, st, f);
                return;
            }
        hipLaunchKernelGGL((heads_kernel<T, CH, HALF, NORM, WHOLE, PLAIN>), grid, dim3(TPB), 0, st, f);
    };
    switch (ch) {
    case 1: return go(std::integral_constant<int, 1>{});
    case 2: return go(std::integral_constant<int, 2>{});
    case 3: return go(std::integral_constant<int, 3>{});
    default: return go(std::integral_constant<int, 4>{});
    }
}

// Vectors to a wave: as few as leave every SIMD some waves, since a wave works out its token's angles whatever it has, and at most four.  us for 1, 2, 3, 4
// and 6: 4680 x 24 heads of 128 bf16 14.3, 13.9, 12.3, 12.3, 12.3; 1560 x 24 5.97, 5.60, 5.60, 5.63, 5.66; 520 x 80 fp32 8.98, 8.77, 8.73, 9.05, 9.47;
// 64 x 24 2.71, 2.87, 3.10, 3.12, 3.12; one token 2.41, 2.55, 2.82, 2.81, 2.81.
constexpr int64_t WAVES = 4096;
// Where a tensor's heads leave room in their one vector, as many tokens in it as leave this many waves (a wave works out its tokens' angles one after
// another).  us for 512, 1024, 2048 waves and one token each: 4680 x (1 + 1) heads of 32 bf16 3.3, 3.3, 4.1, 5.2; 1560 of them 3.0, 3.5, 3.5, 3.5; 4680 x
// (1 + 1) of 128 4.8, 4.8, 4.6, 5.2; 32760 x (2 + 2) of 64 10.1, 10.2, 10.0, 20.9; with all that fit, 520 x (1 + 1) of 128 3.8 instead of 2.9.  bf16
// keys of few heads also beside queries of up to four vectors: 32760 x (12 + 1) of 128 49.3 -> 45.3, 4680 8.0 -> 8.1 (fp32 79.9 -> 78.2, 10.8 -> 11.4: not built).
constexpr int TOKEN_WAVES = 1024;

// Stores that write through the L2, or such with the non-temporal hint.  Nothing is left to write back when the kernel ends with either; written
// through, the last-level cache (256 MB) still has the outputs for attention.  us plain, through, non-temporal, and the same with a copy of the
// outputs behind it:  4680 x 24 heads of 128 bf16 (58 MB in and out) 12.3, 11.1, 11.1 | 24.0, 22.3, 25.7;  1560 x 24 (19 MB) 5.9, 4.8, 4.8 | 13.9, 13.0, 14.1;
// 32760 x 24 (403 MB), more than that cache holds, 79.8, 79.8, 73.8 | 157.6, 157.3, 156.4.
int32_t stores_through(const HeadArgs &a, size_t esz)
{
    size_t bytes = 0;
    for (const Tensor &t : a.t) {
        bytes += 2 * (size_t)a.M * t.heads * a.D * esz;
        // (32-bit offsets from a wave's first token)
        if (((t.heads > 1 ? (t.heads - 1) * t.hs_out : 0) + (a.M > 1 ? 63 * t.ld_out : 0)) * (int64_t)esz > 0x7f000000) return 0;
    }
    return bytes <= ((size_t)256 << 20) ? 1 : 0;
}

bool pieces_ok(const Tensor &t, int32_t M, size_t esz)
{
    const int64_t per = 16 / (int64_t)esz;
    return t.heads == 0 || (qarvd_aligned16(t.x) && qarvd_aligned16(t.out) && (M == 1 || (t.ld % per == 0 && t.ld_out % per == 0)) &&
                            (t.heads == 1 || (t.hs % per == 0 && t.hs_out % per == 0)));
}

template <typename T> qarvd_status launch(const HeadArgs &a, hipStream_t st)
{
    const bool half = a.pairs > 0 && !a.interleaved;
    const bool whole = a.D % 8 == 0 && !(half && a.pairs % 4) && pieces_ok(a.t[0], a.M, sizeof(T)) && pieces_ok(a.t[1], a.M, sizeof(T));
    FastArgs f;
    f.h = a;
    f.rotary_lanes = half ? (a.pairs + 3) / 4 : 0;
    f.lanes = f.rotary_lanes + ((half ? a.D - 2 * a.pairs : a.D) + 7) / 8;
    if (f.lanes <= 64) {
        f.lph_log = ceil_log2(f.lanes);
        f.hpv_log = 6 - f.lph_log;
        for (int i = 0; i < 2; ++i) {
            f.nv[i] = (a.t[i].heads + (1 << f.hpv_log) - 1) >> f.hpv_log;
            f.inv_n[i] = 1.0f / (float)(a.norm == QARVD_NORM_ROW ? (int64_t)a.t[i].heads * a.D : (int64_t)a.D);
        }
        const int most = f.nv[0] > f.nv[1] ? f.nv[0] : f.nv[1];
        for (int i = 0; i < 2; ++i) {
            f.tokens_log[i] = f.nv[i] == 1 && (most == 1 || (sizeof(T) == 2 && most <= 4)) ? f.hpv_log - ceil_log2(a.t[i].heads) : 0;
            while (f.tokens_log[i] && a.M >> f.tokens_log[i] < TOKEN_WAVES) --f.tokens_log[i];
        }
        f.pairs_log = ceil_log2(a.pairs);
        const int64_t vectors = (int64_t)a.M * (f.nv[0] + f.nv[1]);
        const int want = vectors >= 4 * WAVES ? 4 : vectors >= 2 * WAVES ? (int)(vectors / WAVES) : 1;
        const bool row = a.norm == QARVD_NORM_ROW;
        int waves = (most + want - 1) / want;
        if (row && waves > MOST_WAVES) waves = (most + 3) / 4;
        const int ch = (most + waves - 1) / waves;       // evenly
        f.write_through = stores_through(a, sizeof(T));
        if (!row || waves <= MOST_WAVES) {
            f.parts_q = row ? 1 : (f.nv[0] + ch - 1) / ch;
            auto as = [&](auto norm) {
                constexpr int N = decltype(norm)::value;
                if (whole) return half ? launch_fast<T, true, N, true>(f, ch, waves, st) : launch_fast<T, false, N, true>(f, ch, waves, st);
                return half ? launch_fast<T, true, N, false>(f, ch, waves, st) : launch_fast<T, false, N, false>(f, ch, waves, st);
            };
            if (a.norm == QARVD_NORM_NONE) as(std::integral_constant<int, QARVD_NORM_NONE>{});
            else if (row) as(std::integral_constant<int, QARVD_NORM_ROW>{});
            else as(std::integral_constant<int, QARVD_NORM_HEAD>{});
            return qarvd_launch_status();
        }
    }
    hipLaunchKernelGGL((heads_any_kernel<T>), dim3(a.M, a.t[1].heads > 0 ? 2 : 1), dim3(TPB), 0, st, a);
    return qarvd_launch_status();
}

// Tokens of one launch.  It has fewer than 2^32 work-items along x (of a count beyond, only the rest modulo 2^32 would run), and a token has at most
// 1024 of them.
constexpr int64_t MOST_TOKENS = 1 << 21;

// One tensor's pointers and strides.  The strides of a single token or a single head say nothing; otherwise the elements must not overlap:
// a token's heads lie between it and the next, or a head's tokens between it and the next head.
qarvd_status check_tensor(const qarvd_heads *h, size_t esz, int32_t M, int32_t D)
{
    if (!h->x || !h->out || h->heads <= 0) return QARVD_ERR_INVALID_ARG;
    const int64_t lds[2] = {h->ld, h->ld_out}, hss[2] = {h->head_stride, h->head_stride_out};
    for (int i = 0; i < 2; ++i) {
        const bool tokens = M > 1, heads = h->heads > 1;
        if ((tokens && lds[i] < D) || (heads && hss[i] < D)) return QARVD_ERR_INVALID_ARG;
        const int64_t most = (int64_t)1 << 40;
        if ((tokens && lds[i] > most) || (heads && hss[i] > most)) return QARVD_ERR_INVALID_ARG;
        if (tokens && heads && (lds[i] - D) / hss[i] < h->heads - 1 && (hss[i] - D) / lds[i] < M - 1) return QARVD_ERR_INVALID_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(h->x) | reinterpret_cast<uintptr_t>(h->out)) % esz || (reinterpret_cast<uintptr_t>(h->weight) & 3u))
        return QARVD_ERR_UNSUPPORTED;
    return QARVD_OK;
}

}  // namespace

qarvd_status qarvd_heads_check(const qarvd_heads *q, const qarvd_heads *k, qarvd_dtype dt, int32_t M, int32_t D, qarvd_norm norm, float eps,
                               const qarvd_rope *rope)
{
    if (!q || M <= 0 || D <= 0 || !(eps >= 0.0f) || !(eps <= 3.4e38f)) return QARVD_ERR_INVALID_ARG;
    if (norm != QARVD_NORM_NONE && norm != QARVD_NORM_HEAD && norm != QARVD_NORM_ROW) return QARVD_ERR_INVALID_ARG;
    if (dt != QARVD_F32 && dt != QARVD_BF16) return QARVD_ERR_UNSUPPORTED;
    if (D > MAX_D) return QARVD_ERR_UNSUPPORTED;
    const size_t esz = dt == QARVD_F32 ? 4 : 2;
    if (qarvd_status s = check_tensor(q, esz, M, D); s != QARVD_OK) return s;
    if (k)
        if (qarvd_status s = check_tensor(k, esz, M, D); s != QARVD_OK) return s;
    if (rope) {
        if (!rope->pos || !rope->freq || rope->n_axes < 1 || rope->n_axes > 3 || (M > 1 && rope->ldpos < rope->n_axes)) return QARVD_ERR_INVALID_ARG;
        int64_t R = 0;
        for (int i = 0; i < rope->n_axes; ++i) {
            if (rope->axis_dims[i] <= 0 || rope->axis_dims[i] % 2) return QARVD_ERR_INVALID_ARG;
            R += rope->axis_dims[i];
        }
        if (R > D || (rope->interleaved != 0 && rope->interleaved != 1)) return QARVD_ERR_INVALID_ARG;
        if ((reinterpret_cast<uintptr_t>(rope->pos) & 3u) || (reinterpret_cast<uintptr_t>(rope->freq) & 7u)) return QARVD_ERR_UNSUPPORTED;
    }
    return QARVD_OK;
}

extern "C" qarvd_status qarvd_qk_norm_rope(const qarvd_heads *q, const qarvd_heads *k, qarvd_dtype dt, int32_t M, int32_t D, qarvd_norm norm,
                                           float eps, const qarvd_rope *rope, void *stream)
{
    if (qarvd_status s = qarvd_heads_check(q, k, dt, M, D, norm, eps, rope); s != QARVD_OK) return s;
    HeadArgs a = {};
    for (int i = 0; i < (k ? 2 : 1); ++i) {
        const qarvd_heads *h = i ? k : q;
        a.t[i] = Tensor{h->x, h->out, h->weight, h->ld, h->head_stride, h->ld_out, h->head_stride_out, h->heads};
    }
    a.eps = eps; a.D = D; a.norm = (int32_t)norm;
    if (rope) {
        a.pos = rope->pos; a.ldpos = rope->ldpos; a.freq = rope->freq; a.interleaved = rope->interleaved;
        a.end0 = rope->axis_dims[0] / 2;
        a.end1 = a.end0 + (rope->n_axes > 1 ? rope->axis_dims[1] / 2 : 0);
        a.pairs = a.end1 + (rope->n_axes > 2 ? rope->axis_dims[2] / 2 : 0);
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const int64_t esz = dt == QARVD_F32 ? 4 : 2;
    for (int64_t left = M;;) {
        a.M = (int32_t)std::min(left, MOST_TOKENS);
        if (qarvd_status s = dt == QARVD_F32 ? launch<float>(a, st) : launch<uint16_t>(a, st); s != QARVD_OK) return s;
        left -= a.M;
        if (left == 0) return QARVD_OK;
        for (Tensor &t : a.t) {
            if (!t.heads) continue;
            t.x = reinterpret_cast<const char *>(t.x) + MOST_TOKENS * t.ld * esz;
            t.out = reinterpret_cast<char *>(t.out) + MOST_TOKENS * t.ld_out * esz;
        }
        if (a.pos) a.pos += MOST_TOKENS * a.ldpos;
    }
}
