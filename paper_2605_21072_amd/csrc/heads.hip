// Norm of queries and keys and their rotation by position (time, height, width), one pass over both.
//
//     r = 1 / sqrt(mean(x^2) + eps);   x <- x r w;   (a, b) <- (a cos t - b sin t, a sin t + b cos t),   t = pos[axis(i)] freq[i]
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

// Cosine and sine of pos * freq.  The product and its reduction to [-1/2, 1/2] turns are fp64: a position of 2^31 leaves an angle that is off by
// 4e-7.  What remains is split into a whole number of quarter turns and a rest of at most an eighth, which fp32 holds to 2e-8.
__device__ __forceinline__ float2 cos_sin(int pos, double freq)
{
    double t = (double)pos * freq * 0.15915494309189535;
    t -= rint(t);
    const double quarters = rint(4.0 * t);
    const float rest = (float)(4.0 * t - quarters);
    float s, c;
    sincospif(0.5f * rest, &s, &c);
    const int k = (int)quarters & 3;
    const float x = k & 1 ? s : c, y = k & 1 ? c : s;
    return make_float2(k == 1 || k == 2 ? -x : x, k >= 2 ? -y : y);
}
__device__ __forceinline__ int axis_of(const HeadArgs &a, int pair) { return pair < a.end0 ? 0 : pair < a.end1 ? 1 : 2; }

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Any head size, stride and alignment: a workgroup has a token's queries or its keys, a wave every fourth head, and the elements
// are loaded one by one, a second time after the norm is known (the caches hold them).
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

template <typename T> qarvd_status launch(const HeadArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL((heads_any_kernel<T>), dim3(a.M, a.t[1].heads > 0 ? 2 : 1), dim3(TPB), 0, st, a);
    return qarvd_launch_status();
}

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
    a.eps = eps; a.M = M; a.D = D; a.norm = (int32_t)norm;
    if (rope) {
        a.pos = rope->pos; a.ldpos = rope->ldpos; a.freq = rope->freq; a.interleaved = rope->interleaved;
        a.end0 = rope->axis_dims[0] / 2;
        a.end1 = a.end0 + (rope->n_axes > 1 ? rope->axis_dims[1] / 2 : 0);
        a.pairs = a.end1 + (rope->n_axes > 2 ? rope->axis_dims[2] / 2 : 0);
    }
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return dt == QARVD_F32 ? launch<float>(a, st) : launch<uint16_t>(a, st);
}
