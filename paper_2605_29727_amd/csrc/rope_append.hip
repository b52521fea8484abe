// Rotary positions and the append to the KV cache (gfx950): the queries and keys of new rows are rotated at their positions, the keys and
// the values written to their slots of the cache, in its own type, in one pass over the projections' output.
//
// A pair (a, b) of channels turns by t = position * inv_freq[i]:  a' = f (a cos t - b sin t), b' = f (a sin t + b cos t).  t is a number of
// thousands of turns at far positions, of which only the fraction counts: it is formed in fp64 in turns, reduced there, and only the fraction
// (of which fp32 keeps 2^-25) goes to the sine and cosine.  The rotation is in fp32; a result is rounded once, to the type it is stored in.
#include "btv_common.h"

#include <cmath>
#include <type_traits>

namespace {

struct RopeParams {
    const void *Q, *K, *V;
    long long q_stride, k_stride, v_stride;            // elements between rows
    const int32_t *position, *slot;
    const double *inv_freq;
    void *Qout, *Kc, *Vc;
    uint32_t *flag;
    long long num_slots;
    int total, Hq, Hkv, R, interleaved;
    float factor, inv_k, inv_v;                        // E4M3 caches: 1 / scale
};

// The simplest form: a thread per (row, head, pair of channels) and per (row, head, channel) that is not rotated.
template <typename T> __device__ __forceinline__ float load1(const void *p, long long i) { return (float)static_cast<const T *>(p)[i]; }
template <typename T> __device__ __forceinline__ void store1(void *p, long long i, float x)
{
    if constexpr (std::is_same_v<T, uint8_t>) {
        x = x > 448.f ? 448.f : x < -448.f ? -448.f : x;
        static_cast<uint8_t *>(p)[i] = (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xFF);
    } else {
        static_cast<T *>(p)[i] = (T)x;
    }
}

template <typename T, typename C, int D>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeParams p)
{
    const int row = blockIdx.x, heads = p.Hq + 2 * p.Hkv;
    const int slot = p.slot[row];
    const bool stored = slot >= 0 && slot < p.num_slots;
    if (slot >= p.num_slots && threadIdx.x == 0 && p.flag) atomicOr(p.flag, 32u);
    const double pos = (double)p.position[row];
    for (int e = threadIdx.x; e < heads * (D / 2); e += 256) {
        const int head = e / (D / 2), i = e % (D / 2);
        const bool isq = head < p.Hq, isv = head >= p.Hq + p.Hkv;
        const int h = isq ? head : isv ? head - p.Hq - p.Hkv : head - p.Hq;
        if (!isq && !stored) continue;
        const void *src = isq ? p.Q : isv ? p.V : p.K;
        const long long from = (isq ? p.q_stride : isv ? p.v_stride : p.k_stride) * row + (long long)h * D;
        const bool rotated = !isv && i < p.R / 2;
        int a, b;                                      // (channels past the first R and values: two neighbours of what is left)
        if (rotated) { a = p.interleaved ? 2 * i : i; b = p.interleaved ? 2 * i + 1 : i + p.R / 2; }
        else { a = 2 * i; b = 2 * i + 1; }
        float x = load1<T>(src, from + a), y = load1<T>(src, from + b);
        if (rotated) {
            double turns = pos * (p.inv_freq[i] * 0.15915494309189533577);
            turns -= rint(turns);
            float s, c;
            sincospif(2.0f * (float)turns, &s, &c);
            s *= p.factor; c *= p.factor;
            const float u = x * c - y * s;
            y = x * s + y * c;
            x = u;
        }
        if (isq) {
            const long long to = ((long long)row * p.Hq + h) * D;
            store1<T>(p.Qout, to + a, x); store1<T>(p.Qout, to + b, y);
        } else {
            const long long to = ((long long)slot * p.Hkv + h) * D;
            const float f = std::is_same_v<C, uint8_t> ? isv ? p.inv_v : p.inv_k : 1.0f;
            void *cache = isv ? p.Vc : p.Kc;
            store1<C>(cache, to + a, x * f); store1<C>(cache, to + b, y * f);
        }
    }
}

int rope_append(RopeParams p, int dtype, int eb, int D, void *stream)
{
    BTV_REQUIRE(dtype == BTV_F32 || dtype == BTV_BF16, "dtype=%d unsupported", dtype);
    BTV_REQUIRE(p.total >= 0, "total=%d out of range", p.total);
    BTV_REQUIRE(p.Hq >= 1 && p.Hkv >= 1 && p.Hq <= 1024 && p.Hkv <= 1024, "bad heads Hq=%d Hkv=%d", p.Hq, p.Hkv);
    BTV_REQUIRE(D == 64 || D == 128, "D=%d not in {64,128}", D);
    BTV_REQUIRE(p.R >= 0 && p.R <= D && p.R % 16 == 0, "R=%d: a multiple of 16 up to D=%d", p.R, D);
    BTV_REQUIRE(p.interleaved == 0 || p.interleaved == 1, "interleaved=%d: 0 or 1", p.interleaved);
    BTV_REQUIRE(std::isfinite(p.factor), "the factor must be finite");
    BTV_REQUIRE(p.num_slots >= 1 && p.num_slots <= INT32_MAX, "num_slots=%lld out of range", p.num_slots);
    if (p.total == 0) return BTV_OK;
    BTV_REQUIRE(p.Q && p.K && p.V && p.position && p.slot && p.Qout && p.Kc && p.Vc && (p.inv_freq || p.R == 0), "null pointer");
    const int per16 = dtype == BTV_F32 ? 4 : 8;
    BTV_REQUIRE(btv_aligned16(p.Q) && btv_aligned16(p.K) && btv_aligned16(p.V) && btv_aligned16(p.Qout) && btv_aligned16(p.Kc) && btv_aligned16(p.Vc),
                "Q, K, V, Qout and the caches must be 16-byte aligned");
    BTV_REQUIRE((reinterpret_cast<uintptr_t>(p.inv_freq) & 7u) == 0, "inv_freq must be 8-byte aligned");
    BTV_REQUIRE(p.q_stride % per16 == 0 && p.k_stride % per16 == 0 && p.v_stride % per16 == 0, "rows must be multiples of 16 bytes apart");
    BTV_REQUIRE(p.total == 1 || (p.q_stride >= (long long)p.Hq * D && p.k_stride >= (long long)p.Hkv * D && p.v_stride >= (long long)p.Hkv * D), "rows overlap");
    BTV_REQUIRE(p.Qout != p.Q || p.total == 1 || p.q_stride == (long long)p.Hq * D, "Qout may be Q only where its rows follow each other");
    const dim3 grid(p.total);
    hipStream_t st = static_cast<hipStream_t>(stream);
#define BTV_CASE(DT, EB, DD, T, C)                                                                       \
    if (dtype == DT && eb == EB && D == DD) {                                                            \
        hipLaunchKernelGGL((rope_append_kernel<T, C, DD>), grid, dim3(256), 0, st, p);                   \
        BTV_HIP(hipGetLastError());                                                                      \
        return BTV_OK;                                                                                   \
    }
    BTV_CASE(BTV_F32, 4, 64, float, float) BTV_CASE(BTV_F32, 4, 128, float, float)
    BTV_CASE(BTV_BF16, 2, 64, __bf16, __bf16) BTV_CASE(BTV_BF16, 2, 128, __bf16, __bf16)
    BTV_CASE(BTV_BF16, 1, 128, __bf16, uint8_t)
    BTV_CASE(BTV_BF16, 1, 64, __bf16, uint8_t)
#undef BTV_CASE
    return btv_fail(BTV_EINVAL, "an E4M3 cache takes bfloat16 rows");
}

RopeParams params(const void *Q, long long q_stride, const void *K, long long k_stride, const void *V, long long v_stride, int total, int Hq, int Hkv,
                  const int32_t *position, const int32_t *slot, const double *inv_freq, int R, int interleaved, float factor, void *Qout, void *Kc,
                  void *Vc, long long num_slots, void *ws)
{
    RopeParams p = {};
    p.Q = Q; p.K = K; p.V = V; p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
    p.position = position; p.slot = slot; p.inv_freq = inv_freq; p.Qout = Qout; p.Kc = Kc; p.Vc = Vc;
    p.flag = static_cast<uint32_t *>(ws);
    p.num_slots = num_slots; p.total = total; p.Hq = Hq; p.Hkv = Hkv; p.R = R; p.interleaved = interleaved;
    p.factor = factor; p.inv_k = p.inv_v = 1.0f;
    return p;
}

}  // namespace

extern "C" {

int btv_rope_append(const void *Q, long long q_stride, const void *K, long long k_stride, const void *V, long long v_stride, int dtype, int total, int Hq,
                    int Hkv, int D, const int32_t *position, const int32_t *slot, const double *inv_freq, int R, int interleaved, float factor, void *Qout,
                    void *Kcache, void *Vcache, long long num_slots, void *ws, void *stream)
{
    return rope_append(params(Q, q_stride, K, k_stride, V, v_stride, total, Hq, Hkv, position, slot, inv_freq, R, interleaved, factor, Qout, Kcache, Vcache,
                              num_slots, ws), dtype, dtype == BTV_F32 ? 4 : 2, D, stream);
}

int btv_rope_append_fp8kv(const void *Q, long long q_stride, const void *K, long long k_stride, const void *V, long long v_stride, int total, int Hq, int Hkv,
                          int D, const int32_t *position, const int32_t *slot, const double *inv_freq, int R, int interleaved, float factor, void *Qout,
                          void *K8cache, void *V8cache, float k_scale, float v_scale, long long num_slots, void *ws, void *stream)
{
    // (their reciprocals have to be numbers as well)
    BTV_REQUIRE(k_scale >= 1e-37f && k_scale <= 1e37f && v_scale >= 1e-37f && v_scale <= 1e37f, "FP8 K/V scales must lie in [1e-37, 1e37]");
    RopeParams p = params(Q, q_stride, K, k_stride, V, v_stride, total, Hq, Hkv, position, slot, inv_freq, R, interleaved, factor, Qout, K8cache, V8cache,
                          num_slots, ws);
    p.inv_k = 1.0f / k_scale; p.inv_v = 1.0f / v_scale;
    return rope_append(p, BTV_BF16, 1, D, stream);
}

int btv_rope_frequencies(int R, double theta, int scaling, double stretch, double original, double low, double high, double *inv_freq, double *factor)
{
    BTV_REQUIRE(inv_freq && factor, "null pointer");
    BTV_REQUIRE(R >= 2 && R % 2 == 0 && R <= 4096, "R=%d: an even number in [2,4096]", R);
    BTV_REQUIRE(std::isfinite(theta) && theta > 0.0, "theta must be positive and finite");
    BTV_REQUIRE(scaling >= BTV_ROPE_PLAIN && scaling <= BTV_ROPE_YARN, "scaling=%d unknown", scaling);
    if (scaling != BTV_ROPE_PLAIN) BTV_REQUIRE(std::isfinite(stretch) && stretch >= 1.0, "the stretch must be at least 1");
    const bool parts = scaling == BTV_ROPE_PARTS || scaling == BTV_ROPE_YARN;
    if (parts) {
        BTV_REQUIRE(std::isfinite(original) && original > 0.0, "the original length must be positive and finite");
        BTV_REQUIRE(std::isfinite(low) && std::isfinite(high) && low >= 0.0 && low < high, "0 <= low < high turns");
    }
    if (scaling == BTV_ROPE_NTK) {
        BTV_REQUIRE(R > 2, "R=%d: more than one pair", R);
        theta *= std::pow(stretch, (double)R / (R - 2));
    }
    for (int i = 0; i < R / 2; ++i) {
        double w = std::pow(theta, -2.0 * i / R);
        if (scaling == BTV_ROPE_LINEAR) w /= stretch;
        if (parts) {
            const double turns = original * w / 6.283185307179586476925;
            const double keep = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
            w = w * keep + w / stretch * (1.0 - keep);
        }
        inv_freq[i] = w;
    }
    *factor = scaling == BTV_ROPE_YARN ? 0.1 * std::log(stretch) + 1.0 : 1.0;
    return BTV_OK;
}

}  // extern "C"
