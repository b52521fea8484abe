// Rotary positions and the append to the KV cache (gfx950): the queries and keys of new rows are rotated at their positions, the keys and
// the values written to their slots of the cache, in its own type, in one pass over the projections' output.
//
// A pair (a, b) of channels turns by t = position * inv_freq[i]:  a' = f (a cos t - b sin t), b' = f (a sin t + b cos t).  t is a number of
// thousands of turns at far positions, of which only the fraction counts: it is formed in fp64 in turns, reduced there, and only the fraction
// (of which fp32 keeps 2^-25) goes to the sine and cosine.  The rotation is in fp32; a result is rounded once, to the type it is stored in.
#include "btv_common.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace {

constexpr int MOST_ROWS = (1 << 26) - 4;               // (a wavefront each; a launch has fewer than 2^32 threads)

struct Scale { float by, inv; };                       // and its reciprocal
struct RopeParams {
    const void *Q, *K, *V;
    long long q_stride, k_stride, v_stride;            // elements between rows
    const int32_t *position, *slot;
    const double *inv_freq;
    void *Qout, *Kc, *Vc;
    uint32_t *flag;
    long long num_slots;
    int total, Hq, Hkv, R, interleaved;
    int units, inv_units, rotated, heads_per_pass, slices;      // see rope_append_kernel
    float factor;
    Scale scale_k, scale_v;                            // E4M3 caches
};

// Eight neighbouring channels, 16 bytes of bf16 (32 of fp32), as they are loaded and as numbers.
template <typename T> struct Eight { uint4 w[sizeof(T) / 2]; };
template <typename T> __device__ __forceinline__ Eight<T> load8(const T *p)
{
    Eight<T> e;
#pragma unroll
    for (unsigned k = 0; k < sizeof(T) / 2; ++k) e.w[k] = reinterpret_cast<const uint4 *>(p)[k];
    return e;
}
template <typename T> __device__ __forceinline__ void numbers(const Eight<T> &e, float (&x)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            x[4 * k] = __uint_as_float(e.w[k].x); x[4 * k + 1] = __uint_as_float(e.w[k].y);
            x[4 * k + 2] = __uint_as_float(e.w[k].z); x[4 * k + 3] = __uint_as_float(e.w[k].w);
        }
    } else {
        const uint32_t w[4] = { e.w[0].x, e.w[0].y, e.w[0].z, e.w[0].w };
#pragma unroll
        for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(w[k] << 16); x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u); }
    }
}
// (E4M3: x / scale, limited to the largest code; no number stays none.  The product with the reciprocal is off by up to 1.5 of its last bits, which takes some quotients half way between two
// codes to the wrong one; what is missing, in one fused step, times the reciprocal leaves it right to 2^-46 ahead of its one rounding.)
template <typename C> __device__ __forceinline__ void store8(C *p, const float (&x)[8], Scale s)
{
    if constexpr (std::is_same_v<C, uint8_t>) {
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float q = x[4 * k + i] * s.inv, v = fmaf(-fmaf(q, s.by, -x[4 * k + i]), s.inv, q);       // (signs: -0 stays -0)
                y[i] = q > 448.f ? 448.f : q < -448.f ? -448.f : v;
            }
            w[k] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
        }
        *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (sizeof(C) == 4) {
#pragma unroll
        for (int k = 0; k < 2; ++k) reinterpret_cast<float4 *>(p)[k] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    } else {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (__bf16)x[k];
        *reinterpret_cast<bf16x8 *>(p) = y;
    }
}

// A wavefront has one row, or one of `slices` shares of its heads.  A lane has the same channels of head after head, so that its angles are worked out once: eight
// channels, and with halves the eight that they pair up with; channels that are not rotated go in eights of their own.  A pass of the wavefront takes as many heads as
// its lanes have room for (eight of 128 channels, all rotated), the next pass's loads are under way meanwhile.  Bound by HBM: 8191 rows of 32 + 2 x 8 heads of 128 channels, bf16, 201 MB
// in 42 us, 4.8 TB/s (a copy of 1 GiB: 5.2).  16-byte pieces per lane, not whole heads: a lane per pair and the angles anew for every head took 72 us.  E4M3 caches: the two steps that set the
// quotient right are 0 to 4 % of a call (490 such rows 5.20 us without and 5.35, 8191 39.2 and 39.4).
template <typename T, typename C, int D, bool PAIRS_SIDE_BY_SIDE>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeParams p)
{
    constexpr bool SIDE = PAIRS_SIDE_BY_SIDE;
    constexpr int ANGLES = SIDE ? 4 : 8;
    const int wave = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int row = wave / p.slices, slice = wave - row * p.slices;
    if (row >= p.total) return;
    const int slot = p.slot[row];
    const bool stored = slot >= 0 && slot < p.num_slots;
    if (slot >= p.num_slots && slice == 0 && lane == 0 && p.flag) atomicOr(p.flag, 32u);
    const int units = p.units, rotated = p.rotated;                   // of a head: eights (with halves pairs of eights), of which the first are rotated
    const int h0 = (lane * p.inv_units) >> 16, u = lane - h0 * units; // (lane < 64: exact)
    const bool turns_ = u < rotated, live = h0 < p.heads_per_pass;
    const int c0 = turns_ || SIDE ? 8 * u : p.R + 8 * (u - rotated), c1 = c0 + p.R / 2;
    const T *Q = static_cast<const T *>(p.Q) + p.q_stride * row, *K = static_cast<const T *>(p.K) + p.k_stride * row, *V = static_cast<const T *>(p.V) + p.v_stride * row;
    C *Kc = static_cast<C *>(p.Kc) + (long long)slot * p.Hkv * D, *Vc = static_cast<C *>(p.Vc) + (long long)slot * p.Hkv * D;
    T *Qo = static_cast<T *>(p.Qout) + (long long)row * p.Hq * D;
    const int step = p.heads_per_pass * p.slices, heads = p.Hq + (stored ? p.Hkv : 0);

    Eight<T> a = {}, b = {};
    auto load = [&](int h) {
        if (!live || h >= heads) return;
        const T *src = h < p.Hq ? Q + h * D : K + (h - p.Hq) * D;
        a = load8(src + c0);
        if (!SIDE && turns_) b = load8(src + c1);
    };
    int h = slice * p.heads_per_pass + h0;
    load(h);
    // the values, as they are: their loads and stores are under way while the angles are worked out
    if (stored)
        for (int e = slice * 64 + lane; e < p.Hkv * (D / 8); e += 64 * p.slices) {
            float x[8];
            numbers(load8(V + e * 8), x);
            store8(Vc + e * 8, x, p.scale_v);
        }
    float sn[ANGLES], cs[ANGLES];
    if (live && turns_) {
        const double pos = (double)p.position[row];
#pragma unroll
        for (int k = 0; k < ANGLES; ++k) {
            double t = pos * (p.inv_freq[ANGLES * u + k] * 0.15915494309189533577);
            t -= rint(t);
            sincospif(2.0f * (float)t, &sn[k], &cs[k]);
            sn[k] *= p.factor; cs[k] *= p.factor;
        }
    }
    for (; h - h0 < heads; h += step) {
        const Eight<T> a0 = a, b0 = b;
        load(h + step);
        if (!live || h >= heads) continue;
        const bool isq = h < p.Hq;
        float x[8], y[8];
        numbers(a0, x);
        if (turns_) {
            if constexpr (SIDE) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float v = x[2 * k], w = x[2 * k + 1];
                    x[2 * k] = v * cs[k] - w * sn[k];
                    x[2 * k + 1] = v * sn[k] + w * cs[k];
                }
            } else {
                numbers(b0, y);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float v = x[k], w = y[k];
                    x[k] = v * cs[k] - w * sn[k];
                    y[k] = v * sn[k] + w * cs[k];
                }
            }
        }
        if (isq) {
            store8(Qo + h * D + c0, x, Scale{});
            if (!SIDE && turns_) store8(Qo + h * D + c1, y, Scale{});
        } else {
            store8(Kc + (h - p.Hq) * D + c0, x, p.scale_k);
            if (!SIDE && turns_) store8(Kc + (h - p.Hq) * D + c1, y, p.scale_k);
        }
    }
}

int rope_append(RopeParams p, int dtype, int eb, int D, void *stream)
{
    BTV_REQUIRE(dtype == BTV_F32 || dtype == BTV_BF16, "dtype=%d unsupported", dtype);
    BTV_REQUIRE(p.total >= 0 && p.total <= MOST_ROWS, "total=%d outside [0,%d]", p.total, MOST_ROWS);
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
    p.rotated = p.interleaved ? p.R / 8 : p.R / 16;
    p.units = p.rotated + (D - p.R) / 8;
    p.inv_units = (65536 + p.units - 1) / p.units;
    p.heads_per_pass = 64 / p.units;
    // Few rows: a row's passes over several wavefronts, up to two on each of the 1024 SIMDs (of which each works the angles out for itself).  32 + 2 x 8 heads of 128, E4M3
    // cache, us with a wavefront per row and so: 1 row 5.5, 3.3; 128 rows 6.2, 3.7; 490 6.8, 5.4; 1024 8.5, 7.7; 2000 (one again) 10.6, 10.6.
    const int passes = (p.Hq + p.Hkv + p.heads_per_pass - 1) / p.heads_per_pass;
    p.slices = std::max(1, std::min(passes, 2048 / p.total));
    const dim3 grid((unsigned)(((long long)p.total * p.slices + 3) / 4));
    hipStream_t st = static_cast<hipStream_t>(stream);
#define BTV_CASE(DT, EB, DD, T, C)                                                                                       \
    if (dtype == DT && eb == EB && D == DD) {                                                                            \
        if (p.interleaved) hipLaunchKernelGGL((rope_append_kernel<T, C, DD, true>), grid, dim3(256), 0, st, p);          \
        else hipLaunchKernelGGL((rope_append_kernel<T, C, DD, false>), grid, dim3(256), 0, st, p);                       \
        BTV_HIP(hipGetLastError());                                                                                      \
        return BTV_OK;                                                                                                   \
    }
    BTV_CASE(BTV_F32, 4, 64, float, float) BTV_CASE(BTV_F32, 4, 128, float, float)
    BTV_CASE(BTV_BF16, 2, 64, __bf16, __bf16) BTV_CASE(BTV_BF16, 2, 128, __bf16, __bf16)
    BTV_CASE(BTV_BF16, 1, 64, __bf16, uint8_t) BTV_CASE(BTV_BF16, 1, 128, __bf16, uint8_t)
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
    p.factor = factor;
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
    p.scale_k = { k_scale, 1.0f / k_scale }; p.scale_v = { v_scale, 1.0f / v_scale };
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
