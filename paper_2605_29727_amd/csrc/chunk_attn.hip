// Causal attention of the requests' new rows over a paged KV cache (gfx950), bf16 or E4M3 K/V.
#include "btv_common.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace {

constexpr float NEG_BIG = -1.0e30f;

struct ChunkParams {
    const void *Q, *K, *V;
    void *O;
    const int32_t *block_table, *q_offset, *prefix_len;
    uint32_t *flag;
    int batch, total_M, M_max, L_max, Hq, Hkv, G, max_blocks, num_blocks;
    float scale, out_scale;
};

// A workgroup per (row, query head): 256 keys at a time, scores by one thread per key, values by one thread per channel.
template <int D, int EB>
__global__ __launch_bounds__(256) void chunk_attn_simple(ChunkParams p)
{
    constexpr int GROUPS = 256 / D, PER = 256 / GROUPS;
    __shared__ float qs[D], prob[256], red[GROUPS][D], stat[8];
    __shared__ int mine, pages[16];
    const int row = blockIdx.x, hq = blockIdx.y, tid = threadIdx.x, g = hq / p.G;
    if (tid == 0) mine = -1;
    __syncthreads();
    for (int r = tid; r < p.batch; r += 256) {
        const int q0 = p.q_offset[r], q1 = p.q_offset[r + 1], L = p.prefix_len[r];
        const bool ok = q0 >= 0 && q1 >= q0 && q1 - q0 <= p.M_max && q1 <= p.total_M && L >= 0 && L <= p.L_max && (long long)L + (q1 - q0) <= (long long)p.max_blocks * BTV_PAGE;
        if (!ok) { if (row == 0 && hq == 0) atomicOr(p.flag, 2u); continue; }
        if (row >= q0 && row < q1) atomicMax(&mine, r);
    }
    __syncthreads();
    if (mine < 0) return;
    const int r = mine, L = p.prefix_len[r], S = L + (row - p.q_offset[r]) + 1;
    const int32_t *bt = p.block_table + (size_t)r * p.max_blocks;
    if (tid < D) qs[tid] = (float)static_cast<const __bf16 *>(p.Q)[((size_t)row * p.Hq + hq) * D + tid] * p.scale;
    float m = NEG_BIG, l = 0.f, o = 0.f;
    const int d = tid % D, kg = tid / D;
    auto value = [&](const void *pool, int j, int ch) {            // key j of this chunk's 256
        const size_t at = (((size_t)pages[j >> 4] * BTV_PAGE + (j & 15)) * p.Hkv + g) * D + ch;
        if constexpr (EB == 1) {
            const uint32_t c = static_cast<const uint8_t *>(pool)[at];
            return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
        } else {
            return (float)static_cast<const __bf16 *>(pool)[at];
        }
    };
    for (int j0 = 0; j0 < S; j0 += 256) {
        __syncthreads();
        if (tid < 16) pages[tid] = min(max(bt[min((j0 >> 4) + tid, (S - 1) >> 4)], 0), p.num_blocks - 1);
        __syncthreads();
        float s = -INFINITY;
        if (j0 + tid < S) {
            s = 0.f;
            for (int ch = 0; ch < D; ++ch) s = fmaf(qs[ch], value(p.K, tid, ch), s);
        }
        float mx = s;
        for (int x = 32; x >= 1; x >>= 1) mx = fmaxf(mx, __shfl_xor(mx, x));
        if ((tid & 63) == 0) stat[tid >> 6] = mx;
        __syncthreads();
        const float mn = fmaxf(m, fmaxf(fmaxf(stat[0], stat[1]), fmaxf(stat[2], stat[3])));
        const float pj = j0 + tid < S ? expf(s - mn) : 0.f, alpha = expf(m - mn);
        m = mn;
        prob[tid] = pj;
        float sum = pj;
        for (int x = 32; x >= 1; x >>= 1) sum += __shfl_xor(sum, x);
        if ((tid & 63) == 0) stat[4 + (tid >> 6)] = sum;
        __syncthreads();
        l = l * alpha + stat[4] + stat[5] + stat[6] + stat[7];
        o *= alpha;
        for (int j = kg * PER; j < min(kg * PER + PER, S - j0); ++j) o = fmaf(prob[j], value(p.V, j, d), o);
    }
    red[kg][d] = o;
    __syncthreads();
    if (tid < D) {
        float x = red[0][tid];
        for (int k = 1; k < GROUPS; ++k) x += red[k][tid];
        static_cast<__bf16 *>(p.O)[((size_t)row * p.Hq + hq) * D + tid] = (__bf16)(x / l * p.out_scale);
    }
}

constexpr int MOST_ROWS = 1 << 20;

int check_chunk(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    BTV_REQUIRE(batch >= 1 && batch <= 4096, "batch=%d outside [1,4096]", batch);
    BTV_REQUIRE(M_max >= 1 && M_max <= MOST_ROWS, "M_max=%d outside [1,%d]", M_max, MOST_ROWS);
    BTV_REQUIRE(L_max >= 0 && (long long)L_max + M_max < (1ll << 30), "L_max=%d out of range", L_max);
    BTV_REQUIRE(Hq >= 1 && Hkv >= 1 && Hkv <= 1024 && Hq % Hkv == 0 && Hq / Hkv <= 16, "bad heads Hq=%d Hkv=%d", Hq, Hkv);
    BTV_REQUIRE(D == 64 || D == 128, "D=%d not in {64,128}", D);
    return BTV_OK;
}

bool aligned16(const void *a) { return (reinterpret_cast<uintptr_t>(a) & 15u) == 0; }

int chunk_attn(const void *Q, const void *Kpool, const void *Vpool, int num_blocks, const int32_t *block_table, int max_blocks, const int32_t *q_offset,
               const int32_t *prefix_len, int batch, int total_M, int M_max, int L_max, int Hq, int Hkv, int D, int eb, float scale, float k_scale,
               float v_scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(((Q && O) || total_M == 0) && Kpool && Vpool && block_table && q_offset && prefix_len, "null pointer");
    BTV_REQUIRE(aligned16(Q) && aligned16(Kpool) && aligned16(Vpool) && aligned16(O), "Q, K, V and O must be 16-byte aligned");
    int rc = check_chunk(batch, M_max, L_max, Hq, Hkv, D);
    if (rc) return rc;
    BTV_REQUIRE(total_M >= 0 && total_M <= INT32_MAX / Hq, "total_M=%d out of range", total_M);
    BTV_REQUIRE(num_blocks >= 1 && max_blocks >= 1, "bad block counts");
    BTV_REQUIRE((long long)max_blocks * BTV_PAGE >= (long long)L_max + 1, "max_blocks too small for L_max");
    BTV_REQUIRE(std::isfinite(scale) && std::fabs(scale) <= 1e30f, "the scale must be finite");
    rc = btv_check_ws(ws, ws_bytes, BTV_WS_HEADER);
    if (rc) return rc;
    if (total_M == 0) return BTV_OK;
    ChunkParams p = {};
    p.Q = Q; p.K = Kpool; p.V = Vpool; p.O = O; p.block_table = block_table; p.q_offset = q_offset; p.prefix_len = prefix_len;
    p.flag = static_cast<uint32_t *>(ws);
    p.batch = batch; p.total_M = total_M; p.M_max = M_max; p.L_max = L_max; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
    p.max_blocks = max_blocks; p.num_blocks = num_blocks;
    p.scale = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * k_scale;
    p.out_scale = v_scale;
    const dim3 grid(total_M, Hq);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (eb == 1) hipLaunchKernelGGL((chunk_attn_simple<128, 1>), grid, dim3(256), 0, st, p);
    else if (D == 64) hipLaunchKernelGGL((chunk_attn_simple<64, 2>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((chunk_attn_simple<128, 2>), grid, dim3(256), 0, st, p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

}  // namespace

extern "C" {

size_t btv_chunk_attn_paged_workspace(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    return check_chunk(batch, M_max, L_max, Hq, Hkv, D) == BTV_OK ? BTV_WS_HEADER : 0;
}

int btv_chunk_attn_paged(const void *Q, const void *Kpool, const void *Vpool, int num_blocks, const int32_t *block_table, int max_blocks,
                         const int32_t *q_offset, const int32_t *prefix_len, int batch, int total_M, int M_max, int L_max, int Hq, int Hkv, int D,
                         float scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    return chunk_attn(Q, Kpool, Vpool, num_blocks, block_table, max_blocks, q_offset, prefix_len, batch, total_M, M_max, L_max, Hq, Hkv, D, 2, scale, 1.0f,
                      1.0f, O, ws, ws_bytes, stream);
}

size_t btv_chunk_attn_paged_fp8kv_workspace(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    return check_chunk(batch, M_max, L_max, Hq, Hkv, D) == BTV_OK && D == 128 ? BTV_WS_HEADER : 0;
}

int btv_chunk_attn_paged_fp8kv(const void *Q, const void *K8pool, const void *V8pool, float k_scale, float v_scale, int num_blocks,
                               const int32_t *block_table, int max_blocks, const int32_t *q_offset, const int32_t *prefix_len, int batch, int total_M,
                               int M_max, int L_max, int Hq, int Hkv, int D, float scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(D == 128, "FP8 K/V: D=%d, only 128 is built", D);
    BTV_REQUIRE(k_scale > 0.f && k_scale <= 3.0e38f && v_scale > 0.f && v_scale <= 3.0e38f, "FP8 K/V scales must be positive and finite");
    return chunk_attn(Q, K8pool, V8pool, num_blocks, block_table, max_blocks, q_offset, prefix_len, batch, total_M, M_max, L_max, Hq, Hkv, D, 1, scale,
                      k_scale, v_scale, O, ws, ws_bytes, stream);
}

}  // extern "C"
