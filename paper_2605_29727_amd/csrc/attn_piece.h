// What the bf16 MFMA attention kernels share (gfx950): the layout of tiles in LDS and how they are filled, operand reads, the steps of one
// 32-key tile, and attn_piece, a workgroup's rows against a range of tiles.  Included by the translation units of tree attention and of causal
// attention of chunks.
#pragma once
#include "btv_common.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int TK = 32;          // keys per tile = per LDS stage
// Behind a workspace's header: words that attention calls keep from call to call, whatever others do with the rest.
constexpr int MERGE_GROUPS = 128, MERGE_SPLITS = 32;
typedef unsigned long long u64;
struct MergeWords {                                     // of one group: the merge inside one request's kernel
    u64 started[MERGE_SPLITS];                          // tag << 8 | XCD
    u64 near[MERGE_SPLITS], far[MERGE_SPLITS];          // tag << 8 | 1 if it has left
    u64 epoch;
    u64 arrived[31];                                    // chunks: parts of a block that are stored, 0 between calls
};
static_assert(sizeof(MergeWords) == 1024, "whole cache lines per group");
constexpr size_t MERGE_WORDS = MERGE_GROUPS * sizeof(MergeWords);
constexpr float NEG_BIG = -1.0e30f;

struct AttnParams {
    const void *Q, *K, *V;
    void *O;
    const int32_t *parent;        // [total_M], indices local to each request
    const int32_t *block_table;   // paged only
    const int32_t *q_offset;      // paged only, [batch+1]
    const int32_t *prefix_len;    // paged only, [batch]
    _Float16 *Opart;              // [nsplit][total_rows][D]: split partial of O^T's row, divided by its largest magnitude
    float *ML;                    // [nsplit][total_rows][4]: reference max, row sum, that magnitude, unused
    uint32_t *flag;
    unsigned long long *sync;     // one request: words of the merge inside the attention kernel (null: tv_combine_bf16 merges)
    int wait_ticks;               // ... how long a workgroup waits for the others of its group
    int M, L;                     // contiguous: actual sizes; paged: host upper bounds
    int Hq, Hkv, G;
    int ginv;                     // ceil(2^16 / G): (x * ginv) >> 16 = x / G for every packed row x < 4096 (G <= 16)
    int max_blocks, num_blocks;
    int total_rows;               // rows of the partial buffers (>= total_M * Hq)
    int total_M;
    int sps;                      // one request: whole tiles per split (`longer` of them take a round more); batch: tiles per part
    int longer;
    int nsplit;                   // key splits (batch: of the longest request)
    int row_blocks, units;        // row blocks per (split, head, request) unit; number of units
    uint32_t inv_row_blocks, inv_nsplit, inv_sps, inv_Hkv;    // for quotient()
    long long *plan;              // batch only: [batch + 2], where the requests' work starts (see Stretch)
    int batch, teams_log2, pairing, wmin, wr_log2;   // batch only: requests, teams of workgroups, whether a team is a pair, smallest share, rows per block
    float scale;                  // softmax scale
    float scale_log2;             // scale * log2(e) (times the key scale of an FP8 cache)
    float out_scale;              // 1, or the value scale of an FP8 cache
};

// n / d for n >= 0, with inv = reciprocal(d).  (A division by a number that the compiler does not know takes some 30 instructions, and a workgroup
// has three to five of them ahead of its first load.)
__host__ constexpr uint32_t reciprocal(int d) { return d <= 1 ? 0u : (uint32_t)((0x100000000ull + (unsigned)d - 1) / (unsigned)d); }
__device__ __forceinline__ int quotient(int n, int d, uint32_t inv)
{
    const int q = (int)__umulhi((uint32_t)n, inv);      // at most one too many
    return d == 1 ? n : q - (q * d > n);
}

__device__ __forceinline__ uint32_t float_to_bf16_bits(float f)
{   // round to nearest even; inputs here are finite
    uint32_t u = __float_as_uint(f);
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// Request geometry: contiguous calls have one request; paged calls read it from device arrays
// and clamp against the host-provided bounds so that no access can leave its buffer.
struct Req { int q0, M, L; bool ok; };

template <bool PAGED>
__device__ __forceinline__ Req load_req(const AttnParams &p, int r)
{
    Req q;
    if (!PAGED) { q.q0 = 0; q.M = p.M; q.L = p.L; q.ok = true; return q; }
    q.q0 = p.q_offset[r];
    q.M = p.q_offset[r + 1] - q.q0;
    q.L = p.prefix_len[r];
    q.ok = q.M >= 1 && q.M <= p.M && q.L >= 0 && q.L <= p.L && q.q0 >= 0 &&
           q.q0 + q.M <= p.total_M && (long long)q.L + q.M <= (long long)p.max_blocks * BTV_PAGE;
    return q;
}

// Visibility of keys kb..kb+31 for a node: bit c set iff key kb+c is a prefix row, or a tree
// row L+a with a in anc(node).  Bits of anc past the request's node count are zero.
// AncT is either a pointer to the node's BTV_ANC_WORDS words or a register array of them.
template <typename AncT>
__device__ __forceinline__ uint32_t anc_word(const AncT &anc, int w)
{
    uint32_t r = 0u;
#pragma unroll
    for (int k = 0; k < BTV_ANC_WORDS; ++k) r = (k == w) ? anc[k] : r;
    return r;
}

template <typename AncT>
__device__ __forceinline__ uint32_t vis_word(const AncT &anc, int kb, int L)
{
    int off = kb - L;
    if (off <= -32) return 0xFFFFFFFFu;
    if (off < 0) {
        int n = -off;
        return ((1u << n) - 1u) | (anc_word(anc, 0) << n);
    }
    int w = off >> 5, sh = off & 31;
    uint32_t lo = anc_word(anc, w), hi = anc_word(anc, w + 1);
    return sh ? ((lo >> sh) | (hi << (32 - sh))) : lo;
}
// The same for a row of a chunk, which sees all keys up to its own (odd: see take_out).
struct LastKey { int key; bool odd; };
__device__ __forceinline__ uint32_t vis_word(const LastKey &last, int kb, int)
{
    const int n = last.key + 1 - kb;
    return n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
}

// What scores are multiplied with on their way into the exponential: nothing where the queries have taken the softmax scale (trees), or scale * log2(e), in
// fp32, where they come as they are (chunks: an instruction per score, and no rounding of the scaled queries: 2.3e-3 of the result in place of 2.8e-3 by the 2-norm).
struct NoFactor {};
__device__ __forceinline__ float times(float x, NoFactor) { return x; }
__device__ __forceinline__ float times(float x, float c) { return x * c; }

// ------------------------------------------------------------------------------------------------
// bf16 MFMA kernel
//
// LDS holds a ring of NT stages; a stage is one 32-key tile: the K rows and the V rows exactly as
// they lie in memory ([key][channel], 2*D bytes per row).  Stages are filled by direct-to-LDS
// global loads (each lane moves 16 bytes, a wave instruction fills 1 KiB of LDS), so no staging
// registers and no VALU work are spent on data movement and up to NT-1 stages stay in flight.
// Bank conflicts are avoided by choosing which 16-byte chunk of a row each lane fetches: the chunk
// stored at physical position pc of LDS row r is chunk pc ^ f(r) of the source row.
//   K: LDS row i holds key kb + swap_bits_2_3(i) (the MFMA A-row order that makes a lane's 16 score
//      registers two runs of 8 consecutive keys); A operands are 16-byte LDS reads.
//   V: LDS row r holds key kb + r; the V^T A operand (one channel, 8 consecutive keys per lane) comes
//      from two transposing LDS reads (ds_read_b64_tr_b16): a 16-lane group reads 4 keys x 16 channels
//      and every lane receives the 4 keys of its own channel.
// ------------------------------------------------------------------------------------------------
// EB = bytes per K/V element in memory and in LDS: 2 (bf16) or 1 (FP8 E4M3, converted to bf16 in registers after
// the operand reads: every E4M3 number is a bf16 number, so the conversion is exact).
template <int D, int EB = 2>
struct Lds {
    static constexpr int ROWB = EB * D;                      // bytes per K or V row
    static constexpr int TILEB = 32 * ROWB;                  // one K (or V) tile
    static constexpr int STAGE = 2 * TILEB;                  // K tile then V tile
    static constexpr int INSTR = STAGE / 1024;               // wave-wide 1 KiB fills per tile
    static constexpr int CHUNKS = ROWB / 16;                 // 16-byte chunks per row
};

__device__ __forceinline__ int swap_bits_2_3(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }

// bf16 rows (2*D bytes): consecutive rows start on the same bank, so the chunk is rotated by the row number.
// FP8 rows of 128 bytes: even and odd rows already sit in different halves of the 64 banks, so pairs of rows share a
// rotation.
template <int D, int EB = 2> __device__ __forceinline__ int swz_k(int row)
{
    return EB == 2 ? (row & (D / 8 - 1)) : ((row >> 1) & (Lds<D, EB>::CHUNKS - 1));
}
// V rows, bf16: the four rows a 16-lane group of a transposing read touches (row % 4 = 0..3) are moved 64 bytes
// apart.  FP8: a group touches 8 rows x 16 bytes and two groups (32 bytes per row) are served together; the four
// even (and the four odd) rows among them are moved 32 bytes apart.
template <int D, int EB = 2> __device__ __forceinline__ int swz_v(int row)
{
    return EB == 2 ? (((row & 3) << 2) & (D / 8 - 1)) : ((((row >> 1) & 3) << 1) & (Lds<D, EB>::CHUNKS - 1));
}

#define BTV_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

// 16 bytes of every lane straight to LDS, lane after lane from dst on (uniform)
__device__ __forceinline__ void fill_lds(const unsigned char *src, unsigned char *dst)
{
    __builtin_amdgcn_global_load_lds(src, BTV_LDS_PTR(dst), 16, 0, 0);
}

// Per-wave, loop-invariant part of the ring fills.  A wave issues LPW fills per tile; fill jj of wave w is
// instruction j = w*LPW + jj of the tile (K part first).  Lane l of it fills LDS row r, physical chunk pc, with
// source row key_off (relative to the tile's first key) and source chunk pc ^ swizzle(r).  A wave's fills of a tile are ROWS rows of K
// or of V, all in the same half of the tile (the permutation of the K rows stays within 16), so in a paged cache of one page.
template <int D, int WAVES, bool PAGED, int EB = 2>
struct Fill {
    static constexpr int LPW = Lds<D, EB>::INSTR / WAVES, ROWS = 64 / WAVES;
    static_assert(LPW >= 1 && LPW * WAVES == Lds<D, EB>::INSTR, "fills must divide evenly over the waves");
    static_assert(ROWS <= 16 && BTV_PAGE == 16, "a wave's rows are of one half of the tile: of one page");
    const unsigned char *base;      // K or V of this KV head (wave-uniform)
    const int32_t *block_table;     // row of this request (paged)
    uint32_t pages;                 // paged, lane l: page of this wave's rows in tile l of a window of 32 (PGV)
    int num_blocks, S, half;
    uint32_t row_bytes;             // Hkv * D * EB: distance between consecutive keys
    uint32_t lane_off[LPW];         // contiguous: key_off*row_bytes + chunk*16;  paged: (key_off & 15)*row_bytes + chunk*16
    // where the 16 rows of a page begin (an id from the block table is clamped, so that no access can leave the pool)
    __device__ __forceinline__ int valid_page(int id) const { return min(max(id, 0), num_blocks - 1); }
    // The page of the wave's rows in tile st (constant space: a scalar load, so that the vector-memory counter only ever counts the LDS
    // fills).  Past the end it is the last page: rows of the tile's upper half re-read the lower half's last row then.
    __device__ __forceinline__ int page_id(int st) const
    {
        typedef const __attribute__((address_space(4))) int32_t *const_i32;
        const const_i32 bt = reinterpret_cast<const_i32>(reinterpret_cast<uintptr_t>(block_table));
        return bt[__builtin_amdgcn_readfirstlane(min(2 * st + half, (S - 1) >> 4))];
    }
    __device__ __forceinline__ const unsigned char *page(int id) const { return base + (size_t)(uint32_t)id * (BTV_PAGE * row_bytes); }
};

template <int D, int WAVES, bool PAGED, int EB = 2>
__device__ __forceinline__ Fill<D, WAVES, PAGED, EB> make_fill(const void *K, const void *V, const int32_t *bt, int num_blocks,
                                                               int Hkv, int g, int S, int w, int l)
{
    using LD = Lds<D, EB>;
    constexpr int CH = LD::CHUNKS, RPI = 1024 / LD::ROWB;
    Fill<D, WAVES, PAGED, EB> f;
    const bool isv = w >= WAVES / 2;                 // (uniform)
    f.base = static_cast<const unsigned char *>(isv ? V : K) + (size_t)g * D * EB;
    f.block_table = bt; f.num_blocks = num_blocks; f.S = S;
    f.half = (w * f.ROWS & 16) >> 4;
    f.row_bytes = (uint32_t)Hkv * D * EB;
#pragma unroll
    for (int jj = 0; jj < f.LPW; ++jj) {
        const int r = (w * f.LPW + jj) * RPI % 32 + l / CH, pc = l % CH;
        const int key_off = isv ? r : swap_bits_2_3(r);
        const int chunk = pc ^ (isv ? swz_v<D, EB>(r) : swz_k<D, EB>(r));
        f.lane_off[jj] = (uint32_t)(PAGED ? (key_off & 15) : key_off) * f.row_bytes + chunk * 16;
    }
    return f;
}

// Source row (relative to the tile's first key) of lane l in fill jj of wave w: recomputed where it is needed (the
// clamped last tile) rather than kept in registers through the main loop.
template <int D, int WAVES, int EB>
__device__ __forceinline__ int fill_key_off(int w, int jj, int l)
{
    using LD = Lds<D, EB>;
    constexpr int CH = LD::CHUNKS, RPI = 1024 / LD::ROWB, LPW = LD::INSTR / WAVES;
    const int r = (w * LPW + jj) * RPI % 32 + l / CH;
    return w >= WAVES / 2 ? r : swap_bits_2_3(r);
}

// Issue this wave's share of the direct-to-LDS loads of tile `st` (keys 32*st ..) into ring slot `slot`.
// Keys past the end of the sequence re-read the last valid row (finite data; their scores are masked).
// JB .. JE - 1: which of the wave's LPW fills (all by default; the pipelined loop issues them one by one, each behind a
// group of MFMAs, because an issue holds its wave for about a hundred cycles).
// PGV: the page comes from lane `at` of the window in f.pages, else from a scalar load.
// GIVEN: `at` is the page's id.
template <int D, int WAVES, bool PAGED, int EB = 2, int JB = 0, int JE = Lds<D, EB>::INSTR / WAVES, bool PGV = false, bool GIVEN = false>
__device__ __forceinline__ void issue_tile(const Fill<D, WAVES, PAGED, EB> &f, unsigned char *smem, int slot, int st, int w, int l, int at = 0)
{
    using LD = Lds<D, EB>;
    const int kb = st * 32;
    const bool whole = kb + 32 <= f.S;       // uniform: no key of this tile needs clamping
    const unsigned char *src;                // uniform
    if constexpr (!PAGED) src = f.base + (size_t)kb * f.row_bytes;
    else if constexpr (GIVEN) src = f.page(f.valid_page(at));
    else if constexpr (PGV) src = f.page(__builtin_amdgcn_readlane((int)f.pages, at));
    else {
        src = f.page(f.valid_page(f.page_id(st)));
    }
    uint32_t off[JE];
#pragma unroll
    for (int jj = JB; jj < JE; ++jj) off[jj] = f.lane_off[jj];
    if (!whole) {
#pragma unroll
        for (int jj = JB; jj < JE; ++jj) {
            const int ko = fill_key_off<D, WAVES, EB>(w, jj, l), kc = min(kb + ko, f.S - 1) - kb;
            off[jj] += (uint32_t)(PAGED ? (kc & 15) - (ko & 15) : kc - ko) * f.row_bytes;
        }
    }
#pragma unroll
    for (int jj = JB; jj < JE; ++jj) {
        asm volatile("" : "+v"(off[jj]));    // (one branch for all of them: else there is one for each)
        fill_lds(src + off[jj], smem + slot * LD::STAGE + (w * f.LPW + jj) * 1024);
    }
}

// ---- LDS operand reads ---------------------------------------------------------------------------
// All operand reads are raw instructions with explicit counter waits: as ordinary loads / builtins the
// compiler would drain the whole vector-memory queue (the ring fills still in flight) in front of every tile.
// Each wait takes the registers it covers as in/out operands, so no use can be scheduled above it.
//
// K A-operands: lane (c = l%32, h = l/32) reads chunk (2s+h) ^ swz_k(c) of LDS row c for s = 0..D/16-1.  Row
// starts are 2*D-byte aligned, so the address is  (tile + lane part) ^ (s << 5).
template <int D> __device__ __forceinline__ uint32_t lane_k_off(int l)
{
    const int c = l & 31, h = l >> 5;
    return (uint32_t)(c * Lds<D>::ROWB + ((h ^ swz_k<D>(c)) << 4));
}

template <int D> __device__ __forceinline__ void lds_read_k(uint32_t a, u32x4 (&ka)[D / 16])
{
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
        const uint32_t addr = a ^ (uint32_t)(s << 5);
        asm volatile("ds_read_b128 %0, %1" : "=v"(ka[s]) : "v"(addr));
    }
}

template <int DS, int YOUNGER> __device__ __forceinline__ void lds_wait_k(u32x4 (&ka)[DS])
{
    static_assert(DS == 4 || DS == 8, "D in {64,128}");
    if constexpr (DS == 8)
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(ka[0]), "+v"(ka[1]), "+v"(ka[2]), "+v"(ka[3]), "+v"(ka[4]), "+v"(ka[5]), "+v"(ka[6]), "+v"(ka[7])
                     : "n"(YOUNGER));
    else
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(ka[0]), "+v"(ka[1]), "+v"(ka[2]), "+v"(ka[3]) : "n"(YOUNGER));
}

// V^T A-operands (ds_read_b64_tr_b16): lane l sits in 16-lane group l/16 = 2h + dhalf; for (dt, mm, i) it
// supplies the address of key row 16mm + 8h + 4i + (l%16)/4, channels 32dt + 16dhalf + 4(l%4) .. +3, and
// receives keys 16mm + 8h + 4i .. +3 of channel 32dt + (l%32).  With the V swizzle the address is
// ((tile + lane part) ^ (dt << 6)) + (16mm + 4i) * row bytes, the last term an immediate offset.
template <int D> __device__ __forceinline__ uint32_t lane_v_off(int l)
{
    const int h = l >> 5, dhalf = (l >> 4) & 1, rr = (l & 15) >> 2, q = l & 3;
    const int x = 2 * dhalf + (q >> 1);
    return (uint32_t)((8 * h + rr) * Lds<D>::ROWB + ((swz_v<D>(rr) ^ x) << 4) + ((q & 1) << 3));
}

// The reads for keys 16*MM .. 16*MM + 15 (the operands of the PV MFMAs with index mm = MM): 2*D/32 instructions.
template <int D, int MM> __device__ __forceinline__ void lds_read_vt(uint32_t a, bf16x4 (&va)[D / 32][2][2])
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        const uint32_t addr = a ^ (uint32_t)(dt << 6);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2"
                         : "=v"(va[dt][MM][i])
                         : "v"(addr), "n"((16 * MM + 4 * i) * Lds<D>::ROWB));
    }
}

template <int DT>
__device__ __forceinline__ void lds_wait_vt(bf16x4 (&va)[DT][2][2])
{
    static_assert(DT == 2 || DT == 4, "D in {64,128}");
    if constexpr (DT == 4)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(va[0][0][0]), "+v"(va[0][0][1]), "+v"(va[0][1][0]), "+v"(va[0][1][1]), "+v"(va[1][0][0]),
                       "+v"(va[1][0][1]), "+v"(va[1][1][0]), "+v"(va[1][1][1]), "+v"(va[2][0][0]), "+v"(va[2][0][1]),
                       "+v"(va[2][1][0]), "+v"(va[2][1][1]), "+v"(va[3][0][0]), "+v"(va[3][0][1]), "+v"(va[3][1][0]),
                       "+v"(va[3][1][1]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(va[0][0][0]), "+v"(va[0][0][1]), "+v"(va[0][1][0]), "+v"(va[0][1][1]), "+v"(va[1][0][0]),
                       "+v"(va[1][0][1]), "+v"(va[1][1][0]), "+v"(va[1][1][1]));
}

// ---- the arithmetic steps of one 32-key tile of one wave (32 query rows) ---------------------------------
// S^T = K . Q^T
template <int DS>
__device__ __forceinline__ f32x16 qk_tile(const u32x4 (&ka)[DS], const bf16x8 (&qreg)[DS], f32x16 s)
{
#pragma unroll
    for (int k = 0; k < DS; ++k)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, ka[k]), qreg[k], s, 0, 0, 0);
    return s;
}

// largest score of the lane's query over the 32 keys (the other half of the wave holds the other 16)
__device__ __forceinline__ float tile_max(const f32x16 &s)
{
    float t = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) t = fmaxf(t, s[v]);
    auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(t), __float_as_uint(t), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

// Scores arrive in log2 units: the queries were multiplied by scale * log2(e) once, in the prologue, so a
// probability is exp2(score - reference) with no multiply per element.
//
// One half (keys 8 mm .. 8 mm + 7 of the lane's 16) of a tile whose scores already are relative to the reference:
// P = exp2(x) as a B operand, its rounded values added to `sum`.
template <typename C>
__device__ __forceinline__ void exp_half(const f32x16 &x, int mm, bf16x8 &pbm, float &sum, C c)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = { (__bf16)1.0f, (__bf16)1.0f };
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(times(x[mm * 8 + e], c));
        const float p1 = __builtin_amdgcn_exp2f(times(x[mm * 8 + e + 1], c));
        const bf16x2 pp = { (__bf16)p0, (__bf16)p1 };
        pbm[e] = pp[0];
        pbm[e + 1] = pp[1];
        sum = __builtin_amdgcn_fdot2_f32_bf16(pp, ones, sum, false);
    }
}

// The reference of the step-by-step tiles enters through the matrix cores as well: the score accumulator starts from
// -base (negb: the same value in all 16 registers), base being the running maximum once there is one (0 before), so
// the scores arrive relative to it and a probability is exp2 of the accumulator as it stands.  The reference only moves where
// the tile's maximum exceeds it by more than LAZY, so that probabilities stay below 2^LAZY and most tiles rescale nothing; the
// result is the same, numerator and denominator refer to the same m_run.  Where it moves the tile's scores are shifted by hand.
// whole: all rows see all of the tile.  A row that has no score above -infinity there has no reference for the tiles behind it, which do not look for one: it starts
// from -NO_SCORE, far below any maximum, so that its first finite score makes a tile's sum overflow and the tile be done again, and near enough to leave that tile's scores
// 2^-10.  (A row that has met none by the end: attn_piece, behind its loops.)
constexpr float NO_SCORE = 16384.0f;
template <int DT, typename C>
__device__ __forceinline__ void rebase_tile(f32x16 &srel, float &base, f32x16 &negb, float &m_run, float &l_run, f32x16 (&oacc)[DT], C c, bool whole)
{
    constexpr float LAZY = 8.0f;
    const float rmax = tile_max(srel);
    const bool grow = times((rmax + base) - m_run, c) > LAZY, none = whole && m_run < 0.5f * NEG_BIG;
    if (__builtin_amdgcn_ballot_w64(grow || none) != 0ull) {
        const float mnew = grow ? rmax + base : none ? -NO_SCORE : m_run;
        const float alpha = __builtin_amdgcn_exp2f(times(m_run - mnew, c));
        m_run = mnew;
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
        const float nb = m_run > 0.5f * NEG_BIG ? m_run : 0.f;
        const float d = nb - base;
        base = nb;
#pragma unroll
        for (int v = 0; v < 16; ++v) { srel[v] -= d; negb[v] = -nb; }
    }
}

// Probabilities of a tile whose scores are relative to the reference.  The reference has to follow the scores up (rebase_tile)
// where there is none yet or the tile is masked (`exact`); otherwise nothing stands between the scores and their
// exponentials, and the tile's sum tells afterwards whether one of them exceeded 16: then it is done again, against a new one.  (The
// maximum, its exchange between the halves of the wave and the branch on it are 150 cycles of a tile's 1300 to 1800.)
constexpr float GROW = 1048576.0f;       // 2^20: a sum of 16 terms above it means some score > 16
template <int DT, typename C>
__device__ __forceinline__ void probabilities(f32x16 &x, bool exact, float &base, f32x16 &negb, float &m_run, float &l_run, f32x16 (&oacc)[DT],
                                              bf16x8 (&pb)[2], C c, bool whole)
{
    if (exact) rebase_tile<DT>(x, base, negb, m_run, l_run, oacc, c, whole);
    float ts[2] = { 0.f, 0.f };
    exp_half(x, 0, pb[0], ts[0], c);
    exp_half(x, 1, pb[1], ts[1], c);
    float sum = ts[0] + ts[1];
    if (!exact && __builtin_amdgcn_ballot_w64(!(sum <= GROW)) != 0ull) {
        rebase_tile<DT>(x, base, negb, m_run, l_run, oacc, c, false);
        ts[0] = ts[1] = 0.f;
        exp_half(x, 0, pb[0], ts[0], c);
        exp_half(x, 1, pb[1], ts[1], c);
        sum = ts[0] + ts[1];
    }
    l_run += sum;
}

// O^T += V^T . P^T
template <int DT>
__device__ __forceinline__ void pv_tile(const bf16x4 (&va)[DT][2][2], const bf16x8 (&pb)[2], f32x16 (&oacc)[DT])
{
#pragma unroll
    for (int mm = 0; mm < 2; ++mm)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
            const bf16x8 a = __builtin_shufflevector(va[dt][mm][0], va[dt][mm][1], 0, 1, 2, 3, 4, 5, 6, 7);
            oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[mm], oacc[dt], 0, 0, 0);
        }
}

// tree mask of a tile that touches tree rows (or the end of the sequence)
__device__ __forceinline__ void mask_tile(f32x16 &s, uint32_t vis, int h)
{
    vis >>= 8 * h;
    asm volatile("" : "+v"(vis));            // (what follows from the lane alone would be worked out ahead of the loop, in calls without a mask too)
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const int bit = 16 * (v >> 3) + (v & 7);
        if (!((vis >> bit) & 1u)) s[v] = -INFINITY;
    }
}

// Values that are not numbers, in a tile of which some rows see a part only: a probability of 0 times such a value would reach the rows that do
// not see its key.  They are taken out of the operands, and the wavefront remembers that it has met one (rare; found by a product with 0, two values at a time): what they
// do to the rows that see them is added at the end of attn_piece.
template <int DT>
__device__ __forceinline__ bool take_out(bf16x4 (&va)[DT][2][2])
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 zeros = { (__bf16)0.0f, (__bf16)0.0f };
    float t = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bf16x4 x = va[dt][k >> 2][(k >> 1) & 1];
            const bf16x2 y = { x[2 * (k & 1)], x[2 * (k & 1) + 1] };
            t = __builtin_amdgcn_fdot2_f32_bf16(y, zeros, t, false);
        }
    if (__builtin_amdgcn_ballot_w64(!(t == 0.f)) == 0ull) return false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            u32x2 w = __builtin_bit_cast(u32x2, va[dt][k >> 1][k & 1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] &= ~(((((w[i] & 0x7F807F80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xFFFFu);       // (exponents all ones)
            va[dt][k >> 1][k & 1] = __builtin_bit_cast(bf16x4, w);
        }
    return true;
}
template <int DT>
__device__ __forceinline__ bool take_out8(u32x2 (&v8)[DT][2])
{
    auto none = [](uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; };        // (a code without its sign of all ones)
    uint32_t t = 0;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k) t |= none(v8[dt][k >> 1][k & 1]);
    if (__builtin_amdgcn_ballot_w64(t != 0) == 0ull) return false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k) v8[dt][k >> 1][k & 1] &= ~((none(v8[dt][k >> 1][k & 1]) >> 7) * 0xFFu);
    return true;
}

// One whole tile, step after step (no overlap between the steps): used for the tiles that need the mask and
// by the workgroup shapes whose wave pairs alternate over the tiles.  PLAIN: prefix rows only, and not the wave's first tile;
// `exact` (see probabilities) else.
template <int D, bool PLAIN, typename Seen, typename C>
__device__ __forceinline__ void do_tile(uint32_t stage, int kb, int Lr, int l, Seen &seen,
                                        const bf16x8 (&qreg)[D / 16], float &m_run, float &l_run, f32x16 (&oacc)[D / 32],
                                        float &base, f32x16 &negb, bool exact, C c)
{
    constexpr int DS = D / 16, DT = D / 32;
    u32x4 ka[DS];
    bf16x4 va[DT][2][2];
    const uint32_t va_addr = stage + Lds<D>::TILEB + lane_v_off<D>(l);
    lds_read_k<D>(stage + lane_k_off<D>(l), ka);
    lds_read_vt<D, 0>(va_addr, va);
    lds_wait_k<DS, DT * 2>(ka);          // the counter completes in order: K has landed when 2*DT reads remain
    lds_read_vt<D, 1>(va_addr, va);
    f32x16 s = qk_tile<DS>(ka, qreg, negb);
    if (!PLAIN && kb + 32 > Lr) mask_tile(s, vis_word(seen, kb, Lr), l >> 5);
    bf16x8 pb[2];
    probabilities<DT>(s, !PLAIN && exact, base, negb, m_run, l_run, oacc, pb, c, kb + 32 <= Lr);
    lds_wait_vt<DT>(va);
    if constexpr (!PLAIN && std::is_same_v<Seen, LastKey>)
        if (kb + 32 > Lr && take_out<DT>(va)) seen.odd = true;
    pv_tile<DT>(va, pb, oacc);
}

// ---- FP8 (E4M3) K/V: operand reads and exact conversion to bf16 ---------------------------------------
// K: a lane reads 16 consecutive channels (16 bytes) of its key row, channels 32 s + 16 h .. + 15 for s = 0 .. D/32-1,
// and uses the first 8 for contraction step 2s, the last 8 for step 2s+1.  The contraction steps thus take the
// channels in another order than the bf16 layout; the query operands are loaded in the same order, so the sum is
// over the same products.  Address: (tile + lane part) ^ (s << 5), as for bf16 with 128-byte rows.

template <int D> __device__ __forceinline__ uint32_t lane_k8_off(int l)
{
    const int c = l & 31, h = l >> 5;
    return (uint32_t)(c * Lds<D, 1>::ROWB + ((h ^ swz_k<D, 1>(c)) << 4));
}

template <int D> __device__ __forceinline__ void lds_read_k8(uint32_t a, u32x4 (&k8)[D / 32])
{
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        const uint32_t addr = a ^ (uint32_t)(s << 5);
        asm volatile("ds_read_b128 %0, %1" : "=v"(k8[s]) : "v"(addr));
    }
}

template <int YOUNGER> __device__ __forceinline__ void lds_wait_k8(u32x4 (&k8)[4])
{
    asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(k8[0]), "+v"(k8[1]), "+v"(k8[2]), "+v"(k8[3]) : "n"(YOUNGER));
}

// Two E4M3 codes (one 16-bit half of a register) to two bf16, scale 1: exact for every code.
__device__ __forceinline__ uint32_t fp8x2_to_bf16x2(uint32_t w, bool high)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)
                          : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false);
    return __builtin_bit_cast(uint32_t, r);
}

// eight consecutive codes (two registers) -> one bf16 MFMA operand
__device__ __forceinline__ bf16x8 fp8x8_to_bf16x8(uint32_t w0, uint32_t w1)
{
    const u32x4 r = { fp8x2_to_bf16x2(w0, false), fp8x2_to_bf16x2(w0, true), fp8x2_to_bf16x2(w1, false),
                      fp8x2_to_bf16x2(w1, true) };
    return __builtin_bit_cast(bf16x8, r);
}

// V^T operands (ds_read_b64_tr_b8): a 16-lane group reads 8 key rows x 16 channels; lane j of the group supplies
// the address of row j/2, bytes 8 (j%2) .. + 7 of the group's 16 channels, and receives the 8 keys of channel j.
// Lane l sits in group l/16 = 2h + dhalf; for (dt, mm) the group reads keys 16mm + 8h .. + 7, channels
// 32dt + 16dhalf .. + 15, so the lane receives keys 16mm + 8h .. + 7 of channel 32dt + (l%32): one whole operand
// of the PV MFMA with index mm.  With the V swizzle the address is ((tile + lane part) ^ (dt << 5)) + 16mm * row
// bytes, the last term an immediate offset.
template <int D> __device__ __forceinline__ uint32_t lane_v8_off(int l)
{
    const int h = l >> 5, dhalf = (l >> 4) & 1, j = l & 15;
    const int row = 8 * h + (j >> 1);
    return (uint32_t)(row * Lds<D, 1>::ROWB + ((swz_v<D, 1>(row) ^ dhalf) << 4) + ((j & 1) << 3));
}

template <int D, int MM> __device__ __forceinline__ void lds_read_vt8(uint32_t a, u32x2 (&v8)[D / 32][2])
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        const uint32_t addr = a ^ (uint32_t)(dt << 5);
        asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(v8[dt][MM]) : "v"(addr), "n"(16 * MM * Lds<D, 1>::ROWB));
    }
}

__device__ __forceinline__ void lds_wait_vt8(u32x2 (&v8)[4][2])
{
    asm volatile("s_waitcnt lgkmcnt(0)"
                 : "+v"(v8[0][0]), "+v"(v8[0][1]), "+v"(v8[1][0]), "+v"(v8[1][1]), "+v"(v8[2][0]), "+v"(v8[2][1]),
                   "+v"(v8[3][0]), "+v"(v8[3][1]));
}

// One whole tile of an FP8 cache: the same steps as do_tile with half the operand reads and the conversions.
template <int D, bool PLAIN, typename Seen, typename C>
__device__ __forceinline__ void do_tile8(uint32_t stage, int kb, int Lr, int l, Seen &seen,
                                         const bf16x8 (&qreg)[D / 16], float &m_run, float &l_run, f32x16 (&oacc)[D / 32],
                                         float &base, f32x16 &negb, bool exact, C c)
{
    static_assert(D == 128, "FP8 K/V: head dimension 128 only");
    constexpr int DS = D / 16, DT = D / 32;
    u32x4 k8[DS / 2];
    u32x2 v8[DT][2];
    const uint32_t va_addr = stage + Lds<D, 1>::TILEB + lane_v8_off<D>(l);
    lds_read_k8<D>(stage + lane_k8_off<D>(l), k8);
    lds_read_vt8<D, 0>(va_addr, v8);
    lds_wait_k8<DT>(k8);                 // the counter completes in order: K has landed when DT reads remain
    lds_read_vt8<D, 1>(va_addr, v8);
    f32x16 s = negb;
#pragma unroll
    for (int k = 0; k < DS / 2; ++k) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_to_bf16x8(k8[k][0], k8[k][1]), qreg[2 * k], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_to_bf16x8(k8[k][2], k8[k][3]), qreg[2 * k + 1], s, 0, 0, 0);
    }
    if (!PLAIN && kb + 32 > Lr) mask_tile(s, vis_word(seen, kb, Lr), l >> 5);
    bf16x8 pb[2];
    probabilities<DT>(s, !PLAIN && exact, base, negb, m_run, l_run, oacc, pb, c, kb + 32 <= Lr);
    lds_wait_vt8(v8);
    if constexpr (!PLAIN && std::is_same_v<Seen, LastKey>)
        if (kb + 32 > Lr && take_out8<DT>(v8)) seen.odd = true;
#pragma unroll
    for (int mm = 0; mm < 2; ++mm)
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
            oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_to_bf16x8(v8[dt][mm][0], v8[dt][mm][1]), pb[mm],
                                                               oacc[dt], 0, 0, 0);
}

// ---- half-tile operand buffers of the software-pipelined loop ----------------------------------------------
// The loop keeps 16 registers of K operands and 16 of V^T operands (D = 128): half a tile each, refilled right
// after the MFMAs that consumed the previous contents were issued.  Addresses are loop-invariant registers (one
// per contraction step / channel block, the XOR of the swizzle already applied); the ring slot is an immediate
// offset, which reaches SPB slots from one base (the offset field has 16 bits).
template <int OFF> __device__ __forceinline__ void ds_read_k_imm(uint32_t a, u32x4 &r)
{
    static_assert(OFF >= 0 && OFF < 65536, "immediate offset range");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r) : "v"(a), "n"(OFF));
}
template <int OFF> __device__ __forceinline__ void ds_read_vt_imm(uint32_t a, bf16x4 &r)
{
    static_assert(OFF >= 0 && OFF < 65536, "immediate offset range");
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r) : "v"(a), "n"(OFF));
}

// K operands of contraction steps HALF * DS/2 .. + DS/2 - 1 of the tile in slot SLOT (relative to the base in ak).
template <int D, int SLOT, int HALF> __device__ __forceinline__ void read_k_half(const uint32_t (&ak)[D / 16], u32x4 (&kh)[D / 32])
{
#pragma unroll
    for (int s = 0; s < D / 32; ++s) ds_read_k_imm<SLOT * Lds<D>::STAGE>(ak[HALF * (D / 32) + s], kh[s]);
}
// V^T operands of keys 16 MM .. 16 MM + 15 (the PV MFMAs with index MM), all channel blocks.
template <int D, int SLOT, int MM> __device__ __forceinline__ void read_v_half(const uint32_t (&av)[D / 32], bf16x4 (&vh)[D / 32][2])
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        ds_read_vt_imm<SLOT * Lds<D>::STAGE + (16 * MM) * Lds<D>::ROWB>(av[dt], vh[dt][0]);
        ds_read_vt_imm<SLOT * Lds<D>::STAGE + (16 * MM + 4) * Lds<D>::ROWB>(av[dt], vh[dt][1]);
    }
}
// the same reads with the stage address in a register (prologue and epilogue of the loop)
template <int D, int HALF> __device__ __forceinline__ void read_k_half_at(uint32_t a, u32x4 (&kh)[D / 32])
{
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        const uint32_t addr = a ^ (uint32_t)((HALF * (D / 32) + s) << 5);
        asm volatile("ds_read_b128 %0, %1" : "=v"(kh[s]) : "v"(addr));
    }
}
template <int D, int MM> __device__ __forceinline__ void read_v_half_at(uint32_t a, bf16x4 (&vh)[D / 32][2])
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        const uint32_t addr = a ^ (uint32_t)(dt << 6);
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(vh[dt][i]) : "v"(addr), "n"((16 * MM + 4 * i) * Lds<D>::ROWB));
    }
}
// Wait until at most YOUNGER LDS reads issued after these are still in flight (the counter completes in order).
template <int KH, int YOUNGER> __device__ __forceinline__ void wait_k_half(u32x4 (&kh)[KH])
{
    static_assert((KH == 2 || KH == 4) && YOUNGER >= 0 && YOUNGER < 16, "D in {64,128}");
    if constexpr (KH == 4) asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(kh[0]), "+v"(kh[1]), "+v"(kh[2]), "+v"(kh[3]) : "n"(YOUNGER));
    else asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(kh[0]), "+v"(kh[1]) : "n"(YOUNGER));
}
template <int DT, int YOUNGER> __device__ __forceinline__ void wait_v_half(bf16x4 (&vh)[DT][2])
{
    static_assert((DT == 2 || DT == 4) && YOUNGER >= 0 && YOUNGER < 16, "D in {64,128}");
    if constexpr (DT == 4)
        asm volatile("s_waitcnt lgkmcnt(%8)"
                     : "+v"(vh[0][0]), "+v"(vh[0][1]), "+v"(vh[1][0]), "+v"(vh[1][1]), "+v"(vh[2][0]), "+v"(vh[2][1]),
                       "+v"(vh[3][0]), "+v"(vh[3][1])
                     : "n"(YOUNGER));
    else
        asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(vh[0][0]), "+v"(vh[0][1]), "+v"(vh[1][0]), "+v"(vh[1][1]) : "n"(YOUNGER));
}
// half of S^T = K . Q^T: contraction steps HALF * DS/2 .. on top of c
template <int DS, int HALF>
__device__ __forceinline__ f32x16 qk_half(const u32x4 (&kh)[DS / 2], const bf16x8 (&qreg)[DS], f32x16 c)
{
#pragma unroll
    for (int k = 0; k < DS / 2; ++k)
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kh[k]), qreg[HALF * (DS / 2) + k], c, 0, 0, 0);
    return c;
}
// half of O^T += V^T . P^T: the keys of one P operand
template <int DT> __device__ __forceinline__ void pv_half(const bf16x4 (&vh)[DT][2], const bf16x8 &pbm, f32x16 (&oacc)[DT])
{
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        const bf16x8 a = __builtin_shufflevector(vh[dt][0], vh[dt][1], 0, 1, 2, 3, 4, 5, 6, 7);
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pbm, oacc[dt], 0, 0, 0);
    }
}

template <int N> __device__ __forceinline__ void wait_vmcnt()
{
    static_assert(N >= 0 && N < 64, "vmcnt range");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Wait until at most `tiles` (wave-uniform, clamped to [0, MAXT]) tiles of LPW fills each are in flight.
template <int LPW, int MAXT> __device__ __forceinline__ void wait_tiles(int tiles)
{
    static_assert(MAXT * LPW < 64, "vmcnt range");
    if constexpr (MAXT > 0) {
        if (tiles >= MAXT) { wait_vmcnt<MAXT * LPW>(); return; }
        wait_tiles<LPW, MAXT - 1>(tiles);
    } else {
        wait_vmcnt<0>();
    }
}

// LDS map of one workgroup: the ring of NT stages; the query tiles (one per row-wave: its 32 rows as they lie in
// memory, 2*D bytes each, chunk-rotated like a bf16 K tile) in the top of the ring when the prologue's fills leave
// that free, else behind them; 9 KiB for parent[] and the ancestor sets (see PAROFF).  Queries are consumed before the main
// loop's first barrier, after which the ring owns every stage, and so are the sets where they lie in one.  The merge of the
// key-waves re-uses the same memory after the loop.
template <int D, int RW, int KW, int NT, int EB>
struct WgLds {
    static constexpr int STAGE = Lds<D, EB>::STAGE;
    static constexpr int PREFILL = KW == 1 ? (NT - 1 < 3 ? NT - 1 : 3) : NT - KW;   // tiles issued before the main loop
    static constexpr int RING = NT * STAGE;
    static constexpr int QTILE = 32 * D * 2;
    static constexpr int QBYTES = RW * QTILE;
    static constexpr int PRE_B = PREFILL * STAGE;
    static constexpr int QOFF = RING - QBYTES > PRE_B ? RING - QBYTES : PRE_B;
    // parent[] and the ancestor sets.  Shapes with two key-waves read them before the main loop: in stages the prologue leaves free, or
    // behind the query tiles where those leave less than 9 KiB of them (64 channels in the 64-row bf16 shape).  The pipelined shape reads
    // the sets after the plain prefix tiles: behind the ring.
    static constexpr int PARENTS = BTV_MAX_NODES * 4, TREEB = PARENTS + BTV_MAX_NODES * BTV_ANC_WORDS * 4;
    static constexpr int PAROFF = KW == 1 ? (RING > QOFF + QBYTES ? RING : QOFF + QBYTES) : (QOFF - PRE_B >= TREEB ? PRE_B : QOFF + QBYTES);
    static constexpr int USED = (PAROFF + TREEB > QOFF + QBYTES ? PAROFF + TREEB : QOFF + QBYTES) > RING
                                    ? (PAROFF + TREEB > QOFF + QBYTES ? PAROFF + TREEB : QOFF + QBYTES) : RING;
    static_assert(KW == 1 || KW == 2, "the merge is between two key-waves");
    static constexpr int MERGE = KW == 2 ? RW * 2 * ((D / 64) * 16 + 3) * 64 * 4 : 0;    // they exchange half a row each (+ m, l, bound)
    static constexpr int BYTES = USED > MERGE ? USED : MERGE;
    static_assert(QOFF % 1024 == 0 && PAROFF % 1024 == 0 && BYTES <= 160 * 1024, "LDS budget");
};

// Wait until at most n (wave-uniform, clamped to [0, MAXN]) vector-memory operations are in flight.
template <int MAXN> __device__ __forceinline__ void wait_vm_ops(int n)
{
    if constexpr (MAXN > 0) {
        if (n >= MAXN) { wait_vmcnt<MAXN>(); return; }
        wait_vm_ops<MAXN - 1>(n);
    } else {
        wait_vmcnt<0>();
    }
}

// A lane's query row: row r of a KV head's packed rows is node r / G, query head r % G of the group.  Worked out where
// it is needed (mask construction, final store) rather than held in registers through the main loop.  Padding rows
// (r >= rows_g) recompute row 0 and are never written.
struct LaneRow { bool valid; int node; long long orow; };
__device__ __forceinline__ LaneRow lane_row(const AttnParams &p, int r, int rows_g, int g, int q0)
{
    LaneRow x;
    x.valid = r < rows_g;
    const int rr = x.valid ? r : 0;
    x.node = (rr * p.ginv) >> 16;
    x.orow = (long long)(q0 + x.node) * p.Hq + g * p.G + (rr - x.node * p.G);       // row of Q/O as [total_M*Hq, D]
    return x;
}

// Ancestor sets of the request's nodes, set[i] = {i} u set[parent[i]], by the threads of the workgroup, one per node: a thread
// takes over what its node's ancestor has found so far and goes on from where that one has got to, so that what it knows doubles from
// turn to turn: log2 of the depth turns of some 200 cycles, where a walk along parent[] takes as many as the tree is deep (270 each; 2.8 us for a
// random tree of 33 nodes in a workgroup that all others of its group wait for, 7 for one of 60 levels).  The wavefronts do not wait for
// each other: a thread writes its set before the place to go on from, and reads the place before the set (the LDS operations of a wavefront are in
// order), so what it takes is never less than the ancestors down to that place, whoever is ahead.  Every turn moves down: places strictly decrease.
// par: parent[] as staged (entries are checked here), then the places; sets: BTV_ANC_WORDS words per node, the upper half only where
// there are more than 128 nodes.  The sets may be read behind the next barrier.
__device__ __forceinline__ void find_ancestors(const AttnParams &p, uint32_t par, uint32_t sets, int M, int tid)
{
    static_assert(BTV_ANC_WORDS == 8 && BTV_MAX_NODES <= 256, "two 16-byte pieces per set, a thread per node");
    const bool mine = tid < M, big = M > 128;                    // (big: uniform)
    const uint32_t pa = par + 4u * (uint32_t)tid, sa = sets + 32u * (uint32_t)tid;
    int at = -1;
    u32x4 lo, hi;
#pragma unroll
    for (int k = 0; k < 4; ++k) { lo[k] = tid >> 5 == k ? 1u << (tid & 31) : 0u; hi[k] = tid >> 5 == k + 4 ? 1u << (tid & 31) : 0u; }
    if (mine) {
        asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(at) : "v"(pa) : "memory");
        if (at < -1 || at >= tid) { atomicOr(p.flag, 1u); at = -1; }
    }
    auto put = [&]() {                                           // the set, then the place
        if (big) asm volatile("ds_write_b128 %0, %1 offset:16" ::"v"(sa), "v"(hi) : "memory");
        asm volatile("ds_write_b128 %0, %1\n\tds_write_b32 %2, %3" ::"v"(sa), "v"(lo), "v"(pa), "v"(at) : "memory");
    };
    if (mine) put();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();                                // all entries are checked, all sets hold their node
    while (at >= 0) {                                            // (a wavefront: while any of its lanes goes on)
        const uint32_t pb = par + 4u * (uint32_t)at, sb = sets + 32u * (uint32_t)at;
        int next;
        u32x4 l2, h2 = { 0u, 0u, 0u, 0u };
        if (big) asm volatile("ds_read_b32 %0, %3\n\tds_read_b128 %1, %4\n\tds_read_b128 %2, %4 offset:16\n\ts_waitcnt lgkmcnt(0)"
                              : "=&v"(next), "=&v"(l2), "=&v"(h2) : "v"(pb), "v"(sb) : "memory");
        else asm volatile("ds_read_b32 %0, %2\n\tds_read_b128 %1, %3\n\ts_waitcnt lgkmcnt(0)" : "=&v"(next), "=&v"(l2) : "v"(pb), "v"(sb) : "memory");
        lo |= l2; hi |= h2;
        at = next;
        put();
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// The same for up to 64 nodes, by each wavefront for itself: lane i has node i, sets and places stay in registers and move between the lanes
// (log2 of the depth turns of some 100 cycles, no barrier).  lo, hi: the set of `node`.
__device__ __forceinline__ void wave_ancestors(const AttnParams &p, uint32_t par, int M, int l, int node, uint32_t &lo, uint32_t &hi)
{
    int at;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(at) : "v"(par + 4u * (uint32_t)l) : "memory");
    if (l < M && (at < -1 || at >= l)) atomicOr(p.flag, 1u);
    if (l >= M || at >= l) at = -1;
    uint32_t a = l < 32 ? 1u << l : 0u, b = l < 32 ? 0u : 1u << (l & 31);
    while (__builtin_amdgcn_ballot_w64(at >= 0) != 0ull) {
        uint32_t a2, b2;
        int next;
        asm volatile("ds_bpermute_b32 %0, %3, %4\n\tds_bpermute_b32 %1, %3, %5\n\tds_bpermute_b32 %2, %3, %6\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(a2), "=&v"(b2), "=&v"(next) : "v"(at < 0 ? 4 * l : 4 * at), "v"(a), "v"(b), "v"(at));
        a |= a2; b |= b2;                                        // (a lane that is done takes its own)
        at = next;
    }
    asm volatile("ds_bpermute_b32 %0, %2, %3\n\tds_bpermute_b32 %1, %2, %4\n\ts_waitcnt lgkmcnt(0)" : "=&v"(lo), "=&v"(hi) : "v"(4 * node), "v"(a), "v"(b));
}

// Largest finite magnitude of a lane's values: what its row's partials are divided by.  (An infinite one, from a value in the
// cache or a sum past the end of fp32, would leave nothing of the row's other channels.)
template <int B> __device__ __forceinline__ float finite_max(f32x16 (&x)[B])
{
    float a = 0.f;
    // x may be the result of matrix instructions that are still under way, and the compiler puts no wait states ahead of inline assembly
    // (ahead of a vector instruction of its own 12 for a 32x32x16).  The maxima follow these by way of a, the x by being passed through.
#pragma unroll
    for (int b = 1; b < B; ++b) asm volatile("" : "+v"(x[b]));
    asm volatile("s_nop 7\n\ts_nop 3" : "+v"(x[0]), "+v"(a));
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
        for (int v = 0; v < 16; v += 2)              // (fmaxf of fabsf's takes three instructions a value: each is made canonical first)
            asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(a) : "v"(x[b][v]), "v"(x[b][v + 1]));
    if (__builtin_amdgcn_ballot_w64(a > FLT_MAX) != 0ull) {        // (rare)
        a = 0.f;
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) a = fabsf(x[b][v]) <= FLT_MAX ? fmaxf(a, fabsf(x[b][v])) : a;
    }
    return fmaxf(a, __shfl_xor(a, 32));             // the other half of the wave holds the row's other channels
}

// What one workgroup does in one go: rows of row block `by` of (request, KV head g) against the tiles st0 .. st1 - 1.
constexpr int COHERENT = 16;            // of a buffer access: SC1, at the scope of the device
struct Piece {
    int rq, g, by, st0, st1;
    int bx;                       // which partial of its rows this is
    int direct;                   // the only one: O is written
    int grouped;                  // its partial is `pitch` rows on end in the place of the group (merge_group)
    int group, pitch;
    // chunks only
    int node0, nodes;             // the row block's nodes
    int prow0;                    // where its partial's rows begin
};

// A page window (32 tiles' page ids) per 256 bytes, four of them in turn, behind everything else; not where two workgroups
// fill the LDS of a CU to the last byte.
template <int D, int RW, int KW, int NT, bool PAGED, int EB>
struct PageLds {
    static constexpr int BASE = WgLds<D, RW, KW, NT, EB>::BYTES;
    static constexpr int PER_CU = RW * KW <= 4 ? 2 : 1;          // workgroups that are to share a CU
    static constexpr bool USED = PAGED && (BASE + 1024) * PER_CU <= 160 * 1024;
    static constexpr int BYTES = BASE + (USED ? 1024 : 0);
};

// Workgroup = RW row-waves x KW key-waves; wave (rw, kw) owns query rows [32 rw, 32 rw + 32) of the block and,
// in every round of KW consecutive tiles, tile number kw.  LDS ring of NT tiles; one barrier per round.
// begun(): called once the first loads are on their way (by all threads).
// CAUSAL: rows of a chunk of a sequence in place of a tree's.  A row block then holds whole nodes (pc_.nodes from pc_.node0 on, G rows each), a row sees
// every key up to its own, what is plain is what all rows of the block see, and the queries are not scaled.
template <int D, int RW, int KW, int NT, bool PAGED, int EB, bool CAUSAL = false, bool THROUGH = true, typename Begun>
__device__ __forceinline__ void attn_piece(const AttnParams &p, unsigned char *smem, int tid, const Req &rq_, const Piece &pc_, Begun begun)
{
    static_assert(EB == 2 || (EB == 1 && KW >= 2), "FP8 K/V runs in the shapes whose waves alternate over the tiles");
    constexpr int WAVES = RW * KW;
    constexpr int WR = RW * 32;
    constexpr int DS = D / 16;
    constexpr int DT = D / 32;
    constexpr int LPW = Lds<D, EB>::INSTR / WAVES;       // fill instructions per wave and tile
    constexpr int AHEAD = NT - 2 * KW;            // tiles still in flight when a round's tiles have landed
    static_assert(AHEAD >= 0 && AHEAD * LPW < 64, "ring too small or too deep for the counter");
    using LD = Lds<D, EB>;
    using PL = PageLds<D, RW, KW, NT, PAGED, EB>;
    constexpr bool PGV = PL::USED;
    const int w = tid >> 6, l = tid & 63, c = l & 31, h = l >> 5;
    const int kw = w % KW, rw = w / KW;
    const int rq = pc_.rq, g = pc_.g, by = pc_.by, bx = pc_.bx;
    const int Mr = rq_.M, Lr = CAUSAL ? rq_.L + pc_.node0 + 1 : rq_.L;           // (Lr: keys that every row sees)
    const int S = CAUSAL ? rq_.L + pc_.node0 + pc_.nodes : Lr + Mr;
    const int rows_g = Mr * p.G;
    const int st0 = pc_.st0;
    int st1 = pc_.st1;
    const std::conditional_t<CAUSAL, float, NoFactor> cf = [&] { if constexpr (CAUSAL) return p.scale_log2; else return NoFactor{}; }();
    // row x of a chunk's block (as lane_row); whether a row-wave has any
    auto chunk_row = [&](int x) {
        LaneRow r;
        const int n = (x * p.ginv) >> 16;
        r.valid = n < pc_.nodes;
        r.node = r.valid ? pc_.node0 + n : pc_.node0;
        r.orow = (long long)(rq_.q0 + r.node) * p.Hq + g * p.G + (r.valid ? x - n * p.G : 0);
        return r;
    };
    auto has_rows = [&](int wave) {
        if constexpr (CAUSAL) return ((wave * 32 * p.ginv) >> 16) < pc_.nodes;
        else return by * WR + wave * 32 < rows_g;
    };
    if constexpr (!CAUSAL) {   // tree rows past the last node of this row block are invisible to all of its rows: their tiles are dropped
        const int node_hi = ((min((by + 1) * WR, rows_g) - 1) * p.ginv) >> 16;
        st1 = min(st1, max((Lr + node_hi + 1 + 31) / 32, st0 + 1));
    }

    using WL = WgLds<D, RW, KW, NT, EB>;

    // ---- prologue loads, oldest first: the first two page windows, parent[] (one entry per thread), this wave's share of
    // its row-wave's query tile, the first ring tiles.  All are raw instructions counted by hand.
    const int32_t *bt_row = PAGED ? p.block_table + (long long)rq * p.max_blocks : nullptr;
    auto load_window = [&](int g_) {                     // page ids of tiles st0 + 32 g_ .. + 31 (by the first wave)
        const int32_t *src = bt_row + min(2 * (st0 + 32 * g_) + l, (S - 1) >> 4);
        __builtin_amdgcn_global_load_lds(src, BTV_LDS_PTR(smem + PL::BASE + (g_ & 3) * 256), 4, 0, 0);
    };
    if (PGV && __builtin_amdgcn_readfirstlane(w) == 0) { load_window(0); load_window(1); }
    // parent[]: every wave moves 64 entries straight into LDS (index clamped to the request's nodes), whether or not
    // the workgroup reaches the tree rows; entries are checked where they are read.
    if constexpr (!CAUSAL)
#pragma unroll
    for (int i0 = 0; i0 < BTV_MAX_NODES; i0 += WAVES * 64)
        if (tid + i0 < BTV_MAX_NODES) {              // wave-uniform: whole waves
            const int32_t *pp = p.parent + rq_.q0 + min(tid + i0, Mr - 1);
            const int dst = __builtin_amdgcn_readfirstlane(WL::PAROFF + ((tid + i0) >> 6) * 256);
            __builtin_amdgcn_global_load_lds(pp, BTV_LDS_PTR(smem + dst), 4, 0, 0);
        }
    // Query tile: direct-to-LDS like a K tile (each wave instruction moves 1 KiB: whole rows, coalesced); as
    // per-lane operand loads the same bytes cost 64 separate 16-byte pieces per instruction and held the ring fills
    // back by about two microseconds.  The KW waves of a row-wave share the tile's instructions.
    constexpr int QCH = D / 8, QRPI = 1024 / (2 * D), QINSTR = WL::QTILE / 1024, QPW = QINSTR / KW;
    static_assert(QPW * KW == QINSTR, "query tile instructions must divide over the key-waves");
#pragma unroll
    for (int jj = 0; jj < QPW; ++jj) {
        const int j = kw * QPW + jj;
        const int qrow = j * QRPI + l / QCH, pc = l % QCH;
        const int rf = by * WR + rw * 32 + qrow;
        long long of;
        if constexpr (CAUSAL) of = chunk_row(rw * 32 + qrow).orow; else of = lane_row(p, rf, rows_g, g, rq_.q0).orow;
        const unsigned char *src = static_cast<const unsigned char *>(p.Q) + of * (D * 2) + ((pc ^ swz_k<D, 2>(qrow)) << 4);
        // the destination must be wave-uniform: rw and kw are, but the compiler cannot know
        const int dst = __builtin_amdgcn_readfirstlane(WL::QOFF + rw * WL::QTILE + j * 1024);
        __builtin_amdgcn_global_load_lds(src, BTV_LDS_PTR(smem + dst), 16, 0, 0);
    }

    // ---- start filling the ring ------------------------------------------------------------------------
    const int wu = __builtin_amdgcn_readfirstlane(w);
    Fill<D, WAVES, PAGED, EB> fill = make_fill<D, WAVES, PAGED, EB>(p.K, p.V, bt_row, p.num_blocks, p.Hkv, g, S, wu, l);
    // KW == 1: three tiles up front (the first compute needs two), the rest of the ring fills during the first
    // rounds; an issue holds its wave for about a hundred cycles, so a full prefill would only delay the start.
    constexpr int PREFILL = WL::PREFILL;
    int issued = st0, islot = 0;
    if constexpr (CAUSAL) {                              // (the first pages' ids in one round trip: one after the other they are 1.5 us of a piece)
        int id[PREFILL];
#pragma unroll
        for (int k = 0; k < PREFILL; ++k) id[k] = fill.page_id(st0 + k);
#pragma unroll
        for (int k = 0; k < PREFILL; ++k)
            if (issued < st1) {
                issue_tile<D, WAVES, PAGED, EB, 0, LPW, false, true>(fill, smem, islot, issued, wu, l, id[k]);
                ++issued; ++islot;
            }
    } else
#pragma unroll
    for (int k = 0; k < PREFILL; ++k)
        if (issued < st1) {
            issue_tile<D, WAVES, PAGED, EB>(fill, smem, islot, issued, wu, l);
            ++issued; ++islot;
        }
    if (islot >= NT) islot -= NT;

    // ---- parent[] and the query tile have landed when only the ring fills are in flight ------------------------
    wait_vm_ops<PREFILL * LPW>((issued - st0) * LPW);
    // A bare barrier, and raw LDS reads below: with the fence of a full synchronisation, or with ordinary reads of
    // memory that direct-to-LDS loads wrote, the compiler drains the ring fills first.
    __builtin_amdgcn_s_barrier();                    // query tiles (filled by KW waves), parent[] and the page windows are visible
    // The window that tile `issued` belongs to, once per 32 tiles; the first wave asks for the one after it, which is there long
    // before it is read: the ring's waits cover every older load, and a barrier follows each of them.
    auto turn_window = [&]() {
        if constexpr (PGV) {
            const int g_ = (issued - st0) >> 5;
            int v;
            asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)"
                         : "=v"(v) : "v"((uint32_t)(uintptr_t)BTV_LDS_PTR(smem) + PL::BASE + (uint32_t)((g_ & 3) * 256 + (l & 31) * 8 + fill.half * 4)) : "memory");
            fill.pages = (uint32_t)fill.valid_page(v);
            if (g_ > 0 && wu == 0) load_window(g_ + 1);
        }
    };
    auto next_window = [&]() { if (PGV && ((issued - st0) & 31) == 0) turn_window(); };
    // Where tiles follow each other of which all keys exist, a fill is a scalar base, the lane's fixed offset and a stage's address: nothing is tested
    // and, with a page per wave and tile, one id is looked up.  With a test for every fill and both pages of a tile worked out for each, fills
    // were 90 of a trip's 250 instructions in the pipelined loop of a paged cache and several branches (8 requests of 1k to 16k, a layer 163 -> 146 us; FP8
    // 171 -> 149), and 60 of a round's 300 in the contiguous shapes with two key-waves (64 nodes, 2048 keys 11.0 -> 10.6 us; FP8, 5000 keys 14.7 -> 13.5).
    const uint32_t tile_bytes = 32 * fill.row_bytes;
    const unsigned char *ahead = nullptr;                // contiguous: tile `issued`, where whole tiles follow each other
    int ids[KW] = {};                                    // paged without a window: the pages of the next KW tiles, asked for a round ahead
    auto whole_src = [&]() {                             // where this wave's rows of tile `issued` lie, if all of its keys exist
        if constexpr (!PAGED) {
            const unsigned char *src = ahead;
            ahead += tile_bytes;
            asm volatile("" : "+s"(src));                // (a scalar base and the lane's offset; else a pointer per fill and lane is carried along)
            return src;
        } else if constexpr (PGV) {
            const unsigned char *src = fill.page(__builtin_amdgcn_readlane((int)fill.pages, (issued - st0) & 31));
            asm volatile("" : "+s"(src));
            return src;
        } else {
            const unsigned char *src = fill.page(fill.valid_page(ids[0]));
            if (KW > 1) ids[0] = ids[KW - 1];
            ids[KW - 1] = fill.page_id(issued + KW);
            return src;
        }
    };
    auto whole_tiles = [&]() {                           // ahead of the first of a row of them
        if constexpr (!PAGED) ahead = fill.base + (size_t)issued * tile_bytes;
        else if constexpr (!PGV)
#pragma unroll
            for (int k = 0; k < KW; ++k) ids[k] = fill.page_id(issued + k);
    };
    turn_window();
    begun();
    const bool tree_wg = !CAUSAL && st1 * 32 > Lr;   // this workgroup's keys reach the tree rows
    const uint32_t par_lds = (uint32_t)(uintptr_t)BTV_LDS_PTR(smem) + WL::PAROFF, sets_lds = par_lds + WL::PARENTS;
    static_assert(WAVES * 64 >= BTV_MAX_NODES, "find_ancestors: a thread per node");
    if (tree_wg && Mr > 64) find_ancestors(p, par_lds, sets_lds, Mr, tid);
    // Operand s holds the 8 channels that contraction step s takes from this lane's half: 16 s + 8 h .. + 7 for
    // bf16 K, 32 (s/2) + 16 h + 8 (s%2) .. + 7 for FP8 K (the order of its 16-byte operand reads).
    u32x4 qv[DS];
    {
        const uint32_t qa = (uint32_t)(uintptr_t)BTV_LDS_PTR(smem) + WL::QOFF + rw * WL::QTILE + c * (2 * D);
        const int sw = swz_k<D, 2>(c);
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            const int chunk = EB == 2 ? 2 * s + h : 4 * (s / 2) + 2 * h + (s % 2);
            const uint32_t addr = qa + (uint32_t)((chunk ^ sw) << 4);
            asm volatile("ds_read_b128 %0, %1" : "=v"(qv[s]) : "v"(addr));
        }
    }

    // ---- ancestor bitmask of this lane's node, only in workgroups whose keys reach the tree rows ----------
    // Shapes whose waves alternate over the tiles keep the sets inside the ring and read theirs before the main loop; the pipelined
    // shape keeps them behind the ring and reads them after the plain prefix tiles, so that they are not live through that loop.
    uint32_t anc_i[BTV_ANC_WORDS];
    LastKey last = { 0, false };
    if constexpr (!CAUSAL)
#pragma unroll
    for (int k = 0; k < BTV_ANC_WORDS; ++k) anc_i[k] = 0u;
    auto read_mask = [&]() {
        if constexpr (CAUSAL) { last.key = rq_.L + chunk_row(rw * 32 + c).node; return; }
        if (!tree_wg) return;
        const int node = lane_row(p, by * WR + rw * 32 + c, rows_g, g, rq_.q0).node;
        if (Mr <= 64) {
            wave_ancestors(p, par_lds, Mr, l, node, anc_i[0], anc_i[1]);
            return;
        }
        const uint32_t a = sets_lds + (uint32_t)node * (BTV_ANC_WORDS * 4);
        u32x4 lo, hi = { 0u, 0u, 0u, 0u };
        if (Mr > 128) asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:16\n\ts_waitcnt lgkmcnt(0)" : "=&v"(lo), "=&v"(hi) : "v"(a) : "memory");
        else asm volatile("ds_read_b128 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(lo) : "v"(a) : "memory");
#pragma unroll
        for (int k = 0; k < 4; ++k) { anc_i[k] = lo[k]; anc_i[k + 4] = hi[k]; }
    };
    if constexpr (KW > 1) {
        if (tree_wg && Mr > 64) __builtin_amdgcn_s_barrier();    // every wave's sets are there
        read_mask();
    }

    float m_run = NEG_BIG, l_run = 0.f;
    float base = 0.f;                 // what the step-by-step tiles' scores are relative to (rebase_tile)
    f32x16 negb;
#pragma unroll
    for (int v = 0; v < 16; ++v) negb[v] = 0.f;
    f32x16 oacc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) oacc[dt][v] = 0.f;

    bf16x8 qreg[DS];
    if constexpr (DS == 8)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(qv[0]), "+v"(qv[1]), "+v"(qv[2]), "+v"(qv[3]), "+v"(qv[4]), "+v"(qv[5]), "+v"(qv[6]), "+v"(qv[7]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(qv[0]), "+v"(qv[1]), "+v"(qv[2]), "+v"(qv[3]));
    const uint32_t ring = (uint32_t)(uintptr_t)BTV_LDS_PTR(smem);
    auto issue_one = [&]() {                             // the next tile of this split, if there is one
        if (issued < st1) {
            next_window();
            issue_tile<D, WAVES, PAGED, EB, 0, LPW, PGV>(fill, smem, islot, issued, wu, l, (issued - st0) & 31);
            ++issued;
            if (++islot == NT) islot = 0;
        }
    };
    // one half of the wave's fills of the next tile (LPW = 2 in the pipelined shape); the caller advances the counters
    auto issue_part = [&](auto part) {
        constexpr int P = decltype(part)::value;
        constexpr int MID = (LPW + 1) / 2, JB = P == 0 ? 0 : MID, JE = P == 0 ? MID : LPW;
        if constexpr (JB < JE)
            issue_tile<D, WAVES, PAGED, EB, JB, JE, PGV>(fill, smem, islot, issued, wu, l, (issued - st0) & 31);
    };
    // the same of a tile whose 32 keys all exist; src: its first row, or that of the wave's page of it
    auto issue_whole = [&](auto part, auto parts, int slot, const unsigned char *src) {
        constexpr int P = decltype(part)::value, N = decltype(parts)::value;
#pragma unroll
        for (int jj = 0; jj < LPW; ++jj)
            if (N == 1 || (P == 0) == (jj < (LPW + 1) / 2))
                fill_lds(src + fill.lane_off[jj], smem + slot * LD::STAGE + (wu * LPW + jj) * 1024);
    };
    if constexpr (KW == 1) {
        // Every wave has its queries in registers (parent[] and the sets lie behind the ring): the ring owns all stages from here on.
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int k = PREFILL; k < NT - 1; ++k) issue_one();
    }
    // At the top of the round starting at tile st (KW > 1), tiles st+KW .. issued-1 may still be in flight.  The
    // barrier also tells that every wave is done with the previous round, whose KW ring slots the next
    // issues overwrite (in front of the first round: with the queries' tiles and the ancestor sets).
    auto begin_round = [&](int st) {
        if (issued - st - KW == AHEAD) wait_vmcnt<AHEAD * LPW>();
        else wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();
#pragma unroll
        for (int k = 0; k < KW; ++k) issue_one();
    };
    // The first round, of which the queries' scaling (160 instructions) hides the wait or the loads: with four waves the next fills are four to a wave and
    // go out after it (32 nodes over 8192 keys 15.8 -> 15.6 us, 1500 keys 8.9 -> 8.7; FP8, 33 over 12003 18.3 -> 18.0), with eight two and ahead of it
    // (64 and 100 nodes 0.5 % slower the other way).
    constexpr bool SCALED_FIRST = KW > 1 && RW == 2;
    if constexpr (KW > 1 && !SCALED_FIRST) begin_round(st0);
    if constexpr (CAUSAL) {
#pragma unroll
        for (int s = 0; s < DS; ++s) qreg[s] = __builtin_bit_cast(bf16x8, qv[s]);
    } else
    // The queries take the softmax scale and the change of base once (rounded to bf16 again, to nearest even: a
    // relative 2^-9 per element, as if the caller's projection had produced the scaled queries): scores then
    // are in log2 units and a probability costs no multiply.
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const float qs = p.scale_log2;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            u32x4 r;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t wd = qv[s][j];
                const bf16x2 pr = { (__bf16)(__uint_as_float(wd << 16) * qs), (__bf16)(__uint_as_float(wd & 0xFFFF0000u) * qs) };
                r[j] = __builtin_bit_cast(uint32_t, pr);
            }
            qreg[s] = __builtin_bit_cast(bf16x8, r);
            if constexpr (SCALED_FIRST) asm volatile("" : "+v"(qreg[s]));
        }
    }
    if constexpr (SCALED_FIRST) begin_round(st0);
    if constexpr (KW == 1 && EB == 2) {
        // ---- main loop, one tile per round, software-pipelined over the plain prefix tiles ------------------------
        // Local tile j = tile st0 + j lives in ring slot j % NT.  Tiles whose 32 keys all are prefix rows ("plain":
        // no mask) run through a pipeline in which iteration i issues
        //     the PV MFMAs of tile i-1 among the exponentials of tile i,  then the score MFMAs of tile i+1.
        // Scores come out of the matrix cores relative to the running reference (the accumulator starts at minus
        // the reference), so P = exp2(x) with no other arithmetic per element.  The reference is the maximum of
        // the split's first tile and moves only when a tile's row sum shows that some x exceeded 16 (checked on
        // the sum: no maximum per tile); then the tile is redone against its own maximum and everything rescaled.
        // K and V^T operands live in two half-tile buffers, each refilled right after the MFMAs that read it.
        static_assert(NT == 8, "the pipelined loop is written for a ring of 8 stages");
        constexpr int KH = DS / 2;                               // LDS reads per K half (a V^T half takes 2 * DT)
        int Tf = min(st1, Lr / 32) - st0;                        // plain tiles at the start of this split
        if (Tf < 3) Tf = 0;
        int j0 = 0;                                              // first local tile the step-by-step loop below takes
        // A wave whose 32 rows all lie past the request's last row has nothing to compute: it takes its share of the fills and
        // its part in every barrier, and leaves its SIMD to the other wave there.
        if (!has_rows(__builtin_amdgcn_readfirstlane(rw))) {
            if (Tf > 0) {
                wait_tiles<LPW, NT - 4>(issued - st0 - 3);
                __builtin_amdgcn_s_barrier();
                for (int i = 1; i <= Tf - 2; ++i) {
                    wait_tiles<LPW, 3>(issued - st0 - i - 3);
                    __builtin_amdgcn_s_barrier();
                    issue_one();
                }
            }
            for (int j = Tf; j < st1 - st0; ++j) {
                wait_tiles<LPW, NT - 1>(issued - st0 - j - 1);
                __builtin_amdgcn_s_barrier();
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (issued - st0 - j < NT) issue_one();
            }
            wait_vmcnt<0>();
            return;
        }
        if (Tf > 0) {
            const uint32_t kbase = ring + lane_k_off<D>(l), vbase = ring + LD::TILEB + lane_v_off<D>(l);
            auto slot_off = [](int j) { return (uint32_t)((j & (NT - 1)) * LD::STAGE); };      // wave-uniform
            u32x4 kh[KH];
            bf16x4 vh[DT][2];
            f32x16 x;
            bf16x8 pa[2], pc[2];
            float negm;                                          // minus the reference: what the score accumulator starts from
            f32x16 negm16;                                       // ... kept splatted: the first score MFMA of a tile takes it as its
                                                                 // addend and writes x, so no tile pays sixteen moves for it
            // the tile's probabilities against a new reference: its own maximum joins the old one; sums, accumulator follow
            auto regrow = [&](bf16x8 (&pn)[2], float &ts) {
                const float dlt = fmaxf(tile_max(x), 0.f), alpha = __builtin_amdgcn_exp2f(times(-dlt, cf));
                negm -= dlt;
#pragma unroll
                for (int v = 0; v < 16; ++v) negm16[v] = negm;
                l_run *= alpha;
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] -= dlt;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) oacc[dt][v] *= alpha;
                ts = 0.f;
                exp_half(x, 0, pn[0], ts, cf);
                exp_half(x, 1, pn[1], ts, cf);
            };
            // tiles 0 .. 2 have landed when at most the later ones are in flight
            wait_tiles<LPW, NT - 4>(issued - st0 - 3);
            __builtin_amdgcn_s_barrier();
            // ---- prologue: scores of tile 0 set the reference; its probabilities; scores of tile 1 ----
            {
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] = 0.f;
                read_k_half_at<D, 0>(kbase, kh); wait_k_half<KH, 0>(kh); x = qk_half<DS, 0>(kh, qreg, x);
                read_k_half_at<D, 1>(kbase, kh); wait_k_half<KH, 0>(kh); x = qk_half<DS, 1>(kh, qreg, x);
                read_k_half_at<D, 0>(kbase + slot_off(1), kh);
                negm = -tile_max(x);
                negm = negm <= FLT_MAX ? negm : NO_SCORE;        // (a row of which this tile's scores all are -infinity: see rebase_tile)
#pragma unroll
                for (int v = 0; v < 16; ++v) x[v] += negm;
                exp_half(x, 0, pa[0], l_run, cf);                // x <= 0 here: no growth check
                exp_half(x, 1, pa[1], l_run, cf);
#pragma unroll
                for (int v = 0; v < 16; ++v) negm16[v] = negm;
                wait_k_half<KH, 0>(kh); x = qk_half<DS, 0>(kh, qreg, negm16);
                read_k_half_at<D, 1>(kbase + slot_off(1), kh); wait_k_half<KH, 0>(kh); x = qk_half<DS, 1>(kh, qreg, x);
                read_v_half_at<D, 0>(vbase, vh);                 // queue: V(0) first half, K(2) low half
                read_k_half_at<D, 0>(kbase + slot_off(2), kh);
            }
            // ---- iteration i (1 <= i <= Tf - 2): x holds the scores of tile i, pprev the probabilities of tile i-1, pcur
            // receives those of tile i ----
            // On entry the LDS queue holds [V(i-1) first half, K(i+1) low half].
            // Loop-invariant operand addresses for the trips whose ring slots are known at compile time (eight trips
            // unrolled, one per slot): the slot is an immediate offset then, which reaches four slots from one base,
            // and a trip needs no address arithmetic at all (20 instructions of it otherwise).
            uint32_t ak[DS], akh[DS], av[DT], avh[DT];
#pragma unroll
            for (int s2 = 0; s2 < DS; ++s2) { ak[s2] = kbase ^ (uint32_t)(s2 << 5); akh[s2] = ak[s2] + 4u * LD::STAGE; }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) { av[dt] = vbase ^ (uint32_t)(dt << 6); avh[dt] = av[dt] + 4u * LD::STAGE; }
            auto rk = [&](auto slot, auto half) {
                constexpr int S = decltype(slot)::value & 7, H = decltype(half)::value;
                if constexpr (S < 4) read_k_half<D, S, H>(ak, kh); else read_k_half<D, S - 4, H>(akh, kh);
            };
            auto rv = [&](auto slot, auto mm) {
                constexpr int S = decltype(slot)::value & 7, MM = decltype(mm)::value;
                if constexpr (S < 4) read_v_half<D, S, MM>(av, vh); else read_v_half<D, S - 4, MM>(avh, vh);
            };
            // ph: the trip's tile number modulo 8 as a constant, or -1 for a trip with its addresses in registers
            // steady: the tile that this trip asks for exists, and so do all of its keys
            auto iter = [&](bf16x8 (&pprev)[2], bf16x8 (&pcur)[2], int i, auto ph, auto steady) {
                constexpr int PH = decltype(ph)::value;
                constexpr bool STEADY = decltype(steady)::value;
                using C0 = std::integral_constant<int, 0>;
                using C1 = std::integral_constant<int, 1>;
                // tiles <= i+2 are read in this iteration; the barrier also tells that every wave is done with
                // iteration i-1, i.e. with tile i-2, whose slot the next fill takes
                const unsigned char *src = nullptr;
                bool fill_now = true;                            // tile i+6 goes into the slot tile i-2 left
                if constexpr (STEADY) {
                    wait_vmcnt<3 * LPW>();
                    __builtin_amdgcn_s_barrier();
                    if constexpr (((PH + 6) & 7) == 0) next_window();
                    src = whole_src();
                } else {
                    wait_tiles<LPW, 3>(issued - st0 - i - 3);
                    __builtin_amdgcn_s_barrier();
                    fill_now = issued < st1;
                    if (fill_now) next_window();
                }
                auto fill_half = [&](auto part) {
                    if constexpr (STEADY) issue_whole(part, std::integral_constant<int, 2>{}, (PH + 6) & 7, src);
                    else if (fill_now) issue_part(part);
                };
                uint32_t k1 = 0, k2 = 0, v0 = 0, v1 = 0;
                if constexpr (PH < 0) {
                    k1 = kbase + slot_off(i + 1); k2 = kbase + slot_off(i + 2);
                    v0 = vbase + slot_off(i - 1); v1 = vbase + slot_off(i);
                }
                float ts = 0.f;
                wait_v_half<DT, KH>(vh);                          // V(i-1) first half
                pv_half<DT>(vh, pprev[0], oacc);
                fill_half(C0{});                                  // behind four MFMAs: its issue stall is covered
                if constexpr (PH < 0) read_v_half_at<D, 1>(v0, vh);                     // V(i-1) second half  queue: K(i+1)lo, V(i-1)b
                else rv(std::integral_constant<int, PH + 7>{}, C1{});
                __builtin_amdgcn_sched_barrier(0);
                exp_half(x, 0, pcur[0], ts, cf);
                asm volatile("" : "+v"(pcur[0]), "+v"(ts));       // (the exponentials stay between the reads and their wait)
                __builtin_amdgcn_sched_barrier(0);
                wait_v_half<DT, 0>(vh);                           // V(i-1) second half (and K(i+1) low)
                pv_half<DT>(vh, pprev[1], oacc);
                fill_half(C1{});
                if constexpr (PH < 0) read_v_half_at<D, 0>(v1, vh);                     // V(i) first half     queue: V(i)a
                else rv(std::integral_constant<int, PH>{}, C0{});
                __builtin_amdgcn_sched_barrier(0);
                exp_half(x, 1, pcur[1], ts, cf);
                asm volatile("" : "+v"(pcur[1]), "+v"(ts));
                __builtin_amdgcn_sched_barrier(0);
                if (__builtin_amdgcn_ballot_w64(!(ts <= GROW)) != 0ull) regrow(pcur, ts);     // rare
                l_run += ts;
                wait_k_half<KH, 2 * DT>(kh);                      // K(i+1) low (landed above; binds the registers)
                x = qk_half<DS, 0>(kh, qreg, negm16);
                if constexpr (PH < 0) read_k_half_at<D, 1>(k1, kh);                     // K(i+1) high         queue: V(i)a, K(i+1)hi
                else rk(std::integral_constant<int, PH + 1>{}, C1{});
                wait_k_half<KH, 0>(kh);                           // K(i+1) high (and V(i) first half)
                x = qk_half<DS, 1>(kh, qreg, x);
                if constexpr (PH < 0) read_k_half_at<D, 0>(k2, kh);                     // K(i+2) low          queue: K(i+2)lo (V(i)a has landed)
                else rk(std::integral_constant<int, PH + 2>{}, C0{});
                if constexpr (STEADY) ++issued;
                else if (fill_now) { ++issued; if (++islot == NT) islot = 0; }
            };
            // ---- epilogue: tile e = Tf - 1 has its scores, tile e-1 its probabilities (pp); nothing left to overlap ----
            auto drain = [&](bf16x8 (&pp)[2], bf16x8 (&pn)[2]) {
                const int e = Tf - 1;
                const uint32_t ve1 = vbase + slot_off(e - 1), ve = vbase + slot_off(e);
                wait_k_half<KH, 0>(kh);                          // (the low half of tile e+1's K: not used)
                wait_v_half<DT, 0>(vh);                          // V(e-1) first half
                pv_half<DT>(vh, pp[0], oacc);
                read_v_half_at<D, 1>(ve1, vh);
                float ts = 0.f;
                exp_half(x, 0, pn[0], ts, cf);
                exp_half(x, 1, pn[1], ts, cf);
                wait_v_half<DT, 0>(vh);
                pv_half<DT>(vh, pp[1], oacc);
                read_v_half_at<D, 0>(ve, vh);
                if (__builtin_amdgcn_ballot_w64(!(ts <= GROW)) != 0ull) regrow(pn, ts);
                l_run += ts;
                wait_v_half<DT, 0>(vh);
                pv_half<DT>(vh, pn[0], oacc);
                read_v_half_at<D, 1>(ve, vh);
                wait_v_half<DT, 0>(vh);
                pv_half<DT>(vh, pn[1], oacc);
                m_run = -negm;
            };
            // One iteration per trip, the new probabilities copied into place at its end (8 moves): with the roles of
            // two register sets alternating over an unrolled pair the allocator shuffles tuples and spills.
            int i = 1;
            // (the two probability buffers swap roles from trip to trip: no copies inside a group of eight)
            // (one barrier for two trips, with the fills one tile less ahead, measured the same)
#define BTV_TRIP(k, slot, from, to) iter(from, to, i + k, std::integral_constant<int, slot>{}, steady);
#define BTV_TRIPS                                                                                                             \
            BTV_TRIP(0, 1, pa, pc) BTV_TRIP(1, 2, pc, pa) BTV_TRIP(2, 3, pa, pc) BTV_TRIP(3, 4, pc, pa)                       \
            BTV_TRIP(4, 5, pa, pc) BTV_TRIP(5, 6, pc, pa) BTV_TRIP(6, 7, pa, pc) BTV_TRIP(7, 0, pc, pa)
            const int whole = min(st1, S / 32) - st0;            // tiles of this split with all keys
            whole_tiles();
            for (; i + 7 <= Tf - 2 && i + 13 < whole; i += 8) {  // tile i is in ring slot 1 here: eight trips, one per slot
                constexpr std::true_type steady;
                BTV_TRIPS
            }
            for (; i + 7 <= Tf - 2; i += 8) {
                constexpr std::false_type steady;
                BTV_TRIPS
            }
#undef BTV_TRIPS
#undef BTV_TRIP
            for (; i <= Tf - 2; ++i) {
                iter(pa, pc, i, std::integral_constant<int, -1>{}, std::false_type{});
#pragma unroll
                for (int mm = 0; mm < 2; ++mm) pa[mm] = pc[mm];
            }
            drain(pa, pc);
            j0 = Tf;
        }
        // ---- the remaining tiles (those that touch tree rows, or all of a short split), step by step ----
        if (j0 > 0) {                                            // (m_run is a maximum after the pipelined part, or -NO_SCORE)
            base = m_run;
#pragma unroll
            for (int v = 0; v < 16; ++v) negb[v] = -m_run;
        }
        read_mask();                                             // (barriers since the sets were written: those of the prologue)
        for (int j = j0; j < st1 - st0; ++j) {
            wait_tiles<LPW, NT - 1>(issued - st0 - j - 1);       // tile j has landed
            __builtin_amdgcn_s_barrier();                        // ... for every wave, and all are done with tile j-1
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (issued - st0 - j < NT) issue_one();
            if constexpr (CAUSAL) do_tile<D, false>(ring + (j & 7) * LD::STAGE, (st0 + j) * 32, Lr, l, last, qreg, m_run, l_run, oacc, base, negb, true, cf);
            else do_tile<D, false>(ring + (j & 7) * LD::STAGE, (st0 + j) * 32, Lr, l, anc_i, qreg, m_run, l_run, oacc, base, negb, true, cf);
        }
        if constexpr (PAGED) wait_vmcnt<0>();
    } else {
        // ---- main loop: one barrier per round of KW tiles, wave kw takes tile number kw of the round ------
        // (a wave whose 32 rows all lie past the last one only fills)
        const bool live = has_rows(__builtin_amdgcn_readfirstlane(rw));
        const int kwu = wu % KW;                                 // (kw, as a scalar)
        int cslot = kwu, st = st0;
        auto tile = [&](auto plain) {                            // this wave's tile of the round
            constexpr bool PLAIN = decltype(plain)::value;
            const bool exact = !PLAIN && (st == st0 || (st + kwu) * 32 + 32 > Lr);      // (constant in the first round)
            auto with = [&](auto &seen) {
                if constexpr (EB == 2)
                    do_tile<D, PLAIN>(ring + cslot * LD::STAGE, (st + kwu) * 32, Lr, l, seen, qreg, m_run, l_run, oacc, base, negb, exact, cf);
                else
                    do_tile8<D, PLAIN>(ring + cslot * LD::STAGE, (st + kwu) * 32, Lr, l, seen, qreg, m_run, l_run, oacc, base, negb, exact, cf);
            };
            if constexpr (CAUSAL) with(last); else with(anc_i);
        };
        auto next_round = [&]() {
            st += KW;
            cslot += KW;
            if (cslot >= NT) cslot -= NT;
        };
        // Rounds that ask for KW tiles of the prefix with all their keys, and so only take such, have nothing to test for.
        const int plain = min(st1, Lr / 32);
        if (live && st + kwu < st1) tile(std::false_type{});     // (on its own: nothing has to be cleared ahead of it)
        next_round();
        whole_tiles();
        for (; issued + KW <= plain; next_round()) {
            wait_vmcnt<AHEAD * LPW>();
            __builtin_amdgcn_s_barrier();
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                next_window();
                issue_whole(std::integral_constant<int, 0>{}, std::integral_constant<int, 1>{}, islot, whole_src());
                ++issued;
                if (++islot == NT) islot = 0;
            }
            if (live) tile(std::true_type{});
        }
        for (; st < st1; next_round()) {
            begin_round(st);
            if (live && st + kwu < st1) tile(std::false_type{});
        }
    }
    // A row that has met no score above -infinity has no reference, and whatever it is merged with is above it.
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(m_run == -NO_SCORE) != 0ull, 0)) {        // (rare; a maximum of just that has a sum)
        const float sum = l_run + __shfl_xor(l_run, 32);
        if (m_run == -NO_SCORE && sum == 0.f) m_run = NEG_BIG;
    }
    if constexpr (CAUSAL) m_run = fmaxf(times(m_run, cf), NEG_BIG);        // (what stands for no reference stays a number whatever the scale)
    LaneRow lrow;
    if constexpr (CAUSAL) lrow = chunk_row(rw * 32 + c); else lrow = lane_row(p, by * WR + rw * 32 + c, rows_g, g, rq_.q0);
    const bool rvalid = lrow.valid;
    const long long orow = lrow.orow;
    // both halves of a wave hold partial row sums of the same queries
    l_run += __shfl_xor(l_run, 32);

    // ---- merge the key-waves of each row-wave through LDS ---------------------------------------------------
    // Two key-waves: each keeps one half of the channels and hands the other half to its partner, so both merge,
    // scale and store half a row.  dt0 .. dt0 + DTK - 1 are the channel blocks this wave ends up with.
    int dt0 = 0;
    constexpr int DTK = KW == 2 ? DT / 2 : DT;
    float fin[DTK][16];                             // what this wave stores: its rows times `factor`
    float amax;                                     // bound on the row's largest magnitude (for the fp16 partials)
    // Partials travel as fp16 relative to (a bound within a factor two of) the row's largest magnitude, kept in fp32 beside m and l:
    // half the bytes of fp32 to write, flush at the end of the kernel and read back, at a relative error of at most 2^-10 of that
    // magnitude, below the final bf16 rounding.  (The bound stays above LEAST, so that its reciprocal is finite.)
    constexpr float LEAST = 1.0e-36f;
    auto factor = [&]() { return pc_.direct ? p.out_scale / l_run : 1.0f / amax; };
    if constexpr (KW == 2) {
        constexpr int QUADS = DTK * 4, SLOT = (DTK * 16 + 3) * 64;      // floats a wave hands over: groups of four, then m, l, bound
        float *mg = reinterpret_cast<float *>(smem) + rw * 2 * SLOT;
        amax = finite_max<DT>(oacc);
        wait_vmcnt<0>();
        __syncthreads();                            // every wave is done with the ring
        float *out = mg + kw * SLOT;
        auto give = [&](auto first) {               // the channel blocks first .. first + DTK - 1 go to the partner
            constexpr int F = decltype(first)::value;
#pragma unroll
            for (int q = 0; q < QUADS; ++q) {
                const f32x16 &o = oacc[F + q / 4];
                const f32x4 x = { o[4 * (q & 3)], o[4 * (q & 3) + 1], o[4 * (q & 3) + 2], o[4 * (q & 3) + 3] };
                reinterpret_cast<f32x4 *>(out)[q * 64 + l] = x;
            }
        };
        if (kw == 0) give(std::integral_constant<int, DTK>{}); else give(std::integral_constant<int, 0>{});
        out[(DTK * 16) * 64 + l] = m_run;
        out[(DTK * 16 + 1) * 64 + l] = l_run;
        out[(DTK * 16 + 2) * 64 + l] = CAUSAL && last.odd ? -amax : amax;
        __syncthreads();
        const float *in = mg + (kw ^ 1) * SLOT;
        const float m1 = in[(DTK * 16) * 64 + l], l1 = in[(DTK * 16 + 1) * 64 + l];
        float x1 = in[(DTK * 16 + 2) * 64 + l];
        if constexpr (CAUSAL) {                     // (the sign of a magnitude: whether the other has met a value that is no number; a bit, as the magnitude may be 0)
            if (__builtin_amdgcn_ballot_w64(__float_as_uint(x1) >> 31) != 0ull) last.odd = true;
            x1 = fabsf(x1);
        }
        f32x4 other[QUADS];
#pragma unroll
        for (int q = 0; q < QUADS; ++q) other[q] = reinterpret_cast<const f32x4 *>(in)[q * 64 + l];
        const float mn = fmaxf(m_run, m1);
        float a0 = __builtin_amdgcn_exp2f(m_run - mn);
        float a1 = __builtin_amdgcn_exp2f(m1 - mn);
        // both waves must arrive at the same l and bound: sums of the same two products, order fixed by kw
        const float la = kw == 0 ? l_run * a0 : l1 * a1, lb = kw == 0 ? l1 * a1 : l_run * a0;
        const float xa = kw == 0 ? amax * a0 : x1 * a1, xb = kw == 0 ? x1 * a1 : amax * a0;
        m_run = mn;
        l_run = la + lb;
        amax = fminf(fmaxf(xa + xb, LEAST), FLT_MAX);     // >= the merged row's largest (finite) magnitude, at most twice it
        const float f = factor();
        a0 *= f; a1 *= f;
        auto take = [&](auto first) {
            constexpr int F = decltype(first)::value;
#pragma unroll
            for (int dt = 0; dt < DTK; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) fin[dt][v] = fmaf(oacc[F + dt][v], a0, other[dt * 4 + v / 4][v & 3] * a1);
        };
        if (kw == 0) take(std::integral_constant<int, 0>{}); else take(std::integral_constant<int, DTK>{});
        dt0 = kw * DTK;                             // the kept blocks now sit in oacc[0 .. DTK)
    }
    if (!rvalid) return;
    if constexpr (KW == 1) {
        amax = fmaxf(finite_max<DT>(oacc), LEAST);
        const float f = factor();
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) fin[dt][v] = oacc[dt][v] * f;
    }
    if constexpr (CAUSAL)
        if (last.odd) {                             // (rare) the values that take_out has met, added to the rows that see them
            const int k0 = max(st0 * 32, Lr & ~31), k1 = min(st1 * 32, S);
            const unsigned char *V = static_cast<const unsigned char *>(p.V);
            for (int key = k0; key < k1; ++key) {
                const size_t row = (size_t)fill.valid_page(bt_row[key / BTV_PAGE]) * BTV_PAGE + key % BTV_PAGE;
#pragma unroll 1
                for (int dt = 0; dt < DTK; ++dt)
#pragma unroll 1
                    for (int v = 0; v < 16; ++v) {
                        const size_t at = (row * p.Hkv + g) * D + (dt0 + dt) * 32 + 8 * (v / 4) + 4 * h + v % 4;
                        float x;
                        if constexpr (EB == 1) x = __builtin_amdgcn_cvt_f32_fp8((int)V[at], 0);
                        else x = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(V)[at] << 16);
                        const float add = key <= last.key && !(fabsf(x) <= FLT_MAX) ? x : 0.f;
#pragma unroll
                        for (int b = 0; b < DTK; ++b)
#pragma unroll
                            for (int u = 0; u < 16; ++u) fin[b][u] += b == dt && u == v ? add : 0.f;
                    }
            }
        }

    // ---- write: final bf16 rows when this request has a single split, scaled fp16 partials otherwise ---
    // A lane holds channels 8 q + 4 h .. + 3 of its row, the other half of the wave the other four: they exchange every second
    // group, so that each has 8 neighbouring channels and a store instruction touches half as many pieces of rows (there
    // are 32 rows per instruction whatever its width; the stores of a 256-row workgroup took 3 us).
    auto store_rows = [&](unsigned char *row, auto pack) {
#pragma unroll
        for (int dt = 0; dt < DTK; ++dt)
#pragma unroll
            for (int q = 0; q < 4; q += 2) {
                const uint2 a = pack(dt, q), b = pack(dt, q + 1);
                const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false), y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
                *reinterpret_cast<uint4 *>(row + (dt * 32 + (q + h) * 8) * 2) = make_uint4(x[0], y[0], x[1], y[1]);
            }
    };
    if (pc_.direct) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        auto pack = [&](int dt, int q) {
            const b2 lo = { (__bf16)fin[dt][q * 4 + 0], (__bf16)fin[dt][q * 4 + 1] }, hi = { (__bf16)fin[dt][q * 4 + 2], (__bf16)fin[dt][q * 4 + 3] };
            return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
        };
        store_rows(static_cast<unsigned char *>(p.O) + (orow * D + dt0 * 32) * 2, pack);
    } else {
        const size_t prow = CAUSAL ? (size_t)(pc_.prow0 + rw * 32 + c) : pc_.grouped ? (size_t)((pc_.group * p.nsplit + bx) * pc_.pitch + rw * 32 + c) : (size_t)bx * p.total_rows + orow;
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        auto pack = [&](int dt, int q) {
            const h2 lo = { (_Float16)fin[dt][q * 4 + 0], (_Float16)fin[dt][q * 4 + 1] }, hi = { (_Float16)fin[dt][q * 4 + 2], (_Float16)fin[dt][q * 4 + 3] };
            return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
        };
        if constexpr (CAUSAL && THROUGH) {
            // past this XCD's caches: a workgroup elsewhere may merge them (all parts lie within 2^31 bytes)
            const auto rows = __builtin_amdgcn_make_buffer_rsrc(p.Opart, 0, 0x7FFFFFFF, 0x00027000), ml = __builtin_amdgcn_make_buffer_rsrc(p.ML, 0, 0x7FFFFFFF, 0x00027000);
#pragma unroll
            for (int dt = 0; dt < DTK; ++dt)
#pragma unroll
                for (int q = 0; q < 4; q += 2) {
                    const uint2 a = pack(dt, q), b = pack(dt, q + 1);
                    const auto x = __builtin_amdgcn_permlane32_swap(a.x, b.x, false, false), y = __builtin_amdgcn_permlane32_swap(a.y, b.y, false, false);
                    const u32x4 w = { (uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1] };
                    __builtin_amdgcn_raw_buffer_store_b128(w, rows, (int)((prow * D + (dt0 + dt) * 32 + (q + h) * 8) * 2), 0, COHERENT);
                }
            if (h == 0 && kw == 0) {
                const u32x4 w = { __float_as_uint(m_run), __float_as_uint(l_run), __float_as_uint(amax), 0u };
                __builtin_amdgcn_raw_buffer_store_b128(w, ml, (int)(prow * 16), 0, COHERENT);
            }
            return;
        }
        store_rows(reinterpret_cast<unsigned char *>(p.Opart) + (prow * D + dt0 * 32) * 2, pack);
        if (h == 0 && kw == 0) *reinterpret_cast<float4 *>(p.ML + prow * 4) = make_float4(m_run, l_run, amax, 0.f);
    }
}

}  // namespace
