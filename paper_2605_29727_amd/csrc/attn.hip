// Tree-masked attention for gfx950 (MI355X): ancestor bitmask, bf16 MFMA split-K kernels (one request, batches of short
// requests, batches whose workgroups share the work out; bf16 or FP8 K/V), fp32 reference-precision kernel, split-K
// combine, and their C-ABI entry points.
//
// What is computed (App. C, "Linearization and verification mask"): node i attends to the L
// prefix rows of the KV cache and to the tree rows of its ancestors and itself.
//
// bf16 kernel layout.  For one KV head the G = Hq/Hkv query heads of every node are packed
// into rows r = i*G + j, so the whole GQA group shares each K/V byte that is streamed.
// A workgroup (4 or 8 wavefronts of 64 lanes) owns WR rows and a range of 32-key tiles; K and V
// tiles are staged through LDS once per workgroup (ring of stages filled by direct-to-LDS loads).
// Scores are computed transposed, S^T = K . Q^T with 32x32x16 bf16 MFMA: in the accumulator
// layout a lane then holds ONE query column and 16 keys, so the running max / sum of the
// online softmax are per-lane scalars (one cross-half exchange per tile), the P^T tile is
// already in B-operand layout for O^T += V^T . P^T, and the O^T accumulator is rescaled by a
// per-lane factor.  V^T operands come from transposing LDS reads.  The tree mask is applied only on tiles
// that touch tree rows, from a 32-bit visibility word per (query, tile) built from the node's
// ancestor bitmask.
#include "attn_piece.h"

#include <atomic>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

namespace {

// ------------------------------------------------------------------------------------------------
// Ancestor bitmask: anc[i] = {i} u anc[parent[i]].  One workgroup, one thread per node,
// each walking its own chain (parents are strictly decreasing, so the walk ends; an out-of-range
// parent is treated as -1 and flagged).
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void anc_mask_kernel(const int32_t *parent, int M, uint32_t *anc, uint32_t *flag)
{
    __shared__ int32_t par[BTV_MAX_NODES];
    int i = threadIdx.x;
    bool bad = false;
    if (i < M) {
        int pa = parent[i];
        if (pa < -1 || pa >= i) { bad = true; pa = -1; }
        par[i] = pa;
    }
    __syncthreads();
    if (i < M) {
        uint32_t w[BTV_ANC_WORDS];
#pragma unroll
        for (int k = 0; k < BTV_ANC_WORDS; ++k) w[k] = 0u;
        for (int a = i; a >= 0; a = par[a]) {
#pragma unroll
            for (int k = 0; k < BTV_ANC_WORDS; ++k)
                if ((a >> 5) == k) w[k] |= 1u << (a & 31);
        }
        uint4 *dst = reinterpret_cast<uint4 *>(anc + (size_t)i * BTV_ANC_WORDS);
        dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
        dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
    if (bad) atomicOr(flag, 1u);
}

// Fetch every argument now, in one round trip.  Left to the compiler the scalar loads follow the early-exit tests
// in five dependent steps, three of which miss the cache (the argument block spans three lines and is cold in every
// launch): about two microseconds before the first fill is issued.
#define BTV_FETCH_ARGS(p)                                                                                                     \
    asm volatile("" ::"s"(p.Q), "s"(p.K), "s"(p.V), "s"(p.O), "s"(p.parent), "s"(p.block_table), "s"(p.q_offset),              \
                 "s"(p.prefix_len), "s"(p.Opart), "s"(p.ML), "s"(p.flag), "s"(p.sync), "s"(p.M), "s"(p.L), "s"(p.Hq), "s"(p.Hkv), "s"(p.G), "s"(p.ginv), \
                 "s"(p.max_blocks), "s"(p.num_blocks), "s"(p.total_rows), "s"(p.total_M), "s"(p.sps), "s"(p.longer), "s"(p.nsplit), \
                 "s"(p.inv_row_blocks), "s"(p.inv_nsplit), "s"(p.row_blocks), "s"(p.units), "s"(p.scale_log2), "s"(p.out_scale))

// ---- the merge inside the attention kernel --------------------------------------------------------------------------------
// A group = the workgroups whose partials belong to the same rows: the key splits of one (KV head, row block).  Where the
// launch gives every group workgroup ids that are congruent mod 8 they run on one XCD, their partials meet in that XCD's L2, and each of
// them, once all have stored theirs, merges its share of the rows (every nsplit-th) and writes O.  That takes the place of a second
// launch: the write-back of the partials between the kernels, a launch and tv_combine_bf16's own round trips.
//
// Nothing depends on where workgroups run or on whether they run at once:
// * A workgroup writes the XCD it runs on (the hardware's register) beside the call's tag when it starts, and reads its peers' words
//   at its end.  Only if all have started, and on its own XCD, it relies on the L2 ("together"); otherwise its partials are
//   released to the whole device first, and the others' acquired.  A workgroup that is together knows that all its peers are
//   on this XCD, whatever they know themselves.
// * A workgroup says that its partials are stored in a word in the L2 (near; a store of workgroup scope, which stays there), and if it is
//   not together in a word at the memory side as well (far).  It waits until all have, for `wait_ticks` at most.  If that passes it says
//   so in the same words, looks once more, at near and far words alike, and leaves if somebody still is missing.  Whoever stores
//   last sees all words, and who has left among them (each writes its own word, and has it acknowledged, before it looks at the others'), and
//   merges their shares too.  Two that do the same share write the same values.
// * "Not started": where other streams' work holds compute units, a peer may wait for the very units that the waiting workgroups hold.  So after
//   5 us it counts whether all have started, and leaves if not.  A call of 64 nodes over 8192 keys, 21 us alone, beside a kernel that holds
//   64, 128 or 192 of the 256 units: 81, 73 and 151 us with 20 us for all, 65, 58 and 106 with 5 (and 62, 54 and 97 with 2); beside the same
//   calls on another stream, whose workgroups come one after the other: 34 us with 20 or 5, but 46 with 2, as the last one then merges alone
//   what a little more patience has merged by all.  (By a second launch: 32 beside the same calls; beside such a kernel its calls
//   did not run at all until that kernel had ended.)
// * Words carry the call's tag (one more than `epoch`, which every workgroup reads at its start and whoever has seen all of the group
//   moves on), so they are never cleared and a workspace may change its sizes from call to call.
// An exchange between 32 workgroups takes 930 cycles through the L2 and 2300 at the memory side (MI355X, store to all have read).
constexpr int MERGE_WAIT_TICKS = 2000;                  // 20 us of the 100 MHz wall clock
constexpr int MERGE_START_TICKS = 500;                  // (see "not started" above)

__device__ __forceinline__ uint32_t this_xcd() { return (uint32_t)__builtin_amdgcn_s_getreg(20 | (3 << 11)); }     // HW_REG_XCC_ID, bits 3:0

// One of the group's shares: rows of, of + n, .. of the block's `rows`.  16 lanes take a row's partial of one split with one load each
// (a load holds its wave for some 80 cycles whatever its width), 4, 2 or 1 such sets of lanes of a wavefront share a row's splits out,
// by how many rows there are.  Loads go past the L1, to which the group's other workgroups do not write.  The arithmetic is combine_row's, the
// sums over the splits in another order.  What a wavefront spends its time on is one instruction after the other (two wavefronts
// on a SIMD, some 7 cycles each): offsets are worked out before the wait for the others, sums are multiply-adds on the fp16 values as they are.
template <int D, int WAVES> struct Share {
    static constexpr int E = D / 16, SETS = WAVES * 4;  // values per lane; sets of 16 lanes
    int of, count, lp;                                  // first row, number of rows, log2 of the sets per row
    int k, row, ml, part[8];                            // a set's row: which of the share's, of O; byte offsets of what it loads
    __device__ __forceinline__ void begin(int of_, int n, int rows, int tid)
    {
        of = of_;
        count = (rows - of + n - 1) / n;
        lp = 4 * count <= SETS ? 2 : 2 * count <= SETS ? 1 : 0;
        k = (tid >> 4) >> lp;
    }
    __device__ __forceinline__ void find(const AttnParams &p, const Piece &pc, int n, int wr, int tid)
    {
        const int r = of + n * k, rr = pc.by * wr + r, node = (rr * p.ginv) >> 16;
        row = node * p.Hq + pc.g * p.G + (rr - node * p.G);
        ml = (min(tid & ((16 << lp) - 1), n - 1) * pc.pitch + r) * 16;
#pragma unroll
        for (int b = 0; b < 8; ++b) part[b] = part_at(pc, b, 0, n, tid);
    }
    __device__ __forceinline__ int part_at(const Piece &pc, int b, int at, int n, int tid) const
    {
        const int s = at + ((tid >> 4) & ((1 << lp) - 1)) + (b << lp);
        return (min(s, n - 1) * pc.pitch + of + n * k) * (D * 2) + (tid & 15) * (E * 2);
    }
};

template <int D, int WAVES>
__device__ __forceinline__ void merge_share(const AttnParams &p, const Piece &pc, Share<D, WAVES> sh, int n, int wr, float *weights, int tid)
{
    constexpr int E = Share<D, WAVES>::E, PAST_L1 = 16;                 // SC1
    typedef _Float16 hvec __attribute__((ext_vector_type(E)));
    typedef __bf16 bvec __attribute__((ext_vector_type(E)));
    const int lp = sh.lp, set = tid >> 4, sub = set & ((1 << lp) - 1);
    float *wsh = weights + (set >> lp << lp) * MERGE_SPLITS;           // (by the row's first set: no other wavefront's, whatever lp is)
    const uint32_t pitch = (uint32_t)pc.pitch, first = (uint32_t)(pc.group * n) * pitch;
    const auto ml_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ML + (size_t)first * 4, 0, (int)(n * pitch * 16), 0x00027000);
    const auto part_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.Opart + (size_t)first * D, 0, (int)(n * pitch * D * 2), 0x00027000);
    const int s0 = tid & ((16 << lp) - 1), s1 = s0 + 16;                // splits whose weights this lane works out (s1: one set per row)
    while (sh.k < sh.count) {
        auto load_ml = [&](int off) { return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(ml_rsrc, off, 0, PAST_L1)); };
        const float4 m0 = load_ml(sh.ml);
        float4 m1 = make_float4(NEG_BIG, 0.f, 0.f, 0.f);
        if (lp == 0 && n > 16) m1 = load_ml((min(s1, n - 1) * pc.pitch + sh.of + n * sh.k) * 16);
        hvec part[8];
        auto load_parts = [&]() {
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                if constexpr (E == 8) part[b] = __builtin_bit_cast(hvec, __builtin_amdgcn_raw_buffer_load_b128(part_rsrc, sh.part[b], 0, PAST_L1));
                else part[b] = __builtin_bit_cast(hvec, __builtin_amdgcn_raw_buffer_load_b64(part_rsrc, sh.part[b], 0, PAST_L1));
            }
        };
        load_parts();
        auto over_row = [&](float x, auto op) {                         // over the row's 16, 32 or 64 lanes
            x = op(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, false)));      // quad_perm [1,0,3,2]
            x = op(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, false)));      // quad_perm [2,3,0,1]
            x = op(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, false)));     // row_half_mirror
            x = op(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, false)));     // row_mirror
            if (lp >= 1) {
                const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
                x = op(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
            }
            if (lp == 2) {
                const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
                x = op(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
            }
            return x;
        };
        const float x0 = s0 < n ? m0.x : NEG_BIG, x1 = s1 < n ? m1.x : NEG_BIG;
        const float mmax = over_row(lp == 0 ? fmaxf(x0, x1) : x0, [](float u, float v) { return fmaxf(u, v); });
        const float w0 = s0 < n ? __builtin_amdgcn_exp2f(x0 - mmax) : 0.f, w1 = lp == 0 && s1 < n ? __builtin_amdgcn_exp2f(x1 - mmax) : 0.f;
        // weight times the partial's magnitude; 0 past the last split.  (The row's lanes are of one wavefront: no barrier needed.)
        if (s0 < MERGE_SPLITS) wsh[s0] = s0 < n ? w0 * m0.z : 0.f;
        if (lp == 0) wsh[s1] = s1 < n ? w1 * m1.z : 0.f;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const float den = over_row((s0 < n ? w0 * m0.y : 0.f) + (lp == 0 && s1 < n ? w1 * m1.y : 0.f), [](float u, float v) { return u + v; });
        float inv = p.out_scale / den;
        float acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        for (int at = 0;;) {
            float wg[8];
#pragma unroll
            for (int b = 0; b < 8; ++b) wg[b] = wsh[(at + sub + (b << lp)) & (MERGE_SPLITS - 1)];
#pragma unroll
            for (int b = 0; b < 8; ++b)
                if (at + (b << lp) < n) {                               // (a set past the last split: weight 0)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(wg[b], (float)part[b][e], acc[e]);
                }
            at += 8 << lp;
            if (at >= n) break;
#pragma unroll
            for (int b = 0; b < 8; ++b) sh.part[b] = sh.part_at(pc, b, at, n, tid);
            load_parts();
        }
        bvec o;
#pragma unroll
        for (int e = 0; e < E; ++e) {                                   // the row's sets
            if (lp >= 1) {
                const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[e]), __float_as_uint(acc[e]), false, false);
                acc[e] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
            }
            if (lp == 2) {
                const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[e]), __float_as_uint(acc[e]), false, false);
                acc[e] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
            }
            o[e] = (__bf16)(acc[e] * inv);
        }
        if (sub == 0) *reinterpret_cast<bvec *>(static_cast<__bf16 *>(p.O) + (size_t)sh.row * D + (tid & 15) * E) = o;
        sh.k += sh.SETS >> lp;
        if (sh.k < sh.count) sh.find(p, pc, n, wr, tid);
    }
}

// The rest of a workgroup whose partials have been stored (by its threads; not necessarily acknowledged yet).
template <int D, int WAVES, int WR>
__device__ __forceinline__ void merge_group(const AttnParams &p, MergeWords &m, unsigned char *smem, int tid, const Piece &pc, int n, u64 tag)
{
    const int split = pc.bx;
    uint32_t *said = reinterpret_cast<uint32_t *>(smem) + WAVES * 4 * MERGE_SPLITS;      // what the first wavefront has seen (behind merge_share's weights)
    const int lane = tid & 63, peer = min(lane, n - 1), rows = min(WR, p.M * p.G - pc.by * WR);
    u64 begun = 0;
    if (tid < 64) begun = __hip_atomic_load(&m.started[peer], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    Share<D, WAVES> own;                                // found ahead of the wait
    own.begin(split, n, rows, tid);
    own.find(p, pc, n, WR, tid);
    asm volatile("" : "+v"(own.k), "+v"(own.row), "+v"(own.ml), "+v"(own.part[0]), "+v"(own.part[1]), "+v"(own.part[2]), "+v"(own.part[3]),
                 "+v"(own.part[4]), "+v"(own.part[5]), "+v"(own.part[6]), "+v"(own.part[7]));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wavefront's partials are in the L2 ...
    __syncthreads();                                    // ... and all the workgroup's
    if (tid < 64) {
        const bool together = __builtin_amdgcn_ballot_w64(begun != (tag << 8 | this_xcd())) == 0ull;
        if (!together) __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
        auto say = [&](u64 word) {
            if (lane == 0) __hip_atomic_store(&m.near[split], word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (!together) {
                if (lane == 0) __hip_atomic_store(&m.far[split], word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
        };
        u64 left = 0;
        auto look = [&](bool both) {                    // are all there?  Which have left?
            const u64 a = __hip_atomic_load(&m.near[peer], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            const u64 b = both ? __hip_atomic_load(&m.far[peer], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : a;
            const bool in_a = a >> 8 == tag, in_b = b >> 8 == tag;
            left = __builtin_amdgcn_ballot_w64(lane < n && ((in_a && (a & 1)) || (in_b && (b & 1))));
            return __builtin_amdgcn_ballot_w64(!in_a && !in_b) == 0ull;
        };
        say(tag << 8);
        bool all = look(!together);
        if (!all) {
            const long long t0 = (long long)__builtin_amdgcn_s_memrealtime();
            int limit = min(p.wait_ticks, MERGE_START_TICKS);
            do {
                if ((long long)__builtin_amdgcn_s_memrealtime() - t0 > limit) {
                    if (limit < p.wait_ticks) {         // have all started by now?
                        limit = p.wait_ticks;
                        const u64 now = __hip_atomic_load(&m.started[peer], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                        if (__builtin_amdgcn_ballot_w64(now >> 8 != tag) == 0ull) continue;
                    }
                    say(tag << 8 | 1);
                    all = look(true);
                    break;
                }
                __builtin_amdgcn_s_sleep(1);
                all = look(!together);
            } while (!all);
        }
        if (all && !together) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
        if (lane == 0) *reinterpret_cast<uint2 *>(said) = make_uint2(all, (uint32_t)left);
    }
    __syncthreads();
    const uint2 seen = *reinterpret_cast<const uint2 *>(said);
    if (!__builtin_amdgcn_readfirstlane(seen.x)) return;
    merge_share<D, WAVES>(p, pc, own, n, WR, reinterpret_cast<float *>(smem), tid);
    uint32_t left = __builtin_amdgcn_readfirstlane(seen.y) & ~(1u << split);
    while (left) {                                      // (rare) the shares of those that have left
        own.begin(__builtin_ctz(left), n, rows, tid);
        own.find(p, pc, n, WR, tid);
        merge_share<D, WAVES>(p, pc, own, n, WR, reinterpret_cast<float *>(smem), tid);
        left &= left - 1;
    }
    if (tid == 0) __hip_atomic_store(&m.epoch, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// One request: a workgroup per (key split, KV head, row block).  MERGE: the workgroups merge the splits (a kernel of its own: with
// both in one, those that do not merge took 0.2 us longer).
template <int D, int RW, int KW, int NT, int EB, bool MERGE>
__global__ __launch_bounds__(RW * KW * 64, 2) void tv_attn_bf16(AttnParams p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    BTV_FETCH_ARGS(p);
    // Workgroups go to the 8 XCDs round-robin by their linear id.  The row blocks of one (key split, KV head) stream the same K/V
    // bytes, so they get ids that are congruent mod 8 and share one L2; where the merge is done here, so do all splits of a group
    // (p.units counts the (split, head) pairs, or the heads, or the groups that are dealt out to the XCDs; 0: the pairs are dealt
    // out although the merge is done here, so that tests meet a group on several XCDs).
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
    Piece pc = {};
    if constexpr (!MERGE) {
        const int q = quotient(slot, p.row_blocks, p.inv_row_blocks), unit = q * 8 + xcd;
        if (unit >= p.units) return;
        pc.by = slot - q * p.row_blocks; pc.g = quotient(unit, p.nsplit, p.inv_nsplit); pc.bx = unit - pc.g * p.nsplit;
    } else if (p.units == p.Hkv) {
        const int q = quotient(slot, p.row_blocks, p.inv_row_blocks), u = quotient(q, p.nsplit, p.inv_nsplit);
        pc.by = slot - q * p.row_blocks; pc.g = u * 8 + xcd; pc.bx = q - u * p.nsplit;
        if (pc.g >= p.Hkv) return;
    } else if (p.units) {
        const int u = quotient(slot, p.nsplit, p.inv_nsplit), q = u * 8 + xcd;
        pc.g = quotient(q, p.row_blocks, p.inv_row_blocks); pc.by = q - pc.g * p.row_blocks; pc.bx = slot - u * p.nsplit;
        if (pc.g >= p.Hkv) return;
    } else {
        const int q = quotient(slot, p.row_blocks, p.inv_row_blocks), unit = q * 8 + xcd;
        pc.by = slot - q * p.row_blocks; pc.g = quotient(unit, p.nsplit, p.inv_nsplit); pc.bx = unit - pc.g * p.nsplit;
        if (pc.g >= p.Hkv) return;
    }
    const Req rq = load_req<false>(p, 0);
    const int tiles = (rq.L + rq.M + 31) / 32;
    pc.st0 = pc.bx * p.sps + KW * min(pc.bx, p.longer);
    pc.st1 = min(pc.st0 + p.sps + (pc.bx < p.longer ? KW : 0), tiles);
    pc.direct = p.nsplit == 1;
    pc.grouped = MERGE;
    pc.group = pc.g * p.row_blocks + pc.by;
    pc.pitch = min(RW * 32, rq.M * p.G) + 1;            // (rows of the same number lie in different channels)
    if constexpr (MERGE) {
        MergeWords *m = reinterpret_cast<MergeWords *>(p.sync) + pc.group;
        // (a scalar load: nothing writes it before every workgroup of the group has read it)
        const u64 tag = *reinterpret_cast<const __attribute__((address_space(4))) u64 *>(reinterpret_cast<uintptr_t>(&m->epoch)) + 1;
        attn_piece<D, RW, KW, NT, false, EB>(p, smem, threadIdx.x, rq, pc, [&] {
            if (threadIdx.x == 0)
                __hip_atomic_store(&m->started[pc.bx], tag << 8 | this_xcd(), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        });
        merge_group<D, RW * KW, RW * 32>(p, *m, smem, threadIdx.x, pc, p.nsplit, tag);
    } else {
        attn_piece<D, RW, KW, NT, false, EB>(p, smem, threadIdx.x, rq, pc, [] {});
    }
}

// A batch of short requests: a workgroup per (part of at most sps tiles, KV head, request, row block) of the largest request;
// those that a request has no use for leave at once.
template <int D, int RW, int KW, int NT, int EB>
__global__ __launch_bounds__(RW * KW * 64, 2) void tv_attn_short(AttnParams p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    BTV_FETCH_ARGS(p);
    asm volatile("" ::"s"(p.inv_sps), "s"(p.inv_Hkv));
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
    const int uq = quotient(slot, p.row_blocks, p.inv_row_blocks), by = slot - uq * p.row_blocks, unit = uq * 8 + xcd;
    if (unit >= p.units) return;
    Piece pc = {};
    // The part is rotated by the request (and the head).  Without it part i of a head is on the same XCD in every request, or on the
    // same few, and as all requests have a first part and only the longest a last one, some XCDs have most of the work: rotated by the
    // (request, head) number, which comes to the same for an even number of parts, 29 requests of up to 2347 keys with 30 nodes took
    // 69 us, now 61; 31 of up to 3181 with 10 65.5 and 58.
    const int bz = quotient(unit, p.nsplit, p.inv_nsplit);
    pc.rq = quotient(bz, p.Hkv, p.inv_Hkv); pc.g = bz - pc.rq * p.Hkv; pc.by = by;
    const int turned = unit - bz * p.nsplit + 3 * pc.g + pc.rq;
    pc.bx = turned - quotient(turned, p.nsplit, p.inv_nsplit) * p.nsplit;
    const Req rq = load_req<true>(p, pc.rq);
    if (!rq.ok) {
        if (threadIdx.x == 0 && by == 0 && pc.bx == 0 && pc.g == 0) atomicOr(p.flag, 2u);
        return;
    }
    const int tiles = (rq.L + rq.M + 31) >> 5, parts = quotient(tiles + p.sps - 1, p.sps, p.inv_sps);
    if (by * RW * 32 >= rq.M * p.G || pc.bx >= parts) return;
    pc.st0 = pc.bx * p.sps;
    pc.st1 = min(pc.st0 + p.sps, tiles);
    pc.direct = parts == 1;
    attn_piece<D, RW, KW, NT, true, EB>(p, smem, threadIdx.x, rq, pc, [] {});
}

// ---- ragged batches ---------------------------------------------------------------------------------------------------
// The host knows bounds on the requests' sizes only, so the workgroups share the work out themselves: as many as the CUs
// hold, all with about the same time to spend, whatever the lengths.  A request's work for one KV head is a row of
// stretches, one per row block, START + weight * t long for t tiles (START: what starting on a row block and storing its
// rows costs; the weight is WHOLE, or PART where no more than half of the block's rows exist, as a tile goes faster then).
// The stretches lie one after the other, request after request, KV head after KV head (so an XCD keeps to one head or
// two), and team k takes what lies between k w and (k + 1) w; where that cuts a stretch, tv_combine_batch
// merges the parts.  A cut less than MARGIN tiles from where a stretch's tiles begin or end moves there.  A stretch of up to
// SMALL tiles is not cut: the team that its beginning falls to does all of it.  Both make shares uneven by as much as they are long, and that costs
// more than the pieces they save (with 8 and 16 tiles the fullest share of 32 requests of 100 to 4000 tokens was 242 of 174 on average; times below).
// Where trees may take several row blocks a team is a pair of workgroups (neighbours on one XCD, running side by side): a
// stretch stands for two row blocks then, one for each member, over the same tiles, so that the second finds the K/V of the
// first in their L2; an odd last row block is a stretch of half its tiles, each member taking half of every part
// (if it is small, one of them takes it alone).
// Bound by the tiles (0.84 to 0.91 us each in bf16 pieces of more than 128 rows, 0.58 to 0.61 below; FP8 0.49 to 0.51 in pieces of more than 64 rows, 0.32 to 0.34 below), and
// by the pieces: 6 (FP8) to 10.5 us each beyond its tiles (the plan and finding it 1.2 to 1.8, page ids and first tiles 2 to 2.7, the rest of the prologue 1.1, merging
// and storing 1.3 to 2, waiting for the other waves 0.1 to 0.8, the way into and out of the loop 0.5 to 3.2), START comes from that.  us, with START, MARGIN and SMALL of 8, 8 and 16 tiles / 8, 2 and 8 / 10, 2 and 8:
// 8 requests of 1k to 16k, bf16 156 / 155 / 152; 32 of 100 to 4000, FP8 59.7 / 52.8 / 50.9; 5 of up to 8k with 83 nodes 58.5 / 51.8 / 53.8; 9 of up to 9k with
// 12 42.0 / 39.7 / 39.9; 14 of up to 6k, FP8 67.4 / 65.4 / 65.0.  The figures beside the choice of the form
// (short_batch) are the whole call's.
constexpr int WHOLE = 3, PART = 2, START = 10 * WHOLE, MARGIN = 2, SMALL = 8;
// A halved stretch of an odd number of tiles has half a step less for its second member.  A cut one step ahead of its end would leave that
// member's last part empty, nobody would write it, and tv_combine_batch counts it: cuts stay two steps away from the end.
static_assert(MARGIN >= 2, "both members have tiles in every part");
struct Stretch { int t, du, wt, sl, len; };             // tiles; whole stretches; weight of the last; length of the halved one; all
__device__ __forceinline__ Stretch stretch_of(const AttnParams &p, const Req &q)
{
    Stretch s;
    s.t = q.ok ? (q.L + q.M + 31) >> 5 : 0;
    const int rows = q.ok ? q.M * p.G : 0, rb = (rows + (1 << p.wr_log2) - 1) >> p.wr_log2;
    s.du = rb >> p.pairing;
    s.wt = rows - ((rb - 1) << p.wr_log2) <= 1 << p.wr_log2 >> 1 ? PART : WHOLE;
    s.sl = p.pairing && (rb & 1) ? (s.t <= SMALL ? (s.t * s.wt + START + 1) >> 1 : ((s.t + 1) >> 1) * s.wt + START) : 0;
    s.len = s.du * (s.t * (p.pairing ? WHOLE : s.wt) + START) + s.sl;
    return s;
}
__device__ __forceinline__ int wave_incl_scan(int x)
{
    // (rows of 16 by shifts, then the last lane of each row into the rows behind it)
#define BTV_SCAN_STEP(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, ctrl < 0x142)
    BTV_SCAN_STEP(0x111, 0xF); BTV_SCAN_STEP(0x112, 0xF); BTV_SCAN_STEP(0x114, 0xF); BTV_SCAN_STEP(0x118, 0xF);
    BTV_SCAN_STEP(0x142, 0xA); BTV_SCAN_STEP(0x143, 0xC);
#undef BTV_SCAN_STEP
    return x;
}
// 64 lengths: their low and high halves on their own, so that no sum leaves 32 bits
__device__ __forceinline__ long long wave_incl_scan_len(int x)
{
    return ((long long)wave_incl_scan(x >> 16) << 16) + wave_incl_scan(x & 0xFFFF);
}
// Where a team stands.  Every wavefront of its workgroups works this out for itself.
struct Walk {
    long long first, end;                               // the team's share
    long long pos, head;                                // what comes next; where its KV head's work begins
    long long wh;                                       // one head's work
    int h, w;                                           // that KV head; a share
};

// A chunk of 64 requests, one per lane: their stretches, and where they end in a head's work (cum: where the chunk begins).
struct Chunk { Stretch s; long long incl; bool bad; };
__device__ __forceinline__ Chunk load_chunk(const AttnParams &p, int c0, int lane, long long cum)
{
    Chunk c;
    const bool in = c0 + lane < p.batch;
    const Req q = load_req<true>(p, min(c0 + lane, p.batch - 1));
    c.s = stretch_of(p, q);
    c.bad = in && !q.ok;
    c.incl = wave_incl_scan_len(in ? c.s.len : 0) + cum;
    return c;
}
// The first chunk is kept in LDS from one piece to the next.  Loaded again it cost 1.1 us a piece (1.4 to 1.8 pieces a workgroup): its loads
// wait behind the last piece's stores; from LDS 0.5.  8 requests of 1k to 16k, two layers and trees, 303 -> 299 us; 32 of 100 to 4000, FP8, 119.4 -> 115.9; 20 of 1k to
// 6k with 64 channels 181 -> 176.  (Looking for the next piece during this one's first loads, by one wavefront that tells the others: +-1 %.)  Raw
// instructions: ahead of ordinary reads the compiler waits for the stores as well.
constexpr int CHUNK_BYTES = 64 * 32;
__device__ __forceinline__ void keep_chunk(uint32_t kept, int lane, const Chunk &c)
{
    const u32x4 a = { (uint32_t)c.s.t, (uint32_t)c.s.du, (uint32_t)c.s.wt, (uint32_t)c.s.sl }, b = { (uint32_t)c.s.len, (uint32_t)c.incl, (uint32_t)(c.incl >> 32), 0 };
    asm volatile("ds_write_b128 %0, %1\n\tds_write_b128 %0, %2 offset:16\n\ts_waitcnt lgkmcnt(0)" :: "v"(kept + (uint32_t)lane * 32), "v"(a), "v"(b) : "memory");
}
__device__ __forceinline__ Chunk kept_chunk(uint32_t kept, int lane)
{
    u32x4 a, b;
    asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:16\n\ts_waitcnt lgkmcnt(0)" : "=&v"(a), "=&v"(b) : "v"(kept + (uint32_t)lane * 32) : "memory");
    Chunk c;
    c.s.t = (int)a[0]; c.s.du = (int)a[1]; c.s.wt = (int)a[2]; c.s.sl = (int)a[3]; c.s.len = (int)b[0];
    c.incl = (long long)((unsigned long long)b[2] << 32 | b[1]);
    c.bad = false;
    return c;
}
__device__ __forceinline__ long long last_lane(long long x)
{
    return (long long)(((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), 63) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)x, 63));
}

// The share of a team (the `nth` on its XCD), and the first chunk of requests.  The very first workgroup leaves the plan for the merge.
__device__ __forceinline__ Walk share_out(const AttnParams &p, int xcd, int nth, int lane, bool leader, Chunk &c)
{
    Walk k;
    long long begin = 0;
    bool bad = false;
    for (int c0 = ((p.batch - 1) >> 6) << 6; c0 >= 0; c0 -= 64) {         // (the first chunk last; sums of the others do not matter yet)
        c = load_chunk(p, c0, lane, 0);
        bad = bad || c.bad;
        begin += last_lane(c.incl);
    }
    k.wh = begin;
    const long long all = k.wh * p.Hkv;
    const long long w = max((all + (1 << p.teams_log2) - 1) >> p.teams_log2, (long long)p.wmin);
    if (leader) {
        long long cum = 0;
        for (int c0 = 0; c0 < p.batch; c0 += 64) {
            const Chunk d = c0 ? load_chunk(p, c0, lane, cum) : c;
            if (c0 + lane < p.batch) p.plan[2 + c0 + lane] = d.incl - d.s.len;
            cum = last_lane(d.incl);
        }
        if (lane == 0) { p.plan[0] = w; p.plan[1] = k.wh; }
        if (bad) atomicOr(p.flag, 2u);
    }
    k.w = (int)min(w, (long long)INT_MAX);
    // neighbouring shares on one XCD, as many on each: where the work is for a part of the teams, all XCDs have some
    long long per_xcd = (1 << p.teams_log2) >> 3;
    if (w == p.wmin) per_xcd = min(per_xcd, ((all + w - 1) / w + 7) >> 3);
    k.first = k.pos = nth < per_xcd ? min((xcd * per_xcd + nth) * w, all) : all;
    k.end = min(k.first + w, all);
    k.head = 0; k.h = 0;
    return k;
}

// The member's next piece; the walk moves behind it.  False: none left.  c holds the first chunk of requests.
__device__ __forceinline__ bool next_piece(const AttnParams &p, Walk &k, int member, int lane, const Chunk &c, Piece &pc)
{
    while (k.pos < k.end) {
        while (k.pos - k.head >= k.wh) { k.head += k.wh; ++k.h; }
        const long long x = k.pos - k.head;
        Chunk d = c;
        int r0 = 0;
        unsigned long long beyond;
        while ((beyond = __builtin_amdgcn_ballot_w64(x < d.incl)) == 0ull) {
            r0 += 64;
            if (r0 >= p.batch) return false;            // (cannot be: x lies within the head's work)
            d = load_chunk(p, r0, lane, last_lane(d.incl));
        }
        const int src = __builtin_ctzll(beyond);
        Stretch s;
        s.t = __builtin_amdgcn_readlane(d.s.t, src); s.du = __builtin_amdgcn_readlane(d.s.du, src);
        s.wt = __builtin_amdgcn_readlane(d.s.wt, src); s.sl = __builtin_amdgcn_readlane(d.s.sl, src);
        s.len = __builtin_amdgcn_readlane(d.s.len, src);
        const int y = s.len + __builtin_amdgcn_readlane((int)(x - d.incl), src);       // place in the request's work
        const int whole = s.t * (p.pairing ? WHOLE : s.wt) + START, u = min(y / whole, s.du);
        const bool halved = u == s.du;
        const int y0 = y - u * whole;                   // ... in the stretch
        const long long us = k.pos - y0;                // where the stretch begins
        pc.rq = r0 + src;
        pc.g = k.h;
        pc.by = p.pairing ? (halved ? 2 * u : 2 * u + member) : u;
        pc.bx = 0; pc.direct = 1; pc.st0 = 0; pc.st1 = s.t;
        if (s.t <= SMALL) {
            k.pos = us + (halved ? s.sl : whole);
            if (y0 == 0 && (!halved || ((pc.rq ^ k.h) & 1) == member)) return true;
            continue;
        }
        const int wt = halved || !p.pairing ? s.wt : WHOLE;
        const int tl = halved ? (s.t + 1) >> 1 : s.t, cl = tl * wt, cm = MARGIN * wt;  // tiles of the stretch; their length
        const long long ts = us + START;                // they begin here
        int c0 = y0 - START, c1 = (int)min(k.end - ts, (long long)cl);
        if (c0 < cm) c0 = 0; else if (c0 > cl - cm) c0 = cl;
        if (c1 < cm) c1 = 0; else if (c1 > cl - cm) c1 = cl;
        k.pos = c1 < cl ? k.end : ts + cl;
        if (c0 >= c1) continue;
        const int cut = c0 == 0 ? 0 : (c0 - cm) / k.w + 1;
        const int x0 = c0 / wt, x1 = c1 / wt;
        if (!halved) {
            pc.st0 = x0; pc.st1 = x1; pc.bx = cut; pc.direct = c0 == 0 && c1 == cl;
            return true;
        }
        pc.bx = 2 * cut + member; pc.direct = 0;
        pc.st0 = member ? x0 + x1 : 2 * x0;
        pc.st1 = member ? min(2 * x1, s.t) : x0 + x1;
        if (pc.st0 < pc.st1) return true;
    }
    return false;
}

template <int D, int RW, int KW, int NT, int EB>
__global__ __launch_bounds__(RW * KW * 64, 2) void tv_attn_batch(AttnParams p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    BTV_FETCH_ARGS(p);
    asm volatile("" ::"s"(p.plan), "s"(p.batch), "s"(p.teams_log2), "s"(p.pairing), "s"(p.wmin), "s"(p.wr_log2));
    const int xcd = blockIdx.x & 7, slot = blockIdx.x >> 3, member = slot & p.pairing;
    Chunk c;
    Walk k = share_out(p, xcd, slot >> p.pairing, threadIdx.x & 63, blockIdx.x == 0 && threadIdx.x < 64, c);
    const uint32_t kept = (uint32_t)(uintptr_t)BTV_LDS_PTR(smem) + PageLds<D, RW, KW, NT, true, EB>::BYTES;
    if (threadIdx.x < 64) keep_chunk(kept, threadIdx.x, c);     // (barriers before it is read: those of the first piece)
    for (bool again = false;; again = true) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                   // keeps what derives from it (all addresses) from being carried across pieces
        if (again) {
            if (k.pos >= k.end) break;
            c = kept_chunk(kept, tid & 63);
        }
        Piece pc = {};
        if (!next_piece(p, k, member, tid & 63, c, pc)) break;
        attn_piece<D, RW, KW, NT, true, EB>(p, smem, tid, load_req<true>(p, pc.rq), pc, [] {});
        // every wave is done with this piece's LDS, its own fills have landed; the stores may still be on their way
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
    }
}

// Split-K combine: O[row] = sum_s w_s a_s O'_s / sum_s w_s l_s with w_s = exp2((m_s - max m) * scale*log2 e), O'_s the
// fp16 partial and a_s the magnitude it was divided by.
// 8 rows per workgroup, 32 lanes per row, each lane owns D/32 consecutive channels.  Lane j of a row fetches the
// (m, l) pairs of splits j, j + 32, ... and computes their weights; the partial rows of up to 32 splits are fetched
// by independent loads issued before anything is waited for, so the kernel costs about one memory round trip
// whatever the number of splits.  What happens between the lanes of a row stays off the LDS crossbar where it can:
// maximum and sum over the 32 lanes are DPP steps within the rows of 16 and one swap between the two rows (they were
// five dependent ds_bpermute round trips each), and the 32 weights reach every lane through one LDS store and eight
// 16-byte reads of the same address (they were 32 shuffles, each waited for before its multiply-adds).
__device__ __forceinline__ float row32_max(float x, int lane)
{
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, false)));    // quad_perm [1,0,3,2]
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, false)));    // quad_perm [2,3,0,1]
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, false)));   // row_half_mirror
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, false)));   // row_mirror
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(x, __uint_as_float((lane & 16) ? sw[0] : sw[1]));                                               // the other row of 16
}

__device__ __forceinline__ float row32_sum(float x, int lane)
{
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, false));
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return x + __uint_as_float((lane & 16) ? sw[0] : sw[1]);
}

// Over the N = 8, 16 or 32 lanes of a row.
template <int N>
__device__ __forceinline__ float lanes_max(float x)
{
    if (N == 32) return row32_max(x, (int)threadIdx.x);
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, false)));
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, false)));
    x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, false)));
    return N == 8 ? x : fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, false)));
}
template <int N>
__device__ __forceinline__ float lanes_sum(float x)
{
    if (N == 32) return row32_sum(x, (int)threadIdx.x);
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0xB1, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x4E, 0xF, 0xF, false));
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x141, 0xF, 0xF, false));
    return N == 8 ? x : x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x140, 0xF, 0xF, false));
}

// E = 2, 4 or 8 channels per lane
template <int D, int E>
__device__ __forceinline__ void store_row(const AttnParams &p, size_t row, int lane, const float (&acc)[E], float inv)
{
    uint16_t *dst = static_cast<uint16_t *>(p.O) + row * D + lane * E;
    uint32_t x[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) x[e] = float_to_bf16_bits(acc[2 * e] * inv) | (float_to_bf16_bits(acc[2 * e + 1] * inv) << 16);
    if constexpr (E == 8) *reinterpret_cast<uint4 *>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
    else if constexpr (E == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(x[0], x[1]);
    else *reinterpret_cast<uint32_t *>(dst) = x[0];
}

template <int D>
__device__ __forceinline__ void combine_row(const AttnParams &p, size_t row, int nsplit_r, float (&wsh)[8][32])
{
    constexpr int E = D / 32;
    typedef _Float16 hvec __attribute__((ext_vector_type(E)));
    const int rin = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const size_t sstride = (size_t)p.total_rows;
    // reference maximum over all splits: with more than 32 of them it takes a round trip of its own
    float mmax = NEG_BIG;
    for (int s = lane + 32; s < nsplit_r; s += 32) mmax = fmaxf(mmax, p.ML[(s * sstride + row) * 4]);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    float den = 0.f;
    for (int s0 = 0; s0 < nsplit_r; s0 += 32) {     // one pass for up to 32 splits
        const int s_mine = s0 + lane;
        const float4 mlr = *reinterpret_cast<const float4 *>(p.ML + ((size_t)min(s_mine, nsplit_r - 1) * sstride + row) * 4);
        const float4 ml = s_mine < nsplit_r ? mlr : make_float4(NEG_BIG, 0.f, 0.f, 0.f);
        hvec part[32];
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (s0 + 8 * g < nsplit_r) {             // uniform within the row's lanes: whole groups of 8 loads
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    const int s = min(s0 + 8 * g + b, nsplit_r - 1);
                    part[8 * g + b] = *reinterpret_cast<const hvec *>(p.Opart + (s * sstride + row) * D + lane * E);
                }
            }
        if (s0 == 0) mmax = row32_max(fmaxf(mmax, ml.x), (int)threadIdx.x);
        const float w = s_mine < nsplit_r ? __builtin_amdgcn_exp2f(ml.x - mmax) : 0.f;
        den += w * ml.y;
        wsh[rin][lane] = w * ml.z;                              // weight times the partial's magnitude; 0 past the last split
        // (the row's 32 lanes are one half of a wavefront: its LDS operations complete in order, no barrier needed)
        float wgt[32];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float4 x = *reinterpret_cast<const float4 *>(&wsh[rin][4 * q]);
            wgt[4 * q] = x.x; wgt[4 * q + 1] = x.y; wgt[4 * q + 2] = x.z; wgt[4 * q + 3] = x.w;
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (s0 + 8 * g < nsplit_r) {
#pragma unroll
                for (int b = 0; b < 8; ++b) {
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] += wgt[8 * g + b] * (float)part[8 * g + b][e];
                }
            }
    }
    den = row32_sum(den, (int)threadIdx.x);
    const float inv = p.out_scale / den;
    store_row<D, E>(p, row, lane, acc, inv);
}

template <int D>
__global__ __launch_bounds__(256) void tv_combine_bf16(AttnParams p)
{
    __shared__ __attribute__((aligned(16))) float wsh[8][32];
    // every argument in one round trip (the argument block is cold in every launch)
    asm volatile("" ::"s"(p.O), "s"(p.Opart), "s"(p.ML), "s"(p.M), "s"(p.L), "s"(p.Hq), "s"(p.total_rows), "s"(p.nsplit), "s"(p.out_scale));
    const int row = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= p.M * p.Hq) return;
    combine_row<D>(p, (size_t)row, p.nsplit, wsh);
}

// The same for a batch: how many parts a row has follows from where its request's work lies (the plan that the attention's first
// workgroup left).  What bounds it is the chain of the request's place, the parts and the sums: lanes of E channels, the first PARTS
// parts all asked for at once.  With 8 channels a lane has 16-byte loads and half of the wavefronts do, so those of many rows are under way
// together (8 requests of up to 128 nodes, 32 heads: attention and merge 156 -> 153 us, 150 to 156 from run to run; 32 of up to 24, FP8, 51.1 -> 49.1); few rows leave the
// chip room, and D / 32 channels with 16 parts at once are faster (7 requests of 33 nodes, 16 heads, in up to 20 parts: 23.8 and 25.6).
template <int D, int E, int PARTS>
__global__ __launch_bounds__(256) void tv_combine_batch(AttnParams p)
{
    constexpr int LPR = D / E, ROWS = 256 / LPR;             // lanes of a row, rows of a workgroup
    __shared__ __attribute__((aligned(16))) float wsh[ROWS][LPR];
    asm volatile("" ::"s"(p.O), "s"(p.q_offset), "s"(p.prefix_len), "s"(p.Opart), "s"(p.ML), "s"(p.M), "s"(p.L), "s"(p.Hq), "s"(p.G),
                 "s"(p.max_blocks), "s"(p.total_rows), "s"(p.total_M), "s"(p.plan), "s"(p.Hkv), "s"(p.pairing), "s"(p.wr_log2), "s"(p.sps), "s"(p.out_scale));
    const int r = blockIdx.y;
    const Req q = load_req<true>(p, r);
    long long w = 0, wh = 0, at = 0;
    if (!p.sps) { w = p.plan[0]; wh = p.plan[1]; at = p.plan[2 + r]; }
    if (!q.ok) return;
    const int lr = blockIdx.x * ROWS + threadIdx.x / LPR;
    if (lr >= q.M * p.Hq) return;
    int n = 1;
    if (p.sps) {                                        // short requests: equal parts
        n = (((q.L + q.M + 31) >> 5) + p.sps - 1) / p.sps;
    } else {
        const Stretch s = stretch_of(p, q);
        const int node = lr / p.Hq, hq = lr - node * p.Hq, h = hq / p.G, by = (node * p.G + hq - h * p.G) >> p.wr_log2;
        if (s.t <= SMALL) return;                           // written by the attention kernel
        const int u = by >> p.pairing;
        const bool halved = u == s.du;
        const int wt = halved || !p.pairing ? s.wt : WHOLE;
        const int cl = (halved ? (s.t + 1) >> 1 : s.t) * wt, cm = MARGIN * wt;
        const long long ts = h * wh + at + (long long)u * (s.t * WHOLE + START) + START;   // (u = 0 where a team is one workgroup)
        const long long lo = ts + cm, hi = ts + cl - cm;    // where a cut counts
        if (hi >= lo) n += wh * p.Hkv < INT_MAX ? (int)hi / (int)w - ((int)lo - 1) / (int)w : (int)(hi / w - (lo - 1) / w);
        if (halved) n *= 2;
    }
    if (n == 1) return;
    // The first PARTS parts, in groups of four, are all asked for before the first is looked at.
    typedef _Float16 hvec __attribute__((ext_vector_type(E)));
    constexpr int GROUPS = PARTS / 4, TURNS = PARTS > LPR ? PARTS / LPR : 1;
    const int rin = threadIdx.x / LPR, lane = threadIdx.x % LPR;
    const size_t row = (size_t)q.q0 * p.Hq + lr, sstride = (size_t)p.total_rows;
    auto magnitudes = [&](int s) {
        const float4 x = *reinterpret_cast<const float4 *>(p.ML + (min(s, n - 1) * sstride + row) * 4);
        return s < n ? x : make_float4(NEG_BIG, 0.f, 0.f, 0.f);
    };
    const _Float16 *Pp = p.Opart + row * D + lane * E;
    hvec part[GROUPS][4];
    auto load = [&](hvec (&x)[4], int s0) {
#pragma unroll
        for (int b = 0; b < 4; ++b) x[b] = *reinterpret_cast<const hvec *>(Pp + min(s0 + b, n - 1) * sstride * D);
    };
    float4 ml[TURNS];
#pragma unroll
    for (int k = 0; k < TURNS; ++k) ml[k] = magnitudes(k * LPR + lane);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
        if (g == 0 || n > 4 * g) load(part[g], 4 * g);
    float mmax = ml[0].x, den = 0.f;
#pragma unroll
    for (int k = 1; k < TURNS; ++k) mmax = fmaxf(mmax, ml[k].x);
    for (int s = lane + TURNS * LPR; s < n; s += LPR) mmax = fmaxf(mmax, p.ML[(s * sstride + row) * 4]);     // (rare)
    mmax = lanes_max<LPR>(mmax);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    auto weights = [&](const float4 &m, int s0) {           // of the LPR parts from s0 on, one per lane
        const float w = s0 + lane < n ? __builtin_amdgcn_exp2f(m.x - mmax) : 0.f;
        den += w * m.y;
        wsh[rin][lane] = w * m.z;                           // weight times the part's magnitude; 0 past the last part
        // (the row's lanes are in one wavefront: its LDS operations complete in order, no barrier needed)
    };
    auto add = [&](const hvec (&x)[4], int at) {
        const float4 wg = *reinterpret_cast<const float4 *>(&wsh[rin][at]);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += wg.x * (float)x[0][e] + wg.y * (float)x[1][e] + wg.z * (float)x[2][e] + wg.w * (float)x[3][e];
    };
#pragma unroll
    for (int g = 0; g < GROUPS; ++g)
        if (g == 0 || n > 4 * g) {
            if (4 * g % LPR == 0) weights(ml[4 * g / LPR], 4 * g);
            add(part[g], 4 * g % LPR);
        }
#pragma unroll 1
    for (int s0 = PARTS; s0 < n; s0 += 4) {
        if ((s0 & (LPR - 1)) == 0) weights(magnitudes(s0 + lane), s0);
        load(part[0], s0);
        add(part[0], s0 & (LPR - 1));
    }
    const float inv = p.out_scale / lanes_sum<LPR>(den);
    store_row<D, E>(p, row, lane, acc, inv);
}

// ------------------------------------------------------------------------------------------------
// fp32 kernel: one workgroup per (node, query head), over the keys in chunks of CH = 256 (D = 64) or 128 (D = 128; 512
// threads for 256 keys measured the same).
// Precision path, not the fast one; the shapes it sees are small, so what it costs is its chain of steps, a launch for
// the ancestor masks among them once.  A key's score takes D / 64 neighbouring threads, 64 channels each; its
// probability goes to LDS; then a thread owns one channel of 64 of the chunk's keys, whose values are on their way since
// before the scores (one memory round trip per chunk).  The node's ancestors are walked by one thread over parent[] in
// LDS while the keys arrive.  144 keys, 16 nodes, one head: 5.3 us; with a private softmax state of all channels per
// thread, merged by D * 6 shuffles, and the masks' launch it was 12.3.
// ------------------------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void tv_attn_f32(AttnParams p)
{
    constexpr int TPK = D / 64, CH = 256 / TPK, GROUPS = 256 / D, WAVES = 4;   // threads per key, keys per chunk, groups of 64 keys
    static_assert(GROUPS * 64 == CH, "a thread of each group takes 64 of the chunk's keys");
    __shared__ __attribute__((aligned(16))) float qs[D], prob[CH], red[GROUPS][D];
    __shared__ float wmax[WAVES], wsum[WAVES];
    __shared__ int par[BTV_MAX_NODES];
    __shared__ unsigned char seen[BTV_MAX_NODES];
    asm volatile("" ::"s"(p.Q), "s"(p.K), "s"(p.V), "s"(p.O), "s"(p.parent), "s"(p.flag), "s"(p.M), "s"(p.L), "s"(p.Hq), "s"(p.Hkv), "s"(p.G), "s"(p.scale));
    const int i = blockIdx.x, hq = blockIdx.y, tid = threadIdx.x, g = hq / p.G;
    const float *Q = static_cast<const float *>(p.Q) + ((size_t)i * p.Hq + hq) * D;
    const float *K = static_cast<const float *>(p.K) + (size_t)g * D, *V = static_cast<const float *>(p.V) + (size_t)g * D;
    const size_t pitch = (size_t)p.Hkv * D;
    const int S = p.L + p.M;
    const int kk = tid / TPK, part = (tid % TPK) * 64;                         // scores: this thread's key of the chunk, its channels
    const int d = tid % D, kg = tid / D;                                       // values: its channel, its group of keys
    if (tid < D) qs[tid] = Q[tid];
    if (tid < p.M) par[tid] = p.parent[tid];
    seen[tid] = 0;
    float m = NEG_BIG, lsum = 0.f, o = 0.f;
    for (int j0 = 0; j0 < S; j0 += CH) {
        float4 kv[16];
        float vv[64];
        const float *kr = K + (size_t)min(j0 + kk, S - 1) * pitch + part;
#pragma unroll
        for (int u = 0; u < 16; ++u) kv[u] = *reinterpret_cast<const float4 *>(kr + 4 * u);
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (j0 + kg * 64 + b * 16 < S)                                     // (uniform in a wavefront)
#pragma unroll
                for (int u = 0; u < 16; ++u) vv[b * 16 + u] = V[(size_t)min(j0 + kg * 64 + b * 16 + u, S - 1) * pitch + d];
        __syncthreads();                                                       // (also: the last chunk's probabilities have been read)
        if (j0 == 0) {                                                         // the node's ancestors, and every parent's check
            if (tid < p.M && (par[tid] < -1 || par[tid] >= tid)) atomicOr(p.flag, 1u);
            if (tid == 255)
                for (int a = i; a >= 0;) {
                    seen[a] = 1;
                    const int pa = par[a];
                    a = pa < -1 || pa >= a ? -1 : pa;                          // an invalid entry ends the walk (flagged above)
                }
        }
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const float4 q4 = *reinterpret_cast<const float4 *>(&qs[part + 4 * u]);
            s = fmaf(q4.x, kv[u].x, s); s = fmaf(q4.y, kv[u].y, s);
            s = fmaf(q4.z, kv[u].z, s); s = fmaf(q4.w, kv[u].w, s);
        }
        if (TPK == 2) s += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(s), 0xB1, 0xF, 0xF, false));   // the pair's other half
        s *= p.scale;
        __syncthreads();                                                       // seen[]
        const int j = j0 + kk;
        const bool visible = j < p.L || (j < S && seen[j - p.L] != 0);
        float mx = visible ? s : NEG_BIG;
        mx = row32_max(mx, tid);
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        if ((tid & 63) == 0) wmax[tid >> 6] = mx;
        __syncthreads();
        float mn = m;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) mn = fmaxf(mn, wmax[k]);
        const float alpha = expf(m - mn), pj = visible ? expf(s - mn) : 0.f;
        m = mn;
        lsum = lsum * alpha + pj;
        if (part == 0) prob[kk] = pj;
        __syncthreads();
        o *= alpha;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (j0 + kg * 64 + b * 16 < S)
#pragma unroll
                for (int u = 0; u < 16; u += 4) {
                    const float4 pr = *reinterpret_cast<const float4 *>(&prob[kg * 64 + b * 16 + u]);
                    o = fmaf(pr.x, vv[b * 16 + u], o); o = fmaf(pr.y, vv[b * 16 + u + 1], o);
                    o = fmaf(pr.z, vv[b * 16 + u + 2], o); o = fmaf(pr.w, vv[b * 16 + u + 3], o);
                }
    }
    lsum = row32_sum(lsum, tid);
    lsum += __shfl_xor(lsum, 32);
    if ((tid & 63) == 0) wsum[tid >> 6] = lsum;
    red[kg][d] = o;
    __syncthreads();
    if (tid < D) {
        float x = red[0][tid];
#pragma unroll
        for (int k = 1; k < GROUPS; ++k) x += red[k][tid];
        float den = 0.f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) den += wsum[k];
        den *= 1.0f / TPK;                                                     // (every thread of a key counted it)
        static_cast<float *>(p.O)[((size_t)i * p.Hq + hq) * D + tid] = x / den;
    }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
// ---- scratch of the entry point that allocates nothing ---------------------------------------------------------
// One array per GPU, part of the loaded code object (zero until first used), held until the process ends.  Host code
// never uses the array's name as an address: the device address is asked for once per device and kept.
constexpr size_t SCRATCH_BYTES = (size_t)32 << 20;
constexpr size_t MOST_PARTIALS = (size_t)31 << 20;      // bytes of partials that a plan of one request may take: they and the words fit the array
constexpr int SCRATCH_MAX_DEVICES = 64;
static __device__ __align__(256) unsigned char scratch[SCRATCH_BYTES];
void *g_scratch_ptr[SCRATCH_MAX_DEVICES];
std::atomic<bool> g_scratch_known[SCRATCH_MAX_DEVICES];

// Device address of the current device's copy of `scratch` (looked up on the first call per device).
int scratch_address(void **out)
{
    int dev = -1;
    BTV_HIP(hipGetDevice(&dev));
    BTV_REQUIRE(dev >= 0 && dev < SCRATCH_MAX_DEVICES, "device index %d outside [0,%d)", dev, SCRATCH_MAX_DEVICES);
    if (!g_scratch_known[dev].load(std::memory_order_acquire)) {
        void *ptr = nullptr;
        BTV_HIP(hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)));
        BTV_REQUIRE(ptr != nullptr, "no device address for the scratch array");
        g_scratch_ptr[dev] = ptr;                   // (two racing first calls store the same address)
        g_scratch_known[dev].store(true, std::memory_order_release);
    }
    *out = g_scratch_ptr[dev];
    return BTV_OK;
}

// Clears the first `words` 32-bit words at p (a kernel rather than a memset node, so that the call can be captured).
__global__ __launch_bounds__(256) void fill_zero_kernel(uint32_t *p, int words)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < words) p[i] = 0u;
}

constexpr int MOST_SPLITS = 64;                         // that the library chooses by itself
struct Plan { int rw, kw, nt, wr, row_blocks, stages, sps, longer, nsplit; float bytes; };      // (bytes of K and V)

// Whether the workgroups of a plan merge their partials themselves (merge_group): few enough splits and groups for its words; all
// groups' workgroups congruent mod 8, and as many on each XCD; and the chip takes all at once.  Where the KV heads do not share out
// evenly over the XCDs the groups do, and a head's row blocks, on up to 8 XCDs, each read its K/V: 2 .. 4 % faster than the two
// launches for up to 64 MB of such reading (330 plans of 1 to 6 KV heads), 1 .. 3 % slower on average above, 25 % at 140 .. 200 MB.
bool merges_inside(const Plan &pl, int Hkv)
{
    const int groups = Hkv * pl.row_blocks;
    return pl.nsplit > 1 && pl.nsplit <= MERGE_SPLITS && groups <= MERGE_GROUPS &&
           (Hkv % 8 == 0 || (groups % 8 == 0 && pl.bytes * (float)(std::min(8, pl.row_blocks) - 1) <= 64e6f)) &&
           pl.nsplit * groups <= (pl.rw == 2 ? 512 : 256);
}

// Rows of one split's partials, by either merge.
size_t partial_rows(const Plan &pl, int M, int Hq, int Hkv)
{
    return std::max<size_t>((size_t)M * Hq, (size_t)Hkv * pl.row_blocks * (std::min(pl.wr, M * (Hq / Hkv)) + 1));
}

// Splits of `want` parts for a shape: whole rounds of KW tiles, as evenly as they go.
void split_plan(Plan &pl, int L, int want)
{
    // The last split has the tree rows: its workgroups find the ancestor sets and mask tiles (in the pipelined loop those also lose
    // the overlap).  Shared out as if there were `extra` more rounds at the end, it is that much shorter.
    const int tree_tiles = pl.stages - L / TK, rounds = (pl.stages + pl.kw - 1) / pl.kw;
    pl.nsplit = std::max(1, std::min(want, rounds));
    const int extra = std::min(pl.kw == 1 ? (7 * tree_tiles + 9) / 10 : 1, rounds / pl.nsplit - 1);
    const int all = rounds + (pl.nsplit > 1 ? extra : 0);
    pl.sps = all / pl.nsplit * pl.kw;
    pl.longer = all % pl.nsplit;
}

// Shape of the workgroups (64, 128 or 256 packed rows of a KV head; 32 rows per wave, pairs of waves alternating over the
// tiles in the first two, the software-pipelined loop in the third) and number of key splits of one request: those with
// the least estimated time.  The estimate: what a workgroup takes, its start and its tiles (two workgroups of the 64-row shape
// share a CU at 1.3 times the time each), times the rounds in which the CUs of the fullest XCD take the workgroups, but no less than the
// K/V bytes need, some of the smaller of the two on top; and for more than one split the merge.  Its constants are a fit to
// 1200 shapes with splits of equal length, as they were cut then (fitted again to splits that differ by a round: 0.2 %; prefixes of 64 to 32k, 4 to 256 nodes, 2 to 8 KV heads, all three K/V types and head sizes) times all shapes
// and 28 split counts, of the choice and of the time: the choice is 1.2 % behind the best one found on average (fitted to 700 of
// them, 1.1 % on the other 500; with the constants of the merge by a second launch 2.0 %), a rule by row count alone (always
// 256 workgroups where the tiles allow it) was 15 % behind, 70 % for many rows over a short prefix (860 rows over 450 keys: 21 us
// in 256-row blocks and 2 splits, 12 us in 64-row blocks and 5).
// `force_split` > 0 and `force_shape` in 1..3 replace the choice (the tuning entry point passes them).
Plan make_plan(int M, int L, int Hq, int Hkv, int D, int eb = 2, int force_split = 0, int force_shape = 0)
{
    static constexpr struct { int rw, kw, nt; float start, tile[3]; } SHAPES[3] = {      // us; tile: bf16 D = 128, D = 64, FP8
        { 2, 2, 5, 1.90f, { 0.420f, 0.271f, 0.372f } },
        { 4, 2, 8, 2.47f, { 0.494f, 0.294f, 0.495f } },
        { 8, 1, 8, 2.22f, { 0.675f, 0.433f, 0.0f } },
    };
    static constexpr float SHARED_TILE[3] = { 0.596f, 0.337f, 0.517f };                   // two 64-row workgroups on a CU
    static constexpr int SPLITS[] = { 1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 64 };
    const int rows_g = Hq / Hkv * M, kind = eb == 1 ? 2 : D == 64 ? 1 : 0;
    const float bytes = 2.0f * ((float)L + M) * Hkv * D * eb, mem = bytes / 6.73e6f, part = 2.0f * M * Hq * D * 1e-6f;
    Plan best = {};
    float best_t = 0.f;
    for (int k = 0; k < 3; ++k) {
        if (force_shape ? force_shape != k + 1 && !(eb == 1 && force_shape == 3 && k == 1) : eb == 1 && k == 2) continue;
        Plan pl;
        pl.rw = SHAPES[k].rw; pl.kw = SHAPES[k].kw; pl.nt = SHAPES[k].nt;
        pl.wr = pl.rw * 32; pl.bytes = bytes;
        pl.row_blocks = (rows_g + pl.wr - 1) / pl.wr;
        pl.stages = (L + M + TK - 1) / TK;
        auto consider = [&](int want) {
            split_plan(pl, L, want);
            const int n = pl.nsplit, wgs = (n * Hkv + 7) / 8 * 8 * pl.row_blocks;         // (as many as the fullest XCD has, times 8)
            const float cap = k == 0 ? 512.f : 256.f, fill = wgs / cap;
            const float rounds = 0.31f * std::ceil(fill) + 0.69f * std::max(1.f, fill);
            const float comp = rounds * (SHAPES[k].start + (pl.sps + (pl.longer ? pl.kw : 0)) * (k == 0 && wgs > 256 ? SHARED_TILE[kind] : SHAPES[k].tile[kind]));
            float t = std::max(comp, mem) + 0.123f * std::min(comp, mem);
            if (n > 1) t += merges_inside(pl, Hkv) ? 1.67f + 0.70f * n * part : 1.78f + 0.83f * n * part + 0.095f * std::max(0, n - 32);
            if (!best_t || t < best_t) { best = pl; best_t = t; }
        };
        if (force_split > 0) { consider(force_split); continue; }
        // no more splits than tiles, nor partials than the built-in scratch array holds (32 MB are 6 us to write and read)
        const int most = (int)std::min<long long>(std::min(MOST_SPLITS, pl.stages),
                                                  std::max<long long>(1, (long long)(MOST_PARTIALS / (partial_rows(pl, M, Hq, Hkv) * (D * 2 + 16)))));
        for (int want : SPLITS)
            if (want <= most) consider(want);
        for (int cap = 256; cap <= (k == 0 ? 1024 : 512); cap *= 2) {                     // as many as whole rounds take
            const int want = cap / (8 * pl.row_blocks) * 8 / Hkv;
            if (want >= 1 && want <= most) consider(want);
        }
    }
    return best;
}

// A batch: shape of the workgroups by the largest tree's packed rows; in how many parts a row's partials may come; whether a
// merge can be needed at all.  Then either (sps > 0) a workgroup per part of sps tiles, or the plan that the workgroups make
// themselves: how many teams of them the chip holds and the smallest share (slots: a stretch of the longest request gets that
// many parts where the average one is 2.5 times shorter; longer ones larger parts).
struct PlanB { int rw, wr_log2, pairing, teams_log2, slots, wmin, sps, row_blocks; bool merge; };
// The plan that the workgroups make themselves pays where they have much to do (64-row tiles per CU at most, of 128 channels; t: tiles of the longest
// request); below, its larger row blocks and the longer way to the first tile cost more than an even load gives.  us, a grid of parts / the plan.  128 channels: 35
// tiles per CU, t = 142 22.5 / 33.5; 45, t = 242 30.0 / 26.3; 58, t = 124 35.2 / 33.7; 61, t = 63 27.2 / 32.4; 62, t = 333 37.0 / 28.4; 75, t = 240 42.1 / 35.4; 86, t = 185
// 30.4 / 36.9; 101, t = 294 67.6 / 59.9; 104, t = 119 47.5 / 38.0; 115, t = 123 41.0 / 36.2; 150, t = 89 39.2 / 39.4; 178, t = 127 53.2 / 51.7.  64 channels: 60, t = 192
// 21.4 / 26.7; 88, t = 378 27.1 / 30.7; 107, t = 229 27.1 / 26.9; 106, t = 310 28.0 / 24.8; 147, t = 91 33.9 / 28.5; 154, t = 176 35.9 / 29.2; 160, t = 214 28.1 / 29.0; 226, t = 259
// 44.8 / 33.5.  What decides besides is how uneven the lengths are, which the host does not know: of 190 batches the choice is 3.0 % slower than the better form on
// average with 128 channels and 1.1 % with 64, 31 and 19 % at most.  (A line at 60 tiles and t = 80 for 128 channels: 1.5 %, but up to 20 % slower than this one for some.)
bool short_batch(int rows_g, int t, int Hkv, int D, int batch)
{
    const long long tiles_cu = (long long)Hkv * batch * ((rows_g + 63) >> 6) * t / 256;
    return tiles_cu * D < 220 * 128 && !(t >= 90 && tiles_cu * D * t >= 13000ll * 128);
}

PlanB make_batch_plan(int M_max, int L_max, int Hq, int Hkv, int D, int batch, int eb)
{
    PlanB b = {};
    const int G = Hq / Hkv, rows_g = G * M_max, t = (L_max + M_max + TK - 1) / TK;
    if (short_batch(rows_g, t, Hkv, D, batch)) {
        b.rw = 2; b.wr_log2 = 6;
        b.row_blocks = (rows_g + 63) >> 6;
        const int base = Hkv * batch * b.row_blocks;
        // One request: as in the contiguous form.  More: parts of 32 tiles even out the lengths, or of 24 where the workgroups of the
        // whole requests are few (17 requests of up to 1.8k keys with 22 nodes 35.5 us in one part and 26.8 in two, 31 of up to 2.6k
        // with 49, D = 64, 32.6 in two and 27.7 in three; but 30 of up to 2k with 40 49 and 61).  Where that leaves the chip room (it
        // takes 512 of these workgroups at once, but two that share a CU take longer), parts of 4 tiles or more for a workgroup per
        // CU, of 8 or more for two of the longest request, of 16 or more for two rounds of those (2 requests of up to 2.4k with 26
        // nodes took 31 us in 2 parts and take 15 in 9; 7 of up to 1k with 8 13.8 in 3 and 12.0 in 4; 2 of up to 5.7k with 66 26.5
        // in 6 and 23.1 in 8), if a part is more than 10 tiles shorter than the whole: the partials and their merge cost as much
        // (6 of up to 463, D = 64, 9.4 in one and 8.4 in 4; 10 of up to 270 8.7 in one and 10.0 in 3).
        int want = batch == 1 ? std::min((rows_g <= 64 ? 512 : 256) / base, t / 8) : std::min(8, t / (base < 512 ? 24 : 32));
        if (batch > 1 && base < 256) {
            const int one = std::min(256 / base, (t + 3) / 4), two = std::min(512 / base, t / 8);
            const int by = std::min(32, std::max(2 * two >= 3 * one ? two : one, std::min(1024 / base, t / 16)));
            if (by > 1 && t - (t + by - 1) / by > 10) want = std::max(want, by);
        }
        b.sps = ((t + std::max(1, want) - 1) / std::max(1, want) + 1) & ~1;                // whole rounds of two tiles
        b.slots = (t + b.sps - 1) / b.sps;
        b.merge = b.slots > 1;
        return b;
    }
    b.rw = rows_g <= 64 && eb == 1 ? 2 : rows_g <= 128 || eb == 1 ? 4 : 8;
    b.wr_log2 = b.rw == 2 ? 6 : b.rw == 4 ? 7 : 8;
    b.row_blocks = (rows_g + (1 << b.wr_log2) - 1) >> b.wr_log2;
    b.pairing = b.row_blocks > 1;
    b.teams_log2 = (b.rw == 2 ? 9 : 8) - b.pairing;     // (one workgroup per CU, or two of the small ones)
    const long long stretches = (long long)Hkv * batch * ((b.row_blocks + b.pairing) >> b.pairing);
    b.slots = std::min(32, std::max(8, 4 + (int)((5 << b.teams_log2) / (b.pairing ? stretches : 2 * stretches))));
    b.wmin = std::max(2 * START, (t + b.slots - 5) / (b.slots - 4) * WHOLE);
    b.merge = t > SMALL;
    return b;
}

// The merge's words lie at the same place in every workspace of attention calls that hold partials: other calls leave them alone.
struct WsLayout { size_t sync, plan, ml, opart, total; };

WsLayout ws_layout(size_t rows, int D, int nsplit, int batch = 0)
{
    WsLayout w;
    size_t off = BTV_WS_HEADER;
    w.sync = off; off += batch || nsplit > 1 ? MERGE_GROUPS * sizeof(MergeWords) : 0;
    w.plan = off; off += batch ? btv_align_up((size_t)(batch + 2) * sizeof(long long), BTV_WS_ALIGN) : 0;
    size_t ns = nsplit > 1 ? nsplit : 0;
    w.ml = off; off += btv_align_up(ns * rows * 4 * 4, BTV_WS_ALIGN);
    w.opart = off; off += btv_align_up(ns * rows * D * 2, BTV_WS_ALIGN);
    w.total = off;
    return w;
}

// What the workspace queries of one request answer: enough for every call of up to M nodes over up to L keys.  The plan's own need
// is no answer to that: a shorter context or a smaller tree may be cut into more parts, or rows padded to larger blocks (32 nodes of an
// 8B shape: 8.8 MB at 32768 keys, 9.1 at 10208).  No plan of these sizes has more splits than there are tiles, nor than MOST_SPLITS, nor more than
// MOST_PARTIALS bytes in more than one split; partial_rows grows with M.  64 nodes over 8192 keys: 32.6 MB where that call's plan takes 8.6.
size_t enough_for(int M, int L, int Hq, int Hkv, int D, int eb, int force_split = 0, int force_shape = 0)
{
    size_t most = 0;
    const int n = std::min(force_split > 0 ? force_split : MOST_SPLITS, (L + M + TK - 1) / TK);
    for (int k = 1; k <= 3 && n > 1; ++k) {
        if (force_shape ? std::min(force_shape, eb == 1 ? 2 : 3) != k : eb == 1 && k == 3) continue;
        Plan pl = {};
        pl.wr = 32 << k;
        pl.row_blocks = (Hq / Hkv * M + pl.wr - 1) / pl.wr;
        const size_t part = partial_rows(pl, M, Hq, Hkv) * (D * 2 + 16);
        most = std::max(most, force_split > 0 ? n * part : std::min(n * part, MOST_PARTIALS));
    }
    // (the two arrays are aligned one by one)
    static_assert(MOST_PARTIALS + BTV_WS_HEADER + MERGE_GROUPS * sizeof(MergeWords) + 2 * BTV_WS_ALIGN <= SCRATCH_BYTES, "a plan's need fits the built-in array");
    return ws_layout(0, D, n).total + btv_align_up(most, BTV_WS_ALIGN) + (n > 1 ? BTV_WS_ALIGN : 0);
}

// The same for a batch: up to `batch` requests, M_max nodes, L_max keys.  Fewer or smaller requests are cut into more parts, so their
// partials may be the more.  Of make_batch_plan's forms: a short batch takes up to 8 parts of 24 tiles or more; where its grid is
// small, up to 32 parts of 4 tiles or more in no more than 256 workgroups of 64 rows, or of 8 tiles or more in no more than 1024
// (one request: 512 parts in 512); the others 8 parts, or 4 and their share of (5 << teams_log2) pieces, which is 640 row blocks, 1280
// where they go in pairs.  All of it grows with the sizes, and so does what makes a batch one of the others.  8 x 128 nodes over 16k
// keys 124.9 MB, which is that plan's own need.
size_t enough_for_batch(int batch, int M_max, int L_max, int Hq, int Hkv, int D, int eb)
{
    const int rows_g = Hq / Hkv * M_max, t = (L_max + M_max + TK - 1) / TK;
    const long long rows = (long long)batch * M_max * Hq, one = (long long)M_max * Hq;
    long long most = 0;
    if (t >= 48) most = rows * std::min(8, t / 24);
    if (t >= 12) most = std::max(most, std::min<long long>(rows * std::min(32, (t + 3) / 4), 256 * 64));
    if (t >= 16) most = std::max({ most, std::min<long long>(rows * std::min(32, t / 8), 1024 * 64), std::min<long long>(one * std::min(512, t / 8), 512 * 64) });
    if (!short_batch(rows_g, t, Hkv, D, batch)) {
        const long long spread = 640 * 128 * (rows_g <= 128 ? 1 : eb == 1 || rows_g <= 256 ? 2 : 4);
        most = std::max(most, std::min(rows * 32, std::max(rows * 8, rows * 4 + spread)));
    }
    return ws_layout(0, D, 1, batch).total + (most ? btv_align_up((size_t)most * (D * 2 + 16), BTV_WS_ALIGN) + BTV_WS_ALIGN : 0);
}

enum Form { ONE_REQUEST, ONE_MERGED, SHORT_BATCH, LONG_BATCH };

template <int D, int RW, int KW, int NT, Form FORM, int EB = 2>
int launch_bf16(const AttnParams &p, dim3 grid, hipStream_t st)
{
    constexpr int LDS_BYTES = PageLds<D, RW, KW, NT, (FORM > ONE_MERGED), EB>::BYTES + (FORM == LONG_BATCH ? CHUNK_BYTES : 0);
    static_assert(LDS_BYTES * (RW * KW <= 4 ? 2 : 1) <= 160 * 1024, "LDS budget");
    static std::atomic<bool> configured{false};         // (one GPU per process: the attribute is set once)
    void (*kern)(AttnParams);
    if constexpr (FORM == LONG_BATCH) kern = tv_attn_batch<D, RW, KW, NT, EB>;
    else if constexpr (FORM == SHORT_BATCH) kern = tv_attn_short<D, RW, KW, NT, EB>;
    else kern = tv_attn_bf16<D, RW, KW, NT, EB, FORM == ONE_MERGED>;
    if (!configured.load(std::memory_order_acquire)) {
        BTV_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    LDS_BYTES));
        configured.store(true, std::memory_order_release);
    }
    hipLaunchKernelGGL(kern, grid, dim3(RW * KW * 64), LDS_BYTES, st, p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

template <Form FORM>
int dispatch_bf16(const AttnParams &p, int rw, int D, int eb, dim3 grid, hipStream_t st)
{
    if (eb == 1) {      // FP8 K/V
        if (D == 128 && rw == 2) return launch_bf16<128, 2, 2, 5, FORM, 1>(p, grid, st);
        if constexpr (FORM != SHORT_BATCH)
            if (D == 128 && rw == 4) return launch_bf16<128, 4, 2, 8, FORM, 1>(p, grid, st);
        return btv_fail(BTV_EINVAL, "no FP8-KV kernel for D=%d", D);
    }
#define BTV_CASE(DD, RR, KK, NN) \
    if (D == DD && rw == RR) return launch_bf16<DD, RR, KK, NN, FORM>(p, grid, st);
    if constexpr (FORM != LONG_BATCH) { BTV_CASE(128, 2, 2, 5) BTV_CASE(64, 2, 2, 5) }
    if constexpr (FORM != SHORT_BATCH) {
        BTV_CASE(128, 4, 2, 8) BTV_CASE(128, 8, 1, 8) BTV_CASE(64, 4, 2, 8) BTV_CASE(64, 8, 1, 8)
    }
#undef BTV_CASE
    return btv_fail(BTV_EINVAL, "no kernel for D=%d", D);
}

int check_shape(int M, int L, int Hq, int Hkv, int D)
{
    BTV_REQUIRE(M >= 1 && M <= BTV_MAX_NODES, "M=%d outside [1,%d]", M, BTV_MAX_NODES);
    BTV_REQUIRE(L >= 0 && (long long)L + M < (1ll << 30), "L=%d out of range", L);
    BTV_REQUIRE(Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && Hq / Hkv <= 16, "bad heads Hq=%d Hkv=%d", Hq, Hkv);
    BTV_REQUIRE(D == 64 || D == 128, "D=%d not in {64,128}", D);
    return BTV_OK;
}

int check_fp8(int D, float k_scale, float v_scale)
{
    BTV_REQUIRE(D == 128, "FP8 K/V: D=%d, only 128 is built", D);
    BTV_REQUIRE(k_scale > 0.f && k_scale <= 3.0e38f && v_scale > 0.f && v_scale <= 3.0e38f,
                "FP8 K/V scales must be positive and finite");
    return BTV_OK;
}

bool aligned16(const void *a) { return (reinterpret_cast<uintptr_t>(a) & 15u) == 0; }

// eb = bytes per K/V element (2: the dtype's own; 1: E4M3 codes, bf16 Q and O).  The key scale multiplies every
// score, so it joins the softmax scale; the value scale multiplies the weighted sum, so it joins the final division.
void set_scales(AttnParams &p, int D, float scale, float k_scale, float v_scale)
{
    p.scale = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * k_scale;
    p.scale_log2 = p.scale * 1.4426950408889634f;
    p.out_scale = v_scale;
}

int attn_contiguous(const void *Q, const void *K, const void *V, const int32_t *parent, int M, int L, int Hq, int Hkv,
                    int D, int dtype, int eb, float scale, float k_scale, float v_scale, void *O, void *ws,
                    size_t ws_bytes, void *stream, int force_split = 0, int force_shape = 0, uint32_t *flag_out = nullptr,
                    int merge = 0, int wait_ticks = MERGE_WAIT_TICKS)
{
    BTV_REQUIRE(Q && K && V && parent && O, "null pointer");
    BTV_REQUIRE(aligned16(Q) && aligned16(K) && aligned16(V) && aligned16(O), "Q, K, V and O must be 16-byte aligned");
    int rc = check_shape(M, L, Hq, Hkv, D);
    if (rc) return rc;
    hipStream_t st = static_cast<hipStream_t>(stream);
    Plan pl = make_plan(M, L, Hq, Hkv, D, eb, force_split, force_shape);
    if (dtype == BTV_F32) pl.nsplit = 1;
    WsLayout wl = ws_layout(partial_rows(pl, M, Hq, Hkv), D, pl.nsplit);
    rc = btv_check_ws(ws, ws_bytes, wl.total);
    if (rc) return rc;
    unsigned char *w8 = static_cast<unsigned char *>(ws);
    AttnParams p = {};
    p.Q = Q; p.K = K; p.V = V; p.O = O;
    p.ML = reinterpret_cast<float *>(w8 + wl.ml);
    p.Opart = reinterpret_cast<_Float16 *>(w8 + wl.opart);
    p.flag = flag_out ? flag_out : reinterpret_cast<uint32_t *>(w8);
    p.M = M; p.L = L; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.ginv = (65536 + p.G - 1) / p.G;
    p.total_rows = M * Hq; p.total_M = M;
    p.sps = pl.sps; p.longer = pl.longer; p.nsplit = pl.nsplit; p.inv_nsplit = reciprocal(pl.nsplit);
    set_scales(p, D, scale, k_scale, v_scale);
    p.parent = parent;
    if (dtype == BTV_F32) {
        if (D == 64) hipLaunchKernelGGL(tv_attn_f32<64>, dim3(M, Hq), dim3(256), 0, st, p);
        else hipLaunchKernelGGL(tv_attn_f32<128>, dim3(M, Hq), dim3(256), 0, st, p);
        BTV_HIP(hipGetLastError());
        return BTV_OK;
    }
    p.row_blocks = pl.row_blocks; p.inv_row_blocks = reciprocal(pl.row_blocks);
    const bool inside = merge != 1 && merges_inside(pl, Hkv) && (merge || btv_usable_cus(st) >= 256);
    int wgs;
    if (inside) {
        p.sync = reinterpret_cast<unsigned long long *>(w8 + wl.sync);
        p.wait_ticks = wait_ticks;
        p.units = merge == 3 ? 0 : Hkv % 8 == 0 ? Hkv : Hkv * pl.row_blocks;
        wgs = merge == 3 ? (pl.nsplit * Hkv + 7) / 8 * 8 * pl.row_blocks : pl.nsplit * Hkv * pl.row_blocks;
    } else {
        p.units = pl.nsplit * Hkv;
        wgs = ((p.units + 7) / 8) * pl.row_blocks * 8;
    }
    rc = inside ? dispatch_bf16<ONE_MERGED>(p, pl.rw, D, eb, dim3(wgs), st) : dispatch_bf16<ONE_REQUEST>(p, pl.rw, D, eb, dim3(wgs), st);
    if (rc) return rc;
    if (pl.nsplit > 1 && !inside) {
        dim3 cg((M * Hq + 7) / 8, 1);
        if (D == 64) hipLaunchKernelGGL(tv_combine_bf16<64>, cg, dim3(256), 0, st, p);
        else hipLaunchKernelGGL(tv_combine_bf16<128>, cg, dim3(256), 0, st, p);
        BTV_HIP(hipGetLastError());
    }
    return BTV_OK;
}

int attn_paged(const void *Q, const void *Kpool, const void *Vpool, int num_blocks, const int32_t *block_table,
               int max_blocks, const int32_t *q_offset, const int32_t *prefix_len, const int32_t *parent, int batch,
               int total_M, int M_max, int L_max, int Hq, int Hkv, int D, int eb, float scale, float k_scale,
               float v_scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(Q && Kpool && Vpool && block_table && q_offset && prefix_len && parent && O, "null pointer");
    BTV_REQUIRE(aligned16(Q) && aligned16(Kpool) && aligned16(Vpool) && aligned16(O),
                "Q, K, V and O must be 16-byte aligned");
    BTV_REQUIRE(batch >= 1 && batch <= 4096, "batch=%d outside [1,4096]", batch);
    int rc = check_shape(M_max, L_max, Hq, Hkv, D);
    if (rc) return rc;
    BTV_REQUIRE(total_M >= 1 && total_M <= batch * M_max, "total_M=%d inconsistent with batch*M_max", total_M);
    BTV_REQUIRE(num_blocks >= 1 && max_blocks >= 1, "bad block counts");
    BTV_REQUIRE((long long)max_blocks * BTV_PAGE >= (long long)L_max + 1, "max_blocks too small for L_max");
    hipStream_t st = static_cast<hipStream_t>(stream);
    const PlanB pl = make_batch_plan(M_max, L_max, Hq, Hkv, D, batch, eb);
    WsLayout wl = ws_layout((size_t)batch * M_max * Hq, D, pl.slots, batch);
    rc = btv_check_ws(ws, ws_bytes, wl.total);
    if (rc) return rc;
    unsigned char *w8 = static_cast<unsigned char *>(ws);
    AttnParams p = {};
    p.Q = Q; p.K = Kpool; p.V = Vpool; p.O = O;
    p.ML = reinterpret_cast<float *>(w8 + wl.ml);
    p.Opart = reinterpret_cast<_Float16 *>(w8 + wl.opart);
    p.flag = reinterpret_cast<uint32_t *>(w8);
    p.block_table = block_table; p.q_offset = q_offset; p.prefix_len = prefix_len;
    p.max_blocks = max_blocks; p.num_blocks = num_blocks;
    p.M = M_max; p.L = L_max; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.ginv = (65536 + p.G - 1) / p.G;
    p.total_rows = batch * M_max * Hq;    // partial buffers are sized for the bound; rows index by q_offset
    p.total_M = total_M;
    p.plan = reinterpret_cast<long long *>(w8 + wl.plan);
    p.batch = batch; p.teams_log2 = pl.teams_log2; p.pairing = pl.pairing; p.wmin = pl.wmin; p.wr_log2 = pl.wr_log2;
    set_scales(p, D, scale, k_scale, v_scale);
    p.parent = parent;
    p.sps = pl.sps; p.row_blocks = pl.row_blocks; p.inv_row_blocks = reciprocal(pl.row_blocks);
    if (pl.sps) {
        p.nsplit = pl.slots; p.inv_nsplit = reciprocal(pl.slots); p.inv_sps = reciprocal(pl.sps); p.inv_Hkv = reciprocal(Hkv);
        p.units = pl.slots * Hkv * batch;
        rc = dispatch_bf16<SHORT_BATCH>(p, pl.rw, D, eb, dim3(((p.units + 7) / 8) * pl.row_blocks * 8), st);
    } else {
        rc = dispatch_bf16<LONG_BATCH>(p, pl.rw, D, eb, dim3(1 << (pl.teams_log2 + pl.pairing)), st);
    }
    if (rc || !pl.merge) return rc;
    const int rows = M_max * Hq;
    auto combine = [&](auto kern, int per) { hipLaunchKernelGGL(kern, dim3((rows + per - 1) / per, batch), dim3(256), 0, st, p); };
    const bool many = (long long)rows * batch > 12288;
    if (D == 64) many ? combine(tv_combine_batch<64, 8, 8>, 32) : combine(tv_combine_batch<64, 2, 16>, 8);
    else many ? combine(tv_combine_batch<128, 8, 8>, 16) : combine(tv_combine_batch<128, 4, 16>, 8);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

}  // namespace

extern "C" {

int btv_tree_ancestor_mask(const int32_t *parent, int M, uint32_t *anc, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(parent && anc, "null pointer");
    BTV_REQUIRE(M >= 1 && M <= BTV_MAX_NODES, "M=%d outside [1,%d]", M, BTV_MAX_NODES);
    int rc = btv_check_ws(ws, ws_bytes, BTV_WS_HEADER);
    if (rc) return rc;
    hipLaunchKernelGGL(anc_mask_kernel, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream), parent, M, anc, static_cast<uint32_t *>(ws));
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

size_t btv_tree_verify_attn_workspace(int M, int L, int Hq, int Hkv, int D, int dtype)
{
    if (check_shape(M, L, Hq, Hkv, D) != BTV_OK) return 0;
    return dtype == BTV_BF16 ? enough_for(M, L, Hq, Hkv, D, 2) : ws_layout(0, D, 1).total;
}

int btv_tree_verify_attn(const void *Q, const void *K, const void *V, const int32_t *parent, int M, int L, int Hq,
                         int Hkv, int D, int dtype, float scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(dtype == BTV_F32 || dtype == BTV_BF16, "dtype=%d unsupported", dtype);
    return attn_contiguous(Q, K, V, parent, M, L, Hq, Hkv, D, dtype, 2, scale, 1.0f, 1.0f, O, ws, ws_bytes, stream);
}

int btv_tree_verify_attn_noalloc(const void *Q, const void *K, const void *V, const int32_t *parent, int M, int L, int Hq,
                                 int Hkv, int D, int dtype, float scale, void *O, uint32_t *status, void *stream)
{
    BTV_REQUIRE(dtype == BTV_F32 || dtype == BTV_BF16, "dtype=%d unsupported", dtype);
    int rc = check_shape(M, L, Hq, Hkv, D);
    if (rc) return rc;
    void *ws = nullptr;
    rc = scratch_address(&ws);
    if (rc) return rc;
    // the header (data flag, counters) must start at zero whatever an earlier call left behind
    hipLaunchKernelGGL(fill_zero_kernel, dim3(1), dim3(256), 0, static_cast<hipStream_t>(stream),
                       static_cast<uint32_t *>(ws), (int)(BTV_WS_HEADER / 4));
    BTV_HIP(hipGetLastError());
    return attn_contiguous(Q, K, V, parent, M, L, Hq, Hkv, D, dtype, 2, scale, 1.0f, 1.0f, O, ws, SCRATCH_BYTES, stream, 0, 0,
                           status);
}

size_t btv_tree_verify_attn_fp8kv_workspace(int M, int L, int Hq, int Hkv, int D)
{
    if (check_shape(M, L, Hq, Hkv, D) != BTV_OK || D != 128) return 0;
    return enough_for(M, L, Hq, Hkv, D, 1);
}

int btv_tree_verify_attn_fp8kv(const void *Q, const void *K8, const void *V8, float k_scale, float v_scale,
                               const int32_t *parent, int M, int L, int Hq, int Hkv, int D, float scale, void *O,
                               void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_fp8(D, k_scale, v_scale);
    if (rc) return rc;
    return attn_contiguous(Q, K8, V8, parent, M, L, Hq, Hkv, D, BTV_BF16, 1, scale, k_scale, v_scale, O, ws, ws_bytes,
                           stream);
}

size_t btv_tree_verify_attn_tuned_workspace(int M, int L, int Hq, int Hkv, int D, int kv_fp8, int nsplit, int shape)
{
    if (check_shape(M, L, Hq, Hkv, D) != BTV_OK || (kv_fp8 && D != 128) || nsplit < 0 || shape < 0 || shape > 3) return 0;
    return enough_for(M, L, Hq, Hkv, D, kv_fp8 ? 1 : 2, nsplit, shape);
}

int btv_tree_verify_attn_tuned(const void *Q, const void *K, const void *V, int kv_fp8, float k_scale, float v_scale,
                               const int32_t *parent, int M, int L, int Hq, int Hkv, int D, float scale, int nsplit,
                               int shape, void *O, void *ws, size_t ws_bytes, void *stream)
{
    return btv_tree_verify_attn_merge_tuned(Q, K, V, kv_fp8, k_scale, v_scale, parent, M, L, Hq, Hkv, D, scale, nsplit, shape, 0,
                                            MERGE_WAIT_TICKS, O, ws, ws_bytes, stream);
}

int btv_tree_verify_attn_merge_tuned(const void *Q, const void *K, const void *V, int kv_fp8, float k_scale, float v_scale,
                                     const int32_t *parent, int M, int L, int Hq, int Hkv, int D, float scale, int nsplit,
                                     int shape, int merge, int wait_ticks, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(merge >= 0 && merge <= 3, "merge=%d outside [0,3]", merge);
    BTV_REQUIRE(nsplit >= 0 && shape >= 0 && shape <= 3, "nsplit=%d or shape=%d out of range", nsplit, shape);
    if (kv_fp8) {
        int rc = check_fp8(D, k_scale, v_scale);
        if (rc) return rc;
        BTV_REQUIRE(shape != 3, "shape 3 is not built for an FP8 cache");
    }
    return attn_contiguous(Q, K, V, parent, M, L, Hq, Hkv, D, BTV_BF16, kv_fp8 ? 1 : 2, scale, kv_fp8 ? k_scale : 1.0f,
                           kv_fp8 ? v_scale : 1.0f, O, ws, ws_bytes, stream, nsplit, shape, nullptr, merge, wait_ticks);
}

size_t btv_tree_verify_attn_paged_workspace(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    if (batch < 1 || batch > 4096 || check_shape(M_max, L_max, Hq, Hkv, D) != BTV_OK) return 0;
    return enough_for_batch(batch, M_max, L_max, Hq, Hkv, D, 2);
}

int btv_tree_verify_attn_paged(const void *Q, const void *Kpool, const void *Vpool, int num_blocks,
                               const int32_t *block_table, int max_blocks, const int32_t *q_offset,
                               const int32_t *prefix_len, const int32_t *parent, int batch, int total_M, int M_max,
                               int L_max, int Hq, int Hkv, int D, float scale, void *O, void *ws, size_t ws_bytes,
                               void *stream)
{
    return attn_paged(Q, Kpool, Vpool, num_blocks, block_table, max_blocks, q_offset, prefix_len, parent, batch, total_M,
                      M_max, L_max, Hq, Hkv, D, 2, scale, 1.0f, 1.0f, O, ws, ws_bytes, stream);
}

size_t btv_tree_verify_attn_paged_fp8kv_workspace(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    if (batch < 1 || batch > 4096 || check_shape(M_max, L_max, Hq, Hkv, D) != BTV_OK || D != 128) return 0;
    return enough_for_batch(batch, M_max, L_max, Hq, Hkv, D, 1);
}

int btv_tree_verify_attn_paged_fp8kv(const void *Q, const void *K8pool, const void *V8pool, float k_scale,
                                     float v_scale, int num_blocks, const int32_t *block_table, int max_blocks,
                                     const int32_t *q_offset, const int32_t *prefix_len, const int32_t *parent,
                                     int batch, int total_M, int M_max, int L_max, int Hq, int Hkv, int D, float scale,
                                     void *O, void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_fp8(D, k_scale, v_scale);
    if (rc) return rc;
    return attn_paged(Q, K8pool, V8pool, num_blocks, block_table, max_blocks, q_offset, prefix_len, parent, batch,
                      total_M, M_max, L_max, Hq, Hkv, D, 1, scale, k_scale, v_scale, O, ws, ws_bytes, stream);
}

}  // extern "C"
