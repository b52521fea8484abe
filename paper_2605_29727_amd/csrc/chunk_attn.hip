// Causal attention of the requests' new rows over a paged KV cache (gfx950), bf16 or E4M3 K/V: prompts, chunks of them and single tokens in one
// ragged batch.
//
// What is computed: row i of request r, which has L rows in the cache ahead of its new ones, sees the keys 0 .. L + i:
//   O[i,h] = sum_j p_j V[j,g] / sum_j p_j,  p_j = exp2(scale log2(e) (Q[i,h].K[j,g] - m)),  m a reference that follows the largest score.
// One pass over the keys; rows' sums and accumulators stay in fp32 registers (attn_piece.h).  A workgroup takes a row block of whole nodes (node: a new
// token; its G = Hq / Hkv query heads are G packed rows, so that a K/V byte serves all of them) and a range of 32-key tiles.  Long chunks are bound
// by the matrix cores, single tokens by the stream of K/V.
//
// The host knows bounds on the lengths only, so the workgroups share the work out themselves.  A row block is START + weight * keys long (the keys that its last node sees;
// the weight is WHOLE, or PART where no more than half of the block's rows exist and a tile goes faster); blocks lie one after the other, request
// after request, KV head after KV head, and workgroup k takes what lies between k w and (k + 1) w.  Where that cuts a block, each part's rows go to the
// workgroup's own place in the workspace (two at most: a block that it carries on with, one that it begins), and the workgroup that stores the last of them joins them in the order of the keys
// (of 256 rows and longer work a second launch).
// Neighbouring shares are on one XCD, which so keeps to one KV head or two, whose K/V its workgroups meet in their L2.  Where there are fewer blocks than workgroups, blocks go
// in even parts instead, and where there are more, but a few for each workgroup at most and of lengths that come out even, whole blocks in turns.
//
// A chunk of 2048 tokens behind 30720, 64 heads of 128 (8 of K/V): 1.81 ms, 1.18 PFLOP/s (a bf16 product of 8192^3: 1.40), behind 8192 with 32 heads 292 us, 1.06 (7 % more
// on some cards); of a tile's 0.93 us the matrix instructions alone take 0.6 to 0.7 at the clock that they leave, the exponentials and the LDS reads the rest.  32 tokens over 100 to 4000 keys,
// E4M3, 51 MB: 18.4 us.  Blocks of few tiles are bound by a piece's ends (us, 256 rows of 128): finding it 1.4, the first loads 2 to 3, the first scores 1.2, the last products
// 1.1, the masked tiles 1.5, the last sums 1.4, stores 1.
#include "attn_piece.h"

#include <atomic>
#include <climits>

namespace {

typedef long long i64;

constexpr int WHOLE = 3, PART = 2;                              // weights of a key
constexpr int MARGIN = 2, SMALL = 8;                            // tiles: a cut nearer to a block's ends moves there; blocks of up to SMALL are not cut
constexpr int LEAST_PART = 8, LEAST_OF_FEW = 4, UNCUT = 16;     // tiles of the smallest part (of few rows); blocks of up to UNCUT are not worth a merge
constexpr int MOST_ROWS = 1 << 20, MOST_TEAMS = 512;
constexpr int FEW_ROWS = 16;                                   // of single tokens' blocks, whose parts have less room

// The cut block that a workgroup begins, for the merge behind: its parts (0: none), and its first row of Q and O as [total_M].
struct Begun { int parts, row0, nodes, g; };

struct ChunkParams : AttnParams {
    Begun *begun;                 // [teams], for a merge by a launch behind (null: by the workgroups)
    int nb;                       // nodes per row block
    uint32_t inv_nb;              // for quotient()
    int wr;                       // rows per row block
    int teams;                    // workgroups: a power of two
    int start;                    // what a row block costs besides its keys
    int most_keys;                // what a row of the block table has room for
    int weight;                   // of a key, for the largest request's blocks
    int part_rows;                // a workgroup's room for a part's rows
    MergeWords *words;            // how many of a block's parts are stored
    int always_parts;             // few rows: parts whatever the shares would be
    int least_part;               // tiles
};

// 64-bit minimum and maximum of numbers less than 2^62 apart, by the sign of their difference.  (Of values that a wavefront has in common the compiler makes a vector
// comparison and a scalar selection, and has left out what carries the one's result to the other: every share came out as the smallest one.)
__device__ __forceinline__ i64 least(i64 a, i64 b) { return b + ((a - b) & ((a - b) >> 63)); }
__device__ __forceinline__ i64 most(i64 a, i64 b) { return a - ((a - b) & ((a - b) >> 63)); }

__device__ __forceinline__ int part_weight(const ChunkParams &p, int nodes) { return nodes * p.G * 2 <= p.wr ? PART : WHOLE; }
// Length of a request's first b blocks (whole ones)
__device__ __forceinline__ i64 length_to(const ChunkParams &p, int L, int b)
{
    return b * (p.start + (i64)WHOLE * L) + (i64)(WHOLE * p.nb) * (i64)((unsigned long long)((i64)b * (b + 1)) >> 1);
}
__device__ __forceinline__ i64 length_of(const ChunkParams &p, int L, int M)
{
    const int whole = quotient(M, p.nb, p.inv_nb), rest = M - whole * p.nb;
    return length_to(p, L, whole) + (rest ? p.start + (i64)part_weight(p, rest) * (L + M) : 0);
}

// Inclusive sums over the lanes, of numbers below 2^26; of lengths below 2^54 in three pieces.
__device__ __forceinline__ int wave_sums(int x)
{
    // (rows of 16 by shifts, then the last lane of each row into the rows behind it)
#define BTV_SCAN_STEP(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, ctrl < 0x142)
    BTV_SCAN_STEP(0x111, 0xF); BTV_SCAN_STEP(0x112, 0xF); BTV_SCAN_STEP(0x114, 0xF); BTV_SCAN_STEP(0x118, 0xF);
    BTV_SCAN_STEP(0x142, 0xA); BTV_SCAN_STEP(0x143, 0xC);
#undef BTV_SCAN_STEP
    return x;
}
__device__ __forceinline__ i64 wave_sums_of_lengths(i64 x)
{
    constexpr int B = 18;
    const i64 lo = wave_sums((int)x & ((1 << B) - 1)), mid = wave_sums((int)(x >> B) & ((1 << B) - 1)), hi = wave_sums((int)(x >> 2 * B));
    return lo + (mid << B) + (hi << 2 * B);
}
__device__ __forceinline__ int wave_max(int x)             // (not negative)
{
#define BTV_MAX_STEP(ctrl, rows) x = max(x, __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, ctrl < 0x142))
    BTV_MAX_STEP(0x111, 0xF); BTV_MAX_STEP(0x112, 0xF); BTV_MAX_STEP(0x114, 0xF); BTV_MAX_STEP(0x118, 0xF);
    BTV_MAX_STEP(0x142, 0xA); BTV_MAX_STEP(0x143, 0xC);
#undef BTV_MAX_STEP
    return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ i64 lane_value(i64 x, int lane)
{
    return (i64)(((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)x, lane));
}

// 64 requests, one per lane, and where each ends in a KV head's work.
struct Chunk { int q0, L, M, beyond; i64 incl; bool bad; };      // (beyond: the order of whole blocks)
__device__ __forceinline__ Chunk load_chunk(const ChunkParams &p, int c0, int lane, i64 before)
{
    Chunk c;
    const bool in = c0 + lane < p.batch;
    const int r = min(c0 + lane, p.batch - 1);
    const int q1 = p.q_offset[r + 1];
    c.q0 = p.q_offset[r];
    c.L = p.prefix_len[r];
    bool ok = c.q0 >= 0 && q1 >= c.q0 && q1 <= p.total_M && c.L >= 0 && c.L <= p.L;
    c.M = ok ? q1 - c.q0 : 0;
    ok = ok && c.M <= p.M && c.L + c.M <= p.most_keys;
    c.bad = in && !ok;
    if (!in || !ok) c.M = c.L = 0;
    c.incl = wave_sums_of_lengths(c.M ? length_of(p, c.L, c.M) : 0) + before;
    return c;
}
// The first chunk is kept in LDS from one piece to the next, and where each wavefront stands (raw instructions: ahead of ordinary reads the compiler waits for the last
// piece's stores, as it would for registers that it spills), but where two workgroups fill the LDS of a CU to the last byte; there the chunk is loaded again.
constexpr int CHUNK_BYTES = 64 * 32;
template <int D, int RW, int KW, int NT, int EB>
struct ChunkLds {
    using PL = PageLds<D, RW, KW, NT, true, EB>;
    static constexpr bool KEPT = (PL::BYTES + CHUNK_BYTES) * PL::PER_CU <= 160 * 1024;
    static constexpr int BYTES = PL::BYTES + (KEPT ? CHUNK_BYTES : 0);
};
// Where a workgroup stands (every wavefront works it out for itself).
struct Walk {
    i64 pos, end;                 // its share, and what comes next
    i64 head, wh;                 // where the current KV head's work begins; one head's work
    i64 w;                        // a share
    int h, team;                  // that head; the workgroup's place in the order of the shares
    int part;                     // parts: tiles of a part (0: shares or whole blocks)
    int step;                     // whole blocks: tiles of a step in their order (0: shares or parts); pos and end count turns
};

// Places of the lanes' numbers, one array after another, and of the wavefronts' walks.
constexpr int WALK_BYTES = 64, AT_WALKS = CHUNK_BYTES - 8 * WALK_BYTES;
__device__ __forceinline__ void keep_chunk(uint32_t kept, int lane, const Chunk &c)
{
    asm volatile("ds_write_b64 %0, %2\n\tds_write_b32 %1, %3 offset:512\n\tds_write_b32 %1, %4 offset:768\n\tds_write_b32 %1, %5 offset:1024\n\t"
                 "ds_write_b32 %1, %6 offset:1280\n\ts_waitcnt lgkmcnt(0)"
                 :: "v"(kept + (uint32_t)lane * 8), "v"(kept + (uint32_t)lane * 4), "v"(c.incl), "v"(c.L), "v"(c.M), "v"(c.q0), "v"(c.beyond) : "memory");
}
static_assert(AT_WALKS == 1536, "the offsets here");
typedef int int4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void keep_walk(uint32_t kept, int tid, const Walk &k)
{
    const int4v a = { (int)k.pos, (int)(k.pos >> 32), (int)k.end, (int)(k.end >> 32) }, b = { (int)k.head, (int)(k.head >> 32), (int)k.wh, (int)(k.wh >> 32) };
    const int4v c = { k.h, k.team, k.part, k.step }, d = { (int)k.w, (int)(k.w >> 32), 0, 0 };
    if ((tid & 63) == 0)
        asm volatile("ds_write_b128 %0, %1\n\tds_write_b128 %0, %2 offset:16\n\tds_write_b128 %0, %3 offset:32\n\tds_write_b128 %0, %4 offset:48\n\ts_waitcnt lgkmcnt(0)"
                     :: "v"(kept + AT_WALKS + (tid >> 6) * WALK_BYTES), "v"(a), "v"(b), "v"(c), "v"(d) : "memory");
}
__device__ __forceinline__ Chunk kept_chunk(uint32_t kept, int tid, Walk &k)
{
    Chunk c;
    int4v w[4];
    asm volatile("ds_read_b128 %0, %11\n\tds_read_b128 %1, %11 offset:16\n\tds_read_b128 %2, %11 offset:32\n\tds_read_b128 %3, %11 offset:48\n\t"
                 "ds_read_b64 %4, %9\n\tds_read_b32 %5, %10 offset:512\n\tds_read_b32 %6, %10 offset:768\n\tds_read_b32 %7, %10 offset:1024\n\t"
                 "ds_read_b32 %8, %10 offset:1280\n\ts_waitcnt lgkmcnt(0)"
                 : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(c.incl), "=&v"(c.L), "=&v"(c.M), "=&v"(c.q0), "=&v"(c.beyond)
                 : "v"(kept + (uint32_t)(tid & 63) * 8), "v"(kept + (uint32_t)(tid & 63) * 4), "v"(kept + AT_WALKS + (tid >> 6) * WALK_BYTES) : "memory");
    c.bad = false;
    auto word = [&](int i) { return __builtin_amdgcn_readfirstlane(w[i >> 2][i & 3]); };
    auto pair = [&](int i) { return (i64)(((unsigned long long)(uint32_t)word(i + 1) << 32) | (uint32_t)word(i)); };
    k.pos = pair(0); k.end = pair(2); k.head = pair(4); k.wh = pair(6); k.w = pair(12);
    k.h = word(8); k.team = word(9); k.part = word(10); k.step = word(11);
    return c;
}

// The place in the order of `active` shares on each XCD, neighbours on one XCD; the others have no work, but say so.
__device__ __forceinline__ int team_of(int per_xcd)
{
    const int xcd = blockIdx.x & 7, nth = blockIdx.x >> 3;
    return nth < per_xcd ? xcd * per_xcd + nth : 8 * per_xcd + (nth - per_xcd) * 8 + xcd;
}

// n / d for 0 <= n, 1 <= d < 2^22 (the quotient by the reciprocal is off by one at most)
__device__ __forceinline__ int divided(int n, int d, float inv)
{
    int q = (int)((float)n * inv);
    const int r = n - q * d;
    q += r >= d;
    q -= r < 0;
    return q;
}
__device__ __forceinline__ int parts_of(int t, int part, float inv) { return t <= UNCUT ? 1 : divided(t + part - 1, part, inv); }

// The order of whole blocks: the longest first, of all requests, a block's KV heads beside each other.  Turn by turn the workgroups take one each, back and
// forth, so that who had a long one has a short one next; eight neighbours stay in their order, and so on their XCD's KV heads.  Lengths count in 64 steps of
// as many tiles: lane j knows how many blocks (of one KV head) are longer than j steps, and that gives a place in the order its step.
// Shares are even, but each carries on with a block that another has begun, and cuts are merged: whole blocks may take MORE tiles longer (14 prompts of up to 615 tokens, 32 heads
// of 64: 32 us in shares, 21 whole; 26 of up to 1096, 28 heads of 128: 103 and 93; a chunk of 2048 behind 30720, 64 heads: 1900 and 1820.  With 45 tiles more
// 9 chunks of up to 1024 behind 2371 at most took 68 us whole and 62 in shares; with 14 the 26 prompts stayed in shares).
constexpr int TURNS = 8, MORE = 28;
__device__ __forceinline__ int unit_of(const ChunkParams &p, int team, int turn)
{
    return turn * p.teams + ((turn & 1) ? (p.teams - 8 - (team & ~7)) + (team & 7) : team);
}
// How many of a request's blocks are longer than t tiles: whole ones, and one of the rest.
__device__ __forceinline__ int blocks_beyond(const ChunkParams &p, int L, int M, int t)
{
    const int keys = 32 * t + 1 - L;                    // new rows up to and with the last one of such a block, at least
    const int whole = quotient(M, p.nb, p.inv_nb), first = quotient(max(keys, 1) + p.nb - 1, p.nb, p.inv_nb);
    return max(whole - first + 1, 0) + (M > whole * p.nb && M >= keys);
}
__device__ __forceinline__ int step_at(int beyond, int rank) { return __builtin_popcountll(__builtin_amdgcn_ballot_w64(beyond > rank)) - 1; }    // -1: not as many blocks
// Whether whole blocks take no longer than shares: what the first, the middle and the last workgroup have, against a share, a block that it carries on with and the merge.
template <int WAVES>
__device__ __forceinline__ bool whole_blocks(const ChunkParams &p, Walk &k, Chunk &c, int lane, int units, int longest, i64 w, int *counts)
{
    const int most_length = (int)least(w + MORE * 32 * WHOLE, INT_MAX);
    k.step = (longest + 63) >> 6;
    if (longest * (32 * WHOLE) > most_length) return false;
    int n = 0;                                          // the wavefronts share the requests out
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int r = wave; r < p.batch; r += WAVES) n += blocks_beyond(p, __builtin_amdgcn_readlane(c.L, r), __builtin_amdgcn_readlane(c.M, r), lane * k.step);
    counts[wave * 64 + lane] = n;
    __syncthreads();
    c.beyond = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) c.beyond += counts[i * 64 + lane];
    __syncthreads();                                    // (the first fills go there)
    int most_sum = 0;
    for (int s = 0; s < 3; ++s) {
        const int team = s == 0 ? 0 : s == 1 ? p.teams >> 1 : p.teams - 1;
        int sum = 0;
        for (int turn = 0; turn * p.teams < units; ++turn) {
            const int step = step_at(c.beyond, quotient(unit_of(p, team, turn), p.Hkv, p.inv_Hkv));
            if (step >= 0) sum += p.start + (step * k.step + ((k.step + 1) >> 1)) * (32 * WHOLE);
        }
        most_sum = max(most_sum, sum);
    }
    return most_sum <= most_length;
}

// Even parts of 64 rows (single tokens' aside) are weighed with 60 tiles for a block, not 14: where all blocks find a workgroup, the large number keeps them in parts, and in one piece where
// parts would be hardly smaller (29 chunks of up to 96 behind 1313, 28 heads: 30.5 us with 14, so 24.7; 3 prompts of up to 3064: 21.9, 17.2).  Single tokens split at less (16 over up to 1094
// keys, E4M3: 16.3 with 100, with 14 12.0), and shares would count long and short blocks alike (128 single tokens over 100 to 4000 keys, 8 KV heads, bf16: 147 with 60, with 14 130; E4M3 92.4,
// 76.9; 700 over up to 8000, E4M3: 577, 517).
constexpr int MORE_OF_PARTS = (60 - 14) * 32 * WHOLE;
template <bool FEW, int WAVES>
__device__ __forceinline__ Walk share_out(const ChunkParams &p, int lane, bool leader, Chunk &c, int *counts)
{
    Walk k;
    i64 all = 0;
    bool bad = false;
    for (int c0 = ((p.batch - 1) >> 6) << 6; c0 >= 0; c0 -= 64) {       // (the first chunk last; where the others end does not matter yet)
        c = load_chunk(p, c0, lane, 0);
        bad = bad || c.bad;
        all += lane_value(c.incl, 63);
    }
    if (leader && bad) atomicOr(p.flag, 2u);
    k.head = 0; k.h = 0; k.part = 0; k.step = 0; c.beyond = 0;
    k.wh = all; k.w = 0;
    all *= p.Hkv;
    const int teams_log2 = 31 - __builtin_clz(p.teams);
    const i64 w = most((all + p.teams - 1) >> teams_log2, p.wmin);
    if (p.batch <= 64) {
        // Few blocks: every part of at most `part` tiles has a workgroup of its own, with the smallest such number for which there are enough (all blocks of a request go in as
        // many parts as its last).  A share costs its length and START for what it carries on with, a part its tiles and START: where requests differ so
        // much that the longest part takes longer, shares it is.
        const int blocks = quotient(c.M + p.nb - 1, p.nb, p.inv_nb), t = c.M ? (c.L + c.M + 31) >> 5 : 0;
        const int head_blocks = __builtin_amdgcn_readlane(wave_sums(blocks), 63), all_blocks = head_blocks * p.Hkv, longest = wave_max(t);
        if constexpr (!FEW)
            if (all_blocks > p.teams && all_blocks <= TURNS * p.teams && longest > SMALL && longest < 1 << 16
                && whole_blocks<WAVES>(p, k, c, lane, all_blocks, longest, w, counts)) {
                k.team = blockIdx.x;
                k.pos = 0; k.end = (all_blocks + p.teams - 1) >> teams_log2;
                return k;
            }
        k.step = 0;
        if (all_blocks <= p.teams && all_blocks > 0) {
            const int more = FEW && !p.always_parts ? MORE_OF_PARTS : 0;
            // (not below what the work comes to for each, rounded down)
            int lo = max(p.least_part, (int)((float)(all - (i64)all_blocks * p.start) * (0.999f / 32) / (float)(p.weight * p.teams))), n = all_blocks;
            auto count = [&](int part) {
                return __builtin_amdgcn_readlane(wave_sums(t ? blocks * parts_of(t, part, __builtin_amdgcn_rcpf((float)part)) : 0), 63) * p.Hkv;
            };
            // what parts save has to be worth their merge
            if ((longest - lo) * 32 * p.weight < (p.start + more) / 4) lo = max(lo, longest);
            else {
                int hi = longest;
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (count(mid) <= p.teams) hi = mid; else lo = mid + 1;
                }
            }
            const i64 share = most((all + (i64)all_blocks * more + p.teams - 1) >> teams_log2, p.wmin + more);
            if (p.always_parts || ((i64)lo * 32 * p.weight <= share && longest < 1 << 20)) {      // (beyond, a cut's place would leave 32 bits)
                // A part takes its tiles' time, and a while of the merge: the longest block is through the earliest with parts of about the root of its tiles (that
                // ratio, measured).  With the smallest parts that there are workgroups for, of 4 tiles or more, one token over 26907 keys, 2 KV heads, took 66.5 us
                // (now 24); 2 over 20582, E4M3, 28.5 (17.8); a chunk behind 2468 11.8 (8.4).
                lo = max(lo, __builtin_amdgcn_readfirstlane((int)__builtin_amdgcn_sqrtf((p.always_parts ? 1.0f : 1.5f) * (float)longest)));
                n = count(lo);
                k.part = lo;
                k.team = team_of((n + 7) >> 3);
                k.pos = k.team; k.end = n;
                return k;
            }
        }
    }
    // as many shares on each XCD: where the work is for a part of the workgroups, all XCDs have some
    int per_xcd = p.teams >> 3;
    if (w == p.wmin) per_xcd = min(per_xcd, (((int)all + p.wmin - 1) / p.wmin + 7) >> 3);       // (all is teams * wmin at most)
    k.team = team_of(per_xcd);
    k.w = w;
    k.pos = least(k.team * w, all);
    k.end = least(k.pos + w, all);
    return k;
}

// The whole block of the next turn.
__device__ __forceinline__ bool whole_piece(const ChunkParams &p, Walk &k, const Chunk &c, Piece &pc, Req &rq)
{
    const int unit = unit_of(p, k.team, (int)k.pos), rank = quotient(unit, p.Hkv, p.inv_Hkv), step = step_at(c.beyond, rank);
    ++k.pos;
    if (step < 0) { k.pos = k.end; return false; }      // (only the last turn is not full)
    // of the blocks of this step, the requests' in turn
    const int from = blocks_beyond(p, c.L, c.M, step * k.step), longer = step == 63 ? 0 : blocks_beyond(p, c.L, c.M, (step + 1) * k.step), upto = wave_sums(from - longer);
    const int y = rank - __builtin_amdgcn_readlane(wave_sums(longer), 63), src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(y < upto));
    rq.q0 = __builtin_amdgcn_readlane(c.q0, src); rq.L = __builtin_amdgcn_readlane(c.L, src); rq.M = __builtin_amdgcn_readlane(c.M, src);
    const int i = y - __builtin_amdgcn_readlane(upto - (from - longer), src);
    const int b = quotient(rq.M + p.nb - 1, p.nb, p.inv_nb) - __builtin_amdgcn_readlane(from, src) + i;
    pc.rq = src; pc.g = unit - rank * p.Hkv; pc.by = b; pc.bx = 0; pc.node0 = b * p.nb; pc.nodes = min(p.nb, rq.M - pc.node0);
    pc.st0 = 0; pc.st1 = (rq.L + pc.node0 + pc.nodes + 31) >> 5; pc.direct = 1;
    return true;
}

// The only piece of a workgroup in the form of parts: part i of n of a block's tiles, cut behind even numbers of them (a round of two waves).
// n, i: in how many parts the block is, and which this is.
__device__ __forceinline__ bool only_piece(const ChunkParams &p, Walk &k, const Chunk &c, Piece &pc, Req &rq, int &n, int &i)
{
    if (k.pos >= k.end) return false;
    const int parts = c.M ? parts_of((c.L + c.M + 31) >> 5, k.part, __builtin_amdgcn_rcpf((float)k.part)) : 0;
    const int mine = quotient(c.M + p.nb - 1, p.nb, p.inv_nb) * parts, upto = wave_sums(mine), all = __builtin_amdgcn_readlane(upto, 63);
    const int x = (int)k.pos, h = __builtin_amdgcn_readfirstlane(divided(x, all, __builtin_amdgcn_rcpf((float)all))), y = x - h * all;
    const int src = __builtin_ctzll(__builtin_amdgcn_ballot_w64(y < upto));
    const int at = y - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(mine, src)), most_parts = __builtin_amdgcn_readlane(parts, src);
    const int b = __builtin_amdgcn_readfirstlane(divided(at, most_parts, __builtin_amdgcn_rcpf((float)most_parts)));
    i = at - b * most_parts;
    rq.q0 = __builtin_amdgcn_readlane(c.q0, src); rq.L = __builtin_amdgcn_readlane(c.L, src); rq.M = __builtin_amdgcn_readlane(c.M, src);
    const int node0 = b * p.nb, nodes = min(p.nb, rq.M - node0), t = (rq.L + node0 + nodes + 31) >> 5;
    n = t <= UNCUT ? 1 : min(most_parts, t / p.least_part);      // (a block of few keys: fewer parts, the other workgroups have nothing)
    k.pos = k.end;
    if (i >= n) return false;
    const float inv = __builtin_amdgcn_rcpf((float)n);
    auto cut = [&](int at) { return at == 0 ? 0 : at == n ? t : __builtin_amdgcn_readfirstlane(divided(t * at, n, inv)) & ~1; };
    pc.rq = src; pc.g = h; pc.by = b; pc.bx = 0; pc.node0 = node0; pc.nodes = nodes;
    pc.st0 = cut(i); pc.st1 = cut(i + 1);
    pc.direct = n == 1;
    return true;
}
static_assert(LEAST_PART >= 4 && LEAST_OF_FEW >= 4, "a part is of two tiles or more after its cuts are moved to even numbers");

// x / w for 0 <= x, of which the quotient is below 2^16.
__device__ __forceinline__ int shares_in(i64 x, i64 w)
{
    int q = __builtin_amdgcn_readfirstlane((int)((float)x * __builtin_amdgcn_rcpf((float)w)));
    while (q * w > x) --q;
    while ((q + 1) * w <= x) ++q;
    return q;
}
// The next piece; the walk moves behind it.  False: none left.  c holds the first chunk of requests.  n, i: in how many parts the block is, and which this is.
__device__ __forceinline__ bool next_piece(const ChunkParams &p, Walk &k, int lane, const Chunk &c, Piece &pc, Req &rq, int &n, int &i)
{
    while (k.pos < k.end) {
        while (k.pos - k.head >= k.wh) { k.head += k.wh; ++k.h; }
        const i64 x = k.pos - k.head;
        Chunk d = c;
        int r0 = 0;
        unsigned long long beyond;
        while ((beyond = __builtin_amdgcn_ballot_w64(x < d.incl)) == 0ull) {
            r0 += 64;
            if (r0 >= p.batch) return false;            // (cannot be: x lies within the head's work)
            d = load_chunk(p, r0, lane, lane_value(d.incl, 63));
        }
        const int src = __builtin_ctzll(beyond);
        const int L = __builtin_amdgcn_readlane(d.L, src), M = __builtin_amdgcn_readlane(d.M, src), q0 = __builtin_amdgcn_readlane(d.q0, src);
        const i64 y = x - (lane_value(d.incl, src) - length_of(p, L, M));              // place in the request's work
        const int whole = quotient(M, p.nb, p.inv_nb);
        // the block: the largest b with length_to(b) <= y, from the quadratic's root
        int b = 0;
        if (whole > 0) {
            const float q1 = (float)p.start + (float)WHOLE * (float)L + 0.5f * WHOLE * (float)p.nb, yf = (float)y;
            const float root = 2.0f * yf / (q1 + __builtin_amdgcn_sqrtf(q1 * q1 + 2.0f * WHOLE * (float)p.nb * yf));
            b = min(__builtin_amdgcn_readfirstlane((int)root), whole);
            while (b > 0 && length_to(p, L, b) > y) --b;
            while (b < whole && length_to(p, L, b + 1) <= y) ++b;
        }
        const int node0 = b * p.nb, nodes = min(p.nb, M - node0), keys = L + node0 + nodes, t = (keys + 31) >> 5;
        const int wt = b < whole ? WHOLE : part_weight(p, nodes);
        const int y0 = (int)(y - length_to(p, L, b)), cl = wt * keys, cm = MARGIN * 32 * wt;
        const i64 us = k.pos - y0;
        rq.q0 = q0; rq.L = L; rq.M = M;
        pc.rq = r0 + src; pc.g = k.h; pc.by = b; pc.node0 = node0; pc.nodes = nodes;
        pc.bx = 0; pc.st0 = 0; pc.st1 = t; pc.direct = 1;
        if (t <= SMALL) {                               // to the share in which it begins
            k.pos = us + p.start + cl;
            if (y0 == 0) return true;
            continue;
        }
        const i64 ts = us + p.start;
        int c0 = y0 - p.start, c1 = (int)least(k.end - ts, cl);
        c0 = c0 < cm ? 0 : c0 > cl - cm ? cl : c0;
        c1 = c1 < cm ? 0 : c1 > cl - cm ? cl : c1;
        k.pos = c1 < cl ? k.end : ts + cl;
        if (c0 >= c1) continue;
        auto tile = [&](int x) { return wt == WHOLE ? (int)(__umulhi((uint32_t)x, 0xAAAAAAABu) >> 6) : x >> 6; };      // x / (32 wt)
        static_assert(WHOLE == 3 && PART == 2, "the quotients above");
        pc.st0 = tile(c0);
        pc.st1 = c1 == cl ? t : tile(c1);
        const bool first = c0 == 0, last = c1 == cl;
        pc.direct = first && last;
        if (!pc.direct) {
            // the shares that it lies in, but for cuts that were moved to its ends (as above): the first has MARGIN of its keys or more ahead of its end, the last
            // as many behind its beginning
            const i64 here = k.team * k.w;
            i = shares_in(here + k.w - ts - cm, k.w);
            n = i + 1 + shares_in(ts + cl - cm - here, k.w);
        }
        return true;
    }
    return false;
}

// Parts' rows, joined in the order of their keys, each relative to the row's largest reference.  16 lanes per row, R rows per lane; row(i, r): where part i's
// lie.  Parts come in fp16 beside their magnitude (attn_piece.h), sums are fp32.  Up to B parts are asked for at once; the reference follows from B to B.
// THROUGH: past this XCD's caches, to which workgroups elsewhere did not write.
template <int D, int R, int B, bool THROUGH, typename Row, typename Store>
__device__ __forceinline__ void join_parts(const ChunkParams &p, int n, int sub, Row row, Store store)
{
    constexpr int E = D / 16;
    const auto ml_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.ML, 0, 0x7FFFFFFF, 0x00027000);
    const auto part_rsrc = __builtin_amdgcn_make_buffer_rsrc(p.Opart, 0, 0x7FFFFFFF, 0x00027000);
    typedef _Float16 hvec __attribute__((ext_vector_type(E)));
    typedef __bf16 bvec __attribute__((ext_vector_type(E)));
    float mmax[R], den[R], acc[R][E];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mmax[r] = NEG_BIG; den[r] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[r][e] = 0.f;
    }
    for (int i0 = 0; i0 < n; i0 += B) {
        hvec part[R][B];
        float4 ml[R][B];
#pragma unroll
        for (int b = 0; b < B; ++b)
            if (i0 + b < n)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const int at = row(i0 + b, r);
                    constexpr int SCOPE = THROUGH ? COHERENT : 0;
                    ml[r][b] = __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(ml_rsrc, at * 16, 0, SCOPE));
                    if constexpr (E == 8) part[r][b] = __builtin_bit_cast(hvec, __builtin_amdgcn_raw_buffer_load_b128(part_rsrc, at * D * 2 + sub * 16, 0, SCOPE));
                    else part[r][b] = __builtin_bit_cast(hvec, __builtin_amdgcn_raw_buffer_load_b64(part_rsrc, at * D * 2 + sub * 8, 0, SCOPE));
                }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float mn = mmax[r];
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (i0 + b < n) mn = fmaxf(mn, ml[r][b].x);
            const float alpha = __builtin_amdgcn_exp2f(mmax[r] - mn);
            mmax[r] = mn;
            den[r] *= alpha;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] *= alpha;
#pragma unroll
            for (int b = 0; b < B; ++b)
                if (i0 + b < n) {
                    const float w = __builtin_amdgcn_exp2f(ml[r][b].x - mn), wa = w * ml[r][b].z;
                    den[r] += w * ml[r][b].y;
                    // (without a test of the weight: a part that the row sees none of is all zeros, and one whose weight vanishes hands on what is no number, as it would uncut)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[r][e] = fmaf(wa, (float)part[r][b][e], acc[r][e]);
                }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float inv = p.out_scale / den[r];
        bvec o;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = (__bf16)(acc[r][e] * inv);
        store(r, o);
    }
}

// Where part i of the block that `first` begins lies: a workgroup has room for two, one that it carries on with and one that it begins.
__device__ __forceinline__ int part_at(const ChunkParams &p, int first, int i)
{
    return p.always_parts ? (first + i) * p.part_rows : (2 * (first + i) + (i == 0)) * p.part_rows;
}
// The workgroup that stores the last of a block's parts merges them all (each counts itself in, at the block's first share; the count is back at 0 then).  Nothing waits: who is
// not last goes on.  Rows and the count go to the memory side and come from there, where all XCDs see the same (a store is acknowledged when it is there, and only
// then its workgroup counts itself in); with fences of the device in their place every workgroup would write its XCD's L2 back and drop what it holds of others'
// memory.  (Rows and the count are accessed at the scope of the device, and the rows' stores are waited for ahead of the count: that order is all that a release
// and an acquire would add for such accesses on this chip.)  32 single tokens, E4M3, up to 4000 keys: 25.4 us with fences, 18.8 so, 21.3 with a second launch that merges.  With 64 and 128 rows, by a second launch
// and so: 4 prompts of up to 1999, 32 heads of 64 (nothing is cut): 24.5, 23.0; 11 chunks of up to 361 behind 830, 8 heads of 64: 16.8, 14.2.  With 256 one CU reads 64 KB a part: 6 prompts
// of up to 1104, 32 heads of 64: 20.4, 18.0; 8 requests of 1 to 600 rows behind up to 16384: 62.3, 64.3; a chunk of 2048 behind 8192: 286.8, 290.8 (one by one 334, 351).  There the launch
// stays where each workgroup has more than 30 tiles' work.
template <int D, int THREADS>
__device__ __forceinline__ void merge_parts(const ChunkParams &p, const Piece &pc, const Req &rq, int first, int n, uint32_t *said, int tid)
{
    constexpr int ROWS = THREADS / 16;                  // in one go
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // this wavefront's rows are stored ...
    __syncthreads();                                    // ... and all the workgroup's
    if (tid == 0) {
        u64 *count = &p.words[first & (MERGE_GROUPS - 1)].arrived[first / MERGE_GROUPS];
        static_assert(MOST_TEAMS / MERGE_GROUPS <= 31, "a word for every block");
        const bool last = __hip_atomic_fetch_add(count, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (u64)(n - 1);
        if (last) __hip_atomic_store(count, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *said = last;
    }
    __syncthreads();
    if (!*said) return;
    const int sub = tid & 15, rows = pc.nodes * p.G;
    auto join = [&](auto r_, int x0) {
        constexpr int R = decltype(r_)::value;
        join_parts<D, R, R == 1 ? 8 : 4, true>(p, n, sub, [&](int i, int r) { return part_at(p, first, i) + x0 + ROWS * r; }, [&](int r, const auto &o) {
            const int x = x0 + ROWS * r, node = (x * p.ginv) >> 16;
            if (node >= pc.nodes) return;
            const size_t orow = (size_t)(rq.q0 + pc.node0 + node) * p.Hq + pc.g * p.G + (x - node * p.G);
            *reinterpret_cast<std::decay_t<decltype(o)> *>(static_cast<__bf16 *>(p.O) + orow * D + sub * (D / 16)) = o;
        });
    };
    if (rows <= ROWS) {
        if (tid >> 4 < rows) join(std::integral_constant<int, 1>{}, tid >> 4);
    } else
        for (int x0 = 0; x0 < rows; x0 += 4 * ROWS) join(std::integral_constant<int, 4>{}, x0 + (tid >> 4));
}

template <int D, int RW, int KW, int NT, int EB, bool BEHIND>
__global__ __launch_bounds__(RW * KW * 64, 2) void chunk_attn_kernel(ChunkParams p)
{
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    // (every argument in one round trip)
    asm volatile("" ::"s"(p.Q), "s"(p.K), "s"(p.V), "s"(p.O), "s"(p.block_table), "s"(p.q_offset), "s"(p.prefix_len), "s"(p.Opart), "s"(p.ML), "s"(p.flag), "s"(p.M), "s"(p.part_rows), "s"(p.always_parts), "s"(p.least_part),
                 "s"(p.L), "s"(p.Hq), "s"(p.Hkv), "s"(p.G), "s"(p.ginv), "s"(p.max_blocks), "s"(p.num_blocks), "s"(p.total_M), "s"(p.batch), "s"(p.wmin),
                 "s"(p.scale_log2), "s"(p.out_scale), "s"(p.nb), "s"(p.inv_nb), "s"(p.wr), "s"(p.teams), "s"(p.most_keys), "s"(p.start), "s"(p.weight), "s"(p.inv_Hkv), "s"(p.words));
    Chunk c;
    Walk k = share_out<RW == 2, RW * KW>(p, threadIdx.x & 63, blockIdx.x == 0 && threadIdx.x < 64, c, reinterpret_cast<int *>(smem));
    using CL = ChunkLds<D, RW, KW, NT, EB>;
    const uint32_t kept = (uint32_t)(uintptr_t)BTV_LDS_PTR(smem) + CL::PL::BYTES;
    static_assert(CL::PL::BYTES % 16 == 0 && RW * KW <= 8, "what is kept");
    static_assert(RW == 2 || CL::KEPT, "the turns of whole blocks");
    if (CL::KEPT && threadIdx.x < 64) keep_chunk(kept, threadIdx.x, c);     // (barriers before it is read: those of the first piece)
    for (bool again = false;; again = true) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                   // keeps what derives from it (all addresses) from being carried across pieces
        if (again) {
            if constexpr (CL::KEPT) c = kept_chunk(kept, tid, k);
            else c = load_chunk(p, 0, tid & 63, 0);
        }
        Piece pc = {};
        Req rq = {};
        int parts = 1, part = 0;
        bool more;
        if (RW != 2 && k.step) more = whole_piece(p, k, c, pc, rq);
        else if (k.part) more = only_piece(p, k, c, pc, rq, parts, part);
        else more = next_piece(p, k, tid & 63, c, pc, rq, parts, part);
        if (!more) {
            if (BEHIND && tid == 0) p.begun[k.team] = Begun{ 0, 0, 0, 0 };
            return;
        }
        const int first = k.team - part;
        pc.prow0 = part_at(p, first, part);
        const bool last = k.pos >= k.end;
        // (a workgroup begins one cut block at most, with its last piece)
        if (BEHIND && last && tid == 0) p.begun[k.team] = parts > 1 && part == 0 ? Begun{ parts, rq.q0 + pc.node0, pc.nodes, pc.g } : Begun{ 0, 0, 0, 0 };
        if constexpr (CL::KEPT)
            if (!last) keep_walk(kept, tid, k);
        attn_piece<D, RW, KW, NT, true, EB, true, !BEHIND>(p, smem, tid, rq, pc, [] {});
        if (!BEHIND && parts > 1) merge_parts<D, RW * KW * 64>(p, pc, rq, first, parts, reinterpret_cast<uint32_t *>(smem), tid);
        if (last) return;
        // every wave is done with this piece's LDS, its own fills have landed; the stores may still be on their way
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
    }
}

// The blocks of 256 rows that were cut: 16 lanes per row, MERGE_ROWS rows per workgroup; workgroup (k, slice) looks at the block that workgroup k has begun.
constexpr int MERGE_ROWS = 32;
template <int D>
__global__ __launch_bounds__(256) void chunk_merge(ChunkParams p)
{
    asm volatile("" ::"s"(p.begun), "s"(p.part_rows), "s"(p.always_parts), "s"(p.G), "s"(p.ginv), "s"(p.ML), "s"(p.Opart), "s"(p.O), "s"(p.Hq), "s"(p.out_scale));
    const int k = blockIdx.x, sub = threadIdx.x & 15, x0 = blockIdx.y * MERGE_ROWS + (threadIdx.x >> 4);
    const Begun b = p.begun[k];
    if (b.parts == 0 || (int)blockIdx.y * MERGE_ROWS >= b.nodes * p.G) return;
    join_parts<D, MERGE_ROWS / 16, 4, false>(p, b.parts, sub, [&](int i, int r) { return part_at(p, k, i) + x0 + 16 * r; }, [&](int r, const auto &o) {
        const int x = x0 + 16 * r, node = (x * p.ginv) >> 16;
        if (node >= b.nodes) return;
        const size_t orow = (size_t)(b.row0 + node) * p.Hq + b.g * p.G + (x - node * p.G);
        *reinterpret_cast<std::decay_t<decltype(o)> *>(static_cast<__bf16 *>(p.O) + orow * D + sub * (D / 16)) = o;
    });
}

// ---- host side ------------------------------------------------------------------------------------------------------------

int check_chunk(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    BTV_REQUIRE(batch >= 1 && batch <= 4096, "batch=%d outside [1,4096]", batch);
    BTV_REQUIRE(M_max >= 1 && M_max <= MOST_ROWS, "M_max=%d outside [1,%d]", M_max, MOST_ROWS);
    BTV_REQUIRE(L_max >= 0 && (i64)L_max + M_max < (1ll << 29), "L_max=%d out of range", L_max);         // (weighted lengths of a block stay in 32 bits)
    BTV_REQUIRE(Hq >= 1 && Hkv >= 1 && Hkv <= 1024 && Hq % Hkv == 0 && Hq / Hkv <= 16, "bad heads Hq=%d Hkv=%d", Hq, Hkv);
    BTV_REQUIRE(D == 64 || D == 128, "D=%d not in {64,128}", D);
    // the work's length stays below 2^62, and 64 requests' of one head below 2^54 (a request and head has at most M / 4 + 1 blocks)
    const double head = (M_max / 4 + 1) * (8192.0 + (double)WHOLE * ((double)L_max + M_max));
    BTV_REQUIRE(64 * head < 1.8e16 && batch * head * Hkv < 4.6e18, "more work than can be counted");
    return BTV_OK;
}

// Rows per workgroup: at most what the largest request has.
int most_rows(int M_max, int G, int eb)
{
    const i64 rows = (i64)M_max * G;
    return rows <= 64 ? 64 : rows <= 128 || eb == 1 ? 128 : 256;
}
// Many rows read a tile for more of them and are the fastest over long ranges (a chunk of 2048 behind 30720, 64 heads of 128: 256 rows 1834 us, 128 2055), but where they leave
// workgroups without a block, or one in a second turn, the ends of the pieces are most of the time: fewer rows then, as long as the work is short.  By the numbers of
// blocks that the bounds allow (half a block of each request is not full) and the tiles of 256 rows that come to each workgroup.  us with 256, 128, 64 rows:
// 7 prompts of up to 718, 8 heads of 64: 23.3, 16.5, 13.8 (93 blocks of 256 rows, 4 tiles); 7 chunks of up to 215 behind 1598, 64 heads of 128: 42.7, 27.2, 42.1
// (165, 34); 2 prompts of up to 3676, 32 heads of 64: 34.2, 36.5, 44.5 (284, 64); 5 chunks of up to 749 behind 12384, 32 heads of 128: 110, 120, 171 (115, 179);
// E4M3, a chunk of 1938, 8 heads: 16.3 with 128, 12.8 with 64 (10, 1); 22 of up to 110 behind 8711: 34.2, 36.2 (45, 48).
// With 64 channels two workgroups of 128 rows, four waves that take every tile, fit on a CU: of many blocks one's ends pass while the other computes, but each brings its own
// tiles.  us with 256 rows and so: 6 prompts of up to 2348, 16 heads: 41.7, 34.9 (396 blocks, 57 tiles); 26 of up to 125, 32 heads: 17.6, 9.0 (258, 2); 34 chunks of up to
// 545 behind 4275, 16 heads: 65.2, 65.6 (454, 252); 7 of up to 551 behind 25259, 16 heads: 70.2, 76.8 (141, 440).
struct Shape { int rows, key_waves, teams; bool behind; };      // behind: merged by a launch
Shape shape_of(int batch, int total_M, int M_max, int L_max, int G, int Hkv, int D, int eb)
{
    const int most = most_rows(M_max, G, eb);
    const double rows = (double)total_M * G, half = 0.5 * batch;
    const double tiles = (rows / 256 + half) * Hkv * ((double)L_max + 0.5 * M_max) / (32 * 256);
    if ((rows / 64 + half) * Hkv <= 512 && tiles <= 30) return { 64, 2, 512, false };
    if (most <= 64) return { 64, 2, 512, false };
    // (very short ones: a second turn costs as much as the first; 37 prompts of up to 234, 16 heads of 128: 15.4 with 256 rows, 22.9 with 128; 8 of up to 479, 32 heads, where
    // 7 tiles come to each: 26.2, 22.3)
    const bool few = (rows / 256 + half) * Hkv <= 256 && (tiles >= 4 || (rows / 128 + half) * Hkv <= 256);
    if (most == 128 || (few && tiles <= 110)) return { 128, 2, 256, false };
    if (D == 64 && !few && tiles <= 200) return { 128, 1, 512, false };
    return { 256, 1, 256, tiles > 30 };
}
bool cuts(int M_max, int L_max) { return (L_max + M_max + 31) / 32 > SMALL; }

// What a row block costs besides its keys, in tiles of whole blocks: finding it, its first loads, its last steps and stores.  Shares and whole blocks are weighed with
// it.  The stamps say 8 to 12 tiles; that much and half or twice it are within 2 % on average of 120 calls.  With 128 rows 16 is the best (3 chunks of up to 232 behind 4322, 64 heads: 35.8 us
// with 9, so 31.4; E4M3 with 22: 27 of up to 914 behind 623, 91.7, so 77.1).
int start_of(int wr, int D) { return wr == 64 ? 14 : wr == 128 ? 16 : D == 64 ? 12 : 9; }

// Single tokens of requests that have a place on the chip each: always parts.  (With up to four parts per place where the requests alone fill it: 43 requests of up to 2305 keys,
// 8 KV heads, 23.7 us, with one 18.1; 43 of up to 5520, E4M3, 48.8 and 49.6.)
bool few_rows(int batch, int M_max, int G, int Hkv) { return M_max * G <= FEW_ROWS && batch <= 64 && batch * Hkv <= MOST_TEAMS; }

struct WsLayout { size_t begun, ml, opart, total; };
WsLayout ws_layout(int block_rows, int D, bool cut)
{
    WsLayout w;
    size_t off = BTV_WS_HEADER + MERGE_WORDS;
    const size_t rows = cut ? (size_t)block_rows * 2 : 0;               // (of all workgroups; more than MOST_TEAMS * FEW_ROWS, which the parts of few rows take)
    static_assert(512 * 2 * 64 >= MOST_TEAMS * FEW_ROWS, "parts of few rows have room where shares of 64 rows have");
    w.begun = off; off += MOST_TEAMS * sizeof(Begun);
    w.ml = off; off += rows * 16;
    w.opart = off; off += rows * D * 2;
    w.total = btv_align_up(off, BTV_WS_ALIGN);
    return w;
}
size_t enough_for(int M_max, int L_max, int G, int D, int eb)
{
    return ws_layout(most_rows(M_max, G, eb) > 128 ? 256 * 256 : 256 * 128, D, cuts(M_max, L_max)).total;
}

template <int D, int RW, int KW, int NT, int EB, bool BEHIND>
int launch(const ChunkParams &p, hipStream_t st)
{
    constexpr int LDS_BYTES = ChunkLds<D, RW, KW, NT, EB>::BYTES;
    static_assert(LDS_BYTES * (RW * KW <= 4 ? 2 : 1) <= 160 * 1024, "LDS budget");
    static std::atomic<unsigned long long> configured{0};       // a bit per device
    int dev = 0;
    BTV_HIP(hipGetDevice(&dev));
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(configured.load(std::memory_order_acquire) & bit)) {
        BTV_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(chunk_attn_kernel<D, RW, KW, NT, EB, BEHIND>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES));
        configured.fetch_or(bit, std::memory_order_release);
    }
    hipLaunchKernelGGL((chunk_attn_kernel<D, RW, KW, NT, EB, BEHIND>), dim3(p.teams), dim3(RW * KW * 64), LDS_BYTES, st, p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

int chunk_attn(const void *Q, const void *Kpool, const void *Vpool, int num_blocks, const int32_t *block_table, int max_blocks, const int32_t *q_offset,
               const int32_t *prefix_len, int batch, int total_M, int M_max, int L_max, int Hq, int Hkv, int D, int eb, float scale, float k_scale,
               float v_scale, void *O, void *ws, size_t ws_bytes, void *stream)
{
    BTV_REQUIRE(((Q && O) || total_M == 0) && Kpool && Vpool && block_table && q_offset && prefix_len, "null pointer");
    BTV_REQUIRE(btv_aligned16(Q) && btv_aligned16(Kpool) && btv_aligned16(Vpool) && btv_aligned16(O), "Q, K, V and O must be 16-byte aligned");
    int rc = check_chunk(batch, M_max, L_max, Hq, Hkv, D);
    if (rc) return rc;
    BTV_REQUIRE(total_M >= 0 && total_M <= INT_MAX / Hq, "total_M=%d out of range", total_M);
    BTV_REQUIRE(num_blocks >= 1 && max_blocks >= 1, "bad block counts");
    BTV_REQUIRE((i64)max_blocks * BTV_PAGE >= (i64)L_max + 1, "max_blocks too small for L_max");
    BTV_REQUIRE(std::isfinite(scale) && std::fabs(scale) <= 1e30f, "the scale must be finite");
    const float factor = (scale > 0.f ? scale : 1.0f / sqrtf((float)D)) * k_scale * 1.4426950408889634f;
    BTV_REQUIRE(std::isfinite(factor) && factor > 0.f, "the scale must be finite");
    const int G = Hq / Hkv;
    const Shape sh = shape_of(batch, total_M, M_max, L_max, G, Hkv, D, eb);
    const int wr = sh.rows;
    const bool cut = cuts(M_max, L_max);
    const WsLayout wl = ws_layout(sh.teams * wr, D, cut);
    rc = btv_check_ws(ws, ws_bytes, wl.total);
    if (rc) return rc;
    if (total_M == 0) return BTV_OK;
    unsigned char *w8 = static_cast<unsigned char *>(ws);
    ChunkParams p = {};
    p.Q = Q; p.K = Kpool; p.V = Vpool; p.O = O;
    p.block_table = block_table; p.q_offset = q_offset; p.prefix_len = prefix_len;
    p.Opart = reinterpret_cast<_Float16 *>(w8 + wl.opart);
    p.ML = reinterpret_cast<float *>(w8 + wl.ml);
    p.flag = reinterpret_cast<uint32_t *>(w8);
    p.M = M_max; p.L = L_max; p.Hq = Hq; p.Hkv = Hkv; p.G = G; p.ginv = (65536 + G - 1) / G;
    p.inv_Hkv = reciprocal(Hkv);
    p.max_blocks = max_blocks; p.num_blocks = num_blocks; p.total_M = total_M; p.batch = batch;
    p.scale_log2 = factor; p.out_scale = v_scale;
    p.wr = wr; p.nb = wr / G; p.inv_nb = reciprocal(p.nb); p.teams = sh.teams;
    p.weight = (i64)M_max * G * 2 <= wr ? PART : WHOLE;
    p.most_keys = (int)std::min<i64>((i64)max_blocks * BTV_PAGE, INT_MAX);
    const bool few = few_rows(batch, M_max, G, Hkv) && L_max + M_max < 1 << 25;        // (in a part's place tiles times parts stay in 32 bits)
    p.words = reinterpret_cast<MergeWords *>(w8 + BTV_WS_HEADER);
    const bool behind = sh.behind && cut;
    p.begun = behind ? reinterpret_cast<Begun *>(w8 + wl.begun) : nullptr;
    p.start = start_of(wr, D) * 32 * WHOLE;
    p.wmin = p.start + 8 * 32 * WHOLE;
    p.part_rows = wr;
    p.least_part = few ? LEAST_OF_FEW : LEAST_PART;
    if (few) {
        p.always_parts = 1;
        p.part_rows = FEW_ROWS;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
#define BTV_CASE(DD, EE, RR, KK, NN, BB) if (D == DD && eb == EE && wr == RR * 32 && sh.key_waves == KK && behind == BB) rc = launch<DD, RR, KK, NN, EE, BB>(p, st); else
    BTV_CASE(128, 2, 2, 2, 5, false) BTV_CASE(128, 2, 4, 2, 8, false) BTV_CASE(128, 2, 8, 1, 8, false) BTV_CASE(128, 2, 8, 1, 8, true)
    BTV_CASE(64, 2, 2, 2, 5, false) BTV_CASE(64, 2, 4, 2, 8, false) BTV_CASE(64, 2, 4, 1, 8, false) BTV_CASE(64, 2, 8, 1, 8, false) BTV_CASE(64, 2, 8, 1, 8, true)
    BTV_CASE(128, 1, 2, 2, 5, false) BTV_CASE(128, 1, 4, 2, 8, false)
    return btv_fail(BTV_EINVAL, "no kernel for D=%d", D);
#undef BTV_CASE
    if (rc || !behind) return rc;
    const dim3 grid(p.teams, wr / MERGE_ROWS);
    if (D == 64) hipLaunchKernelGGL(chunk_merge<64>, grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL(chunk_merge<128>, grid, dim3(256), 0, st, p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}

}  // namespace

extern "C" {

size_t btv_chunk_attn_paged_workspace(int batch, int M_max, int L_max, int Hq, int Hkv, int D)
{
    return check_chunk(batch, M_max, L_max, Hq, Hkv, D) == BTV_OK ? enough_for(M_max, L_max, Hq / Hkv, D, 2) : 0;
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
    return check_chunk(batch, M_max, L_max, Hq, Hkv, D) == BTV_OK && D == 128 ? enough_for(M_max, L_max, Hq / Hkv, D, 1) : 0;
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
