// Room in a paged cache for the rows that come next (gfx950): from the requests' lengths the pages they still need are taken off a
// free list, and every new row gets its slot and its position.
//
// Two sums over the requests decide everything: of the new rows (where a request's rows begin) and of the pages taken (which pages of
// the free list are its own).  They are sums of up to 4096 numbers that fit the caches, so every workgroup works all of them out for itself:
// one launch, in which no workgroup waits for another.  Then a workgroup writes its share of the rows, one thread per row (the
// request found by bisection in LDS, the page either from the table or straight from the free list, so that nothing waits for the table's new entries
// either), and its share of the requests' new table entries.  Latency bounds it: the launch, the lengths' round trip, the pages' round trip.  8 trees 4.7 us, 700 requests with
// 1 to 500 new rows each (57600 rows) 5.5 us (with the requests' numbers in memory, not LDS, 6.4).
#include "btv_common.h"

#include <atomic>
#include <climits>

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, MOST_REQUESTS = 4096;

struct ExtendParams {
    const int32_t *prefix_len, *n_new, *depth, *n_pages, *free_pages, *n_free;
    int32_t *block_table, *q_offset, *slot, *position, *n_pages_out, *n_free_out;
    uint32_t *flag;
    int batch, total_max, num_blocks, max_blocks, rows_per_wg;
};

// What is kept of a request in LDS for the rows: where its rows begin (2^31 - 1 at most), its length and pages, and how many pages the requests before it ask for, up to
// what the list has (x; ~x, which is negative, where it does not get what it needs).
struct Kept { int32_t *first, *L, *P, *taken; };

// Inclusive sums over the lanes (numbers below 2^54 in three pieces).
__device__ __forceinline__ int wave_sums(int x)
{
#define BTV_SCAN_STEP(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xF, ctrl < 0x142)
    BTV_SCAN_STEP(0x111, 0xF); BTV_SCAN_STEP(0x112, 0xF); BTV_SCAN_STEP(0x114, 0xF); BTV_SCAN_STEP(0x118, 0xF);
    BTV_SCAN_STEP(0x142, 0xA); BTV_SCAN_STEP(0x143, 0xC);
#undef BTV_SCAN_STEP
    return x;
}
__device__ __forceinline__ long long wave_sums(long long x)
{
    constexpr int B = 18;
    const long long lo = wave_sums((int)x & ((1 << B) - 1)), mid = wave_sums((int)(x >> B) & ((1 << B) - 1)), hi = wave_sums((int)(x >> 2 * B));
    return lo + (mid << B) + (hi << 2 * B);
}

__global__ __launch_bounds__(THREADS) void paged_extend_kernel(ExtendParams p)
{
    extern __shared__ int32_t lds[];
    const Kept kept = { lds, lds + p.batch + 1, lds + 2 * p.batch + 1, lds + 3 * p.batch + 1 };
    __shared__ long long sums[2][WAVES], given[WAVES];
    asm volatile("" ::"s"(p.prefix_len), "s"(p.n_new), "s"(p.depth), "s"(p.n_pages), "s"(p.free_pages), "s"(p.n_free), "s"(p.block_table), "s"(p.q_offset), "s"(p.slot),
                 "s"(p.position), "s"(p.n_pages_out), "s"(p.n_free_out), "s"(p.flag), "s"(p.batch), "s"(p.total_max), "s"(p.num_blocks), "s"(p.max_blocks));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int n_free = *p.n_free;
    const bool bad_list = n_free < 0 || n_free > p.num_blocks;
    if (bad_list) n_free = 0;
    bool bad = bad_list;

    // The requests, a turn of one per thread after the other; at, pages: sums up to the turn.
    long long at = 0, pages = 0, taken_all = 0;
    for (int r0 = 0; r0 < p.batch; r0 += THREADS) {
        const int r = r0 + tid, rc = min(r, p.batch - 1);
        const bool in = r < p.batch;
        int L = p.prefix_len[rc], M = p.n_new[rc], P = p.n_pages[rc];
        const long long have = (long long)p.max_blocks * BTV_PAGE;
        const bool ok = L >= 0 && M >= 0 && (long long)L + M <= have && P >= 0 && P <= p.max_blocks && (L + (BTV_PAGE - 1)) / BTV_PAGE <= P;
        M = in ? max(M, 0) : 0;
        const int take = in && ok ? max((int)(((long long)L + M + (BTV_PAGE - 1)) / BTV_PAGE) - P, 0) : 0;
        const long long m = wave_sums((long long)M), t = wave_sums((long long)take);
        if (lane == 63) { sums[0][wave] = m; sums[1][wave] = t; }
        __syncthreads();
        long long row = at + m - M, page = pages + t - take;
        for (int w = 0; w < WAVES; ++w) {
            at += sums[0][w]; pages += sums[1][w];
            if (w < wave) { row += sums[0][w]; page += sums[1][w]; }
        }
        if (in) {
            const bool granted = ok && (take == 0 || page + take <= n_free);
            const int first = row < INT_MAX ? (int)row : INT_MAX;
            kept.first[r] = first; kept.L[r] = L; kept.P[r] = P;
            const int before = page < n_free ? (int)page : n_free;
            kept.taken[r] = granted ? before : ~before;
            if (granted) taken_all += take;
            bad = bad || !granted || row + M > p.total_max;
            if (blockIdx.x == 0) {
                p.q_offset[r] = first;
                p.n_pages_out[r] = granted ? P + take : P;
            }
        }
        __syncthreads();                               // (the sums have been read; behind the last turn: what is kept is there)
    }
    const int total = at < INT_MAX ? (int)at : INT_MAX;
    if (blockIdx.x == 0) {
        taken_all = wave_sums(taken_all);
        if (lane == 63) given[wave] = taken_all;
        __syncthreads();
        if (tid == 0) {
            long long g = 0;
            for (int w = 0; w < WAVES; ++w) g += given[w];
            *p.n_free_out = (int32_t)(n_free - g);
            p.q_offset[p.batch] = total;
        }
    }

    auto row = [&](long long row) {
        int slot = -1, position = 0;
        if (row < total) {
            int lo = 0, hi = p.batch;                  // first[lo] <= row < first[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (kept.first[mid] <= row) lo = mid; else hi = mid;
            }
            const int L = kept.L[lo], P = kept.P[lo], base = kept.taken[lo];
            if (base >= 0) {
                const int j = L + ((int)row - kept.first[lo]), b = j / BTV_PAGE;       // its place in the request
                const int id = b < P ? p.block_table[(size_t)lo * p.max_blocks + b] : p.free_pages[n_free - 1 - base - (b - P)];
                position = p.depth ? L + p.depth[row] - 1 : j;
                if (id >= 0 && id < p.num_blocks) slot = id * BTV_PAGE + j % BTV_PAGE; else bad = true;
            }
        }
        p.slot[row] = slot;
        p.position[row] = position;
    };
    const long long b0 = (long long)blockIdx.x * p.rows_per_wg, b1 = min(b0 + p.rows_per_wg, (long long)p.total_max);
    for (long long x = b0 + tid; x < b1; x += THREADS) row(x);

    // The table's new entries: a wavefront per request.  It takes what lies between its pages and the next one's (rows say nothing here: a request before it may be out of range, and
    // count as more rows than there are numbers).
    for (int r = blockIdx.x * WAVES + wave; r < p.batch; r += gridDim.x * WAVES) {
        const int base = kept.taken[r], P = kept.P[r];
        if (base < 0) continue;
        const int next = r + 1 < p.batch ? kept.taken[r + 1] : pages < n_free ? (int)pages : n_free, take = (next < 0 ? ~next : next) - base;
        for (int k = lane; k < take; k += 64) {
            const int id = p.free_pages[n_free - 1 - base - k];
            bad = bad || id < 0 || id >= p.num_blocks;
            p.block_table[(size_t)r * p.max_blocks + P + k] = id;
        }
    }
    if (bad && p.flag) atomicOr(p.flag, 16u);
}

}  // namespace

extern "C" int btv_paged_extend(const int32_t *prefix_len, const int32_t *n_new, const int32_t *depth, int batch, int total_max,
                                const int32_t *n_pages, const int32_t *free_pages, const int32_t *n_free, int num_blocks,
                                int32_t *block_table, int max_blocks, int32_t *q_offset, int32_t *slot, int32_t *position,
                                int32_t *n_pages_out, int32_t *n_free_out, void *ws, void *stream)
{
    BTV_REQUIRE(prefix_len && n_new && n_pages && free_pages && n_free && block_table && q_offset && n_pages_out && n_free_out, "null pointer");
    BTV_REQUIRE(batch >= 1 && batch <= MOST_REQUESTS, "batch=%d outside [1,%d]", batch, MOST_REQUESTS);
    BTV_REQUIRE(total_max >= 0 && total_max <= (1 << 30), "total_max=%d out of range", total_max);
    BTV_REQUIRE(total_max == 0 || (slot && position), "null pointer");
    BTV_REQUIRE(num_blocks >= 1 && num_blocks <= INT_MAX / BTV_PAGE, "num_blocks=%d out of range", num_blocks);
    BTV_REQUIRE(max_blocks >= 1 && max_blocks <= INT_MAX / BTV_PAGE, "max_blocks=%d out of range", max_blocks);
    BTV_REQUIRE(n_pages_out != n_pages && n_free_out != n_free, "n_pages_out and n_free_out may not be n_pages and n_free");
    ExtendParams p = {};
    p.prefix_len = prefix_len; p.n_new = n_new; p.depth = depth; p.n_pages = n_pages; p.free_pages = free_pages; p.n_free = n_free;
    p.block_table = block_table; p.q_offset = q_offset; p.slot = slot; p.position = position; p.n_pages_out = n_pages_out; p.n_free_out = n_free_out;
    p.flag = static_cast<uint32_t *>(ws);
    p.batch = batch; p.total_max = total_max; p.num_blocks = num_blocks; p.max_blocks = max_blocks;
    // a thread per row while that is two workgroups per CU at most
    const int wgs = total_max <= THREADS ? 1 : total_max <= 512 * THREADS ? (total_max + THREADS - 1) / THREADS : 512;
    p.rows_per_wg = (int)(((long long)total_max + wgs - 1) / wgs);
    const size_t bytes = (4 * (size_t)batch + 1) * sizeof(int32_t);
    if (bytes > 60 * 1024) {                                    // (more than a workgroup gets unasked)
        static std::atomic<unsigned long long> configured{0};   // a bit per device
        int dev = 0;
        BTV_HIP(hipGetDevice(&dev));
        const unsigned long long bit = 1ull << (dev & 63);
        if (!(configured.load(std::memory_order_acquire) & bit)) {
            BTV_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(paged_extend_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (4 * MOST_REQUESTS + 1) * sizeof(int32_t)));
            configured.fetch_or(bit, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(paged_extend_kernel, dim3(wgs), dim3(THREADS), bytes, static_cast<hipStream_t>(stream), p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}
