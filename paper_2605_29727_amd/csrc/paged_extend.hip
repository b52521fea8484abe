// Room in a paged cache for the rows that come next (gfx950): from the requests' lengths the pages they still need are taken off a
// free list, and every new row gets its slot and its position.
//
// Two sums over the requests decide everything: of the new rows (where a request's rows begin) and of the pages taken (which pages of
// the free list are its own).  They are sums of up to 4096 numbers that fit the caches, so every workgroup works all of them out for itself:
// one launch, in which no workgroup waits for another.  Then a workgroup writes its share of the rows, one thread per row (the
// request found by bisection in LDS, the page either from the table or straight from the free list, so that nothing waits for the table's new entries
// either), and its share of the requests' new table entries.  Latency bounds it: the launch, the lengths' round trip, the pages' round trip.
#include "btv_common.h"

#include <climits>

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64, MOST_REQUESTS = 4096, PER_THREAD = MOST_REQUESTS / THREADS;

struct ExtendParams {
    const int32_t *prefix_len, *n_new, *depth, *n_pages, *free_pages, *n_free;
    int32_t *block_table, *q_offset, *slot, *position, *n_pages_out, *n_free_out;
    uint32_t *flag;
    int batch, total_max, num_blocks, max_blocks, rows_per_wg, per_thread;
};

struct Need { int L, M, P, take; bool ok; };

__device__ __forceinline__ Need need_of(const ExtendParams &p, int r)
{
    Need n;
    n.L = p.prefix_len[r]; n.M = p.n_new[r]; n.P = p.n_pages[r];
    const long long have = (long long)p.max_blocks * BTV_PAGE;
    n.ok = n.L >= 0 && n.M >= 0 && (long long)n.L + n.M <= have && n.P >= 0 && n.P <= p.max_blocks && (n.L + (BTV_PAGE - 1)) / BTV_PAGE <= n.P;
    n.M = max(n.M, 0);
    n.take = n.ok ? max((int)(((long long)n.L + n.M + (BTV_PAGE - 1)) / BTV_PAGE) - n.P, 0) : 0;
    return n;
}

__device__ __forceinline__ long long wave_inclusive(long long x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

__global__ __launch_bounds__(THREADS) void paged_extend_kernel(ExtendParams p)
{
    extern __shared__ int32_t lds[];
    int32_t *first = lds;                              // [batch + 1]: where a request's rows begin
    int32_t *taken = lds + p.batch + 1;                // [batch]: pages taken before it, or -1 where it gets none of what it needs
    __shared__ long long sums[2][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int n_free = *p.n_free;
    const bool bad_list = n_free < 0 || n_free > p.num_blocks;
    if (bad_list) n_free = 0;

    // a thread has per_thread neighbouring requests
    const int r0 = tid * p.per_thread, r1 = min(r0 + p.per_thread, p.batch);
    long long rows = 0, pages = 0;
    for (int r = r0; r < r1; ++r) {
        const Need n = need_of(p, r);
        rows += n.M; pages += n.take;
    }
    const long long rows_incl = wave_inclusive(rows, lane), pages_incl = wave_inclusive(pages, lane);
    if (lane == 63) { sums[0][wave] = rows_incl; sums[1][wave] = pages_incl; }
    __syncthreads();
    long long at = rows_incl - rows, page = pages_incl - pages;
    for (int w = 0; w < wave; ++w) { at += sums[0][w]; page += sums[1][w]; }
    bool bad = bad_list;
    long long given = 0;
    for (int r = r0; r < r1; ++r) {
        const Need n = need_of(p, r);
        const bool granted = n.ok && (n.take == 0 || page + n.take <= n_free);
        first[r] = (int32_t)min(at, (long long)INT_MAX);
        taken[r] = granted ? (int32_t)min(page, (long long)n_free) : -1;
        if (granted) given += n.take;
        bad = bad || !granted || at + n.M > p.total_max;
        if (blockIdx.x == 0) {
            p.q_offset[r] = first[r];
            p.n_pages_out[r] = granted ? n.P + n.take : n.P;
        }
        at += n.M; page += n.take;
        if (r == p.batch - 1) {
            first[p.batch] = (int32_t)min(at, (long long)INT_MAX);
            if (blockIdx.x == 0) p.q_offset[p.batch] = first[p.batch];
        }
    }
    given = wave_inclusive(given, lane);
    __syncthreads();                                   // (the sums have been read, first and taken are there)
    if (blockIdx.x == 0) {
        if (lane == 63) sums[0][wave] = given;
        __syncthreads();
        if (tid == 0) {
            long long g = 0;
            for (int w = 0; w < WAVES; ++w) g += sums[0][w];
            *p.n_free_out = (int32_t)(n_free - g);
        }
    }

    // the table's new entries: a wavefront per request
    for (int r = blockIdx.x * WAVES + wave; r < p.batch; r += gridDim.x * WAVES) {
        const int base = taken[r];
        if (base < 0) continue;
        const Need n = need_of(p, r);
        for (int k = lane; k < n.take; k += 64) {
            const int id = p.free_pages[n_free - 1 - base - k];
            bad = bad || id < 0 || id >= p.num_blocks;
            p.block_table[(size_t)r * p.max_blocks + n.P + k] = id;
        }
    }

    const int total = first[p.batch];
    const long long b0 = (long long)blockIdx.x * p.rows_per_wg, b1 = min(b0 + p.rows_per_wg, (long long)p.total_max);
    for (long long row = b0 + tid; row < b1; row += THREADS) {
        int slot = -1, position = 0;
        if (row < total) {
            int lo = 0, hi = p.batch;                  // first[lo] <= row < first[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first[mid] <= row) lo = mid; else hi = mid;
            }
            const int i = (int)row - first[lo], L = p.prefix_len[lo], P = p.n_pages[lo], base = taken[lo];
            const long long j = (long long)L + i;      // its place in the request
            if (base >= 0) {
                position = p.depth ? L + p.depth[row] - 1 : (int)j;
                const int b = (int)(j / BTV_PAGE);
                const int id = b < P ? p.block_table[(size_t)lo * p.max_blocks + b] : p.free_pages[n_free - 1 - base - (b - P)];
                if (id >= 0 && id < p.num_blocks) slot = id * BTV_PAGE + (int)(j % BTV_PAGE); else bad = true;
            }
        }
        p.slot[row] = slot;
        p.position[row] = position;
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
    p.per_thread = (batch + THREADS - 1) / THREADS;
    // a thread per row while that is two workgroups per CU at most
    const int wgs = total_max <= THREADS ? 1 : total_max <= 512 * THREADS ? (total_max + THREADS - 1) / THREADS : 512;
    p.rows_per_wg = (int)(((long long)total_max + wgs - 1) / wgs);
    hipLaunchKernelGGL(paged_extend_kernel, dim3(wgs), dim3(THREADS), (2 * batch + 1) * sizeof(int32_t), static_cast<hipStream_t>(stream), p);
    BTV_HIP(hipGetLastError());
    return BTV_OK;
}
