// Block tables and slot maps from the requests' lengths: the places of a step's new tokens.
//
//   q_start = exclusive sums of new_lens; pages needed = ceil((old + new) / 64) - ceil(old / 64), their exclusive sums say where
//   in the free list a request's pages begin; a place finds its request by bisection in q_start.
//
// One kernel: every block makes both sums for itself, in shared memory (512 requests are one element a thread), because
// the alternative, a second launch behind a kernel of one block, costs more than the sums (a launch that waits for another: 2 to 3 us).
// A page's table entry is written by the place at the page's first token, which exists for every new page: no place waits
// for another.  Launch latency bounds the small calls, 12 bytes written per place the large ones.
#include "splash_common.cuh"

namespace splash {

namespace {

constexpr int kSlotThreads = 512;
constexpr int kPlacesPerThread = 1;       // (until there are two blocks for every SM)

struct SlotParams {
    const int32_t *seq_lens, *new_lens, *free_pages, *free_begin;
    int32_t *table, *positions, *q_start, *new_seq_lens, *counts;
    int64_t *slot_map;
    int64_t num_free, table_stride, num_slots;
    int32_t B, table_width, per_thread;
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens) { return (tokens + kPage - 1) / kPage; }

// Exclusive sum over the block's threads of one value each, and the sum of all.
__device__ __forceinline__ int64_t block_sum(int64_t mine, int64_t *scratch, int64_t &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
    }
    __syncthreads();                                  // the last user of scratch is done
    if (lane == 31) scratch[warp] = sum;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSlotThreads / 32; ++w) {
        const int64_t x = scratch[w];
        if (w < warp) before += x;
        total += x;
    }
    return before + sum - mine;
}

__global__ void __launch_bounds__(kSlotThreads)
kv_slots_kernel(const SlotParams p) {
    extern __shared__ int32_t shared[];
    int32_t *const start = shared;                    // [B + 1]
    int32_t *const first_page = shared + p.B + 1;     // [B] index into the free list of the request's first new page, or -1: refused
    __shared__ int64_t scratch[kSlotThreads / 32];
    __shared__ int refused;
    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x;
    if (tid == 0) refused = 0;
    const int i0 = min(tid * p.per_thread, p.B), i1 = min(i0 + p.per_thread, p.B);
    const int64_t begin = p.free_begin[0];
    const int64_t available = begin >= 0 && begin < p.num_free ? p.num_free - begin : 0;

    int64_t mine = 0, total, pages_total;
    for (int i = i0; i < i1; ++i) mine += max(p.new_lens[i], 0);
    int64_t at = block_sum(mine, scratch, total);
    // pages that a request asks for, if its table row and the places have room for it
    auto need_of = [&](int i, int64_t end) -> int64_t {
        const int64_t old = max(p.seq_lens[i], 0), now = old + max(p.new_lens[i], 0);
        const int64_t want = pages_of(now);
        return want > p.table_width || now > 0x7fffffff || end > p.num_slots ? -1 : want - pages_of(old);
    };
    mine = 0;
    int64_t end = at;
    for (int i = i0; i < i1; ++i) {
        start[i] = (int32_t)min(end, (int64_t)0x7fffffff);
        end += max(p.new_lens[i], 0);
        mine += max(need_of(i, end), (int64_t)0);
    }
    if (tid == 0) start[p.B] = (int32_t)min(total, (int64_t)0x7fffffff);
    int64_t page = block_sum(mine, scratch, pages_total);
    end = at;
    int bad = 0;
    int64_t given = 0;
    for (int i = i0; i < i1; ++i) {
        end += max(p.new_lens[i], 0);
        const int64_t need = need_of(i, end);
        const bool served = need == 0 || (need > 0 && page + need <= available);
        first_page[i] = served ? (int32_t)(need > 0 ? begin + page : 0) : -1;
        bad += !served;
        if (served) given += need;
        if (need > 0) page += need;
    }
    if (bad) atomicAdd(&refused, bad);
    int64_t taken;
    block_sum(given, scratch, taken);                 // (its barriers also publish start, first_page and refused)
    __syncthreads();

    if (blockIdx.x == 0) {
        for (int i = tid; i <= p.B; i += kSlotThreads) p.q_start[i] = start[i];
        for (int i = tid; i < p.B; i += kSlotThreads)
            p.new_seq_lens[i] = first_page[i] >= 0 ? max(p.seq_lens[i], 0) + max(p.new_lens[i], 0) : max(p.seq_lens[i], 0);
        if (tid == 0) {
            p.counts[0] = start[p.B];
            p.counts[1] = (int32_t)taken;
            p.counts[2] = refused;
            p.counts[3] = (int32_t)(begin + taken);
        }
    }
    for (int64_t t = (int64_t)blockIdx.x * kSlotThreads + tid; t < p.num_slots; t += (int64_t)gridDim.x * kSlotThreads) {
        int64_t slot = -1;
        int32_t pos = -1;
        if (t < start[p.B]) {
            int lo = 0, hi = p.B;                     // start[lo] <= t < start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (start[mid] <= t) lo = mid; else hi = mid;
            }
            if (first_page[lo] >= 0) {
                const int32_t old = max(p.seq_lens[lo], 0), have = (int32_t)pages_of(old);
                pos = old + (int32_t)(t - start[lo]);
                const int32_t j = pos / kPage;
                int32_t *const entry = p.table + lo * p.table_stride + j;
                int32_t id;
                if (j < have) {
                    id = *entry;
                } else {
                    id = p.free_pages[first_page[lo] + (j - have)];
                    if (pos % kPage == 0) *entry = id;
                }
                slot = (int64_t)id * kPage + pos % kPage;
            }
        }
        p.slot_map[t] = slot;
        p.positions[t] = pos;
    }
}

}  // namespace

cudaError_t launch_kv_slots(int32_t B, const int32_t *seq_lens, const int32_t *new_lens, const int32_t *free_pages, int64_t num_free,
                            const int32_t *free_begin, int32_t *table, int64_t table_stride, int32_t table_width, int64_t num_slots,
                            int64_t *slot_map, int32_t *positions, int32_t *q_start, int32_t *new_seq_lens, int32_t *counts, int sm_count,
                            cudaStream_t stream) {
    SlotParams p = {seq_lens, new_lens, free_pages, free_begin, table, positions, q_start, new_seq_lens, counts, slot_map, num_free, table_stride,
                    num_slots, B, table_width, (B + kSlotThreads - 1) / kSlotThreads};
    static DeviceOnce once;
    cudaError_t e = once.run([] {
        return cudaFuncSetAttribute(kv_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (2 * SPLASH_KV_SLOTS_MAX_REQUESTS + 1) * 4);
    });
    if (e != cudaSuccess) return e;
    const int64_t blocks = (num_slots + kSlotThreads * kPlacesPerThread - 1) / (kSlotThreads * kPlacesPerThread);
    const unsigned grid = (unsigned)(blocks < 1 ? 1 : blocks > 2 * sm_count ? 2 * sm_count : blocks);
    e = launch_dependent(kv_slots_kernel, dim3(grid), dim3(kSlotThreads), (size_t)(2 * B + 1) * 4, stream, p);
    count_launch();
    return e;
}

}  // namespace splash
