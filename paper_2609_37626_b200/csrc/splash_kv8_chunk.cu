// Attention of more than a few query rows (chunks of prompts, drafted rows) over a paged cache of keys and values in e4m3 with a scale per
// (page, head).
//
// The (row, head) pairs of a request and key head, m = row * group + head, are cut in tiles of 128; an item of work is (request, key head, tile).
// Two blocks of 10 warps share an SM, each with its own item, so that one's queries and outputs pass while the other works:
//   - 4 converter warps, two for keys and two for values, read a page's codes (16 bytes a lane), widen them to fp16 (exact) and lay them out in shared memory, keys K-major and values
//     MN-major in the 128-byte swizzle, two stages each;
//   - 1 warp issues tcgen05.mma: S = Q K^T from shared memory into one of two buffers in tensor memory; O += P V with P read from tensor memory, where the
//     softmax leaves it over S.  While the softmax has page u, S of page u + 1 is there and O of page u - 1 under way;
//   - 4 softmax warps, a thread per row: p = 2^(x - m + 7) with a reference m that moves only when a logit exceeds it by 8 (then O and the sum are
//     rescaled), p rounded to fp16, value scales folded into p as v_scale / U with U the largest so far of pages that the row sees;
//   - 1 scheduler warp walks the worker's share of the cost line and publishes segments (an item's range of pages) and their pages ahead of the others.
// Shared memory bounds it: a page costs 32 KB of stores, 16 KB for K and for V and 32 KB for Q, 768 cycles at 128 bytes, against 640 of MMAs and 512 of
// exponentials (two chunks of 2,048 rows behind 8,192 tokens, 32 heads on 8 of 128: 521 us a call in a loop, 925 TFLOP/s, 16 of them the join; some 2,450 cycles a page and
// block, of which two run.  The first call after a pause takes 585: the same cycles, but at 1.69 GHz; by the tenth 525).
// The line counts pages up to the tile's last causal row, and kOverhead per item (queries, epilogue); items cut by a share's end are joined by the
// combine kernel of the decode path.
#include "splash_kv8.cuh"
#include "splash_umma.cuh"

namespace splash {

namespace {

using namespace kv8;
using namespace umma;

constexpr int kTileRows = 128;
constexpr int kOverhead = 6;                       // cost of an item beside its pages, in pages
constexpr int kMinUnits = 8;                       // least cost of a worker's share
constexpr int kWarpKeys = 4, kWarpValues = 6, kWarpMma = 8, kThreads = 32 * 10;      // (softmax 0 to 3, scheduler 9)
constexpr int kNanBuffers = 8;

enum { kEmptyItem = 1, kEndOfWork = 2 };

struct alignas(16) Segment {
    int request, row0, rows_all, pairs;
    int m0, head, len, lo;             // lo, hi: tokens of the segment that the tile's last row sees
    int hi, t0, pages, slot;           // t0: first token of the first page
    int flags, pad[3];
};

// A page for the converters: the rows of the key head (NULL: no page of the pool, zeros) and their scales.
struct alignas(16) Page {
    const uint8_t *keys, *values;
    float k_scale, v_scale;
    int t0, lo, hi, flags;
};
enum { kPageEdge = 1 /* not all rows see all its tokens */, kPageLast = 2 /* of its segment */, kPageEnd = 4 };

enum {                                 // mbarriers
    kBarKFull = 0, kBarKEmpty = 2, kBarVFull = 4, kBarVEmpty = 6, kBarS = 8 /* [buffer] */, kBarP = 10, kBarO = 12, kBarQ = 14, kBarScale = 15,
    kBarSegFull = 19, kBarSegEmpty = 23, kBarPageFull = 27, kBarPageEmpty = 31, kNumBars = 35
};

template <int D>
struct Layout {
    static constexpr uint32_t kSlabs = D / 64;                             // of 64 fp16 values a row
    static constexpr uint32_t kQSlab = kTileRows * 128, kSlab = kPage * 128, kTile = kSlab * kSlabs;
    static constexpr uint32_t kQ = 0, kK = kQ + kQSlab * kSlabs, kV = kK + 2 * kTile;      // K and V: two stages each
    static constexpr uint32_t kNan = kV + 2 * kTile;                       // [8][128] first token with a NaN in dimension d, per segment
    static constexpr uint32_t kNanAny = kNan + kNanBuffers * 128 * 4;      // [8]
    static constexpr uint32_t kScales = kNanAny + 32;                      // [4] pages: key scale, value scale
    static constexpr uint32_t kSegments = kScales + 32;                    // [4]
    static constexpr uint32_t kPages = kSegments + 4 * sizeof(Segment);    // [4]
    static constexpr uint32_t kBars = kPages + 4 * sizeof(Page);
    static constexpr uint32_t kMisc = kBars + 8 * kNumBars + 8;            // tensor memory address, abort flag
    static constexpr uint32_t kBytes = kMisc + 16 + 1024;
    static constexpr uint32_t kColS = 0, kColO = 128, kColumns = 256;      // tensor memory: two buffers of S (and P over it) of 64 columns, O in D columns
};

// fp16 operands, fp32 sums
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, int b_mn_major) {
    return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t elected, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    umma_bf16(elected, d, a, b, idesc, accumulate);      // kind::f16: the operands' type is in the descriptor
}
// A from tensor memory: row m in lane m, two k to a column
__device__ __forceinline__ void mma_ts(uint32_t elected, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t *r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
// until such a load has arrived: nothing is done with its registers before
__device__ __forceinline__ void tmem_wait_ld32(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
          "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]),
          "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
        :: "memory");
}
__device__ __forceinline__ void tmem_st32u(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
          "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]) : "memory");
}

// ---- the cost line --------------------------------------------------------------------------------------------------------

// Tokens that row tile t of a request sees, and the pages that they lie in: its last row's range.
struct TileRange { int hi, pages; };
__device__ __forceinline__ TileRange tile_range(const AttnParams &p, const Request &r, int t) {
    const int last = (min((t + 1) * kTileRows, r.pairs) - 1) / p.group;
    TileRange x;
    x.hi = min(r.hi, r.len - r.rows_all + last + 1);
    x.pages = x.hi > r.lo ? (x.hi + kPage - 1) / kPage - r.lo / kPage : 0;
    return x;
}
__device__ __forceinline__ int row_tiles(const AttnParams &p, const Request &r) {
    return r.pairs < p.min_pairs || r.pairs > p.max_pairs ? 0 : (r.pairs + kTileRows - 1) / kTileRows;
}
// units of one key head of a request
__device__ __forceinline__ int64_t head_units(const AttnParams &p, const Request &r) {
    int64_t n = 0;
    const int tiles = row_tiles(p, r);
    for (int t = 0; t < tiles; ++t) n += kOverhead + tile_range(p, r, t).pages;
    return n;
}

// The same by a warp, and the row tile that holds unit u of a key head (u becomes its unit of that tile).
__device__ __forceinline__ int64_t head_units_warp(const AttnParams &p, const Request &r, int lane) {
    int64_t n = 0;
    const int tiles = row_tiles(p, r);
    for (int t = lane; t < tiles; t += 32) n += kOverhead + tile_range(p, r, t).pages;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
    return n;
}
__device__ __forceinline__ int tile_of_unit(const AttnParams &p, const Request &r, int64_t &u, int lane) {
    const int tiles = row_tiles(p, r);
    for (int t0 = 0;; t0 += 32) {
        const int cost = t0 + lane < tiles ? kOverhead + tile_range(p, r, t0 + lane).pages : 0;
        int64_t sum = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += x;
        }
        const unsigned behind = __ballot_sync(0xffffffffu, u < sum);      // tiles that end behind u
        const int64_t all = __shfl_sync(0xffffffffu, sum, 31);
        if (behind != 0 || t0 + 32 >= tiles) {
            const int k = behind != 0 ? __ffs(behind) - 1 : 31;
            u -= __shfl_sync(0xffffffffu, sum - cost, k);
            return t0 + k;
        }
        u -= all;
    }
}

struct Share { int64_t begin, end, total, u0; int i0, workers; };

__device__ __forceinline__ Share plan(const AttnParams &p, int worker) {
    __shared__ int64_t sums[kThreads / 32];
    __shared__ int64_t found_u;
    __shared__ int found_i;
    // up to 40 requests: a warp works one's units out, a lane for each of its row tiles; more requests have fewer tiles: a thread each
    constexpr int kFew = 40;
    __shared__ int64_t units[kFew];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.B + kThreads - 1) / kThreads, i0 = min(tid * per, p.B), i1 = min(i0 + per, p.B);
    const bool few = p.B <= kFew;
    if (few) {
        for (int i = warp; i < p.B; i += kThreads / 32) {
            const int64_t n = p.kv_heads * head_units_warp(p, request(p, i), lane);
            if (lane == 0) units[i] = n;
        }
        __syncthreads();
    }
    auto units_of = [&](int i) { return few ? units[i] : p.kv_heads * head_units(p, request(p, i)); };
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += units_of(i);
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += x;
    }
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    Share s;
    s.total = 0;
    int64_t before = sum - mine;
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += sums[w];
        s.total += sums[w];
    }
    // (every worker's share is worth a page at least, so that each from an item's first to its last has a piece of it)
    s.workers = (int)max((int64_t)1, min((int64_t)p.workers, s.total / kMinUnits));
    s.begin = worker < s.workers ? s.total * worker / s.workers : s.total;
    s.end = worker < s.workers ? s.total * (worker + 1) / s.workers : s.total;
    if (s.begin < s.end && before <= s.begin && s.begin < before + mine) {
        int64_t u = s.begin - before;
        int i = i0;
        for (; i < i1; ++i) {
            const int64_t n = units_of(i);
            if (u < n) break;
            u -= n;
        }
        found_i = i;
        found_u = u;
    }
    __syncthreads();
    s.i0 = s.begin < s.end ? found_i : p.B;
    s.u0 = s.begin < s.end ? found_u : 0;
    return s;
}

// ---- roles ----------------------------------------------------------------------------------------------------------------

struct Block {
    const AttnParams &p;
    uint8_t *smem;
    uint32_t base, bars, tmem;         // shared-memory addresses; tensor memory
    Ctx ctx;
    __device__ __forceinline__ uint32_t bar(int id) const { return bars + 8u * (uint32_t)id; }
};

// Published segments by turns: take() waits for the next one, done() gives its place back (by every warp that takes).
struct Segments {
    const Block &b;
    uint32_t offset, at = 0;
    __device__ __forceinline__ const Segment *take() {
        if (!warp_wait(b.ctx, b.bar(kBarSegFull + (at & 3)), (at >> 2) & 1, kBarSegFull)) return nullptr;
        const Segment *const s = reinterpret_cast<const Segment *>(b.smem + offset) + (at & 3);
        return s->flags & kEndOfWork ? nullptr : s;
    }
    __device__ __forceinline__ void done(int lane) {
        __syncwarp();
        if (lane == 0) mbar_arrive(b.bar(kBarSegEmpty + (at & 3)));
        ++at;
    }
};

template <int D>
__device__ __forceinline__ void schedule(const Block &b, const splash_kv8_cache &cache, const Share &share, int worker, int lane) {
    const AttnParams &p = b.p;
    Page *const pages_ring = reinterpret_cast<Page *>(b.smem + Layout<D>::kPages);
    uint32_t page_at = 0;
    Segment *const ring = reinterpret_cast<Segment *>(b.smem + Layout<D>::kSegments);
    uint32_t at = 0;
    bool ok = true, has_cut = false;
    auto publish = [&](const Segment &s) {
        ok = warp_wait(b.ctx, b.bar(kBarSegEmpty + (at & 3)), ((at >> 2) & 1) ^ 1, kBarSegEmpty);
        if (!ok) return;
        if (lane == 0) {
            ring[at & 3] = s;
            mbar_arrive(b.bar(kBarSegFull + (at & 3)));
        }
        __syncwarp();
        ++at;
    };
    // the segment's pages: a lane each finds one and its scales
    auto publish_pages = [&](const Segment &s) {
        for (int j0 = 0; ok && j0 < s.pages; j0 += 32) {
            const int j = j0 + lane;
            Page t = {};
            t.t0 = s.t0 + j * kPage; t.lo = s.lo; t.hi = s.hi;
            if (j < s.pages) {
                const int id = load_l2(p.table + s.request * p.table_stride + t.t0 / kPage);
                if (id >= 0 && id < p.num_pages) {
                    t.keys = static_cast<const uint8_t *>(cache.k_pool) + id * cache.k_page_stride + s.head * cache.k_head_stride;
                    t.values = static_cast<const uint8_t *>(cache.v_pool) + id * cache.v_page_stride + s.head * cache.v_head_stride;
                    t.k_scale = p.k_scales[id * p.k_scale_stride + s.head];
                    t.v_scale = p.v_scales[id * p.v_scale_stride + s.head];
                }
                if (t.t0 < s.lo || t.t0 + kPage > min(s.hi, s.len - s.rows_all + s.m0 / p.group + 1)) t.flags |= kPageEdge;
                if (j + 1 == s.pages) t.flags |= kPageLast;
            }
            for (int k = 0; ok && k < 32 && j0 + k < s.pages; ++k) {
                ok = warp_wait(b.ctx, b.bar(kBarPageEmpty + (page_at & 3)), ((page_at >> 2) & 1) ^ 1, kBarPageEmpty);
                if (!ok) break;
                if (lane == k) {
                    pages_ring[page_at & 3] = t;
                    mbar_arrive(b.bar(kBarPageFull + (page_at & 3)));
                }
                __syncwarp();
                ++page_at;
            }
        }
    };
    int64_t line = share.begin;
    int i = share.i0, head = 0, t = 0;
    if (i < p.B) {
        const Request r = request(p, i);
        const int64_t per_head = head_units_warp(p, r, lane);
        head = (int)(share.u0 / per_head);
        int64_t u = share.u0 - head * per_head;
        t = tile_of_unit(p, r, u, lane);
        line -= u;                                   // where the item begins
    }
    while (ok && i < p.B && line < share.end) {
        const Request r = request(p, i);
        const int tiles = row_tiles(p, r);
        for (; ok && head < p.kv_heads && line < share.end; ++head, t = 0)
            for (; ok && t < tiles && line < share.end; ++t) {
                const TileRange x = tile_range(p, r, t);
                const int64_t first = line + kOverhead, end = first + x.pages;
                const bool mine = line >= share.begin;           // where items are not cut: the worker's that holds its first unit
                const int64_t from = p.whole ? (mine ? first : end) : max(first, share.begin), to = p.whole ? end : min(end, share.end);
                Segment s = {};
                s.request = i; s.row0 = r.row0; s.rows_all = r.rows_all; s.pairs = r.pairs; s.m0 = t * kTileRows; s.head = head; s.len = r.len;
                s.slot = -1;
                if (from < to) {
                    s.pages = (int)(to - from);
                    s.t0 = (r.lo / kPage + (int)(from - first)) * kPage;
                    s.lo = max(r.lo, s.t0);
                    s.hi = to == end ? x.hi : s.t0 + s.pages * kPage;
                    s.slot = from > first ? 2 * worker : to < end ? 2 * worker + 1 : -1;
                    if (from == first && to < end) {
                        if (lane == 0) {
                            const int last = (int)((end * share.workers - 1) / share.total);     // the worker that holds the item's last unit
                            p.cut[2 * worker] = make_int4(last - worker + 1, r.row0, r.pairs, s.m0);
                            p.cut[2 * worker + 1] = make_int4(head, 0, 0, 0);
                        }
                        has_cut = true;
                    }
                    publish(s);
                    publish_pages(s);
                } else if (x.pages == 0 && mine) {
                    s.flags = kEmptyItem;
                    publish(s);
                }
                line = end;
            }
        if (head == p.kv_heads) { ++i; head = 0; t = 0; }
    }
    if (ok) {
        Segment s = {};
        s.flags = kEndOfWork;
        publish(s);
        if (ok) ok = warp_wait(b.ctx, b.bar(kBarPageEmpty + (page_at & 3)), ((page_at >> 2) & 1) ^ 1, kBarPageEmpty);
        if (ok && lane == 0) {
            pages_ring[page_at & 3].flags = kPageEnd;
            mbar_arrive(b.bar(kBarPageFull + (page_at & 3)));
        }
    }
    if (!has_cut && !p.whole && lane == 0) p.cut[2 * worker] = make_int4(0, 0, 0, 0);
}

// (What the converters have written is handed over to the async proxy here, behind the wait for them: a fence of theirs would wait for their loads of
// the next tile, which they have under way all the time.)
template <int D>
__device__ __forceinline__ void issue(const Block &b, int lane) {
    using L = Layout<D>;
    const uint32_t elected = elect_one(), tmem = uniform(b.tmem), base = uniform(b.base);
    constexpr uint32_t kDescS = idesc_f16(kTileRows, kPage, 0), kDescO = idesc_f16(kTileRows, D, 1);
    Segments segments{b, L::kSegments};
    uint32_t pages = 0, seg = 0;                      // pages and segments so far
    bool ok = true;
    // S of a page, when its keys are there
    auto logits = [&](uint32_t page) {
        const uint32_t stage = page & 1;
        if (!warp_wait(b.ctx, b.bar(kBarKFull + stage), (page >> 1) & 1, kBarKFull)) return false;
        fence_proxy_async();
        tcgen05_fence_after();
        const uint64_t q = make_desc(base + L::kQ, 16, 1024), k = make_desc(base + L::kK + stage * L::kTile, 16, 1024);
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
            mma_ss(elected, tmem + L::kColS + stage * 64, q + (((x >> 2) * L::kQSlab + (x & 3) * 32) >> 4), k + (((x >> 2) * L::kSlab + (x & 3) * 32) >> 4), kDescS, x != 0);
        if (elected) {
            umma_commit(b.bar(kBarS + stage));
            umma_commit(b.bar(kBarKEmpty + stage));
        }
        __syncwarp();
        return true;
    };
    while (ok) {
        const Segment *const s = segments.take();
        if (s == nullptr) break;
        const int n = (int)uniform((uint32_t)s->pages);
        if (n > 0) {
            ok = warp_wait(b.ctx, b.bar(kBarQ), seg & 1, kBarQ);
            for (int u = 0; ok && u < min(n, 2); ++u) ok = logits(pages + u);
            for (int u = 0; ok && u < n; ++u) {
                const uint32_t page = pages + u, stage = page & 1;
                ok = warp_wait(b.ctx, b.bar(kBarVFull + stage), (page >> 1) & 1, kBarVFull);
                if (ok) ok = warp_wait(b.ctx, b.bar(kBarP + stage), (page >> 1) & 1, kBarP);
                if (!ok) break;
                fence_proxy_async();
                tcgen05_fence_after();
                const uint64_t v = make_desc(base + L::kV + stage * L::kTile, L::kSlab, 1024);
#pragma unroll
                for (int x = 0; x < kPage / 16; ++x)
                    mma_ts(elected, tmem + L::kColO, tmem + L::kColS + stage * 64 + x * 8, v + ((x * 2048) >> 4), kDescO, (uint32_t)u | (uint32_t)x);
                if (elected) {
                    umma_commit(b.bar(kBarO + stage));
                    umma_commit(b.bar(kBarVEmpty + stage));
                }
                __syncwarp();
                if (u + 2 < n) ok = logits(page + 2);
            }
            pages += n;
            ++seg;
        }
        segments.done(lane);
    }
}

// Codes of one page's keys or values in registers on their way.  Of two warps a lane has 16 bytes of the rows `row` + 16 k in each slab of 64 dimensions, row =
// 8 warp + lane / 4: row mod 8, and with it the swizzle, is the same for all of them, and eight lanes' stores (four chunks of an even and of an odd
// row) meet no bank twice.
template <int D>
struct Codes {
    static constexpr int kSlabs = D / 64, kUnits = 4 * kSlabs;
    uint4 w[kUnits];
    static __device__ __forceinline__ int row_of(int tid) { return (tid >> 5) * 8 + (tid >> 2 & 7); }
    // page NULL: zeros; edge: tokens outside [lo, hi) are zeros too
    __device__ __forceinline__ void load(const uint8_t *page, bool edge, int t0, int lo, int hi, int tid) {
        const int row = row_of(tid), at = row * D + (tid & 3) * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int t = t0 + 16 * k + row;
            const bool there = page != nullptr && (!edge || (t >= lo && t < hi));
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                w[k * kSlabs + x] = make_uint4(0, 0, 0, 0);
                if (there) w[k * kSlabs + x] = *reinterpret_cast<const uint4 *>(page + at + k * 16 * D + x * 64);
            }
        }
    }
    // as fp16 into a stage: rows of 64 values in the 128-byte swizzle, slabs of 64 rows
    __device__ __forceinline__ void store(uint8_t *stage, int tid) const {
        const int row = row_of(tid), unit = 2 * (tid & 3);
        uint8_t *const even = stage + row * 128 + ((unit ^ (row & 7)) << 4), *const odd = stage + row * 128 + (((unit + 1) ^ (row & 7)) << 4);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                const uint4 c = w[k * kSlabs + x];
                uint4 h;
                to_f16x4(c.x, h.x, h.y);
                to_f16x4(c.y, h.z, h.w);
                *reinterpret_cast<uint4 *>(even + x * Layout<D>::kSlab + k * 16 * 128) = h;
                to_f16x4(c.z, h.x, h.y);
                to_f16x4(c.w, h.z, h.w);
                *reinterpret_cast<uint4 *>(odd + x * Layout<D>::kSlab + k * 16 * 128) = h;
            }
    }
    // NaN codes become zeros; the first token with one is noted per dimension
    __device__ __forceinline__ void take_out_nan(int *first, int *any, int t0, int tid) {
        uint32_t found = 0;
#pragma unroll
        for (int k = 0; k < kUnits; ++k)
#pragma unroll
            for (const uint32_t u : {w[k].x, w[k].y, w[k].z, w[k].w}) found |= (u & 0x7f7f7f7fu) + 0x01010101u;
        if ((found & 0x80808080u) == 0) return;
        *any = 1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int x = 0; x < kSlabs; ++x) {
                const uint4 c = w[k * kSlabs + x];
                uint32_t u[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t at = (((u[q] & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u;
                    u[q] &= ~(at * 0xffu);
                    for (int i = 0; i < 4; ++i)
                        if (at >> (8 * i) & 1u) atomicMin(first + x * 64 + (tid & 3) * 16 + q * 4 + i, t0 + 16 * k + row_of(tid));
                }
                w[k * kSlabs + x] = make_uint4(u[0], u[1], u[2], u[3]);
            }
    }
};

// The page behind `page` in the ring (NULL: no more work, or a wait gave up).
__device__ __forceinline__ const Page *page_of_ring(const Block &b, uint32_t offset, uint32_t page) {
    const bool ok = warp_wait(b.ctx, b.bar(kBarPageFull + (page & 3)), (page >> 2) & 1, kBarPageFull);
    const Page *const t = reinterpret_cast<const Page *>(b.smem + offset) + (page & 3);
    return ok && !(t->flags & kPageEnd) ? t : nullptr;
}

// Keys and values are converted by two warps each, so that a page's keys do not wait for the values of the one before.  Codes are fetched a page ahead.
template <int D>
__device__ __forceinline__ void convert_keys(const Block &b, int tid, int lane) {
    using L = Layout<D>;
    float *const scales = reinterpret_cast<float *>(b.smem + L::kScales);
    Codes<D> codes;
    uint32_t page = 0;
    const Page *now = page_of_ring(b, L::kPages, 0);
    if (now != nullptr) codes.load(now->keys, now->flags & kPageEdge, now->t0, now->lo, now->hi, tid);
    while (now != nullptr) {
        const uint32_t stage = page & 1, turn = page & 3;
        if (!warp_wait(b.ctx, b.bar(kBarKEmpty + stage), ((page >> 1) & 1) ^ 1, kBarKEmpty)) return;
        codes.store(b.smem + L::kK + stage * L::kTile, tid);
        if (tid == 0) {
            const float ks = now->k_scale, vs = now->v_scale;
            scales[2 * turn] = isfinite(ks) ? ks : NAN;      // (keys that are infinite, with either sign: their logit is no number)
            scales[2 * turn + 1] = isfinite(vs) ? vs : now->flags & kPageEdge ? 0.f : NAN;
            mbar_arrive(b.bar(kBarScale + turn));
        }
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(b.bar(kBarKFull + stage));
            mbar_arrive(b.bar(kBarPageEmpty + turn));
        }
        now = page_of_ring(b, L::kPages, ++page);
        if (now != nullptr) codes.load(now->keys, now->flags & kPageEdge, now->t0, now->lo, now->hi, tid);
    }
}

template <int D>
__device__ __forceinline__ void convert_values(const Block &b, int tid, int lane) {
    using L = Layout<D>;
    int *const nan = reinterpret_cast<int *>(b.smem + L::kNan), *const nan_any = reinterpret_cast<int *>(b.smem + L::kNanAny);
    Codes<D> codes;
    bool begins = true;
    uint32_t page = 0, seg = 0;
    const Page *now = page_of_ring(b, L::kPages, 0);
    if (now != nullptr) codes.load(now->values, now->flags & kPageEdge, now->t0, now->lo, now->hi, tid);
    while (now != nullptr) {
        const uint32_t stage = page & 1;
        const int flags = now->flags;
        if (begins) {         // a warp is at most two pages ahead of another, and the softmax warps at most two segments behind
            int *const first = nan + ((seg + 2) & (kNanBuffers - 1)) * 128;
            first[tid] = first[tid + 64] = 0x7fffffff;
            if (tid == 0) nan_any[(seg + 2) & (kNanBuffers - 1)] = 0;
        }
        if (!warp_wait(b.ctx, b.bar(kBarVEmpty + stage), ((page >> 1) & 1) ^ 1, kBarVEmpty)) return;
        if (flags & kPageEdge) {                     // 0 * NaN must not reach rows that do not see it
            int *const first = nan + (seg & (kNanBuffers - 1)) * 128, *const any = nan_any + (seg & (kNanBuffers - 1));
            codes.take_out_nan(first, any, now->t0, tid);
            if (!isfinite(now->v_scale)) {           // every value of the page is NaN, for the rows that see a token of it
                for (int d = tid; d < D; d += 64) atomicMin(first + d, max(now->lo, now->t0));
                *any = 1;
            }
        }
        codes.store(b.smem + L::kV + stage * L::kTile, tid);
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(b.bar(kBarVFull + stage));
            mbar_arrive(b.bar(kBarPageEmpty + (page & 3)));
        }
        begins = flags & kPageLast;
        if (begins) ++seg;
        now = page_of_ring(b, L::kPages, ++page);
        if (now != nullptr) codes.load(now->values, now->flags & kPageEdge, now->t0, now->lo, now->hi, tid);
    }
}

// two fp32 values at a time
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t x, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// The warp's rows of O times a factor per row.
template <int D>
__device__ __noinline__ void rescale(uint32_t col, float a) {
    for (int c = 0; c < D; c += 16) {
        float v[16];
        tmem_ld16(col + c, v);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] *= a;
        tmem_st16(col + c, v);
    }
    tmem_wait_st();
}

// The largest of a page's 64 sums, times their factor.
__device__ __noinline__ float largest_logit(uint32_t col, float a) {
    float top = -INFINITY;
    for (int c = 0; c < 64; c += 16) {
        float v[16];
        tmem_ld16(col + c, v);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; ++x) top = fmaxf(top, v[x] * a);
    }
    return top;
}

// The sums of a page's tokens that a row does not see (columns outside [first, last)) become such that their logits are -inf whatever the factor
// (which is changed where no such sum exists); those that it sees become NaN if the factor is.
__device__ __noinline__ float hide(uint32_t col, int first, int last, float a) {
    const bool nan = !(a == a);
    const float hidden = a < 0.f ? INFINITY : -INFINITY;
    for (int c = 0; c < 64; c += 16) {
        float v[16];
        tmem_ld16(col + c, v);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = c + x < first || c + x >= last ? hidden : nan ? NAN : v[x];
        tmem_st16(col + c, v);
    }
    tmem_wait_st();
    return nan ? 1.f : a == 0.f ? 1e-30f : a;
}

// 8 values of a row to out
__device__ __forceinline__ void store8(const AttnParams &p, int64_t at, const float (&v)[8]) {
    if (p.out_f32) {
        float4 *const to = reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at);
        to[0] = make_float4(v[0], v[1], v[2], v[3]);
        to[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.out) + at) =
            p.q_bf16 ? make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]))
                     : make_uint4(pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]), pack_f16x2(v[4], v[5]), pack_f16x2(v[6], v[7]));
    }
}

// The warp's rows of a finished segment, from tensor memory to out or to the workspace; out of line, which leaves the main loop its registers.  Rows of 16-bit
// outputs go through the place of the segment's queries, which no MMA reads any more and of which each warp has that of its own rows, so that lanes side by
// side write consecutive memory (two prompt chunks of 2,048 rows behind 8,192 tokens, 32 heads on 8 of 128: 517 us; inline, 16 bytes of a row a lane: 559).  A
// lane has 64 bytes of an fp32 row at a time, which are whole sectors as they are (by way of shared memory 523).
template <int D>
__device__ __noinline__ void give(const Block &b, const Segment &s, int r, int lane, uint32_t col_o, float scale, const int *nan, int lim) {
    const AttnParams &p = b.p;
    const int m = s.m0 + r, row = m / p.group, g = s.head * p.group + m - row * p.group;
    const bool there = m < s.pairs, wide = s.slot >= 0 || p.out_f32 != 0;
    const int64_t out_at = (s.row0 + (int64_t)row) * p.out_row + g * p.out_head;
    float *const out32 = s.slot < 0 ? static_cast<float *>(p.out) + out_at : p.part_out + ((int64_t)s.slot * kTileRows + r) * D;
    auto place = [&](int row, int k) {                // 16 bytes of it
        return reinterpret_cast<uint4 *>(b.smem + Layout<D>::kQ + (k >> 3) * Layout<D>::kQSlab + row * 128 + (((k & 7) ^ (row & 7)) << 4));
    };
#pragma unroll 1
    for (int c = 0; c < D; c += 16) {
        float v[16];
        tmem_ld16(col_o + c, v);
        tmem_wait_ld();
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            v[x] *= scale;
            if (nan != nullptr && nan[c + x] < lim) v[x] = NAN;
        }
        if (wide) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (there) reinterpret_cast<float4 *>(out32 + c)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float *const u = v + 8 * k;
                *place(r, c / 8 + k) = p.q_bf16 ? make_uint4(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3]), pack_bf16x2(u[4], u[5]), pack_bf16x2(u[6], u[7]))
                                                : make_uint4(pack_f16x2(u[0], u[1]), pack_f16x2(u[2], u[3]), pack_f16x2(u[4], u[5]), pack_f16x2(u[6], u[7]));
            }
        }
    }
    if (wide) return;
    __syncwarp();
    constexpr int kLanes = D / 8;                     // of a row
#pragma unroll 4
    for (int k = 0; k < kLanes; ++k) {
        const int from = k * (32 / kLanes) + lane / kLanes;
        const int64_t to = __shfl_sync(0xffffffffu, there ? out_at : -1, from);
        const uint4 x = *place((r & 96) + from, lane % kLanes);
        if (to >= 0) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.out) + to + 8 * (lane % kLanes)) = x;
    }
    __syncwarp();                                     // the next segment's queries are written behind these reads
}

template <int D>
__device__ __forceinline__ void soften(const Block &b, int r /* row of the tile */, int lane) {
    using L = Layout<D>;
    const AttnParams &p = b.p;
    Segments segments{b, L::kSegments};
    const uint32_t lanes = (uint32_t)(r & 96) << 16;
    const uint32_t col_s = b.tmem + lanes + L::kColS, col_o = b.tmem + lanes + L::kColO;
    const float *const scales = reinterpret_cast<const float *>(b.smem + L::kScales);
    uint32_t pages = 0, seg = 0;
    for (;;) {
        const Segment *const at = segments.take();
        if (at == nullptr) break;
        const Segment &s = *at;
        const int m = s.m0 + r, row = m / p.group, g = s.head * p.group + m - row * p.group;
        const bool there = m < s.pairs;
        const int64_t q_at = (s.row0 + (int64_t)row) * p.q_row + g * p.q_head, out_at = (s.row0 + (int64_t)row) * p.out_row + g * p.out_head;
        if (s.flags & kEmptyItem) {
            if (there) {
                const float zero[8] = {};
#pragma unroll
                for (int d = 0; d < D; d += 8) store8(p, out_at + d, zero);
                p.lse[(s.row0 + (int64_t)row) * p.lse_row + g] = -INFINITY;
            }
            segments.done(lane);
            continue;
        }
        // ---- the row's queries, as fp16 with a power of two that brings the largest to [2^14, 2^15)
        float back;
        {
            uint4 w[D / 8];
            int most = 0;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
                w[k] = make_uint4(0, 0, 0, 0);
                if (there) w[k] = reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.q) + q_at)[k];
            }
            // (the largest finite one, by its 16-bit pattern: patterns of finite values order like their sizes)
            const int inf = p.q_bf16 ? 0x7f80 : 0x7c00;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
                const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int lo = u[x] & 0x7fff, hi = u[x] >> 16 & 0x7fff;
                    if (lo < inf) most = max(most, lo);
                    if (hi < inf) most = max(most, hi);
                }
            }
            const float size = p.q_bf16 ? __int_as_float(most << 16) : __half2float(__ushort_as_half((unsigned short)most));
            const int shift = most == 0 ? 0 : min(14 - ((__float_as_int(size) >> 23) - 127), 100);
            const float factor = __int_as_float((shift + 127) << 23);
            back = p.scale_log2 * __int_as_float((127 - shift) << 23);
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
                const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
                uint32_t h[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float2 f;
                    if (p.q_bf16) f = make_float2(__uint_as_float(u[x] << 16), __uint_as_float(u[x] & 0xffff0000u));
                    else f = __half22float2(*reinterpret_cast<const __half2 *>(&u[x]));
                    h[x] = pack_f16x2(f.x * factor, f.y * factor);
                }
                *reinterpret_cast<uint4 *>(b.smem + L::kQ + (k >> 3) * L::kQSlab + r * 128 + (((k & 7) ^ (r & 7)) << 4)) =
                    make_uint4(h[0], h[1], h[2], h[3]);
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(b.bar(kBarQ));
        }
        const int lim = there ? min(s.hi, s.len - s.rows_all + row + 1) : s.hi;
        const int lim_min = __reduce_min_sync(0xffffffffu, lim);
        const int lo = s.lo, n = s.pages, start = s.t0;
        float ref = kUnset, l = 0.f, unit = 0.f;
        bool ok = true;
        const bool idle = s.m0 + (r & 96) >= s.pairs;
        for (int u = 0; idle && ok && u < n; ++u) {       // none of the warp's rows: what lies in their weights' place is as good as any
            const uint32_t page = pages + u, buffer = page & 1;
            ok = warp_wait(b.ctx, b.bar(kBarS + buffer), (page >> 1) & 1, kBarS);
            if (ok && lane == 0) mbar_arrive(b.bar(kBarP + buffer));
        }
        for (int u = idle ? n : 0; ok && u < n; ++u) {
            const uint32_t page = pages + u, buffer = page & 1;
            const uint32_t col = col_s + buffer * 64;
            ok = warp_wait(b.ctx, b.bar(kBarScale + (page & 3)), (page >> 2) & 1, kBarScale);
            if (!ok) break;
            float a = back * scales[2 * (page & 3)];
            const int tb = start + u * kPage;
            // (a row that sees no token of the page keeps its unit: the page's scale, which may be anything to it, does not move its O)
            const float vs = tb < lim ? scales[2 * (page & 3) + 1] : 0.f;
            ok = warp_wait(b.ctx, b.bar(kBarS + buffer), (page >> 1) & 1, kBarS);
            if (!ok) break;
            tcgen05_fence_after();
            // rescales O, once the MMAs of the page before are done with it
            auto shrink = [&](float factor) {
                ok = warp_wait(b.ctx, b.bar(kBarO + (buffer ^ 1)), ((page - 1) >> 1) & 1, kBarO);
                tcgen05_fence_after();
                rescale<D>(col_o, factor);
            };
            const bool larger = fabsf(vs) > unit;
            if (__any_sync(0xffffffffu, larger)) {
                if (u > 0) shrink(larger ? __fdividef(unit, fabsf(vs)) : 1.f);
                if (larger) unit = fabsf(vs);
            }
            const float f = vs == unit ? 1.f : __fdividef(vs, unit);
            if (tb < lo || tb + kPage > lim_min) a = hide(col, lo - tb, lim - tb, a);
            // y = x - ref, p = 2^y.  Whether a logit exceeds the reference by too much shows while the weights are computed; then they
            // are computed again (the weights' place is that of the sums: they are written when all of them are known to be right).
            uint32_t w[32];
            uint64_t sum[4];
            for (int tries = 0;; ++tries) {
                const uint64_t a2 = pair(a, a), c2 = pair(-ref, -ref), f2 = pair(f, f);
                float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] = 0;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t v[32];
                    tmem_ld32(col + 32 * c, v);
                    tmem_wait_ld32(v);
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        float y0, y1, lo2, hi2;
                        unpair(fma2(pair(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1])), a2, c2), y0, y1);
                        most[x & 3] = fmaxf(fmaxf(most[x & 3], y0), y1);
                        const uint64_t e = pair(fast_exp2(y0), fast_exp2(y1));
                        sum[x & 3] = add2(sum[x & 3], e);
                        unpair(mul2(e, f2), lo2, hi2);
                        w[16 * c + x] = pack_f16x2(lo2, hi2);
                    }
                }
                if (!__any_sync(0xffffffffu, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) > kLift + kSlack) || tries == 1) break;
                const float top = largest_logit(col, a) - kLift;
                const bool grows = top > ref;
                const float factor = grows ? fast_exp2(ref - top) : 1.f;
                l *= factor;
                if (grows) ref = top;
                if (u > 0) shrink(factor);
            }
            tmem_st32u(col, w);
            float lo2, hi2;
            unpair(add2(add2(sum[0], sum[1]), add2(sum[2], sum[3])), lo2, hi2);
            l += lo2 + hi2;
            tmem_wait_st();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(b.bar(kBarP + buffer));
        }
        if (!ok) return;
        // ---- epilogue
        const uint32_t end = pages + n - 1;
        if (!warp_wait(b.ctx, b.bar(kBarO + (end & 1)), (end >> 1) & 1, kBarO)) return;
        tcgen05_fence_after();
        const float scale = l == 0.f ? 0.f : __fdividef(unit, l);
        const float lse2 = l == 0.f ? -INFINITY : ref + __log2f(l);
        const int *const nan = reinterpret_cast<const int *>(b.smem + L::kNan) + (seg & (kNanBuffers - 1)) * 128;
        const bool nans = reinterpret_cast<const volatile int *>(b.smem + L::kNanAny)[seg & (kNanBuffers - 1)] != 0;
        give<D>(b, s, r, lane, col_o, scale, nans ? nan : nullptr, lim);
        if (there) {
            if (s.slot < 0) p.lse[(s.row0 + (int64_t)row) * p.lse_row + g] = lse2 * kLn2;
            else p.part_lse[s.slot * kTileRows + r] = lse2;
        }
        tcgen05_fence_before();
        pages += n;
        segments.done(lane);
        ++seg;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
kv8_chunk_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ splash_kv8_cache cache) {
    using L = Layout<D>;
    extern __shared__ uint8_t raw[];
    uint8_t *const smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, worker = blockIdx.x;
    volatile uint32_t *const misc = reinterpret_cast<volatile uint32_t *>(smem + L::kMisc);
    const uint32_t bars = smem_u32(smem + L::kBars);
    if (tid == 0) {
        for (int k = 0; k < 2; ++k) {
            mbar_init(bars + 8 * (kBarKFull + k), 2); mbar_init(bars + 8 * (kBarKEmpty + k), 1);
            mbar_init(bars + 8 * (kBarVFull + k), 2); mbar_init(bars + 8 * (kBarVEmpty + k), 1);
            mbar_init(bars + 8 * (kBarS + k), 1); mbar_init(bars + 8 * (kBarP + k), 4); mbar_init(bars + 8 * (kBarO + k), 1);
        }
        mbar_init(bars + 8 * kBarQ, 4);
        for (int k = 0; k < 4; ++k) {
            mbar_init(bars + 8 * (kBarScale + k), 1);
            mbar_init(bars + 8 * (kBarSegFull + k), 1); mbar_init(bars + 8 * (kBarSegEmpty + k), 5);
            mbar_init(bars + 8 * (kBarPageFull + k), 1); mbar_init(bars + 8 * (kBarPageEmpty + k), 4);
        }
        misc[1] = 0;
        for (int k = 0; k < kNanBuffers; ++k) reinterpret_cast<int *>(smem + L::kNanAny)[k] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int k = tid; k < kNanBuffers * 128; k += kThreads) reinterpret_cast<int *>(smem + L::kNan)[k] = 0x7fffffff;
    if (warp == kWarpMma) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem + L::kMisc)), "r"(L::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    grid_dependency_wait();
    grid_launch_dependents();
    if (p.clear_status && blockIdx.x == 0 && tid < 4) p.status[tid] = 0;
    const Share share = plan(p, worker);
    const Block b = {p, smem, smem_u32(smem), bars, misc[0], Ctx{misc + 1, p.status}};
    if (warp < kWarpKeys) soften<D>(b, tid, lane);
    else if (warp < kWarpValues) convert_keys<D>(b, tid - 32 * kWarpKeys, lane);
    else if (warp < kWarpMma) convert_values<D>(b, tid - 32 * kWarpValues, lane);
    else if (warp == kWarpMma) issue<D>(b, lane);
    else schedule<D>(b, cache, share, worker, lane);
    if (misc[1]) {
        // a wait has given up: MMAs that were issued must be over before the tensor memory is
        const unsigned long long since = global_timer_ns();
        while (global_timer_ns() - since < 200000ull) __nanosleep(1000);
    }
    tcgen05_fence_before();
    __syncthreads();
    if (warp == kWarpMma) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(misc[0]), "r"(L::kColumns) : "memory");
    }
}

template <int D>
cudaError_t launch_chunk(const AttnParams &p, const splash_kv8_cache &cache, cudaStream_t stream) {
    static DeviceOnce once;
    cudaError_t e = once.run([] { return cudaFuncSetAttribute(kv8_chunk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Layout<D>::kBytes); });
    if (e != cudaSuccess) return e;
    e = launch_dependent(kv8_chunk_kernel<D>, dim3(p.workers), dim3(kThreads), Layout<D>::kBytes, stream, p, cache);
    count_launch();
    return e;
}

}  // namespace

cudaError_t launch_kv8_chunk_combine(const AttnParams &p, int D, cudaStream_t stream);     // (with the combine kernel of the decode path)

int kv8_chunk_rows() { return kTileRows; }
int kv8_chunk_workers(int sm_count) { return 2 * sm_count; }

cudaError_t launch_kv8_chunk(const AttnParams &p, const splash_kv8_cache &cache, cudaStream_t stream) {
    cudaError_t e = cache.head_dim == 128 ? launch_chunk<128>(p, cache, stream) : launch_chunk<64>(p, cache, stream);
    if (e == cudaSuccess && !p.whole) e = launch_kv8_chunk_combine(p, cache.head_dim, stream);
    return e;
}

}  // namespace splash
