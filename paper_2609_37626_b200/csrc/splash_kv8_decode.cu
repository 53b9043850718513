// Attention of few query rows over a paged cache of keys and values in e4m3 with a scale per (page, head).
//
// For a key head the query rows of a request and the heads of the group form (row, head) pairs, m = row * group + head, cut in tiles of up to
// 16 (heads of 64: 32).  An item of work is (request, key head, tile); its pages are streamed once:
//     x = q . K * softmax_scale * log2 e * k_scale,  p = 2^(x - m + 7),  l += p,  O += p * v_scale / U * V
// with a reference m per row that moves only when a logit exceeds it by 8 (then O and l are rescaled) and U the largest
// value scale so far, of the pages that the row sees.  p <= 2^15 is rounded to fp16 for the product with V: 11 bits, for weights down to 2^-21 of the largest.  Queries are scaled to
// fp16's range by a power of two per row, so that bf16 ones lose nothing.
//
// The cache's bytes bound it, 16 KB a page and head of 128: one context of 262,144 tokens on eight key heads takes 92 us, 5.8 TB/s of the 6.5 that a copy
// has; 64 contexts of 1k to 8k tokens 103 us, 5.9 TB/s; from 24 pairs on the MMAs and conversions do (heads of 128, 64 contexts of 4,096 tokens: 8 pairs 92 us,
// 16 pairs 119, 24 pairs 215, 32 pairs 223).  What it takes to stay there:
//   - items are cut where the cost line (pages, and kOverhead per item) of all requests passes a worker's share, so one long
//     context and 512 short ones fill the SMs alike; cut items are joined by a combine kernel.  Three workers per SM;
//   - a producer warp walks the line, 32 pages at once: a lane each finds its page, its scales and its flags; TMA brings
//     keys and values (swizzled against bank conflicts), three or six pages ahead, across items;
//   - four warps take 16 tokens of every page each, with their own m, l, O: they meet only at the end of an item;
//   - tokens and dimensions are the MMAs' m, rows their n: eight rows fill it (rows on m, 16 at a time, were half empty: the same contexts took 128 and 143 us);
//     weights are turned from S's layout to the operand's by movmatrix;
//   - the order of dimensions within an MMA's k does not matter if both operands agree, nor the order of tokens: a lane reads
//     its key and value codes 16 bytes at a time and widens them in registers (e4m3 -> fp16 is exact).  Keys: lane (n, c) of the fragment takes
//     token perm(n) and the 16-byte chunks c, c + 4 of its row, which are the values of the k slots 2c, 2c + 1, 2c + 8, 2c + 9 of successive
//     MMAs; values: tokens c, c + 4, c + 8, c + 12 and the chunk perm(n), bytes of two tokens interleaved.
// mma.sync and not tcgen05: with so few rows the MMAs take a third of the time that the bytes take, and the 8-bit
// operands would have to be widened into shared memory first, twice the bytes over the path that is next in line.
#include <type_traits>

#include "splash_kv8.cuh"
#include "splash_umma.cuh"

namespace splash {

namespace {

using namespace kv8;
using namespace umma;

constexpr int kConsumers = 4;                       // warps, 16 tokens of a page each
constexpr int kThreads = 32 * (kConsumers + 1);
constexpr int kOverhead = 5;                        // cost of an item beside its pages, in pages (512 rollout requests: 98.5 us with 2, 96.5 with 4 to 6, 97.4 with 8)
constexpr int kMinUnits = 2;                        // least cost of a worker's share

enum { kFirst = 1, kLast = 2, kEmpty = 4, kEnd = 8, kEdge = 16, kCausal = 32 };

// What the consumers need to know about a page in the ring, written by the producer.
struct alignas(16) PageInfo {
    int flags;                          // (these four are read at once, for every page)
    float k_scale, v_scale;
    int t0;                             // first token of the page
    int row0, rows_all, pairs, m0;      // the item's rows
    int head, len, lo, hi;              // key head; context; the request's token range
    int slot, pad[3];                   // partial slot or -1
};

// NT: tiles of eight rows
template <int D, int NT>
struct Layout {
    static constexpr int kRows = 8 * NT;
    static constexpr int kCtas = 3;                                        // blocks of an SM
    static constexpr bool kQueryShared = NT > 1;                           // queries as MMA operands in shared memory, or in registers
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr int kHalf = 64 * D;                                   // keys or values of a page
    static constexpr int kPad = D + 4;
    static constexpr int kMerge = kStages * 2 * kHalf;                     // [4][8][D + 4] fp32
    static constexpr int kQuery = kMerge + kConsumers * 8 * kPad * 4;      // [NT][D / 16][32] uint2
    static constexpr int kInfo = kQuery + (kQueryShared ? NT * (D / 16) * 256 : 0);
    static constexpr int kStats = kInfo + kStages * (int)sizeof(PageInfo); // references, sums: [4][rows] each, two sets
    static constexpr int kBars = kStats + 2 * 2 * kConsumers * kRows * 4;
    static constexpr int kBytes = kBars + (2 * kStages + 1) * 8 + 1024;    // (the start is aligned to 1,024)
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// bytes that the barrier's phase is to wait for beside its arrivals
__device__ __forceinline__ void mbar_announce(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// 16-byte chunk `chunk` of row `row` of a [64][D] tile as the TMA unit has swizzled it
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
    return D == 128 ? row * 128 + ((chunk ^ (row & 7)) << 4) : row * 64 + ((chunk ^ (row >> 1 & 3)) << 4);
}

// 16 query values from dimension d on, as fp32
__device__ __forceinline__ void load_q16(const AttnParams &p, int64_t at, bool there, float (&v)[16]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint4 w = make_uint4(0, 0, 0, 0);
        if (there) w = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p.q) + at + half * 8);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float2 f;
            if (p.q_bf16) f = make_float2(__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xffff0000u));
            else f = __half22float2(*reinterpret_cast<const __half2 *>(&u[k]));
            v[half * 8 + 2 * k] = f.x; v[half * 8 + 2 * k + 1] = f.y;
        }
    }
}

// Units of the cost line: (kOverhead + pages) for each (key head, tile) of a request that is this kernel's.
template <int kRows>
__device__ __forceinline__ int64_t units_of(const AttnParams &p, const Request &r) {
    if (r.pairs < p.min_pairs || r.pairs > p.max_pairs || r.pairs == 0) return 0;
    return (int64_t)p.kv_heads * ((r.pairs + kRows - 1) / kRows) * (kOverhead + r.pages());
}

// floor(total * w / W) and, the other way, the worker whose share holds unit x.  A line of less than 2^31 units (all but absurd
// ones) needs no division in 64 bits, which is a subroutine.
__device__ __forceinline__ int64_t share_begin(int64_t total, int w, int W) {
    if (total >> 31) return total * w / W;
    const unsigned t = (unsigned)total, a = t / (unsigned)W, b = t - a * (unsigned)W;
    return a * (unsigned)w + b * (unsigned)w / (unsigned)W;
}
__device__ __forceinline__ int worker_of(int64_t x, int64_t total, int W) { return (int)(((x + 1) * W - 1) / total); }

struct Share { int64_t begin, end, total, u0; int i0, workers; };

// The worker's share of the cost line and where it begins: request i0, unit u0 of it.  All threads.
template <int kRows>
__device__ __forceinline__ Share plan(const AttnParams &p, int worker) {
    __shared__ int64_t sums[kThreads / 32];
    __shared__ int64_t found_u;
    __shared__ int found_i;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.B + kThreads - 1) / kThreads, i0 = min(tid * per, p.B), i1 = min(i0 + per, p.B);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += units_of<kRows>(p, request(p, i));
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
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
        if (w < warp) before += sums[w];
        s.total += sums[w];
    }
    s.workers = (int)max((int64_t)1, min((int64_t)p.workers, s.total / kMinUnits));
    s.begin = worker < s.workers ? share_begin(s.total, worker, s.workers) : s.total;
    s.end = worker < s.workers ? share_begin(s.total, worker + 1, s.workers) : s.total;
    if (before <= s.begin && s.begin < before + mine) {
        int64_t u = s.begin - before;
        int i = i0;
        for (; i < i1; ++i) {
            const int64_t n = units_of<kRows>(p, request(p, i));
            if (u < n) break;
            u -= n;
        }
        found_i = i;
        found_u = u;
    }
    __syncthreads();
    s.i0 = s.begin < s.total ? found_i : p.B;
    s.u0 = s.begin < s.total ? found_u : 0;
    return s;
}

template <int D, int NT>
__device__ __forceinline__ void produce(const AttnParams &p, const Share &share, const CUtensorMap *k_map, const CUtensorMap *v_map, uint8_t *smem, uint32_t bars,
                                        const Ctx &ctx, int worker, int lane) {
    using L = Layout<D, NT>;
    const uint32_t full = bars, empty = bars + 8 * L::kStages;
    PageInfo *const info = reinterpret_cast<PageInfo *>(smem + L::kInfo);
    int stage = 0, i = share.i0;
    uint32_t phase = 0;
    int64_t unit = share.begin, u = share.u0;
    bool ok = true, has_cut = false, more = share.begin < share.end, first = true;
    while (more && ok) {
        // every lane: its unit's item, page and scales
        const int64_t mine = unit + lane;
        int64_t lu = u + lane;
        int li = i;
        Request r = {};
        int64_t n = 0;
        for (; li < p.B; ++li) {
            r = request(p, li);
            n = units_of<L::kRows>(p, r);
            if (lu < n) break;
            lu -= n;
        }
        const bool exists = li < p.B;
        const int pages = r.pages(), cost = kOverhead + pages;
        const int sub = !exists ? 0 : lu >> 31 ? (int)(lu / cost) : (int)((unsigned)lu / (unsigned)cost), pos = exists ? (int)(lu - (int64_t)sub * cost) : 0;
        const int tiles = (r.pairs + L::kRows - 1) / L::kRows;
        const int64_t item = mine - pos;                       // the item's place on the line
        const bool done = !exists || (p.whole ? item >= share.end : mine >= share.end);
        const bool ours = !done && (!p.whole || item >= share.begin);
        const bool data = ours && pos >= kOverhead, blank = ours && pages == 0 && pos == 0;
        const bool cut_front = !p.whole && item + kOverhead < share.begin, cut_back = !p.whole && item + cost > share.end;
        PageInfo a = {};
        int id = 0;
        bool valid = false;
        if (data) {
            const int page = r.lo / kPage + pos - kOverhead;
            id = load_l2(p.table + li * p.table_stride + page);
            valid = id >= 0 && id < p.num_pages;
            a.t0 = page * kPage;
        }
        a.row0 = r.row0; a.rows_all = r.rows_all; a.pairs = r.pairs; a.m0 = exists ? (sub % tiles) * L::kRows : 0;
        a.head = exists ? sub / tiles : 0; a.len = r.len; a.lo = r.lo; a.hi = r.hi;
        a.slot = pages == 0 ? -1 : cut_front ? 2 * worker : cut_back ? 2 * worker + 1 : -1;
        a.k_scale = valid ? p.k_scales[id * p.k_scale_stride + a.head] : 0.f;
        a.v_scale = valid ? p.v_scales[id * p.v_scale_stride + a.head] : 0.f;
        if (data) {
            if (pos == kOverhead || mine == share.begin) a.flags |= kFirst;
            if (pos == cost - 1 || (!p.whole && mine == share.end - 1)) a.flags |= kLast;
            // tokens outside the range, or hidden from some of the rows
            if (a.t0 < r.lo || a.t0 + kPage > r.hi) a.flags |= kEdge;
            if (a.t0 + kPage > r.len - r.rows_all + 1) a.flags |= r.rows_all > 1 ? kEdge | kCausal : kEdge;
        } else {
            a.flags = kEmpty;
        }
        if (data && pos == kOverhead && cut_back) {
            const int pieces = worker_of(item + cost - 1, share.total, share.workers) - worker + 1;
            p.cut[2 * worker] = make_int4(pieces, a.row0, a.pairs, a.m0);
            p.cut[2 * worker + 1] = make_int4(a.head, 0, 0, 0);
        }
        has_cut |= __any_sync(0xffffffffu, data && pos == kOverhead && cut_back);
        unsigned todo = __ballot_sync(0xffffffffu, data || blank);
        auto copy = [&](int to) {
            const uint32_t dst = smem_u32(smem) + to * 2 * L::kHalf;
            mbar_announce(full + 8 * to, 2 * L::kHalf);
            tma_load_4d(dst, k_map, full + 8 * to, 0, 0, a.head, valid ? id : p.num_pages);      // (behind the pool: zeros)
            tma_load_4d(dst + L::kHalf, v_map, full + 8 * to, 0, 0, a.head, valid ? id : p.num_pages);
        };
        unsigned sent = 0;
        if (first) {
            // the ring is empty: the copies of the first pages do not wait for these pages' scales, which are still on their way
            unsigned ahead = todo;
            for (int to = 0; to < L::kStages && ahead != 0; ++to, ahead &= ahead - 1) {
                const int j = __ffs(ahead) - 1;
                if (lane == j && data) copy(to);
                sent |= 1u << j;
            }
            first = false;
        }
        while (todo != 0) {
            const int j = __ffs(todo) - 1;
            todo &= todo - 1;
            ok = warp_wait(ctx, empty + 8 * stage, phase ^ 1, 100 + stage);
            if (!ok) break;
            if (lane == j) {
                if (data && !(sent >> j & 1u)) copy(stage);
                info[stage] = a;
                mbar_arrive(full + 8 * stage);
            }
            __syncwarp();
            if (++stage == L::kStages) { stage = 0; phase ^= 1; }
        }
        more = !__shfl_sync(0xffffffffu, (int)done, 31);
        i = __shfl_sync(0xffffffffu, li, 31);
        u = __shfl_sync(0xffffffffu, lu, 31) + 1;
        unit += 32;
    }
    if (ok) ok = warp_wait(ctx, empty + 8 * stage, phase ^ 1, 120);
    if (ok && lane == 0) {
        info[stage].flags = kEnd;
        mbar_arrive(full + 8 * stage);
    }
    if (!p.whole && !has_cut && lane == 0) p.cut[2 * worker] = make_int4(0, 0, 0, 0);
    if (!ok) {
        // a wait has given up: the copies still in flight must land before the block's shared memory goes to another one
        for (int s = 0; s < L::kStages; ++s) {
            const uint32_t parity = s < stage ? phase : phase ^ 1;         // of the stage's last use
            for (int k = 0; k < 100000 && !mbar_test_wait(full + 8 * s, parity); ++k) {}
        }
    }
}

// All consumer warps meet; false: one of them has given up.
__device__ __forceinline__ bool meet(const Ctx &ctx, uint32_t bar, uint32_t &phase, int lane) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
    const bool ok = warp_wait(ctx, bar, phase, 130);
    phase ^= 1;
    return ok;
}

__device__ __forceinline__ void store4(const AttnParams &p, int64_t at, const float4 &v) {
    if (p.out_f32) {
        *reinterpret_cast<float4 *>(static_cast<float *>(p.out) + at) = v;
    } else {
        const uint2 h = p.q_bf16 ? make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)) : make_uint2(pack_f16x2(v.x, v.y), pack_f16x2(v.z, v.w));
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p.out) + at) = h;
    }
}

// transposes an 8 x 8 matrix of 16-bit values that lies in the warp's registers, two to a lane
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ float number(float x) { return fabsf(x) == INFINITY ? NAN : x; }

// What a row that is done is multiplied with where the unit grows from `from` to `to`: its result O * unit / l stays, and so does its sum, with l times
// 2^shift and the reference less by that.  Three eighths of the growth go to l and the rest to O, however many steps it takes, so that neither leaves
// fp32's range (l is below 2^45, O in the order of 2^7; from 2^-7 to 2^127 l grows by 2^50 and O falls by 2^84).
struct Done { float o, l, shift; };
__device__ __forceinline__ Done done_row(float from, float to) {
    const int a = __float_as_int(from), b = __float_as_int(to), grown = (b >> 23) - (a >> 23), shift = (3 * (b >> 23) >> 3) - (3 * (a >> 23) >> 3);
    const float mantissas = __fdividef(__int_as_float((a & 0x7fffff) | 0x3f800000), __int_as_float((b & 0x7fffff) | 0x3f800000));
    Done d;
    d.o = from == 0.f ? 0.f : mantissas * __int_as_float(max(127 - (grown - shift), 0) << 23);
    d.l = __int_as_float((127 + shift) << 23);
    d.shift = (float)shift;
    return d;
}

template <int D, int NT>
__device__ __forceinline__ void consume(const AttnParams &p, uint8_t *smem, uint32_t bars, const Ctx &ctx, int warp, int lane) {
    using L = Layout<D, NT>;
    constexpr int kK = D / 16, kM = D / 16;                 // MMAs along the dimensions: as k of the logits, as m of the outputs
    constexpr bool kQueryShared = L::kQueryShared;
    const uint32_t full = bars, empty = bars + 8 * L::kStages, group_bar = bars + 16 * L::kStages;
    const PageInfo *const infos = reinterpret_cast<const PageInfo *>(smem + L::kInfo);
    float *const merge = reinterpret_cast<float *>(smem + L::kMerge);
    uint2 *const query = reinterpret_cast<uint2 *>(smem + L::kQuery);
    // references and sums of the warps' rows, in two sets by turns: a warp may be at the end of the next item while another still reads these
    float *stat_m = reinterpret_cast<float *>(smem + L::kStats);
    const int n = lane >> 2, c = lane & 3;
    const int perm = D == 128 ? (n >> 1) | (n & 1) << 2 : n;
    // tokens (of the warp's 16) whose logits the lane holds: perm and perm + 8; whose values it reads: these four
    const int tok_a = D == 128 ? c : 2 * c, tok_b = D == 128 ? c + 4 : 2 * c + 1;
    const int tok[4] = {tok_a, tok_b, tok_a + 8, tok_b + 8};

    float o[NT][kM][4], ref[NT][2], l[NT][2], rs[NT][2], unit = 0.f, per_unit = 0.f;      // of the rows 2c, 2c + 1 of each tile of eight
    uint32_t qf[kQueryShared ? 1 : NT][kK][2];
    int lim[NT][2];
    int stage = 0;
    uint32_t phase = 0, group_phase = 0;
    for (;;) {
        if (!warp_wait(ctx, full + 8 * stage, phase, 140 + stage)) break;
        const PageInfo &info = infos[stage];
        const int4 page = *reinterpret_cast<const int4 *>(&info);
        const int flags = page.x;
        if (flags & kEnd) break;
        if (flags & (kFirst | kEmpty)) {
            // the item's queries, as fp16 with a power of two per row that brings the largest of a row to [2^14, 2^15)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float v[D / 64][16];
                const int mm = info.m0 + nt * 8 + n;
                const bool there = mm < info.pairs && !(flags & kEmpty);
                const int row = mm / p.group, g = mm - row * p.group;
                const int64_t at = (info.row0 + row) * p.q_row + (info.head * p.group + g) * p.q_head;
                int most = 0;
#pragma unroll
                for (int h = 0; h < D / 64; ++h) {
                    load_q16(p, at + h * 64 + 16 * c, there, v[h]);
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const int b = __float_as_int(v[h][k]) & 0x7fffffff;
                        if (b < 0x7f800000) most = max(most, b);
                    }
                }
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                const int shift = most == 0 ? 0 : min(14 - ((most >> 23) - 127), 100);
                const float factor = __int_as_float((shift + 127) << 23), back = p.scale_log2 * __int_as_float((127 - shift) << 23);
                const int limit = there ? min(info.hi, info.len - info.rows_all + row + 1) : info.hi;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    rs[nt][e] = __shfl_sync(0xffffffffu, back, 4 * (2 * c + e));
                    lim[nt][e] = __shfl_sync(0xffffffffu, limit, 4 * (2 * c + e));
                    ref[nt][e] = kUnset;
                    l[nt][e] = 0.f;
                }
#pragma unroll
                for (int k = 0; k < kK; ++k) {
                    const int h = k / 4, x = 4 * (k % 4);
                    const uint2 b = make_uint2(pack_f16x2(v[h][x] * factor, v[h][x + 1] * factor), pack_f16x2(v[h][x + 2] * factor, v[h][x + 3] * factor));
                    if constexpr (!kQueryShared) { qf[nt][k][0] = b.x; qf[nt][k][1] = b.y; }
                    else if (k % kConsumers == warp) query[(nt * kK + k) * 32 + lane] = b;
                }
#pragma unroll
                for (int j = 0; j < kM; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) o[nt][j][x] = 0.f;
            }
            unit = per_unit = 0.f;
            if (kQueryShared && !meet(ctx, group_bar, group_phase, lane)) break;
        }
        if (!(flags & kEmpty)) {
            const uint8_t *const keys = smem + stage * 2 * L::kHalf, *const values = keys + L::kHalf;
            // ---- logits of 16 tokens (m) and eight rows at a time (n)
            constexpr int kChains = NT == 1 && D == 128 ? 2 : 1;     // sums side by side: an MMA waits for the one before it in its sum
            float parts[kChains][NT][4] = {}, (&s)[NT][4] = parts[0];
            uint32_t kw[2][kK];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int h = 0; h < D / 64; ++h) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(keys + chunk_at<D>(16 * warp + 8 * t + perm, c + 4 * h));
                    kw[t][4 * h] = w.x; kw[t][4 * h + 1] = w.y; kw[t][4 * h + 2] = w.z; kw[t][4 * h + 3] = w.w;
                }
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                uint32_t a[2][2];
#pragma unroll
                for (int t = 0; t < 2; ++t) to_f16x4(kw[t][k], a[t][0], a[t][1]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    uint2 b;
                    if constexpr (!kQueryShared) b = make_uint2(qf[nt][k][0], qf[nt][k][1]);
                    else b = query[(nt * kK + k) * 32 + lane];
                    mma_f16(parts[k % kChains][nt], a[0][0], a[1][0], a[0][1], a[1][1], b.x, b.y);
                }
            }
            if constexpr (kChains == 2) {
#pragma unroll
                for (int x = 0; x < 4; ++x) s[0][x] += parts[kChains - 1][0][x];
            }
            // ---- values of the tokens a, b, a + 8, b + 8
            uint32_t vw[4][D / 32];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = 16 * warp + tok[t];
                if constexpr (D == 128) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(values + chunk_at<D>(row, perm));
                    vw[t][0] = w.x; vw[t][1] = w.y; vw[t][2] = w.z; vw[t][3] = w.w;
                } else {
                    const uint2 w = *reinterpret_cast<const uint2 *>(values + chunk_at<D>(row, n >> 1) + (n & 1) * 8);
                    vw[t][0] = w.x; vw[t][1] = w.y;
                }
            }
            // ---- weights, in base 2 relative to the row's reference, and relative to the largest value scale so far
            // (an infinite scale counts as NaN: keys that are infinite, with either sign, have a logit that is no number)
            const float ks = number(__int_as_float(page.y)), vs = number(__int_as_float(page.z));
            if (fabsf(vs) > unit) {
                per_unit = __fdividef(1.f, fabsf(vs));
                const float a = unit * per_unit;
                if (!(flags & kCausal)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < kM; ++j)
#pragma unroll
                            for (int x = 0; x < 4; ++x) o[nt][j][x] *= a;
                } else {
                    // (a row that sees no token of the page, nor of a later one, is done: the page's scale may be anything to it)
                    const Done done = done_row(unit, fabsf(vs));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float b = a;
                            if (lim[nt][e] <= page.w) { b = done.o; l[nt][e] *= done.l; ref[nt][e] -= done.shift; }
#pragma unroll
                            for (int j = 0; j < kM; ++j) { o[nt][j][e] *= b; o[nt][j][2 + e] *= b; }
                        }
                }
                unit = fabsf(vs);
            }
            const float f = vs == unit ? 1.f : vs * per_unit;
            uint32_t hidden = 0;                     // logits of tokens that the row does not see, a bit each
            if (flags & kEdge) {
                const int base = page.w + 16 * warp, lo = info.lo, hi = info.hi;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int at = base + perm + 8 * (x >> 1);
                        if (at < lo || at >= lim[nt][x & 1]) hidden |= 1u << (4 * nt + x);
                    }
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (base + tok[t] < lo || base + tok[t] >= hi) {
#pragma unroll
                        for (int q = 0; q < D / 32; ++q) vw[t][q] = 0;
                    }
            }
            float y[NT][4], most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            auto relative = [&] {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) y[nt][x] = fmaf(s[nt][x], rs[nt][x & 1] * ks, -ref[nt][x & 1]);
                if (hidden != 0) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            if (hidden >> (4 * nt + x) & 1u) y[nt][x] = -INFINITY;
                }
            };
            relative();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int x = 0; x < 4; ++x) most[x] = fmaxf(most[x], y[nt][x]);
            if (__any_sync(0xffffffffu, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) > kLift + kSlack)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = -INFINITY;
#pragma unroll
                        for (int x = e; x < 4; x += 2)
                            if (!(hidden >> (4 * nt + x) & 1u)) top = fmaxf(top, s[nt][x] * (rs[nt][e] * ks));
#pragma unroll
                        for (int sh = 4; sh < 32; sh <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sh));
                        top -= kLift;
                        if (top > ref[nt][e]) {
                            const float a = fast_exp2(ref[nt][e] - top);
                            ref[nt][e] = top;
                            l[nt][e] *= a;
#pragma unroll
                            for (int j = 0; j < kM; ++j) { o[nt][j][e] *= a; o[nt][j][2 + e] *= a; }
                        }
                    }
                relative();
            }
            uint32_t pf[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float w[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) w[x] = fast_exp2(y[nt][x]);
                l[nt][0] += w[0] + w[2];
                l[nt][1] += w[1] + w[3];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    pf[nt][t] = pack_f16x2(w[2 * t] * f, w[2 * t + 1] * f);
                    if (!(f == f))                               // a scale that is NaN, for the rows that see the token
                        pf[nt][t] = (y[nt][2 * t] == -INFINITY ? 0u : 0x7fffu) | (y[nt][2 * t + 1] == -INFINITY ? 0u : 0x7fff0000u);
                    pf[nt][t] = transpose8x8(pf[nt][t]);         // tokens to k, rows to n
                }
            }
            // ---- a NaN value in a page where some rows do not see every token: products 0 * NaN must not reach the rows that do
            // not see it.  Values without NaN go on; rows that see one get it by counting (weights 1 and 0) instead.
            if (flags & kCausal) {
                uint32_t nan = 0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int q = 0; q < D / 32; ++q) nan |= ((vw[t][q] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
                if (__any_sync(0xffffffffu, nan != 0)) {
                    uint32_t sees[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            sees[nt][t] = transpose8x8((hidden >> (4 * nt + 2 * t) & 1u ? 0u : 0x3c00u) | (hidden >> (4 * nt + 2 * t + 1) & 1u ? 0u : 0x3c000000u));
#pragma unroll
                    for (int q = 0; q < D / 32; ++q) {
                        uint32_t nw[4];
#pragma unroll
                        for (int t = 0; t < 4; ++t) {
                            const uint32_t at = (((vw[t][q] & 0x7f7f7f7fu) + 0x01010101u) >> 7) & 0x01010101u;
                            nw[t] = at * 0x38u;                         // 1.0
                            vw[t][q] &= ~(at * 0xffu);
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const uint32_t sel = half ? 0x7362 : 0x5140;
                            uint32_t a0, a1, a2, a3;
                            to_f16x4(__byte_perm(nw[0], nw[1], sel), a0, a1);
                            to_f16x4(__byte_perm(nw[2], nw[3], sel), a2, a3);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                float count[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_f16(count, a0, a1, a2, a3, sees[nt][0], sees[nt][1]);
#pragma unroll
                                for (int x = 0; x < 4; ++x)
                                    if (count[x] > 0.f) o[nt][2 * q + half][x] = NAN;
                            }
                        }
                    }
                }
            }
            // ---- outputs: 16 dimensions (m), eight rows (n)
#pragma unroll
            for (int q = 0; q < D / 32; ++q)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t sel = half ? 0x7362 : 0x5140;
                    uint32_t a0, a1, a2, a3;
                    to_f16x4(__byte_perm(vw[0][q], vw[1][q], sel), a0, a1);
                    to_f16x4(__byte_perm(vw[2][q], vw[3][q], sel), a2, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][2 * q + half], a0, a1, a2, a3, pf[nt][0], pf[nt][1]);
                }
        }
        if (flags & (kLast | kEmpty)) {
            // ---- the four warps' parts of the item
            const int m0 = info.m0, pairs = info.pairs, row0 = info.row0, head = info.head, slot = info.slot;
            float *const stat_l = stat_m + kConsumers * L::kRows;
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * stage);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int sh = 4; sh < 32; sh <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], sh);
                    if (n == 0) {
                        stat_m[warp * L::kRows + nt * 8 + 2 * c + e] = ref[nt][e];
                        stat_l[warp * L::kRows + nt * 8 + 2 * c + e] = l[nt][e];
                    }
                }
            if (!meet(ctx, group_bar, group_phase, lane)) break;
            bool ok = true;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (m0 + nt * 8 >= pairs) break;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = nt * 8 + 2 * c + e;
                    float top = kUnset;
#pragma unroll
                    for (int w = 0; w < kConsumers; ++w) top = fmaxf(top, stat_m[w * L::kRows + r]);
                    const float a = fast_exp2(ref[nt][e] - top);
                    float *const to = merge + (warp * 8 + 2 * c + e) * L::kPad + (D == 128 ? perm * 16 : n * 8);
#pragma unroll
                    for (int j = 0; j < kM; j += 2)
                        *reinterpret_cast<float4 *>(to + 2 * j) =
                            make_float4(o[nt][j][e] * a, o[nt][j][2 + e] * a, o[nt][j + 1][e] * a, o[nt][j + 1][2 + e] * a);
                }
                if (!(ok = meet(ctx, group_bar, group_phase, lane))) break;
                const int tid = warp * 32 + lane, r8 = tid >> 4, r = nt * 8 + r8, mm = m0 + r;
                if (mm < pairs) {
                    float top = kUnset, sum = 0.f;
#pragma unroll
                    for (int w = 0; w < kConsumers; ++w) top = fmaxf(top, stat_m[w * L::kRows + r]);
#pragma unroll
                    for (int w = 0; w < kConsumers; ++w) sum += stat_l[w * L::kRows + r] * fast_exp2(stat_m[w * L::kRows + r] - top);
                    const float scale = sum == 0.f ? 0.f : unit / sum;
                    // (the sum's exponent goes to the reference, exactly: of its logarithm a mantissa's is left)
                    const int sum_bits = __float_as_int(sum);
                    const float mantissa = __int_as_float((sum_bits & 0x7fffff) | 0x3f800000);
                    const float lse2 = sum == 0.f ? -INFINITY : sum < INFINITY ? top + (float)((sum_bits >> 23) - 127) + __log2f(mantissa) : sum;
                    const int row = mm / p.group, g = head * p.group + mm - row * p.group;
#pragma unroll
                    for (int q = 0; q < D / 64; ++q) {
                        const int d = 4 * ((tid & 15) + 16 * q);
                        float4 v = *reinterpret_cast<const float4 *>(merge + r8 * L::kPad + d);
#pragma unroll
                        for (int w = 1; w < kConsumers; ++w) {
                            const float4 x = *reinterpret_cast<const float4 *>(merge + (w * 8 + r8) * L::kPad + d);
                            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
                        }
                        v.x *= scale; v.y *= scale; v.z *= scale; v.w *= scale;
                        if (slot < 0) store4(p, (row0 + row) * p.out_row + g * p.out_head + d, v);
                        else *reinterpret_cast<float4 *>(p.part_out + ((int64_t)slot * L::kRows + r) * D + d) = v;
                    }
                    if ((tid & 15) == 0) {
                        if (slot < 0) p.lse[(row0 + row) * p.lse_row + g] = lse2 * kLn2;
                        else p.part_lse[slot * L::kRows + r] = lse2;
                    }
                }
                if (nt + 1 < NT && m0 + nt * 8 + 8 < pairs && !(ok = meet(ctx, group_bar, group_phase, lane))) break;
            }
            if (!ok) break;
            stat_m = reinterpret_cast<float *>(smem + L::kStats) + (stat_m == reinterpret_cast<float *>(smem + L::kStats) ? 2 * kConsumers * L::kRows : 0);
        } else {
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * stage);
        }
        if (++stage == L::kStages) { stage = 0; phase ^= 1; }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, Layout<D, NT>::kCtas)
kv8_decode_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using L = Layout<D, NT>;
    extern __shared__ uint8_t raw[];
    __shared__ uint32_t abort_flag;
    uint8_t *const smem = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
    const uint32_t bars = smem_u32(smem + L::kBars);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, worker = blockIdx.x;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int s = 0; s < L::kStages; ++s) { mbar_init(bars + 8 * s, 1); mbar_init(bars + 8 * (L::kStages + s), kConsumers); }
        mbar_init(bars + 16 * L::kStages, kConsumers);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x < 4) p.status[threadIdx.x] = 0;
    const Share share = plan<L::kRows>(p, worker);      // (its barriers publish the mbarriers too)
    const Ctx ctx = {&abort_flag, p.status};
    if (warp == kConsumers) produce<D, NT>(p, share, &k_map, &v_map, smem, bars, ctx, worker, lane);
    else consume<D, NT>(p, smem, bars, ctx, warp, lane);
}

// Pieces of the cut items, [piece][row][D] with their base-2 lse: out = sum_j 2^(lse_j - lse) out_j.  The pieces of an item lie in the
// last slot of its first worker and the first slots of the following ones.  Block (worker, 4 / kWarps rows), kWarps warps to a row that share
// its pieces: one where there are items for all workers, so that most have a piece or two; four where a few items are spread over all of them (one
// context over all workers has 55 pieces for each of eight heads, which a warp alone walks through in 16 us).
// The next kernel on the stream is let in at the end and not at the start: blocks of the next call's decode kernel that come in
// beside these, three to an SM where there is room for fewer, cost that call more (64 contexts of 1k to 8k tokens: 127 us a call) than the launch that
// is hidden gives (106).
template <int D, int kRows, int kWarps>
__global__ void __launch_bounds__(128, 8)
kv8_combine_kernel(const __grid_constant__ AttnParams p) {
    constexpr int kPer = D / 32, kBatch = 8;
    __shared__ float sums[4], tops[4], parts[4][D];
    grid_dependency_wait();
    const int worker = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int4 cut = p.cut[2 * worker];           // pieces, first query row, (row, head) pairs, first pair of the tile
    const int head = p.cut[2 * worker + 1].x;
    const int pieces = cut.x, r = blockIdx.y * (4 / kWarps) + warp / kWarps, mm = cut.w + r;
    if (pieces == 0) return;
    const bool there = mm < cut.z;
    auto slot = [&](int j) { return j == 0 ? 2 * worker + 1 : 2 * (worker + j); };
    float top = kUnset, acc[kPer] = {}, sum = 0.f;
    if (there) {
        for (int j0 = warp % kWarps; j0 < pieces; j0 += kWarps * kBatch) {
            float w[kBatch], v[kBatch][kPer], most = kUnset;
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int j = j0 + kWarps * k;
                w[k] = -INFINITY;
                if (j < pieces) {
                    const int64_t at = (int64_t)slot(j) * kRows + r;
                    w[k] = p.part_lse[at];
                    if constexpr (kPer == 4) {
                        const float4 x = *reinterpret_cast<const float4 *>(p.part_out + at * D + lane * 4);
                        v[k][0] = x.x; v[k][1] = x.y; v[k][2] = x.z; v[k][3] = x.w;
                    } else {
                        const float2 x = *reinterpret_cast<const float2 *>(p.part_out + at * D + lane * 2);
                        v[k][0] = x.x; v[k][1] = x.y;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) most = fmaxf(most, w[k]);
            if (most > top) {
                const float a = fast_exp2(top - most);
                top = most;
                sum *= a;
#pragma unroll
                for (int x = 0; x < kPer; ++x) acc[x] *= a;
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (j0 + kWarps * k < pieces) {
                    w[k] = fast_exp2(w[k] - top);
                    sum += w[k];
#pragma unroll
                    for (int x = 0; x < kPer; ++x) acc[x] += w[k] * v[k][x];
                }
        }
    }
    if constexpr (kWarps > 1) {
        if (lane == 0) { sums[warp] = sum; tops[warp] = top; }
#pragma unroll
        for (int x = 0; x < kPer; ++x) parts[warp][lane * kPer + x] = acc[x];
        __syncthreads();
        if (warp % kWarps != 0) return;
        float most = top;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) most = fmaxf(most, tops[warp + w]);
        const float a = fast_exp2(top - most);
        sum *= a;
#pragma unroll
        for (int x = 0; x < kPer; ++x) acc[x] *= a;
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            const float b = fast_exp2(tops[warp + w] - most);
            sum += sums[warp + w] * b;
#pragma unroll
            for (int x = 0; x < kPer; ++x) acc[x] += parts[warp + w][lane * kPer + x] * b;
        }
        top = most;
    }
    if (!there) return;
    const float scale = sum == 0.f ? 0.f : 1.f / sum;
    const int row = mm / p.group, g = head * p.group + mm - row * p.group;
    const int64_t at = (int64_t)(cut.y + row) * p.out_row + g * p.out_head + lane * kPer;
    if constexpr (kPer == 4) {
        store4(p, at, make_float4(acc[0] * scale, acc[1] * scale, acc[2] * scale, acc[3] * scale));
    } else if (p.out_f32) {
        *reinterpret_cast<float2 *>(static_cast<float *>(p.out) + at) = make_float2(acc[0] * scale, acc[1] * scale);
    } else {
        *reinterpret_cast<uint32_t *>(static_cast<uint16_t *>(p.out) + at) =
            p.q_bf16 ? pack_bf16x2(acc[0] * scale, acc[1] * scale) : pack_f16x2(acc[0] * scale, acc[1] * scale);
    }
    if (lane == 0) p.lse[(int64_t)(cut.y + row) * p.lse_row + g] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

bool make_pool_map(CUtensorMap *map, const splash_kv8_cache &c, const void *pool, int64_t page_stride, int64_t head_stride) {
    EncodeTiledFn fn = encode_tiled();
    if (!fn) { set_error("cuTensorMapEncodeTiled is not available"); return false; }
    const uint64_t D = (uint64_t)c.head_dim;
    cuuint64_t dims[4] = {D, 64, (cuuint64_t)c.num_kv_heads, (cuuint64_t)c.num_pages};
    // (strides of dimensions of one element are the caller's own business)
    cuuint64_t strides[3] = {D, (cuuint64_t)(c.num_kv_heads > 1 ? head_stride : 64 * D), (cuuint64_t)(c.num_pages > 1 ? page_stride : 64 * D)};
    cuuint32_t box[4] = {(cuuint32_t)D, 64, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(pool), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) set_error("cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
    return r == CUDA_SUCCESS;
}

template <int D, int kRows, int kWarps>
cudaError_t launch_combine_of(const AttnParams &p, cudaStream_t stream) {
    static DeviceOnce once;
    cudaError_t e = once.run([] {
        // (an SM that had to change its shared memory between the two kernels would have to run empty first)
        return cudaFuncSetAttribute(kv8_combine_kernel<D, kRows, kWarps>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    });
    if (e != cudaSuccess) return e;
    e = launch_dependent(kv8_combine_kernel<D, kRows, kWarps>, dim3(p.workers, kRows * kWarps / 4), dim3(128), 0, stream, p);
    count_launch();
    return e;
}

// `items`: no more of them are cut
template <int D, int kRows>
cudaError_t launch_combine(const AttnParams &p, int items, cudaStream_t stream) {
    return p.workers / items >= 8 ? launch_combine_of<D, kRows, 4>(p, stream) : launch_combine_of<D, kRows, 1>(p, stream);
}

template <int D, int NT>
cudaError_t launch_decode(const AttnParams &p, int items, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream) {
    using L = Layout<D, NT>;
    static DeviceOnce once;
    cudaError_t e = once.run([] {
        return cudaFuncSetAttribute(kv8_decode_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
    });
    if (e != cudaSuccess) return e;
    e = launch_dependent(kv8_decode_kernel<D, NT>, dim3(p.workers), dim3(kThreads), L::kBytes, stream, p, k_map, v_map);
    count_launch();
    if (e != cudaSuccess || p.whole) return e;
    return launch_combine<D, L::kRows>(p, items, stream);
}

}  // namespace

// Rows of a tile for requests of at most `pairs` (row, head) pairs, and the workers that the line is cut for (the blocks that the GPU holds).  Three
// blocks an SM leave 128 registers, which only tiles of eight rows, and of 16 rows of 64 dimensions, keep to.  16 rows of 128 dimensions spill 116 bytes, 24 and 32 rows of 64
// dimensions 76 and 348; more than 16 of 128 dimensions cost more than the second tile (32: 47 us where two of 16 take 37), 24 rows of 64 dimensions as one
// tile as much as two of 16 (37 us), 32 rows 135 us as one tile and 146 as two.
void kv8_decode_shape(int64_t pairs, int head_dim, int sm_count, int *rows, int *workers) {
    const int64_t most = head_dim == 64 ? 32 : 16, tiles = (pairs + most - 1) / most;
    *rows = (int)((pairs + tiles - 1) / tiles + 7) / 8 * 8;
    *workers = 3 * sm_count;
}

bool kv8_pool_maps(const splash_kv8_cache &c, CUtensorMap *k_map, CUtensorMap *v_map) {
    return make_pool_map(k_map, c, c.k_pool, c.k_page_stride, c.k_head_stride) && make_pool_map(v_map, c, c.v_pool, c.v_page_stride, c.v_head_stride);
}

// of the kernel for many rows: a warp to a row, whatever is cut
cudaError_t launch_kv8_chunk_combine(const AttnParams &p, int D, cudaStream_t stream) {
    return D == 128 ? launch_combine_of<128, 128, 1>(p, stream) : launch_combine_of<64, 128, 1>(p, stream);
}

cudaError_t launch_kv8_decode(const AttnParams &p, int D, int rows, const CUtensorMap &k_map, const CUtensorMap &v_map, cudaStream_t stream) {
    const int64_t pairs = (int64_t)p.max_rows * p.group, tiles = ((pairs < p.max_pairs ? pairs : p.max_pairs) + rows - 1) / rows, all = tiles * p.kv_heads * p.B;
    const int items = (int)(all < 0x7fffffff ? all : 0x7fffffff);        // at most
    auto of = [&](auto d) {
        constexpr int kD = decltype(d)::value;
        if constexpr (kD == 64) {
            if (rows == 24) return launch_decode<kD, 3>(p, items, k_map, v_map, stream);
            if (rows == 32) return launch_decode<kD, 4>(p, items, k_map, v_map, stream);
        }
        return rows == 8 ? launch_decode<kD, 1>(p, items, k_map, v_map, stream) : launch_decode<kD, 2>(p, items, k_map, v_map, stream);
    };
    return D == 128 ? of(std::integral_constant<int, 128>{}) : of(std::integral_constant<int, 64>{});
}

}  // namespace splash
