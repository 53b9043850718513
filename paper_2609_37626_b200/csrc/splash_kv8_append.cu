// Keys and values of new tokens into the paged e4m3 cache, a power-of-two scale per (page, head).
//
//   a = max |x| over a run (the new rows of one page) of a head;  need = min { 2^e : a <= 448 * 2^e }
//   s' = need for a page that begins here, max(s, need) for one begun earlier;  code = e4m3(x / s')
//   and older codes of a page whose scale moves: c' = e4m3(c * s / s')
//
// Division by a power of two is a product with its reciprocal, exact, so that a code is rounded once; an older code that moves
// is rounded again only where it falls below the normal range.  Bytes bound it: two read and one written per value (four prompts of 8,192 tokens, eight heads of
// 128: 201 MB).  A block takes the runs that BEGIN in its window of tokens, for one head of keys or of values, and follows the last
// one past the window's end, so that each row is read once, stays in registers between the maximum and the codes, and no
// block waits for another.
#include "splash_kv8.cuh"

namespace splash {

namespace {

using namespace kv8;

constexpr int kAppendThreads = 256;
constexpr int kTokens = 128;          // a window of up to 64 tokens and what its last run may have behind it

struct AppendParams {
    const uint16_t *x[2];
    uint8_t *pool[2];
    float *scales[2];
    int64_t row_stride[2], head_stride[2], page_stride[2], pool_head_stride[2], scale_stride[2];
    const int64_t *slot_map;
    int64_t rows;
    int32_t num_pages, window;
};

// smallest 2^e with a <= 448 * 2^e = 1.75 * 2^(e + 8); a is finite and not negative
__device__ __forceinline__ float scale_for(float a) {
    const int bits = __float_as_int(a);
    const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return __int_as_float((max(e, kMinExp) + 127) << 23);
}

template <bool kBf16>
__device__ __forceinline__ float widen(uint32_t h) {
    if constexpr (kBf16) return __uint_as_float(h << 16);
    else return __half2float(__ushort_as_half((unsigned short)h));
}

// x / s: the reciprocal of a power of two is exact
__device__ __forceinline__ float over(float x, float s, float inv, bool exact) { return exact ? x * inv : __fdiv_rn(x, s); }
// (positive, and with a reciprocal that is a normal number)
__device__ __forceinline__ bool power_of_two(float s) { const int e = __float_as_int(s) >> 23; return (__float_as_int(s) & 0x7fffff) == 0 && e >= 1 && e <= 253; }
__device__ __forceinline__ float reciprocal(float power) { return __int_as_float((254 << 23) - __float_as_int(power)); }

template <int D, bool kBf16>
__global__ void __launch_bounds__(kAppendThreads)
kv8_append_kernel(const AppendParams p) {
    constexpr int kLanes = D / 8;                         // 16 bytes of a row each
    constexpr int kRowsAtOnce = kAppendThreads / kLanes;
    constexpr int kSteps = kTokens / kRowsAtOnce;
    constexpr uint32_t kInf = kBf16 ? 0x7f80 : 0x7c00;    // 16-bit pattern: at or above it, a value is not finite
    __shared__ uint32_t starts[kTokens / 32], breaks[kTokens / 32];
    __shared__ int32_t page_of[kTokens];                  // page of the token's row, or -1: not this block's
    __shared__ int8_t offset_of[kTokens], run_of[kTokens];
    __shared__ int32_t most[64];                          // per run: 16-bit pattern of the largest finite |x|
    __shared__ float scale[64], old_scale[64];
    __shared__ int32_t moved_page[64];
    __shared__ int8_t moved_rows[64], moved_run[64];
    __shared__ int num_moved;

    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int head = blockIdx.y, which = blockIdx.z;
    const int64_t first = (int64_t)blockIdx.x * p.window;
    float *const scales = p.scales[which] + head;
    uint8_t *const pool = p.pool[which] + head * p.pool_head_stride[which];

    if (tid == 0) num_moved = 0;
    if (tid < 64) most[tid] = 0;
    int64_t slot = -1;
    bool begins = false;
    float before = 0.f;
    if (tid < kTokens) {
        const int64_t t = first + tid;
        bool valid = false;
        if (t < p.rows) {
            slot = p.slot_map[t];
            valid = slot >= 0 && slot / kPage < p.num_pages;
            begins = valid && (slot % kPage == 0 || t == 0 || p.slot_map[t - 1] != slot - 1);
        }
        const uint32_t s = __ballot_sync(0xffffffffu, begins), b = __ballot_sync(0xffffffffu, begins || !valid);
        if (lane == 0) { starts[warp] = s; breaks[warp] = b; }
        if (begins && tid < p.window && slot % kPage != 0) before = scales[slot / kPage * p.scale_stride[which]];     // (used behind the maxima)
    }
    __syncthreads();
    if (tid < kTokens) {
        // the run's first token: the last break at or before this one
        int at = -1, run = 0;
#pragma unroll
        for (int w = 0; w < kTokens / 32; ++w) {
            const uint32_t upto = w < warp ? 0xffffffffu : w == warp ? 0xffffffffu >> (31 - lane) : 0u;
            if (breaks[w] & upto) at = w * 32 + 31 - __clz(breaks[w] & upto);
        }
        bool mine = at >= 0 && at < p.window && (starts[at >> 5] >> (at & 31) & 1u);
        if (mine) {
            for (int w = 0; w < (at >> 5); ++w) run += __popc(starts[w]);
            run += __popc(starts[at >> 5] & ((1u << (at & 31)) - 1u));
        }
        page_of[tid] = mine ? (int32_t)(slot / kPage) : -1;
        offset_of[tid] = (int8_t)(slot % kPage);
        run_of[tid] = (int8_t)run;
    }
    __syncthreads();

    const int row = tid / kLanes, col = tid % kLanes;
    const uint16_t *const x = p.x[which] + head * p.head_stride[which] + col * 8;
    uint4 data[kSteps];
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int j = row + k * kRowsAtOnce;
        if (page_of[j] >= 0) data[k] = *reinterpret_cast<const uint4 *>(x + (first + j) * p.row_stride[which]);
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int j = row + k * kRowsAtOnce;
        uint32_t a = 0;
        if (page_of[j] >= 0) {
            const uint32_t w[4] = {data[k].x, data[k].y, data[k].z, data[k].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = w[i] & 0x7fff, hi = w[i] >> 16 & 0x7fff;
                if (lo < kInf) a = max(a, lo);
                if (hi < kInf) a = max(a, hi);
            }
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
        if (col == 0 && page_of[j] >= 0) atomicMax(&most[run_of[j]], (int)a);      // a maximum: the order does not matter
    }
    __syncthreads();
    if (begins && tid < p.window) {
        const int run = run_of[tid], r0 = offset_of[tid];
        const float need = scale_for(widen<kBf16>(most[run]));
        const bool moves = r0 == 0 || !(before >= need);
        scale[run] = moves ? need : before;
        old_scale[run] = before;
        if (moves) scales[(int64_t)page_of[tid] * p.scale_stride[which]] = need;
        if (moves && r0 > 0) {
            const int k = atomicAdd(&num_moved, 1);       // (the order of the list does not change what is written)
            moved_page[k] = page_of[tid]; moved_rows[k] = (int8_t)r0; moved_run[k] = (int8_t)run;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int j = row + k * kRowsAtOnce;
        if (page_of[j] < 0) continue;
        const float s = scale[run_of[j]];
        const bool exact = power_of_two(s);
        const float unit = exact ? reciprocal(s) : 0.f;
        const uint32_t w[4] = {data[k].x, data[k].y, data[k].z, data[k].w};
        uint32_t code[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t lo = w[i] & 0xffff, hi = w[i] >> 16;
            if ((lo & 0x7fff) >= kInf) lo = 0x7fff;       // infinities are stored as NaN
            if ((hi & 0x7fff) >= kInf) hi = 0x7fff;
            code[i] = to_e4m3x2(over(widen<kBf16>(lo), s, unit, exact), over(widen<kBf16>(hi), s, unit, exact));
        }
        *reinterpret_cast<uint2 *>(pool + page_of[j] * p.page_stride[which] + offset_of[j] * D + col * 8) =
            make_uint2(code[0] | code[1] << 16, code[2] | code[3] << 16);
    }
    // older rows of pages whose scale has moved: a warp each
    for (int m = warp; m < num_moved; m += kAppendThreads / 32) {
        const float from = old_scale[moved_run[m]], s = scale[moved_run[m]];
        const float unit = reciprocal(s);                 // s is a new scale: a power of two
        uint4 *const at = reinterpret_cast<uint4 *>(pool + moved_page[m] * p.page_stride[which]);
        const int n = moved_rows[m] * (D / 16);
        for (int i = lane; i < n; i += 32) {
            const uint4 c = at[i];
            uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t out = 0, h2[2];
                to_f16x4(w[q], h2[0], h2[1]);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&h2[half]));
                    out |= to_e4m3x2(v.x * from * unit, v.y * from * unit) << (16 * half);
                }
                w[q] = out;
            }
            at[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

}  // namespace

cudaError_t launch_kv8_append(const splash_kv8_cache &cache, int32_t dtype, int64_t rows, const void *k, int64_t k_row, int64_t k_head, const void *v,
                              int64_t v_row, int64_t v_head, const int64_t *slot_map, int sm_count, cudaStream_t stream) {
    AppendParams p;
    p.x[0] = static_cast<const uint16_t *>(k); p.x[1] = static_cast<const uint16_t *>(v);
    p.pool[0] = static_cast<uint8_t *>(cache.k_pool); p.pool[1] = static_cast<uint8_t *>(cache.v_pool);
    p.scales[0] = cache.k_scales; p.scales[1] = cache.v_scales;
    p.row_stride[0] = k_row; p.row_stride[1] = v_row; p.head_stride[0] = k_head; p.head_stride[1] = v_head;
    p.page_stride[0] = cache.k_page_stride; p.page_stride[1] = cache.v_page_stride;
    p.pool_head_stride[0] = cache.k_head_stride; p.pool_head_stride[1] = cache.v_head_stride;
    p.scale_stride[0] = cache.k_scale_stride; p.scale_stride[1] = cache.v_scale_stride;
    p.slot_map = slot_map; p.rows = rows; p.num_pages = cache.num_pages;
    // a decode step has a run per row: small windows until there are blocks for every SM a few times over
    p.window = 8;
    while (p.window < 64 && (rows + p.window - 1) / p.window * cache.num_kv_heads * 2 > 16 * sm_count) p.window *= 2;
    const int64_t blocks = (rows + p.window - 1) / p.window;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)blocks, (unsigned)cache.num_kv_heads, 2);
    auto launch = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kAppendThreads), 0, stream, p); };
    const bool bf16 = dtype == SPLASH_DTYPE_BF16;
    const cudaError_t e = cache.head_dim == 128 ? (bf16 ? launch(kv8_append_kernel<128, true>) : launch(kv8_append_kernel<128, false>))
                                                : (bf16 ? launch(kv8_append_kernel<64, true>) : launch(kv8_append_kernel<64, false>));
    count_launch();
    return e;
}

}  // namespace splash
