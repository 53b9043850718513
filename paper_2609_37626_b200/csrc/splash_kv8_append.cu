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
    int32_t num_pages, window, heads;
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

// Division by a power of two is a product with its reciprocal, and exact.
// (positive, and with a reciprocal that is a normal number)
__device__ __forceinline__ bool power_of_two(float s) { const int e = __float_as_int(s) >> 23; return (__float_as_int(s) & 0x7fffff) == 0 && e >= 1 && e <= 253; }
__device__ __forceinline__ float reciprocal(float power) { return __int_as_float((254 << 23) - __float_as_int(power)); }

template <bool kBf16>
__device__ __forceinline__ float2 widen2(uint32_t w) {
    if constexpr (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2 *>(&w));
}

// Codes of eight values over a scale that is no power of two.
template <bool kBf16>
__device__ __noinline__ uint2 divided(uint4 x, float s) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t c[4];
    for (int i = 0; i < 4; ++i) {
        const float2 f = widen2<kBf16>(w[i]);
        c[i] = to_e4m3x2(__fdiv_rn(f.x, s), __fdiv_rn(f.y, s));
    }
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
}

// infinities are stored as NaN
__device__ __forceinline__ void not_finite_to_nan(uint32_t (&w)[4], uint32_t inf) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7fff) >= inf) w[i] |= 0x7fff;
        if ((w[i] >> 16 & 0x7fff) >= inf) w[i] |= 0x7fff0000u;
    }
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <int D, bool kBf16>
__global__ void __launch_bounds__(kAppendThreads, 4)
kv8_append_kernel(const AppendParams p) {
    constexpr int kLanes = D / 8;                         // 16 bytes of a row each
    constexpr int kRowsAtOnce = kAppendThreads / kLanes;
    constexpr int kSteps = 64 / kRowsAtOnce;              // of a window
    constexpr uint32_t kInf = kBf16 ? 0x7f80 : 0x7c00;    // 16-bit pattern: at or above it, a value is not finite
    __shared__ uint32_t starts[kTokens / 32], breaks[kTokens / 32];
    __shared__ int64_t place_of[kTokens];                 // where in a head's pages the token's row goes, in bytes, or -1: it is not this block's
    __shared__ int8_t run_of[kTokens];
    __shared__ int last_ends;                             // the window's last run ends with it
    // of one head, in two sets by turns: a warp may have begun the next head while another still writes this one's codes
    __shared__ int32_t most[2][64];                       // per run: 16-bit pattern of the largest finite |x|
    __shared__ float2 scale[2][64];                       // the scale, and its reciprocal or 0 if that is not exact
    __shared__ float old_scale[2][64];
    __shared__ int32_t moved_page[2][64];
    __shared__ int8_t moved_rows[2][64], moved_run[2][64];
    __shared__ int num_moved[2], odd[2];                  // odd: something among the rows is not finite

    grid_dependency_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int which = blockIdx.z;
    const int64_t first = (int64_t)blockIdx.x * p.window;
    const int row = tid / kLanes, col = tid % kLanes;

    if (tid < 2) { num_moved[tid] = 0; odd[tid] = 0; }
    if (tid < 128) most[tid >> 6][tid & 63] = 0;
    // The window's rows are fetched while its slots still are (most of them turn out to be this block's), and those of the next head while
    // one is worked on.
    uint4 data[kSteps];
    const int64_t row_stride = p.row_stride[which], head_stride = p.head_stride[which];
    const uint16_t *const x0 = p.x[which] + (first + row) * row_stride + col * 8;
    const int rows = (int)min((int64_t)p.window, p.rows - first);
    auto fetch = [&](int head) {
        const uint16_t *x = x0 + head * head_stride;
#pragma unroll
        for (int k = 0; k < kSteps; ++k, x += kRowsAtOnce * row_stride)
            if (row + k * kRowsAtOnce < rows) data[k] = *reinterpret_cast<const uint4 *>(x);
    };
    fetch(blockIdx.y);
    int64_t slot = -1;
    bool begins = false;
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
        begins = begins && tid < p.window;                // (those behind it are another block's)
    }
    const int32_t page = (int32_t)(slot / kPage), offset = (int32_t)(slot & (kPage - 1));      // (of a valid slot)
    const float *const old_at = p.scales[which] + page * p.scale_stride[which];
    float before = 0.f;                                   // the scale of a page that was begun earlier
    if (begins && offset != 0) before = old_at[blockIdx.y];
    __syncthreads();
    int run = 0;
    if (tid < kTokens) {
        // the run's first token: the last break at or before this one
        int at = -1;
#pragma unroll
        for (int w = 0; w < kTokens / 32; ++w) {
            const uint32_t upto = w < warp ? 0xffffffffu : w == warp ? 0xffffffffu >> (31 - lane) : 0u;
            if (breaks[w] & upto) at = w * 32 + 31 - __clz(breaks[w] & upto);
        }
        const bool mine = at >= 0 && at < p.window && (starts[at >> 5] >> (at & 31) & 1u);
        if (mine) {
            for (int w = 0; w < (at >> 5); ++w) run += __popc(starts[w]);
            run += __popc(starts[at >> 5] & ((1u << (at & 31)) - 1u));
        }
        if (tid == p.window) last_ends = !mine;           // (tokens behind the window are of its last run until that ends)
        place_of[tid] = mine ? page * p.page_stride[which] + offset * D : -1;
        run_of[tid] = (int8_t)run;
    }
    __syncthreads();

    int turn = 0;
    for (int head = blockIdx.y; head < p.heads; head += gridDim.y, turn ^= 1) {
        uint8_t *const pool = p.pool[which] + head * p.pool_head_stride[which];
        // Rows behind the window, of its last run: they are read again for their codes.
        auto behind = [&](auto &&with) {
            const uint16_t *x = x0 + p.window * row_stride + head * head_stride;
            for (int j = p.window + row; j < kTokens && !last_ends; j += kRowsAtOnce, x += kRowsAtOnce * row_stride) {
                const int64_t place = place_of[j];
                if (!__any_sync(0xffffffffu, place >= 0)) break;
                uint4 d = make_uint4(0, 0, 0, 0);
                if (place >= 0) d = *reinterpret_cast<const uint4 *>(x);
                with(j, d, place);
            }
        };
        // 16-bit patterns of values without their signs order like the values: two are compared at a time
        auto largest = [&](int j, const uint4 &d, int64_t place) {
            const bool mine = place >= 0;
            const uint32_t w[4] = {d.x & 0x7fff7fffu, d.y & 0x7fff7fffu, d.z & 0x7fff7fffu, d.w & 0x7fff7fffu};
            const uint32_t both = mine ? max_u16x2(max_u16x2(w[0], w[1]), max_u16x2(w[2], w[3])) : 0u;
            uint32_t a = max(both & 0xffff, both >> 16);
            if (a >= kInf) {                              // (a row with something that is not finite: without it)
                odd[turn] = 1;
                a = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if ((w[i] & 0xffff) < kInf) a = max(a, w[i] & 0xffff);
                    if (w[i] >> 16 < kInf) a = max(a, w[i] >> 16);
                }
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
            if (col == 0 && mine) atomicMax(&most[turn][run_of[j]], (int)a);      // a maximum: the order does not matter
        };
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int j = row + k * kRowsAtOnce;
            largest(j, data[k], j < p.window ? place_of[j] : -1);
        }
        behind(largest);
        __syncthreads();
        if (tid == 0) { num_moved[turn ^ 1] = 0; odd[turn ^ 1] = 0; }      // (everybody is done with the head before)
        if (begins) {
            const int r0 = offset;
            const float need = scale_for(widen<kBf16>(most[turn][run]));
            most[turn][run] = 0;
            const bool moves = r0 == 0 || !(before >= need);
            const float s = moves ? need : before;
            scale[turn][run] = make_float2(s, power_of_two(s) ? reciprocal(s) : 0.f);
            old_scale[turn][run] = before;
            if (moves) p.scales[which][page * p.scale_stride[which] + head] = need;
            if (moves && r0 > 0) {
                const int k = atomicAdd(&num_moved[turn], 1);       // (the order of the list does not change what is written)
                moved_page[turn][k] = page; moved_rows[turn][k] = (int8_t)r0; moved_run[turn][k] = (int8_t)run;
            }
            if (r0 > 0 && head + (int)gridDim.y < p.heads) before = old_at[head + gridDim.y];
        }
        uint4 now[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) now[k] = data[k];
        if (head + (int)gridDim.y < p.heads) fetch(head + gridDim.y);
        __syncthreads();
        const bool some_odd = odd[turn] != 0;
        auto write = [&](int j, const uint4 &d, int64_t place) {
            if (place < 0) return;
            const float2 s = scale[turn][run_of[j]];
            uint32_t w[4] = {d.x, d.y, d.z, d.w};
            if (some_odd) not_finite_to_nan(w, kInf);
            uint2 code;
            if (s.y != 0.f) {
                uint32_t c[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = widen2<kBf16>(w[i]);
                    c[i] = to_e4m3x2(f.x * s.y, f.y * s.y);
                }
                code = make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
            } else {
                code = divided<kBf16>(make_uint4(w[0], w[1], w[2], w[3]), s.x);
            }
            *reinterpret_cast<uint2 *>(pool + place + col * 8) = code;
        };
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int j = row + k * kRowsAtOnce;
            write(j, now[k], j < p.window ? place_of[j] : -1);
        }
        behind(write);
        // older rows of pages whose scale has moved: a warp each
        for (int m = warp; m < num_moved[turn]; m += kAppendThreads / 32) {
            const float from = old_scale[turn][moved_run[turn][m]], unit = scale[turn][moved_run[turn][m]].y;      // (a new scale: a power of two)
            uint4 *const at = reinterpret_cast<uint4 *>(pool + moved_page[turn][m] * p.page_stride[which]);
            const int n = moved_rows[turn][m] * (D / 16);
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
    p.slot_map = slot_map; p.rows = rows; p.num_pages = cache.num_pages; p.heads = cache.num_kv_heads;
    // A window of 64 tokens is a page where a prompt is written (smaller ones read a run's rows behind the window twice: 33 MB of prompts
    // take 53 us, with windows of 32 107; 3,000 rows of ragged chunks 5.3 and 6.5).  In a decode step every row is a run, and more blocks are sooner done
    // (64 rows 3.6 us with windows of 16, 4.2).  Once there are eight blocks for every SM, a block takes more heads of its window one after the other,
    // which saves it the window's slots (those prompts: 53 us, a block per head 66).
    p.window = rows <= 512 ? 16 : 64;
    const int64_t blocks = (rows + p.window - 1) / p.window;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    int groups = cache.num_kv_heads;
    while (groups > 1 && blocks * ((groups + 1) / 2) * 2 >= 8 * sm_count) groups = (groups + 1) / 2;
    const dim3 grid((unsigned)blocks, (unsigned)groups, 2);
    auto launch = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kAppendThreads), 0, stream, p); };
    const bool bf16 = dtype == SPLASH_DTYPE_BF16;
    const cudaError_t e = cache.head_dim == 128 ? (bf16 ? launch(kv8_append_kernel<128, true>) : launch(kv8_append_kernel<128, false>))
                                                : (bf16 ? launch(kv8_append_kernel<64, true>) : launch(kv8_append_kernel<64, false>));
    count_launch();
    return e;
}

}  // namespace splash
