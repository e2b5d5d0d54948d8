// The learned relative position bias as a tensor and the gradient of its table (definition in position.hpp).  Both are bound by
// memory: one writes heads * q_len * k_len values, the other reads batch times as many.
//
//   bias[h, i, j] = table[bucket(j - i - offset), h]
//   dtable[n, h]  = sum over b, i, j with bucket(j - i - offset) = n of dbias[b, h, i, j]
#include "position.hpp"

namespace egeria {

namespace {

constexpr int kRows = 8;            // rows of a thread's patch: kRows x 16 bytes, kRows + values - 1 distances

// LDS word of entry i of a table that the 64 lanes of a wave read 8 entries apart: one word of padding every 64 keeps them on
// different banks.
__device__ __forceinline__ int spread(int i) { return i + (i >> 6); }

template <typename T> struct Unit;
template <> struct Unit<float> {
    static constexpr int N = 4;
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Unit<uint16_t> {
    static constexpr int N = 8;
    typedef uint16_t vec __attribute__((ext_vector_type(8), aligned(2)));
};
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(uint16_t v) { return bf16_to_f32(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float v)
{
    return __builtin_bit_cast(uint16_t, (__bf16)v);
}

// Where a thread's patches lie: 2^lg units of 16 bytes side by side (32 to 256 of them, so that half a wave has one row of patches),
// 256 / 2^lg patches below each other: `rows` rows to a workgroup, and `cols` times these columns one after the other, so that what
// a workgroup writes or reads lies close together (long rows in pieces of 4 KiB, 64 of them below each other, were written at
// 4.9 TB/s; 8 whole rows of 8 KiB at 5.6).
struct Deal {
    int lg, rows, cols;
    uint32_t row_blocks, col_blocks, shares;
};

template <typename T>
__global__ __launch_bounds__(256) void position_bias_kernel(Buckets b, const float *__restrict__ table, int heads, int q_len, int k_len,
                                                            int offset, Deal deal, T *__restrict__ out)
{
    constexpr int N = Unit<T>::N;
    typedef typename Unit<T>::vec vec;
    extern __shared__ float lut[];
    const uint32_t p = xcd_piece(blockIdx.x, gridDim.x);
    const uint32_t cb = p % deal.col_blocks, rb = p / deal.col_blocks % deal.row_blocks, h = p / deal.col_blocks / deal.row_blocks;
    const int entries = b.both ? 2 * b.far + 1 : b.far + 1;
    const int rows = b.both ? 2 * b.n : b.n;
    Span *spans = (Span *)(lut + ((spread(entries) + 1) & ~1));
    float *value = (float *)(spans + rows);
    find_spans(b, rows, 0, spans);
    if ((int)threadIdx.x < rows) value[threadIdx.x] = table[threadIdx.x * heads + h];
    __syncthreads();
    each_entry(spans, rows, [&](int n, int e) { lut[spread(e)] = value[n]; });
    __syncthreads();
    const int i0 = (int)rb * deal.rows + (int)(threadIdx.x >> deal.lg) * kRows;
    const int last = (int)rb * deal.rows + deal.rows < q_len ? (int)rb * deal.rows + deal.rows : q_len;
    for (int c = 0; c < deal.cols; ++c) {
        const int j0 = (int)(((cb * deal.cols + c) << deal.lg) + (threadIdx.x & ((1 << deal.lg) - 1))) * N;
        if (j0 >= k_len) return;
        T v[kRows + N - 1];                                        // distances first, first + 1, ...
        const int first = j0 - (i0 + kRows - 1) - offset;
#pragma unroll
        for (int e = 0; e < kRows + N - 1; ++e) v[e] = narrow<T>(lut[spread(distance_index(b, first + e))]);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (i0 + r >= last) break;
            T *dst = out + ((int64_t)h * q_len + i0 + r) * k_len + j0;
            if (j0 + N <= k_len) {
                vec w;
#pragma unroll
                for (int e = 0; e < N; ++e) w[e] = v[kRows - 1 - r + e];
                *(vec *)dst = w;
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (j0 + e < k_len) dst[e] = v[kRows - 1 - r + e];
            }
        }
    }
}

// One workgroup: the same piece of the rows and columns, summed over its share of the batch.  A thread adds up its patch along the
// diagonals in registers, over the batch, then the diagonals' sums go to a table by distance of its half wave in LDS.  The lanes of
// half a wave add to different entries at each step and a wave's additions are in order: the result does not depend on timing.
// WHOLE: rows are whole units of 16 bytes.  Else a row's 16 bytes come from the two whole units that hold them: loads at other
// addresses cost 24 % where those are multiples of 4, and at odd multiples of 2 run at a fifth of the rate (13 x 22 x 1142 x 391 in bf16
// 199 us, now 51).
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void position_bias_backward_kernel(Buckets b, const T *__restrict__ dbias, int64_t batch, int heads,
                                                                     int q_len, int k_len, int offset, Deal deal, int rows_of_table,
                                                                     float *__restrict__ partials)
{
    constexpr int N = Unit<T>::N;
    extern __shared__ float sums[];                                // [8 half waves][entries]
    const uint32_t p = xcd_piece(blockIdx.x, gridDim.x);
    const uint32_t cb = p % deal.col_blocks, rb = p / deal.col_blocks % deal.row_blocks, sh = p / deal.col_blocks / deal.row_blocks % deal.shares;
    const uint32_t h = p / deal.col_blocks / deal.row_blocks / deal.shares;
    const int entries = b.both ? 2 * b.far + 1 : b.far + 1;
    Span *spans = (Span *)(sums + 8 * entries);
    find_spans(b, rows_of_table, 0, spans);
    for (int i = threadIdx.x; i < 8 * entries; i += 256) sums[i] = 0.0f;
    __syncthreads();
    float *mine = sums + (threadIdx.x >> 5) * entries;
    const int64_t b0 = batch * sh / deal.shares, b1 = batch * (sh + 1) / deal.shares;
    const int i0 = (int)rb * deal.rows + (int)(threadIdx.x >> deal.lg) * kRows;
    const int last = (int)rb * deal.rows + deal.rows < q_len ? (int)rb * deal.rows + deal.rows : q_len;
    const int64_t total = batch * heads * q_len * (int64_t)k_len;
    double left = 0.0, right = 0.0;                                // distances beyond the table: long sums, of values that may cancel
    const int hi = b.both ? b.far : 0;
    for (int c = 0; c < deal.cols; ++c) {
        const int j0 = (int)(((cb * deal.cols + c) << deal.lg) + (threadIdx.x & ((1 << deal.lg) - 1))) * N;
        float d[kRows + N - 1];
#pragma unroll
        for (int e = 0; e < kRows + N - 1; ++e) d[e] = 0.0f;
        if (j0 < k_len && i0 < last)
            for (int64_t n = b0; n < b1; ++n) {
                // row r of the workgroup's first patches as a buffer up to the tensor's end, from the unit that holds its beginning
                const int64_t row0 = ((n * heads + h) * q_len + (int)rb * deal.rows) * k_len;
                const int down = (i0 - (int)rb * deal.rows) * k_len + j0;        // (0 + j0, or a few short rows and j0)
                v4u lo[kRows], up[kRows];
                int s[kRows];
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const char *base = (const char *)(dbias + row0 + (int64_t)r * k_len);
                    const int off = WHOLE ? 0 : (int)((uintptr_t)base & 15u), at = off + down * (int)sizeof(T);
                    const int64_t left = ((const char *)(dbias + total) - base + off) & ~(int64_t)3;        // (below 0: a row behind the tensor)
                    const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base - off), 0,
                                                                                          left < 0 ? 0 : (left > 0x7fffffff ? 0x7fffffff : (int)left), kBufferWord);
                    s[r] = WHOLE ? 0 : at & 15;
                    const int unit = i0 + r < last ? at - s[r] : (int)0x80000000;
                    lo[r] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rows, unit, 0, 0));
                    if (!WHOLE) up[r] = __builtin_bit_cast(v4u, __builtin_amdgcn_raw_buffer_load_b128(rows, unit + 16, 0, 0));
                }
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    union { v4u u; T e[N]; } x;
                    x.u = WHOLE ? lo[r] : from_byte(lo[r], up[r], s[r]);
#pragma unroll
                    for (int e = 0; e < N; ++e) d[kRows - 1 - r + e] += j0 + e < k_len ? widen(x.e[e]) : 0.0f;
                }
                if (!WHOLE && sizeof(T) == 2 && (total & 1) && n == batch - 1 && (int)h == heads - 1 && last == q_len && j0 + N >= k_len) {
                    // the tensor's last value shares no whole word with another: it is beyond the buffer
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (i0 + r == q_len - 1 && j0 + e == k_len - 1) d[kRows - 1 - r + e] += widen(dbias[total - 1]);
                }
            }
        const int first = j0 - (i0 + kRows - 1) - offset;
        if (first >= hi || first + kRows + N - 2 <= -b.far) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < kRows + N - 1; ++e) s += (double)d[e];
            if (first >= hi) right += s;
            else left += s;
        } else {
#pragma unroll
            for (int e = 0; e < kRows + N - 1; ++e) {
                const int rel = first + e;
                // entries inside the table are different in every lane of the half; what lies beyond its ends is the lane's own sum
                if (rel <= -b.far) left += (double)d[e];
                else if (rel >= hi) right += (double)d[e];
                else mine[rel + b.far] += d[e];
                asm volatile("" ::: "memory");                  // the next entry is another lane's: no read of it before this write
            }
            wave_lds_turn();                                       // the next patch's lanes add where others of this one have
        }
    }
    left = wave_sum(left);
    right = wave_sum(right);
    wave_lds_turn();
    if ((threadIdx.x & 63) == 0) {
        mine[0] += (float)left;                                    // the ends of the table have the same buckets as what lies beyond
        mine[entries - 1] += (float)right;
    }
    const int64_t part = ((int64_t)sh * deal.row_blocks + rb) * deal.col_blocks + cb, parts = (int64_t)deal.shares * deal.row_blocks * deal.col_blocks;
    bucket_sums(spans, sums, 8, entries, entries, rows_of_table, partials + ((int64_t)h * parts + part) * rows_of_table);
}

constexpr int kReduceThreads = 1024;
__global__ __launch_bounds__(kReduceThreads) void table_reduce_kernel(const float *__restrict__ partials, int heads, int64_t parts, int buckets,
                                                           float *__restrict__ dtable)
{
    __shared__ double memory[kReduceThreads];
    reduce_table<kReduceThreads>(partials, heads, parts, buckets, dtable, blockIdx.x, memory);
}

// How rows, columns and, for the gradient, the batch are dealt to workgroups: one row of patches for each thread, up to four pieces of
// the columns where that leaves 2048 workgroups, and the batch in shares where rows and columns alone do not give 1024.
Deal make_deal(int64_t batch, int heads, int q_len, int k_len, int per_unit)
{
    Deal p;
    const int64_t units = ((int64_t)k_len + per_unit - 1) / per_unit;
    p.lg = 5;
    while (p.lg < 8 && (1 << p.lg) < units) ++p.lg;
    p.rows = kRows << (8 - p.lg);
    p.row_blocks = (uint32_t)(((int64_t)q_len + p.rows - 1) / p.rows);
    const int64_t pieces = (units + (1 << p.lg) - 1) >> p.lg, rows = (int64_t)p.row_blocks * heads;
    p.cols = 1;
    while (p.cols < 4 && p.cols < pieces && (pieces + p.cols) / (p.cols + 1) * rows >= 2048) ++p.cols;
    p.col_blocks = (uint32_t)((pieces + p.cols - 1) / p.cols);
    const int64_t blocks = p.col_blocks * rows;
    int64_t shares = blocks > 0 ? (1024 + blocks - 1) / blocks : 1;
    shares = shares > batch ? batch : shares;
    p.shares = (uint32_t)(shares < 1 ? 1 : shares);
    return p;
}

bool valid_sizes(const egeria_position_table *t, int32_t heads, int32_t q_len, int32_t k_len, int32_t offset, egeria_dtype dt)
{
    if (!t || !valid_position_table(t) || heads < 1 || heads > 65535 || q_len < 0 || k_len < 0) return false;
    if (dt != EGERIA_F32 && dt != EGERIA_BF16) return false;
    return offset >= -(1 << 29) && offset <= (1 << 29) && q_len <= (1 << 28) && k_len <= (1 << 28);
}

int64_t parts_of(const Deal &p) { return (int64_t)p.shares * p.row_blocks * p.col_blocks; }

}  // namespace

hipError_t launch_table_reduce(const float *partials, int heads, int64_t parts, int buckets, float *dtable, hipStream_t st)
{
    return launch_k(EGERIA_KERNEL_NONE, table_reduce_kernel, dim3((unsigned)heads), dim3(kReduceThreads), 0, st, partials, heads, parts, buckets, dtable);
}

}  // namespace egeria

using namespace egeria;

extern "C" {

egeria_status egeria_position_bias(const egeria_position_table *t, int32_t heads, int32_t q_len, int32_t k_len, int32_t offset,
                                   void *bias, egeria_dtype dt, void *stream)
{
    if (!valid_sizes(t, heads, q_len, k_len, offset, dt)) return EGERIA_ERR_INVALID_ARG;
    if (q_len == 0 || k_len == 0) return EGERIA_OK;
    if (!bias || ((uintptr_t)bias & 15u)) return EGERIA_ERR_INVALID_ARG;
    const Buckets b = make_buckets(t);
    const Deal p = make_deal(1, heads, q_len, k_len, dt == EGERIA_F32 ? 4 : 8);
    const int64_t blocks = (int64_t)p.row_blocks * p.col_blocks * heads;
    if (blocks * 256 > kMostThreads) return EGERIA_ERR_UNSUPPORTED;
    const int entries = distance_entries(b);
    const size_t lds = 4 * (size_t)(entries + entries / 64 + 2) + t->buckets * (sizeof(Span) + 4);
    auto go = [&](auto kernel, auto *out) {
        return launch_k(EGERIA_KERNEL_NONE, kernel, dim3((unsigned)blocks), dim3(256), lds, (hipStream_t)stream, b, t->table, (int)heads,
                        (int)q_len, (int)k_len, (int)offset, p, out);
    };
    const hipError_t e = dt == EGERIA_F32 ? go(position_bias_kernel<float>, (float *)bias) : go(position_bias_kernel<uint16_t>, (uint16_t *)bias);
    return e == hipSuccess ? EGERIA_OK : EGERIA_ERR_HIP;
}

size_t egeria_position_bias_workspace_bytes(const egeria_position_table *t, int32_t batch, int32_t heads, int32_t q_len, int32_t k_len,
                                            egeria_dtype dt)
{
    if (!valid_sizes(t, heads, q_len, k_len, 0, dt) || batch < 0) return 0;
    const Deal p = make_deal(batch, heads, q_len, k_len, dt == EGERIA_F32 ? 4 : 8);
    return align_up((size_t)parts_of(p) * heads * t->buckets * 4, 256) + 256;
}

egeria_status egeria_position_bias_backward(const egeria_position_table *t, const void *dbias, egeria_dtype dt, int32_t batch, int32_t heads,
                                            int32_t q_len, int32_t k_len, int32_t offset, float *dtable, void *ws, size_t ws_bytes,
                                            void *stream)
{
    if (!valid_sizes(t, heads, q_len, k_len, offset, dt) || batch < 0 || !dtable || ((uintptr_t)dtable & 15u)) return EGERIA_ERR_INVALID_ARG;
    const bool none = batch == 0 || q_len == 0 || k_len == 0;
    if (!none && (!dbias || ((uintptr_t)dbias & 15u))) return EGERIA_ERR_INVALID_ARG;
    if (!ws || ((uintptr_t)ws & 15u)) return EGERIA_ERR_INVALID_ARG;
    if (ws_bytes < egeria_position_bias_workspace_bytes(t, batch, heads, q_len, k_len, dt)) return EGERIA_ERR_WORKSPACE_TOO_SMALL;
    hipStream_t st = (hipStream_t)stream;
    float *partials = (float *)ws;
    if (none) return launch_table_reduce(partials, heads, 0, t->buckets, dtable, st) == hipSuccess ? EGERIA_OK : EGERIA_ERR_HIP;
    const Buckets b = make_buckets(t);
    const Deal p = make_deal(batch, heads, q_len, k_len, dt == EGERIA_F32 ? 4 : 8);
    const int64_t blocks = parts_of(p) * heads;
    if (blocks * 256 > kMostThreads) return EGERIA_ERR_UNSUPPORTED;
    const size_t lds = 32 * (size_t)distance_entries(b) + t->buckets * sizeof(Span);
    auto go = [&](auto kernel, auto *src) {
        return launch_k(EGERIA_KERNEL_NONE, kernel, dim3((unsigned)blocks), dim3(256), lds, st, b, src, (int64_t)batch, (int)heads, (int)q_len,
                        (int)k_len, (int)offset, p, (int)t->buckets, partials);
    };
    const bool whole = k_len % (dt == EGERIA_F32 ? 4 : 8) == 0;
    hipError_t e;
    if (dt == EGERIA_F32) e = whole ? go(position_bias_backward_kernel<float, true>, (const float *)dbias) : go(position_bias_backward_kernel<float, false>, (const float *)dbias);
    else e = whole ? go(position_bias_backward_kernel<uint16_t, true>, (const uint16_t *)dbias) : go(position_bias_backward_kernel<uint16_t, false>, (const uint16_t *)dbias);
    if (e == hipSuccess) e = launch_table_reduce(partials, heads, parts_of(p), t->buckets, dtable, st);
    return e == hipSuccess ? EGERIA_OK : EGERIA_ERR_HIP;
}

}  // extern "C"
