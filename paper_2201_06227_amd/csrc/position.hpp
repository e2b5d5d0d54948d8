// The learned relative position bias: buckets of the distance between a key and a query, shared by the attention kernels and
// by the kernels that make the bias and its gradient as tensors.
//
// A side has n buckets (half of them where both sides have their own).  With e = n / 2 and m = n - e, a distance below e has a
// bucket to itself; bucket e + k holds the distances from e (M / e)^(k/m) on, up to the next border, and the last one all that
// follow.  So a bucket is an interval of distances, and from the last border on (`far`, below the limit M) every distance has the
// same one: a table of the distances -far ... far holds the whole function.
#pragma once
#include "common.hpp"
#include <math.h>

namespace egeria {

constexpr int kMaxBuckets = 128;            // rows of a position table
constexpr int kMaxDistance = 1024;          // largest max_distance: the tables by distance have to fit LDS
constexpr int64_t kMostThreads = 0xffffffffLL;          // of a launch

struct Buckets {
    int32_t n;                              // buckets of one side
    int32_t e;                              // distances below e have buckets of their own
    int32_t both;                           // the two sides have buckets of their own
    int32_t far;                            // first distance of the last bucket
    int16_t border[kMaxBuckets];            // first distance of bucket e + k (launch arguments are copied: as short as they can be)
};

inline int position_rows(const egeria_position_table *t) { return t ? t->buckets : 0; }

inline bool valid_position_table(const egeria_position_table *t)
{
    if (t->buckets < (t->bidirectional ? 4 : 2) || t->buckets > kMaxBuckets || (t->bidirectional && (t->buckets & 1))) return false;
    const int n = t->bidirectional ? t->buckets / 2 : t->buckets;
    return t->max_distance > n / 2 && t->max_distance <= kMaxDistance && t->table && !((uintptr_t)t->table & 15u);
}

// Borders in fp64; one that is within 1e-12 of a whole number is that number (they are whole where the power is, and pow() may
// miss it by a rounding).
inline Buckets make_buckets(const egeria_position_table *t)
{
    Buckets b;
    b.both = t->bidirectional ? 1 : 0;
    b.n = b.both ? t->buckets / 2 : t->buckets;
    b.e = b.n / 2;
    const int m = b.n - b.e;
    for (int k = 0; k < kMaxBuckets; ++k) b.border[k] = 0x7fff;
    for (int k = 0; k < m; ++k) {
        const double x = (double)b.e * pow((double)t->max_distance / b.e, (double)k / m), near = rint(x);
        b.border[k] = (int16_t)(fabs(x - near) <= 1e-12 * x ? near : ceil(x));
    }
    b.far = b.border[m - 1];
    return b;
}

// Entries of the table by distance: index clamp(distance, -far, hi) + far with hi = far or, one-sided, 0.
inline int distance_entries(const Buckets &b) { return b.both ? 2 * b.far + 1 : b.far + 1; }

#ifdef __HIPCC__
// The 16 bytes from byte s of two units of 16 (s even; words chosen one by one, since a chosen index would send them through memory).
__device__ __forceinline__ v4u from_byte(v4u a, v4u b, int s)
{
    const bool two = s & 8, one = s & 4, half = s & 2;
    const uint32_t x0 = two ? a[2] : a[0], x1 = two ? a[3] : a[1], x2 = two ? b[0] : a[2], x3 = two ? b[1] : a[3], x4 = two ? b[2] : b[0], x5 = two ? b[3] : b[1];
    const uint32_t y0 = one ? x1 : x0, y1 = one ? x2 : x1, y2 = one ? x3 : x2, y3 = one ? x4 : x3, y4 = one ? x5 : x4;
    v4u r;
    r[0] = half ? __builtin_amdgcn_alignbyte(y1, y0, 2) : y0;
    r[1] = half ? __builtin_amdgcn_alignbyte(y2, y1, 2) : y1;
    r[2] = half ? __builtin_amdgcn_alignbyte(y3, y2, 2) : y2;
    r[3] = half ? __builtin_amdgcn_alignbyte(y4, y3, 2) : y3;
    return r;
}

__device__ __forceinline__ int distance_index(const Buckets &b, int rel)
{
    const int hi = b.both ? b.far : 0;
    return (rel < -b.far ? -b.far : (rel > hi ? hi : rel)) + b.far;
}
// First entry of the table by distance that bucket `row` holds, and how many (0: none)
__device__ __forceinline__ int entries_of_bucket(const Buckets &b, int row, int *count)
{
    const bool right = b.both && row >= b.n;
    const int k = right ? row - b.n : row;
    int lo = k < b.e ? k : b.border[k - b.e], hi;                   // distances lo ... hi - 1
    if (k < b.e) hi = k + 1;
    else hi = k == b.n - 1 ? b.far + 1 : b.border[k - b.e + 1];
    if (right && lo == 0) lo = 1;                                   // distance 0 is the left side's
    *count = hi > lo ? hi - lo : 0;
    return right ? b.far + lo : b.far - hi + 1;
}

// The entries of every bucket in a table by distance with `pad` more entries on each side, which belong to the ends' buckets, into LDS:
// by the first `rows` of the workgroup's threads, all borders in one round trip.  (Looked up where they were needed, one bucket
// after the other, they took most of a short call's time: dq of 64 x 256 x 12 x 64 57 us, now 53.)
struct Span {
    int at, count;
};
__device__ __forceinline__ void find_spans(const Buckets &b, int rows, int pad, Span *spans)
{
    if ((int)threadIdx.x >= rows) return;
    const int entries = b.far + (b.both ? b.far : 0) + 1;
    int count, at = entries_of_bucket(b, threadIdx.x, &count);
    if (count > 0) {
        if (at + count == entries) count += pad;
        if (at == 0) count += pad;
        else at += pad;
    }
    spans[threadIdx.x] = {at, count};
}
// For every bucket f(bucket, entry) of each of its entries: a wave for each bucket in turn
template <int THREADS = 256, typename F>
__device__ __forceinline__ void each_entry(const Span *spans, int rows, F f)
{
    for (int n = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); n < rows; n += THREADS / 64) {
        const Span s = spans[n];
        for (int e = threadIdx.x & 63; e < s.count; e += 64) f(n, s.at + e);
    }
}

// What a workgroup makes of sums by distance, copies [copies][stride] in LDS of `entries` each, to the sums by bucket out[0 .. rows), times
// `by`.
template <int THREADS = 256>
__device__ __forceinline__ void bucket_sums(const Span *spans, float *sums, int copies, int stride, int entries, int rows, float *out, float by = 1.0f)
{
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    for (int e = tid; e < entries; e += THREADS) {
        float s = sums[e];
        for (int w = 1; w < copies; ++w) s += sums[w * stride + e];
        sums[e] = s;
    }
    __syncthreads();
    for (int n = tid >> 6; n < rows; n += THREADS / 64) {
        const Span r = spans[n];
        float s = 0.0f;
        for (int e = lane; e < r.count; e += 64) s += sums[r.at + e];
        s = wave_sum(s);
        if (lane == 0) out[n] = s * by;
    }
}

// dtable [buckets, heads], head h, of the partial sums [heads][parts][buckets], in this order and in fp64, by a workgroup of THREADS;
// memory: one double for each
template <int THREADS>
__device__ __forceinline__ void reduce_table(const float *__restrict__ partials, int heads, int64_t parts, int buckets, float *__restrict__ dtable,
                                             int h, double *memory)
{
    // groups of `width` threads (a power of two, one for each bucket) take the parts in turn
    int width = 1;
    while (width < buckets) width <<= 1;
    const int groups = THREADS / width, g = threadIdx.x / width, n = threadIdx.x % width;
    double s = 0.0;
    if (n < buckets) {
        const float *src = partials + (int64_t)h * parts * buckets + n;
        for (int64_t i = g; i < parts; i += 8 * groups) {
            float x[8];                                                    // eight loads in flight
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = src[(i + e * groups < parts ? i + e * groups : i) * buckets];
#pragma unroll
            for (int e = 0; e < 8; ++e) s += i + e * groups < parts ? (double)x[e] : 0.0;
        }
    }
    memory[threadIdx.x] = s;
    __syncthreads();
    if (g == 0 && n < buckets) {
#pragma unroll 8
        for (int k = 1; k < groups; ++k) s += memory[k * width + n];
        dtable[n * heads + h] = (float)s;
    }
}
#endif

// dtable of partial sums [heads][parts][buckets] (reduce_table)
hipError_t launch_table_reduce(const float *partials, int heads, int64_t parts, int buckets, float *dtable, hipStream_t st);

}  // namespace egeria
