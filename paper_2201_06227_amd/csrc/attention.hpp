// What the attention kernels share: arguments, operand tiles in LDS, matrix-core fragments.
#pragma once
#include "position.hpp"

namespace egeria {

struct View {
    char *p;
    int64_t sb, st, sh;                     // strides in elements
};

struct AttnArgs {
    View q, k, v, o, d_o, dq, dk, dv;
    float *lse;                             // [batch, heads, q_len]
    float *delta;                           // [batch, heads, q_len], backward
    float *partials;                        // [heads][batch * parts * row tiles][buckets], backward with a table gradient
    float *dtable;                          // [buckets, heads] out, or null
    float *split_o, *split_ml;              // forward split over keys: partial outputs and row statistics
    float *part_q, *part_kv;                // backward in parts: [parts][batch, heads, q_len][D], [parts][batch, kv_heads, k_len][dk, dv][D]
    const int32_t *q_lens, *k_lens;
    const float *table;                     // null: no bias
    int32_t table_rows;
    int32_t batch, heads, kv_heads, group, q_len, k_len, dim, causal;
    int32_t splits, q_parts, kv_parts;
    int32_t whole;                          // one pass: key heads of the batch that are not done in (kv_parts) parts
    int64_t table_parts;                    // partial sums of each head in `partials`
    float scale;
    Buckets b;
};

constexpr int kRowTile = 128;               // queries (or keys, in the dk / dv kernel) of a workgroup
constexpr int kKeyTile = 64;                // keys (queries) of one step
constexpr int kFewRows = 32;                // rows of a workgroup of the kernel for few rows
constexpr int kFewKeys = 32;                // keys that a wave of it takes at a time

hipError_t launch_attention_forward(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st);
// few rows: a.splits workgroups share a row tile's keys; more than one leaves partial results (split_o, split_ml) that a second
// launch joins
hipError_t launch_attention_few(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st);
// dq, delta and the partial sums of the table's gradient; then dk, dv and the table's gradient; then, in parts, their sums
hipError_t launch_attention_backward(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st);
// everything in one pass, for at most kOnePassKeys keys and heads of at most 64 (one_pass_lds(...) <= kMostLds)
constexpr int kOnePassKeys = 256;
constexpr size_t kMostLds = 156 * 1024;
size_t one_pass_lds(const egeria_attention_desc *d, bool table_grad);
inline int one_pass_queries(int32_t dtype) { return dtype == EGERIA_F32 ? 32 : 64; }       // queries of a step
hipError_t launch_attention_one_pass(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st);

// Joins parts of sums: one of up to three tensors [batch, heads, len, ..] in each blockIdx.y.
struct JoinJob {
    View out;
    const float *sum;                       // [parts][rows][stride]
    int64_t rows;                           // of the heads from number `first` on
    int32_t heads, len, parts, stride, first;
};
struct JoinJobs {
    JoinJob job[3];
    int n = 0;
    int64_t most = 0;                       // rows
    void add(const JoinJob &j)
    {
        if (j.parts < 2 || j.rows == 0) return;
        job[n++] = j;
        most = j.rows > most ? j.rows : most;
    }
};
hipError_t launch_join_parts(const JoinJobs &jobs, int dim, egeria_dtype dt, bool vec, hipStream_t st);

// A launcher's instance for the type, the head size and how the rows are read.  D: the head size in whole blocks of 32, which is what
// the products cost; tiles in LDS have rows of 64 or 128 values (heads of 96 in products of 128: causal 2 x 4096 x 16 (4) x 96
// forward 156 us, now 132, backward 518 / 444).
#define EG_PICK_DIM(go, T, vec, a, ...)                                                                              \
    (a.dim <= 32 ? (vec ? go<T, 32, true>(__VA_ARGS__) : go<T, 32, false>(__VA_ARGS__))                               \
                 : a.dim <= 64 ? (vec ? go<T, 64, true>(__VA_ARGS__) : go<T, 64, false>(__VA_ARGS__))                 \
                 : a.dim <= 96 ? (vec ? go<T, 96, true>(__VA_ARGS__) : go<T, 96, false>(__VA_ARGS__))                 \
                               : (vec ? go<T, 128, true>(__VA_ARGS__) : go<T, 128, false>(__VA_ARGS__)))
#define EG_PICK(go, a, dt, vec, st) (dt == EGERIA_F32 ? EG_PICK_DIM(go, float, vec, a, a, st) : EG_PICK_DIM(go, uint16_t, vec, a, a, st))
inline int64_t padded_dim(int32_t dim) { return (dim + 31) / 32 * 32; }
constexpr int row_values(int d) { return d <= 64 ? 64 : 128; }

#ifdef __HIPCC__

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kHidden = -1e30f;           // table entries up to this hide their pairs

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
typedef __attribute__((address_space(3))) v4u lds_v4u;
typedef __attribute__((address_space(3))) float lds_f32;

// Which piece of the launch a workgroup takes.  Its `units` have `per` pieces each.  Workgroup ids go round the 8 XCDs: a unit's pieces go
// to one of them, where the rows that several of them read are in its L2; neighbouring units, which are as long as each other where
// the batch is sorted by length, go to different ones.  The units left over when eight at a time have been dealt are spread over all
// XCDs.  Two ways:
//   like pieces (no causal mask): a unit is a sequence, whose heads lie side by side in memory, and its pieces come one after the
//   other (forward of 64 x 256 x 12 x 64 26 us; with a key head as the unit 33);
//   pieces of which the first take longest (causal): a unit is a key head, and kMixed units are taken together, their first pieces
//   first, so that what ends last is short (causal 2 x 4096 x 16 (4) x 128 unit after unit / this way: forward 216 / 170 us, dq 247 /
//   226, dk and dv 459 / 364).
struct Piece {
    uint32_t unit, rest;
};
constexpr uint32_t kMixed = 4;
__device__ __forceinline__ Piece deal_units(uint32_t blk, uint32_t units, uint32_t per, bool alike)
{
    const uint32_t mine = units >> 3, left = units & 7u;
    if (blk < 8 * mine * per) {
        const uint32_t n = blk >> 3, x = blk & 7u;
        if (alike) {
            const uint32_t u = n / per;
            return {u * 8 + x, n - u * per};
        }
        const uint32_t turn = n / (kMixed * per), in = n - turn * kMixed * per;
        const uint32_t m = turn * kMixed + kMixed > mine ? mine - turn * kMixed : kMixed, rest = in / m;
        return {(turn * kMixed + in - rest * m) * 8 + x, rest};
    }
    uint32_t n = blk - 8 * mine * per;
    if (alike) {
        n = xcd_piece(n, left * per);
        const uint32_t u = n / per;
        return {8 * mine + u, n - u * per};
    }
    const uint32_t rest = n / left;
    return {8 * mine + n - rest * left, rest};
}
// The pieces of kernels that have `tiles` tiles for each of `each` things (heads, parts) of a key head: key head of the batch, number of
// the thing, and tile.
struct HeadPiece {
    uint32_t head, which, tile;
};
__device__ __forceinline__ HeadPiece deal_heads(uint32_t blk, uint32_t batch, uint32_t kv_heads, uint32_t each, uint32_t tiles, bool alike)
{
    if (alike) {
        const Piece p = deal_units(blk, batch, kv_heads * each * tiles, true);
        const uint32_t n = p.rest / tiles, g = n / each;
        return {p.unit * kv_heads + g, n - g * each, p.rest - n * tiles};
    }
    const Piece p = deal_units(blk, batch * kv_heads, each * tiles, false);
    const uint32_t tile = p.rest / each;
    return {p.unit, p.rest - tile * each, tile};
}

struct v8f {
    float v[8];
};

template <int N> struct Const {
    static constexpr int value = N;
};

__device__ __forceinline__ int clamped(const int32_t *lens, int b, int most)
{
    const int n = lens ? lens[b] : most;
    return n < 0 ? 0 : (n > most ? most : n);
}

// Operand fragments of a 32 x 32 x 16 product: lane l holds row (A) or column (B) l % 32, eight consecutive values of the reduced
// dimension from 8 (l / 32) on.  bf16: one instruction.  fp32: eight of depth two, which take element e of both halves: the same
// sixteen products, so one layout serves both types.
template <typename T> struct FragOf;
template <> struct FragOf<uint16_t> { typedef v8bf type; };
template <> struct FragOf<float> { typedef v8f type; };

__device__ __forceinline__ v16f mma(v8bf a, v8bf b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v16f mma(const v8f &a, const v8f &b, v16f c)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}

// sum of the lane's products
__device__ __forceinline__ float dot(v8bf a, v8bf b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf((float)a[e], (float)b[e], s);
    return s;
}
__device__ __forceinline__ float dot(const v8f &a, const v8f &b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(a.v[e], b.v[e], s);
    return s;
}

// A 32 x 32 result holds, in register r of lane l, row 8 (r / 4) + 4 (l / 32) + r % 4 of column l % 32.  Registers 8 s ... 8 s + 7 are
// therefore, for the lane's column, the rows 16 s + {4 half + 0..3, 8 + 4 half + 0..3}: an operand of the next product over those 16
// rows, if the other operand is read in the same order (col_frag).  So probabilities go from one product to the next in
// registers.
template <typename T> __device__ __forceinline__ typename FragOf<T>::type pack(const v16f &c, int s);
template <> __device__ __forceinline__ v8bf pack<uint16_t>(const v16f &c, int s)
{
    v8bf f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (__bf16)c[8 * s + e];
    return f;
}
template <> __device__ __forceinline__ v8f pack<float>(const v16f &c, int s)
{
    v8f f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = c[8 * s + e];
    return f;
}
__device__ __forceinline__ int row_of(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// Tiles of rows of D values in LDS, read along rows (row_frag: 16 bytes of 32 rows) and across them (col_frag: 4 rows of 32 columns,
// transposed by the read itself for bf16).  A row is kept in units of 16 bytes, unit u of row r at slot u ^ turn(r).  The 64 banks
// of 4 bytes hold 256 bytes, i.e. 16 units: the 16 rows that a quarter of a wave reads a unit of have 16 different (row, slot) places
// if turn() takes different values over the rows that share a place; and of the four rows that half a wave reads 4 units of each
// across (col_frag; other ways across a tile may have conflicts), those that share places have turn() differ in the bits above the lowest two.  Rows of 128 bytes (two to a line of banks): the
// bits of r / 2 in reverse; longer rows: r with its lowest two bits on top.
constexpr int kTileAlign = 512;             // of LDS that holds tiles: a whole number of rows (Lane)
template <typename T, int D>
struct Tile {
    static constexpr int kUnits = D * (int)sizeof(T) / 16, kRowBytes = D * (int)sizeof(T);
    static_assert(kTileAlign % kRowBytes == 0, "bits of a unit are changed in an address");
    static __device__ __forceinline__ int turn(int r)
    {
        if constexpr (kUnits == 8) return ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1 | ((r >> 3) & 1);
        else return (r & 3) << 2 | ((r >> 2) & 3);
    }
    static __device__ __forceinline__ uint32_t at(int r, int u) { return (uint32_t)(r * kRowBytes + ((u ^ turn(r)) << 4)); }

    typedef typename FragOf<T>::type frag;

    // Where a lane reads: what depends on the lane, once; everything else of an address is an exclusive-or or a sum with constants,
    // since rows 16 apart have the same turn and units are numbered by bits: those of a row's bytes, so tiles begin at whole rows in LDS,
    // the kernel's dynamic memory at kTileAlign whatever static memory lies before it.  (With addresses worked out per read, a step
    // of the forward kernel for heads of 128 had 41 additions beside 32 reads, and their terms overflowed the registers.)
    struct Lane {
        uint32_t row, col;
    };
    static __device__ __forceinline__ Lane lane_at(uint32_t lds, int lane)
    {
        const int half = lane >> 5;
        if constexpr (sizeof(T) == 2) {
            // across: in each group of 16 lanes, lane i addresses 4 columns of row i / 4 and receives column i of the four rows
            return {lds + at(lane & 31, half), lds + at(4 * half + ((lane & 15) >> 2), ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8};
        } else {
            return {lds + at(lane & 31, 2 * half), lds + (uint32_t)(4 * half * kRowBytes + ((((lane & 31) >> 2) ^ half) << 4) + (lane & 3) * 4)};
        }
    }
    // rows R0 ... R0 + 31, values 16 kk ... 16 kk + 15 of the tile `off` bytes behind the lane's
    static __device__ __forceinline__ frag row_frag(const Lane &l, uint32_t off, int r0, int kk)
    {
        const uint32_t more = off + (uint32_t)(r0 * kRowBytes);
        if constexpr (sizeof(T) == 2) {
            return __builtin_bit_cast(v8bf, *(const lds_v4u *)(uintptr_t)((l.row ^ (uint32_t)(kk << 5)) + more));
        } else {
            const v4u lo = *(const lds_v4u *)(uintptr_t)((l.row ^ (uint32_t)(kk << 6)) + more), hi = *(const lds_v4u *)(uintptr_t)((l.row ^ (uint32_t)(kk << 6 | 16)) + more);
            v8f f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f.v[e] = __uint_as_float(lo[e]);
                f.v[4 + e] = __uint_as_float(hi[e]);
            }
            return f;
        }
    }
    // columns 32 db ... 32 db + 31 of the 16 rows from r0 on, in the order of pack()
    static __device__ __forceinline__ frag col_frag(const Lane &l, uint32_t off, int r0, int db)
    {
        const uint32_t more = off + (uint32_t)(r0 * kRowBytes);
        if constexpr (sizeof(T) == 2) {
            constexpr uint32_t kTurn8 = kUnits == 8 ? 16 : 32;             // turn() of a row 8 further
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(uintptr_t)((l.col ^ (uint32_t)(db << 6)) + more));
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(uintptr_t)((l.col ^ ((uint32_t)(db << 6) ^ kTurn8)) + more + 8 * kRowBytes));
            return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v8f f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t unit = (uint32_t)(8 * db) ^ (uint32_t)((e & 3) << 2) ^ (uint32_t)((e >> 2) << 1);
                f.v[e] = *(const lds_f32 *)(uintptr_t)((l.col ^ (unit << 4)) + more + (uint32_t)(((e & 3) + 8 * (e >> 2)) * kRowBytes));
            }
            return f;
        }
    }
};

// Reads rows of one head of a tensor [.., token, .., feature].
// VEC: rows start on 16 bytes, hold a whole number of 16-byte units, do not overlap, and kRowTile of them span less than 2 GiB:
// 16-byte loads, into tiles as buffer loads straight into LDS.  A unit beyond the row's end or of a token at or beyond `tokens` is asked
// for beyond the buffer and arrives as zeros.  Otherwise: element by element.
template <int ALIGN> struct AnyUnit;
template <> struct AnyUnit<2> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct AnyUnit<4> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
template <typename T, int D, bool VEC>
struct Rows {
    const char *base;
    int64_t row_bytes;
    int tokens, dim;

    __device__ __forceinline__ void open(const View &v, int b, int h, int n, int d)
    {
        base = v.p + ((int64_t)b * v.sb + (int64_t)h * v.sh) * (int64_t)sizeof(T);
        row_bytes = v.st * (int64_t)sizeof(T);
        tokens = n;
        dim = d;
    }
    // 16 bytes: unit u of token t, zeros beyond the row and the tokens.  The load itself is unconditional, from a place that exists (the
    // tensor is not empty): under a condition each would be awaited before the next is asked for.
    __device__ __forceinline__ v4u unit(int t, int u) const
    {
        constexpr int N = 16 / (int)sizeof(T);
        const bool ok = t < tokens && u * N < dim;
        const int row = t < tokens ? t : (tokens > 0 ? tokens - 1 : 0);
        const char *p = base + (int64_t)row * row_bytes;
        v4u w;
        if constexpr (VEC) w = *(const v4u *)(p + (u * N < dim ? u * 16 : 0));
        else if (dim >= N) {
            // at any address; a unit that the row ends in: the row's last 16 bytes, moved down
            const int at = u * N <= dim - N ? u * N : dim - N, over = (u * N - at) * (int)sizeof(T);
            w = *(const typename AnyUnit<sizeof(T)>::type *)(p + at * (int)sizeof(T));
            w = from_byte(w, v4u(0), over < 16 ? over : 0);
        } else {
            union { v4u w; T e[N]; } x;
            x.w = v4u(0);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const T v = ((const T *)p)[e < dim ? e : 0];
                x.e[e] = e < dim ? v : (T)0;
            }
            w = x.w;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = ok ? w[k] : 0u;
        return w;
    }
    // fragment of the 32 tokens from t0 on, values 16 kk ...
    __device__ __forceinline__ typename FragOf<T>::type frag(int t0, int kk, int lane) const
    {
        const int t = t0 + (lane & 31), half = lane >> 5;
        if constexpr (sizeof(T) == 2) return __builtin_bit_cast(v8bf, unit(t, 2 * kk + half));
        else {
            const v4u lo = unit(t, 4 * kk + 2 * half), hi = unit(t, 4 * kk + 2 * half + 1);
            v8f f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f.v[e] = __uint_as_float(lo[e]);
                f.v[4 + e] = __uint_as_float(hi[e]);
            }
            return f;
        }
    }
};

// Brings N tokens at a time of such rows into tiles, by the THREADS threads numbered tid (whole waves); the requests of the VEC form
// are outstanding until an explicit wait.  Rows at or beyond `tokens` lie beyond the buffer's extent (rows do not overlap: VEC).
template <typename T, int D, bool VEC, int N, int THREADS>
struct Feed {
    typedef Tile<T, row_values(D)> tile;
    static constexpr int kUnits = tile::kUnits, kSteps = N * kUnits / THREADS, kRowsPer = THREADS / kUnits;
    static_assert(N * kUnits % THREADS == 0, "whole requests");
    Rows<T, D, VEC> rows;
    uint32_t off;                           // the lane's place in the first request
    int tid;

    __device__ __forceinline__ uint32_t place(int i) const
    {
        const int n = i * THREADS + tid, r = n / kUnits, u = (n % kUnits) ^ tile::turn(r);
        return u < rows.dim * (int)sizeof(T) / 16 ? (uint32_t)r * (uint32_t)rows.row_bytes + (uint32_t)u * 16u : 0x80000000u;
    }
    __device__ __forceinline__ void open(const View &v, int b, int h, int n, int d, int id)
    {
        rows.open(v, b, h, n, d);
        tid = id;
        if constexpr (VEC) off = place(0);
    }
    __device__ __forceinline__ void load(uint32_t lds, int t0) const
    {
        if constexpr (VEC) {
            const uint64_t at = (uint64_t)(rows.base + (int64_t)t0 * rows.row_bytes);
            const int64_t left = (int64_t)(rows.tokens - t0) * rows.row_bytes;
            v4i rsrc;
            rsrc[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)at);
            rsrc[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xffff);
            rsrc[2] = __builtin_amdgcn_readfirstlane(left < 0 ? 0 : (left > 0x7fffffff ? 0x7fffffff : (int)left));
            rsrc[3] = kBufferWord;
            const uint32_t first = lds + (uint32_t)__builtin_amdgcn_readfirstlane(tid & ~63) * 16u;
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
                // rows 16 apart have the same turn: one place, and a multiple of the stride (added to a place outside it stays there)
                load_to_lds_b128(rsrc, first + (uint32_t)(i * THREADS * 16),
                                 kRowsPer % 16 == 0 ? off + (uint32_t)(i * kRowsPer) * (uint32_t)rows.row_bytes : place(i));
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int n = i * THREADS + tid, r = n / kUnits, u = n % kUnits;
                *(lds_v4u *)(uintptr_t)(lds + tile::at(r, u)) = rows.unit(t0 + r, u);
            }
        }
    }
};

// Writes four values: features f ... f + 3 of a token
template <typename T, bool VEC>
__device__ __forceinline__ void store4(T *row, int f, int dim, float x0, float x1, float x2, float x3)
{
    if constexpr (sizeof(T) == 2) {
        union { v2u w; __bf16 e[4]; } x;
        x.e[0] = (__bf16)x0, x.e[1] = (__bf16)x1, x.e[2] = (__bf16)x2, x.e[3] = (__bf16)x3;
        if constexpr (VEC) {
            if (f < dim) *(v2u *)(row + f) = x.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (f + e < dim) ((__bf16 *)row)[f + e] = x.e[e];
        }
    } else {
        const float x[4] = {x0, x1, x2, x3};
        if constexpr (VEC) {
            if (f < dim) *(float4 *)(row + f) = make_float4(x0, x1, x2, x3);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (f + e < dim) row[f + e] = x[e];
        }
    }
}

// The 32 rows of a wave, columns of a result across lanes (row i of the wave in lanes i and i + 32), times `by`, into rows t0 ... of a
// tensor's head as far as `rows` goes.  VEC: through 32 rows of a tile in LDS that the wave has to itself (`lds`, its own after a
// barrier), so that a request covers whole rows instead of 8 or 16 bytes of 32 of them: with those, the address unit worked a few
// microseconds on a workgroup's results (forward of 64 x 256 x 12 x 64 30.6 us, now 26).
template <typename T, int D, bool VEC>
__device__ __forceinline__ void store_rows(const v16f (&x)[D / 32], float by, const View &v, int b, int h, int t0, int rows, int dim, uint32_t lds, int lane)
{
    typedef Tile<T, row_values(D)> tile;
    const int half = lane >> 5, mine = lane & 31;
    T *base = (T *)v.p + ((int64_t)b * v.sb + (int64_t)h * v.sh);
    if constexpr (!VEC) {
        if (t0 + mine >= rows) return;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                store4<T, VEC>(base + (int64_t)(t0 + mine) * v.st, 32 * n + row_of(r, half), dim, x[n][r] * by, x[n][r + 1] * by, x[n][r + 2] * by, x[n][r + 3] * by);
    } else {
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int f = 32 * n + row_of(r, half);
                if constexpr (sizeof(T) == 2) {
                    union { v2u w; __bf16 e[4]; } y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y.e[e] = (__bf16)(x[n][r + e] * by);
                    *(__attribute__((address_space(3))) v2u *)(uintptr_t)(lds + tile::at(mine, f >> 3) + 8 * half) = y.w;
                } else {
                    v4u y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = __float_as_uint(x[n][r + e] * by);
                    *(lds_v4u *)(uintptr_t)(lds + tile::at(mine, f >> 2)) = y;
                }
            }
        wave_lds_turn();
        constexpr int kPer = 64 / tile::kUnits;                             // rows of a request
        const int u = lane % tile::kUnits;
#pragma unroll
        for (int n = 0; n < 32 / kPer; ++n) {
            const int r = n * kPer + lane / tile::kUnits;
            const v4u y = *(const lds_v4u *)(uintptr_t)(lds + tile::at(r, u));
            if (t0 + r < rows && u * 16 < dim * (int)sizeof(T)) *(v4u *)((char *)(base + (int64_t)(t0 + r) * v.st) + u * 16) = y;
        }
        wave_lds_turn();
    }
}

// The bias of one head by distance, in LDS: table entries in units of the scores' base-2 exponent (hidden ones minus infinity), from
// distance -far - kPad to hi + kPad.  A block of at most 64 keys and 32 queries that reaches into [-far, hi] has no distance outside, so
// its pairs are looked up without clamping, four neighbouring distances at a time; every other block has one bias for all of
// its pairs.
constexpr int kPad = 96;
__device__ __forceinline__ float table_value(const float *table, int row, int heads, int h)
{
    const float t = table[row * heads + h];
    return t <= kHidden ? -INFINITY : t * kLog2e;
}
inline size_t bias_lut_floats(const Buckets &b) { return align_up((size_t)distance_entries(b) + 2 * kPad, 4) + 3 * kMaxBuckets; }
inline size_t bias_lut_floats(const AttnArgs &a) { return a.table ? bias_lut_floats(a.b) : 0; }

typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

struct BiasLut {
    float *lut;
    Span *spans;                            // entries of every bucket
    float *value;
    int far, hi;                            // ends of the table: distances beyond them have the bias of the nearest end
    bool on;

    __device__ __forceinline__ int count() const { return far + hi + 1 + 2 * kPad; }
    __device__ __forceinline__ int room() const { return (count() + 3) & ~3; }
    __device__ __forceinline__ void open(const AttnArgs &a, float *memory)
    {
        on = a.table != nullptr;
        far = a.b.far;
        hi = a.b.both ? a.b.far : 0;
        lut = memory;
        spans = (Span *)(lut + room());
        value = (float *)(spans + kMaxBuckets);
        if (on) find_spans(a.b, a.table_rows, kPad, spans);
    }
    __device__ __forceinline__ float *end() const { return value + kMaxBuckets; }
    // by all threads: read(), a barrier, fill(); the caller synchronises after it
    __device__ __forceinline__ void read(const AttnArgs &a, int h) const
    {
        if (on && (int)threadIdx.x < a.table_rows) value[threadIdx.x] = table_value(a.table, threadIdx.x, a.heads, h);
    }
    template <int THREADS = 256>
    __device__ __forceinline__ void fill(const AttnArgs &a) const
    {
        if (on) each_entry<THREADS>(spans, a.table_rows, [&](int n, int e) { lut[e] = value[n]; });
    }
    // a block of pairs with distances lo ... top: one bias for all of them, which is it
    __device__ __forceinline__ bool left(int top) const { return top <= -far; }
    __device__ __forceinline__ bool one(int lo, int top) const { return !on || left(top) || lo >= hi; }
    __device__ __forceinline__ float the_one(int top) const { return !on ? 0.0f : lut[left(top) ? 0 : count() - 1]; }
    __device__ __forceinline__ v4f_any four(int rel) const { return *(const v4f_any *)(lut + (rel + far + kPad)); }
};

template <typename K>
inline hipError_t allow_lds(K kernel, size_t bytes, bool (&done)[kMaxDevices])
{
    const int dev = current_device();
    if (dev < 0) return hipErrorInvalidDevice;
    if (done[dev] || bytes <= 65536) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMostLds);
    if (e == hipSuccess) done[dev] = true;
    return e;
}

#endif

}  // namespace egeria
