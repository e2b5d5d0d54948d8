// Attention forward: out = softmax(scale q k^T + bias) v and the log-sum-exp of every row, in one pass over the keys.
//
// A wave keeps 32 queries.  Per step of 64 keys it forms S^T = K Q^T (keys down, queries across: a lane has one query and half of the
// step's keys, so row maxima and sums need one exchange with the lane's partner), raises the running maximum m and rescales what is
// summed so far where it grew, and adds V^T P^T to O^T, P^T going from result to operand in registers (pack).  All exponents
// are base 2: t = s * (scale log2 e) + bias log2 e, p = 2^(t - m), L = (m + log2 sum p) ln 2.
#include "attention.hpp"

namespace egeria {

namespace {

// Queries of one wave: what the two kernels below do with one step of keys.
template <typename T, int D>
struct RowState {
    static constexpr int kDepth = D / 16, kBlocks = D / 32;
    typedef Tile<T, row_values(D)> tile;
    typename tile::frag q[kDepth];
    v16f o[kBlocks];
    float m, l;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) o[i] = v16f(0.0f);
        m = -INFINITY;
        l = 0.0f;
    }
    // S^T of N blocks of 32 keys
    template <int N>
    __device__ __forceinline__ void scores(v16f (&s)[N], const typename tile::Lane &at, uint32_t k_off) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = v16f(0.0f);
        if constexpr (N == 1) {
            // a chain of its own for every other product: with one, a wave alone on its SIMD waits for each to end
            v16f odd = v16f(0.0f);
#pragma unroll
            for (int kk = 0; kk < kDepth; kk += 2) {
                s[0] = mma(tile::row_frag(at, k_off, 0, kk), q[kk], s[0]);
                odd = mma(tile::row_frag(at, k_off, 0, kk + 1), q[kk + 1], odd);
            }
            s[0] += odd;
        } else {
#pragma unroll
            for (int kk = 0; kk < kDepth; ++kk)
#pragma unroll
                for (int n = 0; n < N; ++n) s[n] = mma(tile::row_frag(at, k_off, 32 * n, kk), q[kk], s[n]);
        }
    }
    // The reference that exponents are taken against after a step with maximum `top` (both lanes of a query agree on it).  It follows
    // the maximum only when that has grown by more than kSlack: until then p <= 2^kSlack, which costs neither fp32 sums nor bf16
    // operands precision, and what is summed so far need not be rescaled.  (Following it always, some query of a wave has a
    // new maximum in most steps: causal 2 x 8192 x 16 (4) x 128 561 us, now 542; 8 x 2048 x 12 x 64 136 / 131.)
    static constexpr float kSlack = 8.0f;
    __device__ __forceinline__ float raise(float top)
    {
        top = fmaxf(top, lane_xor<32>(top));
        if (__any(top > m + kSlack || (m == -INFINITY && top > m))) {
            asm volatile("" ::: "memory");                                 // a branch, not 64 speculated products
            const float to = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.0f : to));
            l *= keep;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= keep;
            m = to;
        }
        return m == -INFINITY ? 0.0f : m;
    }
    template <int N>
    __device__ __forceinline__ void add(const v16f (&p)[N], const typename tile::Lane &at, uint32_t v_off)
    {
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const typename tile::frag f = pack<T>(p[n], s);
#pragma unroll
                for (int i = 0; i < kBlocks; ++i) o[i] = mma(tile::col_frag(at, v_off, 32 * n + 16 * s, i), f, o[i]);
            }
    }
};

template <int N>
__device__ __forceinline__ float largest(const v16f (&s)[N])
{
    float top = -INFINITY;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[n][r]);
    return top;
}

// Four features of a row: its sums over the sum of its weights, zeros if nothing was added (whatever was taken 0 times)
template <typename T, bool VEC>
__device__ __forceinline__ void store_row(const AttnArgs &a, int b, int i, int h, int f, const float (&o)[4], float l)
{
    const float inv = 1.0f / l;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = l == 0.0f ? 0.0f : o[e] * inv;
    store4<T, VEC>((T *)a.o.p + ((int64_t)b * a.o.sb + (int64_t)i * a.o.st + (int64_t)h * a.o.sh), f, a.dim, x[0], x[1], x[2], x[3]);
}
// L of a row from its reference and its sum against that: minus infinity if nothing was added; NaN, from a score that is NaN or
// infinite, stays
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2; }

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) * row_values(D) == 512 ? 1 : 2) void attention_forward_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(kTileAlign))) char smem[];
    typedef Tile<T, row_values(D)> tile;
    constexpr int kTileBytes = kKeyTile * tile::kRowBytes;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tiles = (uint32_t)(a.q_len + kRowTile - 1) / kRowTile;
    const HeadPiece piece = deal_heads(blockIdx.x, (uint32_t)a.batch, (uint32_t)a.kv_heads, (uint32_t)a.group, tiles, !a.causal);
    // the longest rows of a causal head first
    const int q0 = (int)(tiles - 1 - piece.tile) * kRowTile, b = (int)(piece.head / (uint32_t)a.kv_heads);
    const int h = (int)(piece.head % (uint32_t)a.kv_heads) * a.group + (int)piece.which;
    const int nq = clamped(a.q_lens, b, a.q_len), nk = clamped(a.k_lens, b, a.k_len), shift = a.causal ? nk - nq : 0;
    const int rows = nq - q0 < kRowTile ? nq - q0 : kRowTile;               // live rows of the tile (may be negative)
    int keys = rows > 0 ? nk : 0;
    if (a.causal && keys > q0 + rows + shift) keys = q0 + rows + shift;     // the last live row sees keys up to itself
    const int steps = keys > 0 ? (keys + kKeyTile - 1) / kKeyTile : 0;

    const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)smem;
    BiasLut bias;
    bias.open(a, (float *)(smem + 4 * kTileBytes));
    bias.read(a, h);

    Rows<T, D, VEC> qr;
    qr.open(a.q, b, h, nq, a.dim);
    Feed<T, D, VEC, kKeyTile, 256> kr, vr;
    kr.open(a.k, b, h / a.group, nk, a.dim, tid);
    vr.open(a.v, b, h / a.group, nk, a.dim, tid);
    if (steps > 0) {
        kr.load(lds, 0);
        vr.load(lds + kTileBytes, 0);
    }
    const typename tile::Lane at = tile::lane_at(lds, lane);
    const int qw = q0 + 32 * wave, i = qw + (lane & 31);
    RowState<T, D> st;
    st.clear();
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) st.q[kk] = qr.frag(qw, kk, lane);
    const float c = a.scale * kLog2e;
    if (bias.on) __syncthreads();
    bias.fill(a);

    auto one_step = [&](auto buffer, int step) __attribute__((always_inline)) {
        constexpr uint32_t now = decltype(buffer)::value * 2 * kTileBytes, next = 2 * kTileBytes - now;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();                                                    // this step's tiles are there, the other pair is free
        const int j0 = step * kKeyTile;
        if (step + 1 < steps) {
            kr.load(lds + next, j0 + kKeyTile);
            vr.load(lds + next + kTileBytes, j0 + kKeyTile);
        }
        if (qw >= nq || (a.causal && j0 > qw + 31 + shift)) return;         // no pair of the wave is visible
        v16f s[2];
        st.scores(s, at, now);
        const int lo = j0 - (qw + 31) - shift, hi = j0 + kKeyTile - 1 - qw - shift;       // distances of the wave's pairs
        const bool edge = j0 + kKeyTile > nk || (a.causal && hi > 0);
        const bool one = bias.one(lo, hi);
        // scores times `by` plus `beta`, unless they have to be worked out pair by pair (both ways end in the same code: as two of
        // their own the compiler copied the whole sum to and fro)
        float by = c, beta = bias.the_one(hi);
        if (!one || edge || !(c > 0.0f)) {
            const int rel = j0 + 4 * half - i - shift;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    v4f_any t = v4f_any(beta);
                    if (!one) t = bias.four(rel + 32 * n + row_of(r, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][r + e] = fmaf(s[n][r + e], c, t[e]);
                }
            if (edge) {
                const int live = nk - j0 - 4 * half, most = a.causal && -rel < live - 1 ? -rel + 1 : live;
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * n + row_of(r, 0) >= most) s[n][r] = -INFINITY;
            }
            by = 1.0f;
            beta = 0.0f;
        }
        const float off = beta - st.raise(fmaf(largest(s), by, beta));
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], by, off));
                sum += s[n][r];
            }
        st.l += sum;
        st.add(s, at, now + kTileBytes);
    };
    for (int step = 0; step < steps; step += 2) {
        one_step(Const<0>(), step);
        if (step + 1 < steps) one_step(Const<1>(), step + 1);
    }

    const float total = st.l + lane_xor<32>(st.l), l = i < nq ? total : 0.0f;
    if (half == 0 && i < a.q_len)
        a.lse[((int64_t)b * a.heads + h) * a.q_len + i] = log_sum(st.m, l);
    __syncthreads();                                                        // the tiles have been read
    if (l == 0.0f) {                                                        // (a weight of 0 does not make zeros of values that are not finite)
#pragma unroll
        for (int n = 0; n < D / 32; ++n) st.o[n] = v16f(0.0f);
    }
    store_rows<T, D, VEC>(st.o, l == 0.0f ? 0.0f : 1.0f / l, a.o, b, h, qw, a.q_len, a.dim, lds + 32 * wave * tile::kRowBytes, lane);
}

// ---- few rows ---------------------------------------------------------------------------------------------------
// One token (or a few) per sequence: the time is that of reading the keys and values once.  The rows of all heads that share a key
// head are packed into tiles of 32 (row r: head r / q_len of the group, query r % q_len), the four waves of a workgroup take 32 keys
// each in turn, with tiles and running statistics of their own, and join at the end; and `splits` workgroups share a tile's keys
// where there are few tiles, joined by a second launch.

template <typename T, int D> struct FewLayout {
    static constexpr int kTileBytes = kFewKeys * Tile<T, row_values(D)>::kRowBytes;
    static constexpr int kBuffers = 4 * 2 * 2 * kTileBytes <= 128 * 1024 ? 2 : 1;
    static constexpr int kWaveBytes = 2 * kBuffers * kTileBytes;
    static constexpr int kRowFloats = D + 4;                                // rows of the joined outputs, on different banks
    static constexpr int kStage = 4 * kWaveBytes, kJoin = 4 * kFewRows * kRowFloats * 4;
    static constexpr int kMain = kStage > kJoin ? kStage : kJoin;
};

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void attention_few_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(kTileAlign))) char smem[];
    typedef FewLayout<T, D> L;
    __shared__ float stat[2][4][kFewRows];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t rows = (uint32_t)a.group * (uint32_t)a.q_len, tiles = (rows + kFewRows - 1) / kFewRows;
    const Piece piece = deal_units(blockIdx.x, (uint32_t)(a.batch * a.splits), tiles * (uint32_t)a.kv_heads, true);
    const uint32_t split = piece.unit % (uint32_t)a.splits, rt = piece.rest / (uint32_t)a.kv_heads;
    const int g = (int)(piece.rest % (uint32_t)a.kv_heads), b = (int)(piece.unit / (uint32_t)a.splits);
    const int nq = clamped(a.q_lens, b, a.q_len), nk = clamped(a.k_lens, b, a.k_len), shift = a.causal ? nk - nq : 0;
    const uint32_t r0 = rt * kFewRows, r1 = r0 + kFewRows < rows ? r0 + kFewRows : rows;
    const int h0 = (int)(r0 / (uint32_t)a.q_len), h1 = (int)((r1 - 1) / (uint32_t)a.q_len);        // heads of the group in this tile
    // keys that any row of the tile sees, dealt to the splits in whole rounds of the four waves
    int keys = nk, last = h0 == h1 ? (int)((r1 - 1) % (uint32_t)a.q_len) : a.q_len - 1;
    if (last >= nq) last = nq - 1;
    if (a.causal && keys > last + shift + 1) keys = last + shift + 1;
    if (nq == 0 || keys < 0) keys = 0;
    const int per = ((keys + a.splits - 1) / a.splits + 4 * kFewKeys - 1) / (4 * kFewKeys) * (4 * kFewKeys);
    const int64_t first = (int64_t)split * per;
    const int k0 = first < keys ? (int)first : keys, k1 = keys - k0 < per ? keys : k0 + per;

    const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)smem + (uint32_t)wave * L::kWaveBytes;
    float *tab = (float *)(smem + L::kMain);                               // [heads of the tile][table rows]
    Span *spans = (Span *)(tab + (((h1 - h0 + 1) * a.table_rows + 1) & ~1));
    uint8_t *lut = (uint8_t *)(spans + a.table_rows);                      // bucket of every distance
    const int lut_hi = a.b.both ? a.b.far : 0;
    if (a.table) {
        for (int n = tid; n < (h1 - h0 + 1) * a.table_rows; n += 256)
            tab[n] = table_value(a.table, n % a.table_rows, a.heads, g * a.group + h0 + n / a.table_rows);
        find_spans(a.b, a.table_rows, 0, spans);
        __syncthreads();
        each_entry(spans, a.table_rows, [&](int n, int e) { lut[e] = (uint8_t)n; });
    }
    const uint32_t r = r0 + (lane & 31), rr = r < rows ? r : rows - 1;
    const int hl = (int)(rr / (uint32_t)a.q_len), i = (int)(rr % (uint32_t)a.q_len), h = g * a.group + hl;
    const bool live = r < rows && i < nq;
    RowState<T, D> st;
    st.clear();
    {
        Rows<T, D, VEC> qr;
        qr.open(a.q, b, h, live ? nq : 0, a.dim);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) st.q[kk] = qr.frag(i - (lane & 31), kk, lane);
    }
    const float c = a.scale * kLog2e;
    const float *my_tab = tab + (hl - h0) * a.table_rows;
    Feed<T, D, VEC, kFewKeys, 64> kr, vr;
    kr.open(a.k, b, g, nk, a.dim, lane);
    vr.open(a.v, b, g, nk, a.dim, lane);
    const typename Tile<T, row_values(D)>::Lane at_lane = Tile<T, row_values(D)>::lane_at(lds, lane);
    if (a.table) __syncthreads();
    const float beta_left = a.table ? my_tab[lut[0]] : 0.0f, beta_right = a.table ? my_tab[lut[a.b.far + lut_hi]] : 0.0f;
    constexpr int kLoads = 2 * kFewKeys * Tile<T, row_values(D)>::kUnits / 64;         // requests of one step
    int j0 = k0 + kFewKeys * wave;
    auto stage = [&](uint32_t to, int j) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                 // the buffer has been read
        kr.load(lds + to, j);
        vr.load(lds + to + L::kTileBytes, j);
    };
    auto one_step = [&](auto buffer, int j0) __attribute__((always_inline)) {
        constexpr uint32_t now = decltype(buffer)::value * 2 * L::kTileBytes, next = 2 * L::kTileBytes - now;
        if (L::kBuffers == 2) {
            if (j0 + 4 * kFewKeys < k1) {
                stage(next, j0 + 4 * kFewKeys);
                if (VEC) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
            } else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        } else {
            stage(now, j0);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        wave_lds_turn();
        v16f s[1];
        st.scores(s, at_lane, now);
        const int rel = j0 - i - shift;                                     // distances rel ... rel + 31
        const bool edge = j0 + kFewKeys > nk || (a.causal && __any(rel + kFewKeys - 1 > 0));
        float beta = beta_right;
        bool far = true;
        if (a.table) {
            const bool left = rel + kFewKeys - 1 <= -a.b.far, right = rel >= lut_hi;
            far = __all(left || right);
            if (left) beta = beta_left;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int at = rel + row_of(e, half);
            if (!far) beta = my_tab[lut[distance_index(a.b, at)]];
            const bool seen = !edge || (j0 + row_of(e, half) < nk && (!a.causal || at <= 0));
            s[0][e] = seen ? fmaf(s[0][e], c, beta) : -INFINITY;
        }
        const float base = st.raise(largest(s));
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            s[0][e] = __builtin_amdgcn_exp2f(s[0][e] - base);
            sum += s[0][e];
        }
        st.l += sum;
        st.add(s, at_lane, now + L::kTileBytes);
    };
    if (L::kBuffers == 2 && j0 < k1) stage(0, j0);
    for (; j0 < k1; j0 += 4 * kFewKeys) {
        one_step(Const<0>(), j0);
        if (L::kBuffers == 2) {
            j0 += 4 * kFewKeys;
            if (j0 < k1) one_step(Const<1>(), j0);
        }
    }
    __syncthreads();                                                        // every wave is done with its tiles
    st.l += lane_xor<32>(st.l);
    if (half == 0) {
        stat[0][wave][lane] = st.m;
        stat[1][wave][lane] = st.l;
    }
    float *join = (float *)smem;                                           // [wave][row][feature]
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
            *(float4 *)(join + (wave * kFewRows + (lane & 31)) * L::kRowFloats + 32 * n + row_of(e, half)) =
                make_float4(st.o[n][e], st.o[n][e + 1], st.o[n][e + 2], st.o[n][e + 3]);
    __syncthreads();
    for (int n = tid; n < kFewRows * (D / 4); n += 256) {
        const int row = n / (D / 4), f = n % (D / 4) * 4;
        if (r0 + row >= rows) break;
        float top = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[0][w][row]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float k = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(stat[0][w][row] - top);
            const float4 x = *(const float4 *)(join + (w * kFewRows + row) * L::kRowFloats + f);
            l = fmaf(stat[1][w][row], k, l);
            o[0] = fmaf(x.x, k, o[0]);
            o[1] = fmaf(x.y, k, o[1]);
            o[2] = fmaf(x.z, k, o[2]);
            o[3] = fmaf(x.w, k, o[3]);
        }
        const int head = g * a.group + (int)((r0 + row) / (uint32_t)a.q_len), qi = (int)((r0 + row) % (uint32_t)a.q_len);
        if (a.splits == 1) {
            if (qi >= nq) l = 0.0f;
            store_row<T, VEC>(a, b, qi, head, f, o, l);
            if (f == 0) a.lse[((int64_t)b * a.heads + head) * a.q_len + qi] = log_sum(top, l);
        } else {
            const int64_t at = ((((int64_t)b * a.kv_heads + g) * tiles + rt) * a.splits + split) * kFewRows + row;
            *(float4 *)(a.split_o + at * D + f) = make_float4(o[0], o[1], o[2], o[3]);
            if (f == 0) {
                a.split_ml[2 * at] = top;
                a.split_ml[2 * at + 1] = l;
            }
        }
    }
}

// Joins the splits of the rows: a thread has four features of one row.
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, uint32_t row_tiles)
{
    constexpr uint32_t per = 256 / (D / 4);
    const uint32_t rows = (uint32_t)a.group * (uint32_t)a.q_len;
    if (threadIdx.x >= per * (D / 4)) return;
    const int64_t n = (int64_t)xcd_piece(blockIdx.x, gridDim.x) * per + threadIdx.x / (D / 4);       // row of all tiles
    const int f = threadIdx.x % (D / 4) * 4;
    const int64_t tile = n / kFewRows;
    const uint32_t row = (uint32_t)(tile % row_tiles) * kFewRows + (uint32_t)(n % kFewRows);
    const int64_t bg = tile / row_tiles;
    if (bg >= (int64_t)a.batch * a.kv_heads || row >= rows) return;
    const int b = (int)(bg / a.kv_heads), g = (int)(bg % a.kv_heads);
    const int head = g * a.group + (int)(row / (uint32_t)a.q_len), qi = (int)(row % (uint32_t)a.q_len);
    const int64_t at = tile * a.splits * kFewRows + n % kFewRows;
    // eight splits at a time, their statistics and values asked for together.  A split without a maximum is empty, with sums of 0, or its
    // scores are NaN, and so are its sums: it is added like any other, against a reference of 0.  What is read in place of a split that
    // does not exist (finite or not) counts as 0.
    float top = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < a.splits; s0 += 8) {
        float2 ml[8];
        float4 x[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int64_t p = at + (int64_t)(s0 + s < a.splits ? s0 + s : s0) * kFewRows;
            ml[s] = *(const float2 *)(a.split_ml + 2 * p);
            x[s] = *(const float4 *)(a.split_o + p * D + f);
            if (s0 + s >= a.splits) {
                ml[s] = make_float2(-INFINITY, 0.0f);
                x[s] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
        }
        float to = top;
#pragma unroll
        for (int s = 0; s < 8; ++s) to = fmaxf(to, ml[s].x);
        const float base = to == -INFINITY ? 0.0f : to, keep = __builtin_amdgcn_exp2f(top - base);
        l *= keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] *= keep;
        top = to;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float k = __builtin_amdgcn_exp2f(ml[s].x - base);
            l = fmaf(ml[s].y, k, l);
            o[0] = fmaf(x[s].x, k, o[0]);
            o[1] = fmaf(x[s].y, k, o[1]);
            o[2] = fmaf(x[s].z, k, o[2]);
            o[3] = fmaf(x[s].w, k, o[3]);
        }
    }
    if (qi >= clamped(a.q_lens, b, a.q_len)) l = 0.0f;
    store_row<T, VEC>(a, b, qi, head, f, o, l);
    if (f == 0) a.lse[((int64_t)b * a.heads + head) * a.q_len + qi] = log_sum(top, l);
}

template <typename T, int D, bool VEC>
hipError_t go(const AttnArgs &a, hipStream_t st)
{
    static bool done[kMaxDevices] = {};
    const size_t lds = 4 * (size_t)kKeyTile * Tile<T, row_values(D)>::kRowBytes + 4 * bias_lut_floats(a);
    const hipError_t e = allow_lds(attention_forward_kernel<T, D, VEC>, lds, done);
    if (e != hipSuccess) return e;
    const int64_t blocks = (int64_t)a.batch * a.heads * ((a.q_len + kRowTile - 1) / kRowTile);
    return launch_k(EGERIA_KERNEL_ATTENTION, attention_forward_kernel<T, D, VEC>, dim3((unsigned)blocks), dim3(256), lds, st, a);
}

template <typename T, int D, bool VEC>
hipError_t go_few(const AttnArgs &a, hipStream_t st)
{
    static bool done[kMaxDevices] = {};
    const int64_t rows = (int64_t)a.group * a.q_len, tiles = (rows + kFewRows - 1) / kFewRows, all = (int64_t)a.batch * a.kv_heads * tiles;
    const int64_t heads = rows < kFewRows ? a.group : (kFewRows + a.q_len - 2) / a.q_len + 1;       // most heads of a tile
    const size_t lds = FewLayout<T, D>::kMain + (a.table ? (size_t)(heads * a.table_rows + 1) * 4 + a.table_rows * sizeof(Span) + align_up((size_t)distance_entries(a.b), 16) : 0);
    hipError_t e = allow_lds(attention_few_kernel<T, D, VEC>, lds, done);
    if (e != hipSuccess) return e;
    e = launch_k(EGERIA_KERNEL_ATTENTION, attention_few_kernel<T, D, VEC>, dim3((unsigned)(all * a.splits)), dim3(256), lds, st, a);
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t per = 256 / (D / 4);
    return launch_k(EGERIA_KERNEL_NONE, attention_join_kernel<T, D, VEC>, dim3((unsigned)((all * kFewRows + per - 1) / per)), dim3(256), 0, st, a,
                    (uint32_t)tiles);
}

}  // namespace

hipError_t launch_attention_forward(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st) { return EG_PICK(go, a, dt, vec, st); }
hipError_t launch_attention_few(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st) { return EG_PICK(go_few, a, dt, vec, st); }

}  // namespace egeria
