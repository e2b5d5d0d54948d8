// Attention backward: dq, dk, dv and the gradient of the position table from the saved output and log-sum-exp; the probabilities are
// recomputed.  Two kernels, each the owner of what it writes, so there are no atomics on results and sums have one order: dq (and the
// table's partial sums) by rows of queries, dk and dv by rows of keys.  Seven products of 2 * pairs * dim instead of the five that a
// single kernel with atomic sums would do.
//
//   dq:  S^T = K Q^T and dP^T = V dO^T (queries across, as in the forward pass), ds = p (dP - D), dQ^T += K^T dS^T
//   dkv: S = Q K^T and dP = dO V^T (keys across), dV^T += dO^T P, dK^T += Q^T dS
// In both, P and dS go from result to operand in registers (pack).
#include "attention.hpp"
#include "attention_diagonals.hpp"

namespace egeria {

namespace {

// Keys of a step of the dq kernel: half as many where a step would leave no LDS for the sums by distance.
template <typename T, int D>
constexpr int dq_keys() { return sizeof(T) * row_values(D) == 512 ? kKeyTile / 2 : kKeyTile; }

// ---- dq ---------------------------------------------------------------------------------------------------------

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) * row_values(D) == 512 ? 1 : 2) void attention_dq_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(kTileAlign))) char smem[];
    typedef Tile<T, row_values(D)> tile;
    constexpr int kKeys = dq_keys<T, D>(), kTileBytes = kKeys * tile::kRowBytes;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tiles = (uint32_t)(a.q_len + kRowTile - 1) / kRowTile;
    const HeadPiece piece = deal_heads(blockIdx.x, (uint32_t)a.batch, (uint32_t)a.kv_heads, (uint32_t)(a.group * a.q_parts), tiles, !a.causal);
    const uint32_t rt = tiles - 1 - piece.tile;                             // the longest rows of a causal head first
    const int part = (int)(piece.which % (uint32_t)a.q_parts), b = (int)(piece.head / (uint32_t)a.kv_heads);
    const int h = (int)(piece.head % (uint32_t)a.kv_heads) * a.group + (int)(piece.which / (uint32_t)a.q_parts);
    const int q0 = (int)rt * kRowTile, bh = b * a.heads + h;
    const int nq = clamped(a.q_lens, b, a.q_len), nk = clamped(a.k_lens, b, a.k_len), shift = a.causal ? nk - nq : 0;
    const int rows = nq - q0 < kRowTile ? nq - q0 : kRowTile;
    int keys = rows > 0 ? nk : 0;
    if (a.causal && keys > q0 + rows + shift) keys = q0 + rows + shift;
    const int all = keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
    const int begin = (int)((int64_t)all * part / a.q_parts), steps = (int)((int64_t)all * (part + 1) / a.q_parts);

    const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)smem;
    BiasLut bias;
    bias.open(a, (float *)(smem + 4 * kTileBytes));
    bias.read(a, h);
    const int entries = bias.count();
    float *sums = bias.end();                                               // [wave][half]: sums of ds by distance, laid out as the bias
    if (a.partials)
        for (int i = tid; i < 8 * entries; i += 256) sums[i] = 0.0f;
    float *mine = sums + (2 * wave + half) * entries;

    Rows<T, D, VEC> qr, gr, orow;
    qr.open(a.q, b, h, nq, a.dim);
    gr.open(a.d_o, b, h, nq, a.dim);
    orow.open(a.o, b, h, nq, a.dim);
    Feed<T, D, VEC, kKeys, 256> kr, vr;
    kr.open(a.k, b, h / a.group, nk, a.dim, tid);
    vr.open(a.v, b, h / a.group, nk, a.dim, tid);
    if (begin < steps) {
        kr.load(lds, begin * kKeys);
        vr.load(lds + kTileBytes, begin * kKeys);
    }
    const typename tile::Lane at = tile::lane_at(lds, lane);
    const int qw = q0 + 32 * wave, i = qw + (lane & 31);
    const int64_t row = ((int64_t)b * a.heads + h) * a.q_len + i;
    typename tile::frag q[D / 16], g[D / 16];
    double sum = 0.0;                                                       // (a row's error in delta stays in the table's long sums: not one chain of D)
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        q[kk] = qr.frag(qw, kk, lane);
        g[kk] = gr.frag(qw, kk, lane);
        sum += (double)dot(g[kk], orow.frag(qw, kk, lane));
        g[kk] = turned(g[kk], lane);
    }
    float delta = (float)(sum + __shfl_xor(sum, 32));
    if (half == 0 && i < a.q_len && part == 0) a.delta[row] = delta;
    const float lse = i < nq ? a.lse[row] : -INFINITY;
    // p 2^whole is what the exponential gives; its factor is in the difference that it is multiplied by (none for rows without a pair and
    // those whose log-sum-exp would swallow it)
    const float whole = fabsf(lse) > kFine ? 0.0f : fminf(fmaxf(rintf(lse * kLog2e), -64.0f), 64.0f), by_p = __builtin_amdgcn_exp2f(-whole);
    const float base = lse == -INFINITY ? INFINITY : lowered(lse, whole), c = a.scale * kLog2e, sign = sign_of<typename tile::frag>(lane) * by_p;
    delta *= by_p;
    v16f dq[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dq[n] = v16f(0.0f);
    double left = 0.0, right = 0.0;                                         // sums of ds beyond the table by distance: long ones, of values that cancel
    if (bias.on) __syncthreads();
    bias.fill(a);

    auto one_step = [&](auto buffer, int step) __attribute__((always_inline)) {
        constexpr uint32_t now = decltype(buffer)::value * 2 * kTileBytes, next = 2 * kTileBytes - now;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        const int j0 = step * kKeys;
        if (step + 1 < steps) {
            kr.load(lds + next, j0 + kKeys);
            vr.load(lds + next + kTileBytes, j0 + kKeys);
        }
        if (qw >= nq) return;
#pragma unroll
        for (int n = 0; n < kKeys / 32; ++n) {
            const int jn = j0 + 32 * n;
            if (jn >= nk || (a.causal && jn > qw + 31 + shift)) break;      // no pair of the wave is visible
            v16f s = v16f(0.0f), d = v16f(0.0f);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                s = mma(tile::row_frag(at, now, 32 * n, kk), q[kk], s);
                d = mma(tile::row_frag(at, now + kTileBytes, 32 * n, kk), g[kk], d);
            }
            const int lo = jn - (qw + 31) - shift, hi = jn + 31 - qw - shift;             // distances of the wave's pairs
            const bool edge = jn + 32 > nk || (a.causal && hi > 0);
            const bool one = bias.one(lo, hi);
            const float beta = bias.the_one(hi);
            const int rel = jn + 4 * half - i - shift;
            if (one) {
                const float off = beta - base;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, off));
            } else {
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const v4f_any t = bias.four(rel + row_of(r, 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r + e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], c, t[e] - base));
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] *= fmaf(sign, d[r], -delta);
            if (edge) {
                const int live = nk - jn - 4 * half, most = a.causal && -rel < live - 1 ? -rel + 1 : live;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (row_of(r, 0) >= most) s[r] = 0.0f;
            }
            if (a.partials) {
                if (one) {
                    if (bias.left(hi)) left += (double)sum16(s);
                    else right += (double)sum16(s);
                } else add_diagonals<1>(s, mine + (jn - qw - shift + bias.far + kPad), lane);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const typename tile::frag f = pack<T>(s, k);
#pragma unroll
                for (int m = 0; m < D / 32; ++m) dq[m] = mma(tile::col_frag(at, now, 32 * n + 16 * k, m), f, dq[m]);
            }
        }
    };
    for (int step = begin; step < steps; step += 2) {
        one_step(Const<0>(), step);
        if (step + 1 < steps) one_step(Const<1>(), step + 1);
    }

    const float by = a.scale;
    if (lse == -INFINITY) {                                                 // (a row without a pair: 0 times a difference that is not finite is no zero)
#pragma unroll
        for (int n = 0; n < D / 32; ++n) dq[n] = v16f(0.0f);
    }
    __syncthreads();                                                        // the tiles have been read
    if (a.q_parts == 1) store_rows<T, D, VEC>(dq, by, a.dq, b, h, qw, a.q_len, a.dim, lds + 32 * wave * tile::kRowBytes, lane);
    else if (i < a.q_len) {
        float *sum = a.part_q + (((int64_t)part * a.batch * a.heads + bh) * a.q_len + i) * D;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(float4 *)(sum + 32 * n + row_of(r, half)) = make_float4(dq[n][r] * by, dq[n][r + 1] * by, dq[n][r + 2] * by, dq[n][r + 3] * by);
    }
    if (a.partials) {
        left = wave_sum(left);
        right = wave_sum(right);
        if (lane == 0) {                                                   // the wave's own table: in order after its additions
            mine[0] += (float)left;
            mine[entries - 1] += (float)right;
        }
        bucket_sums(bias.spans, sums, 8, entries, entries, a.table_rows, a.partials + (((int64_t)h * a.batch + b) * a.q_parts * tiles + part * tiles + rt) * a.table_rows);
    }
}

// Queries of a step of the dk / dv kernel.  Heads of 128: the values of the workgroup's keys stay in LDS, since their fragments beside
// the keys' and two sums of 128 x 32 would overflow a wave's 256 registers; with steps of 32 queries two workgroups still share a
// compute unit.
template <int D>
constexpr int dkv_queries() { return D > 64 ? 32 : kKeyTile; }

// ---- dk, dv -------------------------------------------------------------------------------------------------------

template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256, sizeof(T) * row_values(D) == 512 ? 1 : 2) void attention_dkv_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(kTileAlign))) char smem[];
    typedef Tile<T, row_values(D)> tile;
    constexpr int kQueries = dkv_queries<D>(), kTileBytes = kQueries * tile::kRowBytes;
    constexpr bool kValuesInLds = D > 64;
    __shared__ float stat[2][2][kQueries];                                  // base-2 log-sum-exp and -delta of a step's queries
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the table's gradient, whose partial sums the dq kernel has left: the first workgroups
    const uint32_t extra = a.dtable ? (uint32_t)a.heads : 0u;
    if (blockIdx.x < extra) {
        reduce_table<256>(a.partials, a.heads, a.table_parts, a.table_rows, a.dtable, (int)blockIdx.x, (double *)smem);
        return;
    }
    const uint32_t tiles = (uint32_t)(a.k_len + kRowTile - 1) / kRowTile;
    // (workgroups that read the same queries: a part of those of a key head)
    Piece piece;
    if (a.causal) piece = deal_units(blockIdx.x - extra, (uint32_t)(a.batch * a.kv_heads * a.kv_parts), tiles, false);
    else {
        const HeadPiece p = deal_heads(blockIdx.x - extra, (uint32_t)a.batch, (uint32_t)a.kv_heads, (uint32_t)a.kv_parts, tiles, true);
        piece = {p.head * (uint32_t)a.kv_parts + p.which, p.tile};
    }
    const int part = (int)(piece.unit % (uint32_t)a.kv_parts), bh = (int)(piece.unit / (uint32_t)a.kv_parts);
    const int k0 = (int)piece.rest * kRowTile, hk = bh % a.kv_heads, b = bh / a.kv_heads;
    const int nq = clamped(a.q_lens, b, a.q_len), nk = clamped(a.k_lens, b, a.k_len), shift = a.causal ? nk - nq : 0;
    // queries that see a key of the tile: from `first` on; the same for every head of the group
    int first = a.causal && k0 > shift ? (k0 - shift) / kQueries * kQueries : 0;
    const int per_head = k0 < nk && first < nq ? (nq - first + kQueries - 1) / kQueries : 0;
    const int64_t all = (int64_t)per_head * a.group;
    const int begin = (int)(all * part / a.kv_parts), steps = (int)(all * (part + 1) / a.kv_parts);

    const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)smem;
    constexpr int kStage = 4 * kTileBytes + (kValuesInLds ? kRowTile * tile::kRowBytes : 0);
    BiasLut bias;
    bias.open(a, (float *)(smem + kStage));
    const int jw = k0 + 32 * wave, j = jw + (lane & 31);
    const float c = a.scale * kLog2e;
    Rows<T, D, VEC> kr, vr;
    kr.open(a.k, b, hk, nk, a.dim);
    vr.open(a.v, b, hk, nk, a.dim);
    const typename tile::Lane at = tile::lane_at(lds, lane);
    typename tile::frag k[D / 16], v[kValuesInLds ? 1 : D / 16];
    v16f dk[D / 32], dv[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = v16f(0.0f);

    // stages the queries of a step: rows into LDS, statistics into registers (the caller stores them once the step before is done)
    float next_base = 0.0f, next_delta = 0.0f;
    Feed<T, D, VEC, kQueries, 256> qr, gr;
    qr.open(a.q, b, 0, nq, a.dim, tid);
    gr.open(a.d_o, b, 0, nq, a.dim, tid);
    const char *q_base = qr.rows.base, *g_base = gr.rows.base;
    auto stage = [&](uint32_t to, int step) __attribute__((always_inline)) {
        const int h = hk * a.group + step / per_head, i0 = first + step % per_head * kQueries;
        qr.rows.base = q_base + (int64_t)h * a.q.sh * (int64_t)sizeof(T);
        gr.rows.base = g_base + (int64_t)h * a.d_o.sh * (int64_t)sizeof(T);
        qr.load(to, i0);
        gr.load(to + kTileBytes, i0);
        if (tid < kQueries) {
            const int i = i0 + tid < nq ? i0 + tid : nq - 1;
            const int64_t row = ((int64_t)b * a.heads + h) * a.q_len + i;
            next_base = a.lse[row];
            next_delta = a.delta[row];
            if (i0 + tid >= nq) next_base = -INFINITY;
        }
    };
    auto keep = [&](int buffer) {
        if (tid < kQueries) {
            stat[buffer][0][tid] = next_base == -INFINITY ? INFINITY : next_base * kLog2e;
            stat[buffer][1][tid] = -next_delta;
        }
    };
    if (begin < steps) {
        if constexpr (kValuesInLds) {
            Feed<T, D, VEC, kRowTile, 256> values;
            values.open(a.v, b, hk, nk, a.dim, tid);
            values.load(lds + 4 * kTileBytes, k0);
        }
        stage(lds, begin);
        keep(0);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            k[kk] = kr.frag(jw, kk, lane);
            if constexpr (!kValuesInLds) v[kk] = vr.frag(jw, kk, lane);
        }
    }
    int lut_head = -1;
    const typename tile::Lane at_v = tile::lane_at(lds + 4 * kTileBytes + 32 * wave * tile::kRowBytes, lane);
    auto one_step = [&](auto buffer, int step) __attribute__((always_inline)) {
        constexpr int kBuffer = decltype(buffer)::value;
        constexpr uint32_t now = kBuffer * 2 * kTileBytes, next = 2 * kTileBytes - now;
        const int h = hk * a.group + step / per_head, i0 = first + step % per_head * kQueries;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (a.table && h != lut_head) {                                     // the next head of the group
            bias.read(a, h);
            __syncthreads();
            bias.fill(a);
            lut_head = h;
            __syncthreads();
        }
        if (step + 1 < steps) stage(lds + next, step + 1);
#pragma unroll
        for (int n = 0; n < kQueries / 32; ++n) {
            const int in = i0 + 32 * n;
            if (in >= nq || jw >= nk || (a.causal && jw > in + 31 + shift)) continue;
            // dP - delta: the sum of the products starts at -delta (and no bias, no addition of it: causal 2 x 4096 x 16 (4) x 128 557 us,
            // now 539)
            v16f s = v16f(0.0f), d;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 delta = *(const float4 *)&stat[kBuffer][1][32 * n + row_of(r, half)];
                d[r] = delta.x, d[r + 1] = delta.y, d[r + 2] = delta.z, d[r + 3] = delta.w;
            }
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                s = mma(tile::row_frag(at, now, 32 * n, kk), k[kk], s);
                if constexpr (kValuesInLds)
                    d = mma(tile::row_frag(at, now + kTileBytes, 32 * n, kk), tile::row_frag(at_v, 0, 0, kk), d);
                else d = mma(tile::row_frag(at, now + kTileBytes, 32 * n, kk), v[kk], d);
            }
            const int lo = jw - (in + 31) - shift, hi = jw + 31 - in - shift;             // distances of the wave's pairs
            const bool one = bias.one(lo, hi);
            const float beta = bias.the_one(hi);
            const int rel = j - in - 4 * half - shift;
            v16f p;
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 base = *(const float4 *)&stat[kBuffer][0][32 * n + row_of(r, half)];
                const float bs[4] = {base.x, base.y, base.z, base.w};
                if (!bias.on) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[r + e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], c, -bs[e]));
                    continue;
                }
                v4f_any t;
                if (one) t = v4f_any(beta);
                else t = bias.four(rel - row_of(r, 0) - 3);                // of the keys' distances from four queries, the last first
#pragma unroll
                for (int e = 0; e < 4; ++e) p[r + e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], c, t[3 - e] - bs[e]));
            }
            if (a.causal && hi > 0) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (rel - row_of(r, 0) > 0) p[r] = 0.0f;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = p[r] * d[r];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const typename tile::frag fp = pack<T>(p, e), fs = pack<T>(s, e);
#pragma unroll
                for (int m = 0; m < D / 32; ++m) {
                    dv[m] = mma(tile::col_frag(at, now + kTileBytes, 32 * n + 16 * e, m), fp, dv[m]);
                    dk[m] = mma(tile::col_frag(at, now, 32 * n + 16 * e, m), fs, dk[m]);
                }
            }
        }
        if (step + 1 < steps) keep(1 - kBuffer);
    };
    for (int step = begin; step < steps; step += 2) {
        one_step(Const<0>(), step);
        if (step + 1 < steps) one_step(Const<1>(), step + 1);
    }

    __syncthreads();                                                        // the tiles have been read
    if (!(j < nk)) {                                                        // (columns of their own, and anything may be in them)
#pragma unroll
        for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = v16f(0.0f);
    }
    if (a.kv_parts == 1) {
        const uint32_t room = lds + 32 * wave * tile::kRowBytes;
        store_rows<T, D, VEC>(dk, a.scale, a.dk, b, hk, jw, a.k_len, a.dim, room, lane);
        store_rows<T, D, VEC>(dv, 1.0f, a.dv, b, hk, jw, a.k_len, a.dim, room, lane);
    } else if (j < a.k_len) {
        float *sum = a.part_kv + (((int64_t)part * a.batch * a.kv_heads + bh) * a.k_len + j) * (2 * D);
        const float by = a.scale;
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int f = 32 * n + row_of(r, half);
                *(float4 *)(sum + f) = make_float4(dk[n][r] * by, dk[n][r + 1] * by, dk[n][r + 2] * by, dk[n][r + 3] * by);
                *(float4 *)(sum + D + f) = make_float4(dv[n][r], dv[n][r + 1], dv[n][r + 2], dv[n][r + 3]);
            }
    }
}

// a thread for four features of a row
template <typename T, int D, bool VEC>
__global__ __launch_bounds__(256) void attention_join_parts_kernel(JoinJobs jobs, int dim)
{
    const JoinJob &j = jobs.job[blockIdx.y];
    constexpr int kPer = 256 / (D / 4);
    const int f = threadIdx.x % (D / 4) * 4;
    const int64_t row = (int64_t)blockIdx.x * kPer + threadIdx.x / (D / 4);
    if (threadIdx.x >= kPer * (D / 4) || row >= j.rows) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int p = 0; p < j.parts; ++p) {
        const float4 x = *(const float4 *)(j.sum + ((int64_t)p * j.rows + row) * j.stride + f);
        s.x += x.x, s.y += x.y, s.z += x.z, s.w += x.w;
    }
    const int i = (int)(row % j.len), bh = j.first + (int)(row / j.len), h = bh % j.heads, b = bh / j.heads;
    T *out = (T *)j.out.p + ((int64_t)b * j.out.sb + (int64_t)i * j.out.st + (int64_t)h * j.out.sh);
    store4<T, VEC>(out, f, dim, s.x, s.y, s.z, s.w);
}

template <typename T, int D, bool VEC>
hipError_t go_join(const JoinJobs &jobs, int dim, hipStream_t st)
{
    if (jobs.n == 0) return hipSuccess;
    const int64_t per = 256 / (D / 4);
    return launch_k(EGERIA_KERNEL_NONE, attention_join_parts_kernel<T, D, VEC>, dim3((unsigned)((jobs.most + per - 1) / per), (unsigned)jobs.n), dim3(256), 0,
                    st, jobs, dim);
}

template <typename T, int D, bool VEC>
hipError_t go_backward(const AttnArgs &a, hipStream_t st)
{
    static bool done_q[kMaxDevices] = {}, done_kv[kMaxDevices] = {};
    const size_t row = (size_t)Tile<T, row_values(D)>::kRowBytes, lut = bias_lut_floats(a);
    const int64_t q_blocks = (int64_t)a.batch * a.heads * ((a.q_len + kRowTile - 1) / kRowTile) * a.q_parts;
    const int64_t k_blocks = (int64_t)a.batch * a.kv_heads * ((a.k_len + kRowTile - 1) / kRowTile) * a.kv_parts + (a.dtable ? a.heads : 0);
    if (q_blocks > 0) {
        const size_t lds = 4 * dq_keys<T, D>() * row + 4 * (lut + (a.partials ? 8 * ((size_t)distance_entries(a.b) + 2 * kPad) : 0));
        hipError_t e = allow_lds(attention_dq_kernel<T, D, VEC>, lds, done_q);
        if (e != hipSuccess) return e;
        e = launch_k(EGERIA_KERNEL_ATTENTION, attention_dq_kernel<T, D, VEC>, dim3((unsigned)q_blocks), dim3(256), lds, st, a);
        if (e != hipSuccess) return e;
    }
    if (k_blocks > 0) {
        const size_t lds = 4 * dkv_queries<D>() * row + (D > 64 ? kRowTile * row : 0) + 4 * lut;
        hipError_t e = allow_lds(attention_dkv_kernel<T, D, VEC>, lds, done_kv);
        if (e != hipSuccess) return e;
        e = launch_k(EGERIA_KERNEL_ATTENTION, attention_dkv_kernel<T, D, VEC>, dim3((unsigned)k_blocks), dim3(256), lds, st, a);
        if (e != hipSuccess) return e;
    }
    JoinJobs jobs;
    const int64_t rows = (int64_t)a.batch * a.heads * a.q_len, keys = (int64_t)a.batch * a.kv_heads * a.k_len;
    jobs.add({a.dq, a.part_q, rows, a.heads, a.q_len, a.q_parts, D, 0});
    jobs.add({a.dk, a.part_kv, keys, a.kv_heads, a.k_len, a.kv_parts, 2 * D, 0});
    jobs.add({a.dv, a.part_kv + D, keys, a.kv_heads, a.k_len, a.kv_parts, 2 * D, 0});
    return go_join<T, D, VEC>(jobs, a.dim, st);
}

}  // namespace

hipError_t launch_join_parts(const JoinJobs &jobs, int dim, egeria_dtype dt, bool vec, hipStream_t st)
{
    const AttnArgs a = {.dim = dim};
    return dt == EGERIA_F32 ? EG_PICK_DIM(go_join, float, vec, a, jobs, dim, st) : EG_PICK_DIM(go_join, uint16_t, vec, a, jobs, dim, st);
}
hipError_t launch_attention_backward(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st) { return EG_PICK(go_backward, a, dt, vec, st); }

}  // namespace egeria
