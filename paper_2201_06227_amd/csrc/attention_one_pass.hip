// Attention backward in one pass, for sequences of few keys (at most 256, heads of at most 64): a workgroup has all keys of a key
// head, a wave 32 of them, and goes through the queries of the head's group.  Per step it forms S, P, dS once, adds to dK and dV as
// the dk / dv kernel does, and leaves dS in LDS, from which its waves make the step's dQ: five products where two kernels need seven, one
// exponential where they need two, and every tensor is read once.  That is what counts at these lengths: 64 x 256 x 12 x 64 in bf16
// has 177 MB of tensors; with a table's gradient two kernels and the sums take 105 us, this one and the table's launch 100; without a table
// 88 and 81.  The reads of keys and dS for dQ (Across) go down rows 4 or 8 apart, which two lanes of a half find on the same banks:
// conflicts take 28 % (bf16) and 37 % (fp32) of the kernel's LDS cycles.
#include "attention.hpp"
#include "attention_diagonals.hpp"

namespace egeria {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

// Fragments of a 16 x 16 x (32 or 16) product from tiles of 64 columns (values) or 128 bytes a row, across the rows: lane l has column
// l % 16; bf16: eight rows from 8 (l / 16) on, fp32: four from 4 (l / 16) on.
template <typename T, int UNITS> struct Across;
template <int UNITS> struct Across<uint16_t, UNITS> {
    static constexpr int kRows = 32;
    typedef Tile<uint16_t, UNITS * 8> tile;
    typedef v8bf frag;
    static __device__ __forceinline__ uint32_t lane_at(uint32_t lds, int lane)
    {
        return lds + tile::at(8 * (lane >> 4) + ((lane & 15) >> 2), (lane & 3) >> 1) + (lane & 1) * 8;
    }
    static __device__ __forceinline__ frag get(uint32_t at, int r0, int cb)
    {
        static_assert(UNITS == 8, "a row of 128 bytes");
        const uint32_t more = (uint32_t)(r0 * tile::kRowBytes);
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(uintptr_t)((at ^ (uint32_t)(cb << 5)) + more));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(uintptr_t)((at ^ (uint32_t)(cb << 5 ^ 32)) + more + 4 * tile::kRowBytes));
        return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
template <int UNITS> struct Across<float, UNITS> {
    static constexpr int kRows = 16;
    typedef Tile<float, UNITS * 4> tile;
    typedef v4f frag;
    static __device__ __forceinline__ uint32_t lane_at(uint32_t lds, int lane)
    {
        const int g = lane >> 4, turned = UNITS == 8 ? (g & 1) << 1 | g >> 1 : g;
        return lds + (uint32_t)(4 * g * tile::kRowBytes + ((((lane & 15) >> 2) ^ turned) << 4) + (lane & 3) * 4);
    }
    static __device__ __forceinline__ frag get(uint32_t at, int r0, int cb)
    {
        v4f f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t unit = (uint32_t)(4 * cb) ^ (uint32_t)(UNITS == 8 ? (e >> 1) << 2 : e << 2);
            f[e] = *(const lds_f32 *)(uintptr_t)((at ^ (unit << 4)) + (uint32_t)((r0 + e) * tile::kRowBytes));
        }
        return f;
    }
};
__device__ __forceinline__ v4f mma16(v8bf a, v8bf b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ v4f mma16(v4f a, v4f b, v4f c)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// LDS of a workgroup: keys, dS of a step, two pairs of query tiles, then the bias and the sums by distance
template <typename T, int WAVES> struct OnePass {
    static constexpr int kQueries = 128 / (int)sizeof(T);           // queries of a step: a row of dS^T has 128 bytes
    typedef Tile<T, 64> tile;
    typedef Tile<T, kQueries> ds_tile;
    static constexpr int kTileBytes = kQueries * tile::kRowBytes, kKeyBytes = 32 * WAVES * tile::kRowBytes, kDsBytes = 32 * WAVES * 128;
    static constexpr int kStage = kKeyBytes + kDsBytes + 4 * kTileBytes;
};

template <typename T, int D, bool VEC, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attention_one_pass_kernel(AttnArgs a)
{
    extern __shared__ __attribute__((aligned(kTileAlign))) char smem[];
    typedef OnePass<T, WAVES> L;
    typedef typename L::tile tile;
    constexpr int kQueries = L::kQueries, kTileBytes = L::kTileBytes, kThreads = 64 * WAVES;
    constexpr int kLanesPerRow = tile::kUnits, kRowsAtOnce = kThreads / kLanesPerRow, kRounds = kQueries / kRowsAtOnce;
    __shared__ float stat[2][2][kQueries];                                  // base-2 log-sum-exp and delta of a step's queries
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the key heads that are left over when every compute unit has had the same number are done in parts
    const int over = (int)blockIdx.x - a.whole, parts = over < 0 ? 1 : a.kv_parts, part = over < 0 ? 0 : over % parts;
    const int bh = over < 0 ? (int)blockIdx.x : a.whole + over / parts, hk = bh % a.kv_heads, b = bh / a.kv_heads;
    const int nq = clamped(a.q_lens, b, a.q_len), nk = clamped(a.k_lens, b, a.k_len), shift = a.causal ? nk - nq : 0;
    const int per_head = nk > 0 ? (nq + kQueries - 1) / kQueries : 0, all = per_head * a.group;
    const int begin = (int)((int64_t)all * part / parts), steps = (int)((int64_t)all * (part + 1) / parts);
    const int chunks = (nk + Across<T, 8>::kRows - 1) / Across<T, 8>::kRows;

    const uint32_t lds = (uint32_t)(uintptr_t)(lds_byte *)smem, lds_ds = lds + L::kKeyBytes, lds_q = lds_ds + L::kDsBytes;
    BiasLut bias;
    bias.open(a, (float *)(smem + L::kStage));
    const int entries = bias.count();
    float *sums = bias.end(), *mine = sums + (2 * wave + half) * entries;  // [wave][half]: sums of ds by distance
    const int jw = 32 * wave, j = jw + (lane & 31);
    const float c = a.scale * kLog2e, sign = sign_of<typename tile::frag>(lane);
    // p and dS are 2^whole times what they should be, and so are all sums of them
    const int whole = nk > 1 ? 31 - __builtin_clz(nk) : 0;
    const float by_p = __uint_as_float((uint32_t)(127 - whole) << 23);

    Feed<T, D, VEC, kQueries, kThreads> qr, gr;
    qr.open(a.q, b, 0, nq, a.dim, tid);
    gr.open(a.d_o, b, 0, nq, a.dim, tid);
    Rows<T, D, VEC> orow;
    orow.open(a.o, b, 0, nq, a.dim);
    const char *q_base = qr.rows.base, *g_base = gr.rows.base, *o_base = orow.base;
    v4u next_g[kRounds], next_o[kRounds];
    float next_lse[kRounds];
    int next_h = hk * a.group + (per_head > 0 ? begin / per_head : 0), next_i = (per_head > 0 ? begin % per_head : 0) * kQueries;                                  // head and first query of the next step to be staged
    int now_h = next_h, now_i = next_i;                                     // of the step at hand
    auto stage = [&](uint32_t to) __attribute__((always_inline)) {
        const int h = next_h, i0 = next_i;
        next_i += kQueries;
        if (next_i >= nq) next_i = 0, ++next_h;
        qr.rows.base = q_base + (int64_t)h * a.q.sh * (int64_t)sizeof(T);
        gr.rows.base = g_base + (int64_t)h * a.d_o.sh * (int64_t)sizeof(T);
        orow.base = o_base + (int64_t)h * a.o.sh * (int64_t)sizeof(T);
        qr.load(to, i0);
        gr.load(to + kTileBytes, i0);
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int i = i0 + r * kRowsAtOnce + tid / kLanesPerRow;
            next_g[r] = gr.rows.unit(i, tid % kLanesPerRow);
            next_o[r] = orow.unit(i, tid % kLanesPerRow);
            next_lse[r] = i < nq ? a.lse[((int64_t)b * a.heads + h) * a.q_len + i] : -INFINITY;
        }
    };
    auto keep = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            float s;
            if constexpr (sizeof(T) == 2) s = dot(__builtin_bit_cast(v8bf, next_g[r]), __builtin_bit_cast(v8bf, next_o[r]));
            else {
                s = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fmaf(__uint_as_float(next_g[r][e]), __uint_as_float(next_o[r][e]), s);
                s += lane_xor<8>(s);
            }
            s += lane_xor<4>(s);
            s += lane_xor<2>(s);
            s += lane_xor<1>(s);
            if (tid % kLanesPerRow == 0) {
                const int row = r * kRowsAtOnce + tid / kLanesPerRow;
                stat[buffer][0][row] = next_lse[r] == -INFINITY ? INFINITY : lowered(next_lse[r], (float)whole);
                stat[buffer][1][row] = s;
            }
        }
    };
    typename tile::frag k[D / 16], v[D / 16];
    v16f dk[D / 32], dv[D / 32];
#pragma unroll
    for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = v16f(0.0f);
    if (begin < steps) {
        Feed<T, D, VEC, 32 * WAVES, kThreads> keys;
        keys.open(a.k, b, hk, nk, a.dim, tid);
        keys.load(lds, 0);
        stage(lds_q);
        Rows<T, D, VEC> kr, vr;
        kr.open(a.k, b, hk, nk, a.dim);
        vr.open(a.v, b, hk, nk, a.dim);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
            k[kk] = kr.frag(jw, kk, lane);
            v[kk] = turned(vr.frag(jw, kk, lane), lane);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        keep(0);
    }
    const typename tile::Lane at = tile::lane_at(lds_q, lane);
    const uint32_t at_k = Across<T, tile::kUnits>::lane_at(lds, lane), at_ds = Across<T, 8>::lane_at(lds_ds, lane);
    double left = 0.0, right = 0.0;                                         // sums of ds beyond the table by distance: long ones, of values that cancel
    int lut_head = -1;
    auto table_sums = [&](int h, int q) { return a.partials + (((int64_t)h * a.batch + b) * a.kv_parts + q) * a.table_rows; };
    auto finish_head = [&](int h) {                                         // the sums by bucket of a head whose queries are done
        left = wave_sum(left);
        right = wave_sum(right);
        if (lane == 0) {
            mine[0] += (float)left;
            mine[entries - 1] += (float)right;
        }
        bucket_sums<kThreads>(bias.spans, sums, 2 * WAVES, entries, entries, a.table_rows, table_sums(h, part), by_p);
        left = right = 0.0;
        __syncthreads();
    };

    auto one_step = [&](auto buffer, int step) __attribute__((always_inline)) {
        constexpr int kBuffer = decltype(buffer)::value;
        constexpr uint32_t now = kBuffer * 2 * kTileBytes, next = 2 * kTileBytes - now;
        const int h = now_h, i0 = now_i;
        now_i += kQueries;
        if (now_i >= nq) now_i = 0, ++now_h;
        if (a.table && h != lut_head) {                                     // the next head of the group
            if (a.partials) {
                if (lut_head >= 0) finish_head(lut_head);
                for (int n = tid; n < 2 * WAVES * entries; n += kThreads) sums[n] = 0.0f;
            }
            bias.read(a, h);
            __syncthreads();
            bias.template fill<kThreads>(a);
            lut_head = h;
        }
        __syncthreads();                                                    // this step's tiles are there; dS has been read
        if (step + 1 < steps) stage(lds_q + next);
        if (jw < nk) {
#pragma unroll
            for (int n = 0; n < kQueries / 32; ++n) {
                const int in = i0 + 32 * n;
                const bool any = in < nq && !(a.causal && jw > in + 31 + shift);
                v16f s = v16f(0.0f), p = v16f(0.0f);
                if (any) {
                    v16f d = v16f(0.0f);
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        s = mma(tile::row_frag(at, now, 32 * n, kk), k[kk], s);
                        d = mma(tile::row_frag(at, now + kTileBytes, 32 * n, kk), v[kk], d);
                    }
                    const int lo = jw - (in + 31) - shift, hi = jw + 31 - in - shift;
                    const bool one = bias.one(lo, hi);
                    const float beta = bias.the_one(hi);
                    const int rel = j - in - 4 * half - shift;
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const float4 base = *(const float4 *)&stat[kBuffer][0][32 * n + row_of(r, half)];
                        const float bs[4] = {base.x, base.y, base.z, base.w};
                        v4f_any t;
                        if (one) t = v4f_any(beta);
                        else t = bias.four(rel - row_of(r, 0) - 3);
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[r + e] = __builtin_amdgcn_exp2f(fmaf(s[r + e], c, t[3 - e] - bs[e]));
                    }
                    // keys at or beyond the length enter dq and the table's sums here; a column of its own in dk and dv
                    if (jw + 32 > nk || (a.causal && hi > 0)) {
                        const int least = j >= nk ? 1 << 30 : (a.causal ? rel : -(1 << 30));
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (row_of(r, 0) < least) p[r] = 0.0f;
                    }
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const float4 delta = *(const float4 *)&stat[kBuffer][1][32 * n + row_of(r, half)];
                        const float ds[4] = {delta.x, delta.y, delta.z, delta.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[r + e] = p[r + e] * fmaf(sign, d[r + e], -ds[e]);
                    }
                    if (a.partials) {
                        if (one) {
                            if (bias.left(hi)) left += (double)sum16(s);
                            else right += (double)sum16(s);
                        } else add_diagonals<-1>(s, mine + (jw - in - shift + bias.far + kPad), lane);
                    }
                }
                // dS^T: the lane's key, four queries at a time
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int q = 32 * n + 8 * g + 4 * half;
                    if constexpr (sizeof(T) == 2) {
                        union { v2u w; __bf16 e[4]; } x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x.e[e] = (__bf16)s[4 * g + e];
                        *(__attribute__((address_space(3))) v2u *)(uintptr_t)(lds_ds + L::ds_tile::at(j, q >> 3) + (q & 7) * 2) = x.w;
                    } else {
                        v4u x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = __float_as_uint(s[4 * g + e]);
                        *(lds_v4u *)(uintptr_t)(lds_ds + L::ds_tile::at(j, q >> 2)) = x;
                    }
                }
                if (any) {
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
            }
        }
        // the next step's tiles, before this step's dq is written: a wait behind those stores would be one for them
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (step + 1 < steps) keep(1 - kBuffer);
        __syncthreads();
        // dQ^T of the step, 16 features of 16 queries at a time, over all keys: a wave's blocks have the same features, so they share
        // the keys' fragments; several chunks of keys are read ahead of their products (one at a time the waits for LDS made this 1.5 us
        // of a step's 5).  bf16 in workgroups of four waves, which have twice the blocks each: two, since with four a wave's registers
        // overflow (200 x 128 x 8 x 64 82 us, now 65).
        constexpr int kWide = D / 16, kBlocks = kWide * (kQueries / 16), kMine = kBlocks > WAVES ? kBlocks / WAVES : 1, kAhead = sizeof(T) == 2 && WAVES == 4 ? 2 : 4;
        const int mb = wave % kWide;
        v4f x[kMine];
#pragma unroll
        for (int t = 0; t < kMine; ++t) x[t] = v4f(0.0f);
        for (int n0 = 0; n0 < chunks && wave < kBlocks; n0 += kAhead) {
            typename Across<T, 8>::frag fk[kAhead], fd[kMine][kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) {
                const int r0 = (n0 + n < chunks ? n0 + n : n0) * Across<T, 8>::kRows;
                fk[n] = Across<T, tile::kUnits>::get(at_k, r0, mb);
#pragma unroll
                for (int t = 0; t < kMine; ++t) fd[t][n] = Across<T, 8>::get(at_ds, r0, (wave + WAVES * t) / kWide);
            }
#pragma unroll
            for (int n = 0; n < kAhead; ++n)
                if (n0 + n < chunks) {
#pragma unroll
                    for (int t = 0; t < kMine; ++t) x[t] = mma16(fk[n], fd[t][n], x[t]);
                }
        }
#pragma unroll
        for (int t = 0; t < kMine; ++t) {
            const int i = i0 + 16 * ((wave + WAVES * t) / kWide) + (lane & 15);
            if (wave < kBlocks && i < nq && i + shift >= 0) {
                T *out = (T *)a.dq.p + ((int64_t)b * a.dq.sb + (int64_t)i * a.dq.st + (int64_t)h * a.dq.sh);
                const float sc = a.scale * by_p;
                store4<T, VEC>(out, 16 * mb + 4 * (lane >> 4), a.dim, x[t][0] * sc, x[t][1] * sc, x[t][2] * sc, x[t][3] * sc);
            }
        }
    };
    for (int step = begin; step < steps; step += 2) {
        one_step(Const<0>(), step);
        if (step + 1 < steps) one_step(Const<1>(), step + 1);
    }
    if (a.partials) {
        __syncthreads();
        if (begin < steps) finish_head(lut_head);
        // heads and parts that have not been written
        const int h0 = hk * a.group, seen0 = begin < steps ? h0 + begin / per_head : h0, seen1 = begin < steps ? lut_head + 1 : h0;
        for (int n = tid; n < a.group * a.table_rows; n += kThreads) {
            const int h = h0 + n / a.table_rows;
            for (int q = part; q < a.kv_parts; q += parts)
                if (q != part || h < seen0 || h >= seen1) table_sums(h, q)[n % a.table_rows] = 0.0f;
        }
    }
    // dq of queries that see no key, which in a step would be sums of 0 times anything
    const int live1 = nk > 0 ? nq : 0, live0 = shift < 0 && nk > 0 ? -shift : 0, none = a.q_len - (live1 - live0);
    for (int64_t n = tid; part == 0 && n < (int64_t)none * a.group * (D / 4); n += kThreads) {
        const int f = (int)(n % (D / 4)) * 4, h = hk * a.group + (int)(n / (D / 4) % a.group), m = (int)(n / (D / 4) / a.group);
        const int i = m < live0 ? m : m + (live1 - live0);
        store4<T, VEC>((T *)a.dq.p + ((int64_t)b * a.dq.sb + (int64_t)i * a.dq.st + (int64_t)h * a.dq.sh), f, a.dim, 0.0f, 0.0f, 0.0f, 0.0f);
    }
    __syncthreads();                                                        // the keys have been read
    if (j >= nk) {                                                          // (columns of their own, and anything may be in them)
#pragma unroll
        for (int n = 0; n < D / 32; ++n) dk[n] = dv[n] = v16f(0.0f);
    }
    if (parts == 1) {
        const uint32_t room = lds + 32 * wave * tile::kRowBytes;
        store_rows<T, D, VEC>(dk, a.scale * by_p, a.dk, b, hk, jw, a.k_len, a.dim, room, lane);
        store_rows<T, D, VEC>(dv, by_p, a.dv, b, hk, jw, a.k_len, a.dim, room, lane);
    } else if (j < a.k_len) {
        const float by = a.scale * by_p;
        float *sum = a.part_kv + (((int64_t)part * (a.batch * a.kv_heads - a.whole) + (bh - a.whole)) * a.k_len + j) * (2 * D);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int f = 32 * n + row_of(r, half);
                *(float4 *)(sum + f) = make_float4(dk[n][r] * by, dk[n][r + 1] * by, dk[n][r + 2] * by, dk[n][r + 3] * by);
                *(float4 *)(sum + D + f) = make_float4(dv[n][r] * by_p, dv[n][r + 1] * by_p, dv[n][r + 2] * by_p, dv[n][r + 3] * by_p);
            }
    }
}

template <typename T, int WAVES>
size_t lds_of(const Buckets *b, bool table_grad)
{
    size_t n = OnePass<T, WAVES>::kStage;
    if (b) n += 4 * (bias_lut_floats(*b) + (table_grad ? 2 * WAVES * ((size_t)distance_entries(*b) + 2 * kPad) : 0));
    return n;
}

template <typename T, int D, bool VEC, int WAVES>
hipError_t go_one_pass(const AttnArgs &a, hipStream_t st)
{
    static bool done[kMaxDevices] = {};
    const size_t lds = lds_of<T, WAVES>(a.table ? &a.b : nullptr, a.partials != nullptr);
    hipError_t e = allow_lds(attention_one_pass_kernel<T, D, VEC, WAVES>, lds, done);
    if (e != hipSuccess) return e;
    const int64_t over = (int64_t)a.batch * a.kv_heads - a.whole;
    e = launch_k(EGERIA_KERNEL_ATTENTION, attention_one_pass_kernel<T, D, VEC, WAVES>, dim3((unsigned)(a.whole + over * a.kv_parts)), dim3(64 * WAVES), lds,
                 st, a);
    if (e != hipSuccess) return e;
    JoinJobs jobs;
    jobs.add({a.dk, a.part_kv, over * a.k_len, a.kv_heads, a.k_len, a.kv_parts, 2 * D, a.whole});
    jobs.add({a.dv, a.part_kv + D, over * a.k_len, a.kv_heads, a.k_len, a.kv_parts, 2 * D, a.whole});
    e = launch_join_parts(jobs, a.dim, sizeof(T) == 4 ? EGERIA_F32 : EGERIA_BF16, VEC, st);
    if (e != hipSuccess || !a.dtable) return e;
    return launch_table_reduce(a.partials, a.heads, a.table_parts, a.table_rows, a.dtable, st);
}

}  // namespace

size_t one_pass_lds(const egeria_attention_desc *d, bool table_grad)
{
    Buckets b = {};
    if (d->bias) b = make_buckets(d->bias);
    const Buckets *p = d->bias ? &b : nullptr;
    if (d->dtype == EGERIA_F32) return d->k_len <= 128 ? lds_of<float, 4>(p, table_grad) : lds_of<float, 8>(p, table_grad);
    return d->k_len <= 128 ? lds_of<uint16_t, 4>(p, table_grad) : lds_of<uint16_t, 8>(p, table_grad);
}

namespace {

template <typename T, int D, bool VEC>
hipError_t go_keys(const AttnArgs &a, hipStream_t st) { return a.k_len <= 128 ? go_one_pass<T, D, VEC, 4>(a, st) : go_one_pass<T, D, VEC, 8>(a, st); }
template <typename T>
hipError_t go_dim(const AttnArgs &a, bool vec, hipStream_t st)
{
    if (a.dim <= 32) return vec ? go_keys<T, 32, true>(a, st) : go_keys<T, 32, false>(a, st);
    return vec ? go_keys<T, 64, true>(a, st) : go_keys<T, 64, false>(a, st);
}

}  // namespace

hipError_t launch_attention_one_pass(const AttnArgs &a, egeria_dtype dt, bool vec, hipStream_t st)
{
    return dt == EGERIA_F32 ? go_dim<float>(a, vec, st) : go_dim<uint16_t>(a, vec, st);
}

}  // namespace egeria
