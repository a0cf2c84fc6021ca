// Gradient of differential attention (jv_diff_attn_bwd): row sums of dO against both outputs, dQ with the rows kept and the keys
// streamed, dK and dV with the keys kept and the rows streamed, and the gradients of lambda's vectors.  Scores are formed again
// in both passes, so no sum needs an atomic and the order of every sum is fixed.
#include <math.h>

#include <algorithm>

#include "jv_diff_attn.h"

namespace jv {

// What both passes need of a query, from the rows of O and P2 V that the forward pass left in the element type
// (P1 V = O + lambda P2 V) and its references and sums: a.stats holds
//     [0], [1]   -log2(denominator of map m) / c, which a score product starts from: the weight is 2^(c sum), 0 in a map without a weight
//     [2]        -D1            [3]   -lambda (D1 - D2),    Dm = rowsum(dO o (Pm V)),
// and for fp32 tensors, whose weights e inv with e = 2^(c score - m) keep the reference m and the sum 1 / inv apart (their logarithm, rounded, would
// cost the weights 2^-24 of its size),
//     [0], [1]   -m1, -m2;      [2], [3]   f1 = inv1, h1 = -D1 inv1;      [4], [5]   f2 = -lambda inv2, h2 = lambda D2 inv2;      [6]   D2:
// dS1 = e1 (f1 dP + h1), dS2 = e2 (f2 dP + h2), P1 - lambda P2 = e1 f1 + e2 f2.
// A row takes as many lanes as it has 16-byte pieces.  Bound by memory: 131 072 rows of 128 in bf16 21 us (101 MB, 4.8 TB/s).
template <typename T, int W>
__global__ void __launch_bounds__(256) diff_attn_rows_kernel(DiffArgs a) {
    constexpr int PER = 16 / (int)sizeof(T), LANES = W / PER;
    const int lane = threadIdx.x & 63;
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int ch = (threadIdx.x % LANES) * PER;
    const bool live = at < diff_rows(a);
    const long long row = live ? at : diff_rows(a) - 1;
    const int bh = (int)((unsigned)row / (unsigned)a.n_q), qi = (int)((unsigned)row - (unsigned)bh * a.n_q), b = (unsigned)bh / (unsigned)a.heads, h = bh - b * a.heads;
    // (rows of a wavefront may belong to two heads and more)
    const float lam = diff_lambda_of<W>(a, __builtin_amdgcn_readfirstlane(bh), __builtin_amdgcn_readlane(bh, 63), bh, lane);
    float d1 = 0.f, d2 = 0.f;
    if (qi < DiffLengths(a, b).q) {
        const u32x4 go = *(const u32x4 *)((const T *)a.d_o.ptr + b * a.d_o.sb + h * a.d_o.sh + qi * a.d_o.sn + ch);
        const u32x4 o = *(const u32x4 *)((const T *)a.o.ptr + b * a.o.sb + h * a.o.sh + qi * a.o.sn + ch);
        const u32x4 o2 = *(const u32x4 *)((const T *)a.o2 + row * W + ch);
        auto add = [&](float x, float y, float y2) {
            d1 = fmaf(x, fmaf(lam, y2, y), d1);
            d2 = fmaf(x, y2, d2);
        };
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                add(bf16_lo(go[e]), bf16_lo(o[e]), bf16_lo(o2[e]));
                add(bf16_hi(go[e]), bf16_hi(o[e]), bf16_hi(o2[e]));
            }
        } else {
            const f32x4 x = __builtin_bit_cast(f32x4, go), y = __builtin_bit_cast(f32x4, o), y2 = __builtin_bit_cast(f32x4, o2);
#pragma unroll
            for (int e = 0; e < 4; ++e) add(x[e], y[e], y2[e]);
        }
    }
#pragma unroll
    for (int x = 1; x < LANES; x *= 2) {
        d1 += __shfl_xor(d1, x);
        d2 += __shfl_xor(d2, x);
    }
    constexpr int STATS = sizeof(T) == 2 ? 4 : 7;
    if (!live || ch >= STATS * PER) return;
    const long long n = diff_rows(a);
    const int which = ch / PER;  // a statistic a lane
    const int map = sizeof(T) == 2 ? which & 1 : which < 2 ? which : which < 4 ? 0 : 1;  // whose reference and sum it is made of
    const float m = qi < DiffLengths(a, b).q ? a.ml[2 * map * n + row] : INFINITY, l = a.ml[(2 * map + 1) * n + row];  // m = +inf: no weight in this map
    float stat;
    if constexpr (sizeof(T) == 2) {
        if (which == 2) stat = -d1;
        else if (which == 3) stat = -lam * (d1 - d2);
        else stat = m == INFINITY ? -INFINITY : -(m + log2f(l)) / a.c;
    } else if (which == 6) {
        stat = d2;
    } else if (m == INFINITY) {
        stat = which < 2 ? -INFINITY : 0.f;
    } else if (which < 2) {
        stat = -m;
    } else {
        const float inv = 1.f / l;
        stat = inv * (which == 2 ? 1.f : which == 3 ? -d1 : which == 4 ? -lam : lam * d2);
    }
    a.stats[which * n + row] = stat;
}

// One of a.parts equal parts of `total`: [from, to).
__device__ inline void diff_part(const DiffArgs &a, int part, int total, int *from, int *to) {
    *from = (unsigned)total * part / (unsigned)a.parts;  // (at most 2^25 tiles and a head's share of one each, 16 parts)
    *to = (unsigned)total * (part + 1) / (unsigned)a.parts;
}

// What the query pass knows of a query: its weights are e inv with e = 2^(c score - m), formed as the forward pass did (DiffScaling; scores have its
// bits: the same operands in the same order), and the gradients of its logits
// dS1 = e1 (dP f1 + h1), dS2 = e2 (dP f2 + h2).
struct DiffRowGrad {
    float minus_m1, minus_m2, f1, h1, f2, h2;
    float c1, c2;  // DiffScaling::then
    float inv2;  // bf16 tensors
    float d2;    // fp32 tensors
    __device__ void load(const DiffArgs &a, long long row, bool sees, float lam) {
        minus_m1 = minus_m2 = -INFINITY;
        f1 = h1 = f2 = h2 = inv2 = 0.f;
        if (!sees) return;
        const long long n = diff_rows(a);
        minus_m1 = -a.ml[row];
        minus_m2 = -a.ml[2 * n + row];
        f1 = minus_m1 == -INFINITY ? 0.f : 1.f / a.ml[n + row];  // (a map without a weight)
        inv2 = minus_m2 == -INFINITY ? 0.f : 1.f / a.ml[3 * n + row];
        const float minus_d1 = a.stats[2 * n + row], lam_d2 = a.stats[3 * n + row] - lam * minus_d1;
        h1 = minus_d1 * f1;
        f2 = -lam * inv2;
        h2 = lam_d2 * inv2;
    }
    __device__ void load_f32(const DiffArgs &a, long long row, bool sees) {
        minus_m1 = minus_m2 = -INFINITY;
        f1 = h1 = f2 = h2 = d2 = 0.f;
        if (!sees) return;
        const long long n = diff_rows(a);
        const float *stat = a.stats + row;
        minus_m1 = stat[0];
        minus_m2 = stat[n];
        f1 = stat[2 * n];
        h1 = stat[3 * n];
        f2 = stat[4 * n];
        h2 = stat[5 * n];
        d2 = stat[6 * n];
    }
};

// dQ of a wavefront's queries, or its part of it, and the workgroup's sum of P2 o dP.  Queries that see no key went along with weights of zero, which
// K and V that are not finite turn into NaN: zeros are written for them.
template <typename T, int W>
__device__ inline void diff_finish_dq(const DiffArgs &a, const f32x16 (&acc)[W / 32], float lam_sum, bool sees, int b, int h, int block, int part, float (&wave_lam)[4], int tid) {
    const int lane = tid & 63, g = lane >> 5, wave = tid >> 6, qi = (block * 4 + wave) * 32 + (lane & 31);
    const long long bh = (long long)b * a.heads + h;
    if (qi < a.n_q) {
        float *partial = a.dq_part + ((long long)part * diff_rows(a) + bh * a.n_q + qi) * W;
        T *dq = (T *)const_cast<void *>(a.dq.ptr) + b * a.dq.sb + h * a.dq.sh + qi * a.dq.sn;
#pragma unroll
        for (int cb = 0; cb < W / 32; ++cb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &x = acc[cb];
                f32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = sees ? x[4 * q4 + e] * a.scale : 0.f;
                const int ch = 32 * cb + 8 * q4 + 4 * g;
                if (a.parts > 1) diff_store4(partial + ch, y);
                else diff_store4(dq + ch, y);
            }
    }
    lam_sum = wave_sum(sees ? lam_sum : 0.f);
    if (lane == 0) wave_lam[wave] = lam_sum;
    __syncthreads();
    if (tid == 0) a.lam_part[(bh * a.blocks + block) * a.parts + part] = (wave_lam[0] + wave_lam[1]) + (wave_lam[2] + wave_lam[3]);
}

// Where a workgroup of the query pass stands: 128 queries of a head, a part of the keys.
struct DiffQueries {
    int part, block, b, h, kv, qi, limit, most, least, tile, tile_end;
    long long row;
    bool row_live;
    __device__ bool find(const DiffArgs &a, int (&wave_most)[4], int wave, int lane) {
        DiffItem item;
        if (!item.find(a, a.B * a.heads, a.parts, true)) return false;
        part = item.part;
        block = item.block;
        const int bh = item.bh;
        b = (unsigned)bh / (unsigned)a.heads;
        h = bh - b * a.heads;
        kv = (unsigned)h / (unsigned)a.group;
        qi = (block * 4 + wave) * 32 + (lane & 31);
        row_live = qi < a.n_q;
        row = (long long)bh * a.n_q + qi;
        const DiffLengths len(a, b);
        limit = row_live ? len.limit(a, qi) : 0;
        most = limit;
        least = limit > 0 ? limit : a.n_k + kDiffTile;  // (rows without a key have weights of zero without a mask)
#pragma unroll
        for (int x = 1; x < 32; x *= 2) {
            most = max(most, __shfl_xor(most, x));
            least = min(least, __shfl_xor(least, x));
        }
        if (lane == 0) wave_most[wave] = most;
        __syncthreads();
        most = __builtin_amdgcn_readfirstlane(max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3])));
        least = __builtin_amdgcn_readfirstlane(least);
        diff_part(a, part, (most + kDiffTile - 1) / kDiffTile, &tile, &tile_end);
        return true;
    }
};

// Scores and dP of a tile (rows: keys) become the gradients of the logits, in place; returns the lane's sum of e2 dP.
// For lambda, bf16 tensors add these up, tile by tile (one sum over 2 048 products was off four times as far): their D2 holds the rounding of P2 V's
// weights and rows, which shows in a sum of so many signs.  fp32 tensors add up D2 (diff_attn_dq_f32_kernel).
__device__ inline float diff_logit_grads(f32x16 &s1, f32x16 &s2, const f32x16 &dp, const DiffRowGrad &r, float c, bool far) {
    float sum = 0.f;
    if (far) {  // in place: without the branch's two outcomes side by side in registers
        const DiffScaling to1(c, diff_far(r.minus_m1)), to2(c, diff_far(r.minus_m2));
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            s1[v] *= to1.first;
            s2[v] *= to2.first;
        }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const float e1 = __builtin_amdgcn_exp2f(fmaf(s1[v], r.c1, r.minus_m1)), e2 = __builtin_amdgcn_exp2f(fmaf(s2[v], r.c2, r.minus_m2));
        sum = fmaf(e2, dp[v], sum);
        s1[v] = e1 * fmaf(dp[v], r.f1, r.h1);
        s2[v] = e2 * fmaf(dp[v], r.f2, r.h2);
    }
    return sum;
}
// dQ, and the sums of P2 o dP (for lambda): a wavefront keeps 32 queries of one head, their dO and their dQ, and walks the keys.
// A tile takes W / 16 score products, as many of V with dO, and as many of K^T with the gradients of the logits.  Tiles come straight
// into two LDS stages, the next tile's under this one's arithmetic.  Bound by the issue of matrix and vector instructions: 4 x 4 096 tokens x 8 heads of
// 128 465 us (0.89 PFLOP/s).
template <int W>
__global__ void __launch_bounds__(256, 2) diff_attn_dq_bf16_kernel(DiffArgs a) {
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = kDiffTile * 2 * W, STAGE = 2 * TILE;  // a stage: K rows, then V rows
    __shared__ __align__(1024) unsigned char smem[2 * STAGE];
    __shared__ int wave_most[4];
    __shared__ float wave_lam[4];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffQueries p;
    if (!p.find(a, wave_most, wave, lane)) return;  // whole workgroup
    const int len_k = DiffLengths(a, p.b).k;
    DiffDma<W, 4> kload, vload;
    kload.start(a.k.ptr, p.b * a.k.sb + p.kv * a.k.sh, a.k.sn, wave, lane);
    vload.start(a.v.ptr, p.b * a.v.sb + p.kv * a.v.sh, a.v.sn, wave, lane);
    auto issue = [&](int t, int stage) {
        kload.issue(smem + stage * STAGE, t * kDiffTile, len_k, wave, lane);
        vload.issue(smem + stage * STAGE + TILE, t * kDiffTile, len_k, wave, lane);
    };
    int tile = p.tile;
    if (tile < p.tile_end) issue(tile, 0);
    const float lam = diff_lambda<W>(a, p.h, lane).value;
    bf16x8 q[2 * KS], go[2 * KS];
    DiffRowGrad r;
    {
        const int at = p.row_live ? p.qi : 0;
        const __bf16 *row = (const __bf16 *)a.q.ptr + p.b * a.q.sb + p.h * a.q.sh + at * a.q.sn;
        const __bf16 *grow = (const __bf16 *)a.d_o.ptr + p.b * a.d_o.sb + p.h * a.d_o.sh + at * a.d_o.sn;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) {
            q[ks] = diff_global_frag(row, ks, g, p.limit > 0);
            go[ks] = diff_global_frag(grow, ks, g, p.limit > 0);
        }
        r.load(a, p.row, p.limit > 0, lam);
    }
    // Every other query works with -dO and -dP: the matrix unit's sums lie a little low (2e-10 of their terms), whatever their sign, which the sums for
    // lambda would add up over all queries and heads.
    if (lane & 1) {
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) go[ks] = as_bf16x8(as_u32x4(go[ks]) ^ 0x80008000u);
        r.f1 = -r.f1;
        r.f2 = -r.f2;
        r.inv2 = -r.inv2;
    }
#pragma unroll
    for (int ks = 0; ks < 2 * KS; ++ks) asm volatile("" : "+v"(q[ks]), "+v"(go[ks]));  // (waited for here, not inside the loop)
    asm volatile("" : "+v"(r.minus_m1), "+v"(r.minus_m2), "+v"(r.f1), "+v"(r.h1), "+v"(r.f2), "+v"(r.h2), "+v"(r.inv2));
    const bool far = __builtin_amdgcn_ballot_w64(diff_far(r.minus_m1) || diff_far(r.minus_m2)) != 0;
    r.c1 = DiffScaling(a.c, diff_far(r.minus_m1)).then;
    r.c2 = DiffScaling(a.c, diff_far(r.minus_m2)).then;
    f32x16 acc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) diff_zero(acc[cb]);
    float lam_sum = 0.f;
    const unsigned rows0 = Lds::rows(lds_address(smem), lane), cols0 = Lds::cols(lds_address(smem), lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    for (int stage = 0; tile < p.tile_end; ++tile, stage ^= 1) {
        if (tile + 1 < p.tile_end) issue(tile + 1, stage ^ 1);
        const unsigned rows = rows0 + stage * STAGE, cols = cols0 + stage * STAGE;
        f32x16 s1, s2, dp;
        diff_zero(s1);
        diff_zero(s2);
        diff_zero(dp);
        u32x4 x[KS], y[KS];
        Lds::template read_rows<0>(x, rows, 0);
        diff_landed(x);
        Lds::template read_rows<0>(y, rows, KS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s1 = mfma32(as_bf16x8(x[ks]), q[ks], s1);
        diff_landed(y);
        Lds::template read_rows<TILE>(x, rows, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s2 = mfma32(as_bf16x8(y[ks]), q[KS + ks], s2);
        diff_landed(x);
        Lds::template read_rows<TILE>(y, rows, KS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma32(as_bf16x8(x[ks]), go[ks], dp);
        diff_landed(y);
        u32x2 c0[2 * CB];
        Lds::template read_cols<0, 0>(c0, cols);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) dp = mfma32(as_bf16x8(y[ks]), go[KS + ks], dp);
        if ((tile + 1) * kDiffTile > p.least) diff_hide_keys(s1, s2, tile * kDiffTile, p.limit > 0 ? p.limit : a.n_k + kDiffTile, g);
        lam_sum += diff_logit_grads(s1, s2, dp, r, a.c, far);
        bf16x8 ds1[2], ds2[2];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            ds1[kk] = diff_block_frag(s1, kk);
            ds2[kk] = diff_block_frag(s2, kk);
        }
        diff_landed(c0);
        u32x2 c1[2 * CB];
        Lds::template read_cols<0, 1>(c1, cols);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] = mfma32(diff_join2(c0[2 * cb], c0[2 * cb + 1]), cb < CB / 2 ? ds1[0] : ds2[0], acc[cb]);
        diff_landed(c1);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] = mfma32(diff_join2(c1[2 * cb], c1[2 * cb + 1]), cb < CB / 2 ? ds1[1] : ds2[1], acc[cb]);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile, for every wavefront, and every wavefront done with this one
        lds_barrier();
    }
    asm("" : "+v"(lam_sum));
    diff_finish_dq<__bf16, W>(a, acc, lam_sum * r.inv2, p.limit > 0, p.b, p.h, p.block, p.part, wave_lam, tid);
}

// The same for fp32 tensors, on operands of three bf16 numbers.  For lambda D2 is added up, once a row: the matrix unit's dP, a sum of so many small
// terms, lies a little low whatever its sign (1e-8 of its size), and Sum P2 o dP, where signs cancel, was 1e-4 off at 4 096 tokens through it.
// 2 x 1 024 tokens x 8 heads of 128 87 us (0.89 PFLOP/s of bf16 products), 2 x 576 x 12 of 64 32 us.
template <int W>
__global__ void __launch_bounds__(256, 1) diff_attn_dq_f32_kernel(DiffArgs a) {
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = DiffTile<W>::kBytes, STAGE = 6 * TILE;  // a stage: three planes of K rows, three of V rows
    __shared__ __align__(1024) unsigned char smem[2 * STAGE];
    __shared__ int wave_most[4];
    __shared__ float wave_lam[4];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffQueries p;
    if (!p.find(a, wave_most, wave, lane)) return;  // whole workgroup
    const int len_k = DiffLengths(a, p.b).k;
    DiffDma3<W, 4> kload, vload;
    kload.start(a.planes[1], ((long long)p.b * a.kv_heads + p.kv) * a.n_k, wave, lane);
    vload.start(a.planes[2], ((long long)p.b * a.kv_heads + p.kv) * a.n_k, wave, lane);
    auto issue = [&](int t, int stage) {
        kload.issue(smem + stage * STAGE, t * kDiffTile, len_k, wave, lane);
        vload.issue(smem + stage * STAGE + 3 * TILE, t * kDiffTile, len_k, wave, lane);
    };
    int tile = p.tile;
    if (tile < p.tile_end) issue(tile, 0);
    DiffPlanes q[2 * KS], go[2 * KS];
    DiffRowGrad r;
    {
        const long long at = (p.row_live ? p.row : 0) * 3 * W;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) {
            q[ks] = diff_global_planes<W>(a.planes[0] + at, ks, g, p.limit > 0);
            go[ks] = diff_global_planes<W>(a.planes[3] + at, ks, g, p.limit > 0);
        }
        r.load_f32(a, p.row, p.limit > 0);
    }
#pragma unroll
    for (int ks = 0; ks < 2 * KS; ++ks)  // (waited for here, not inside the loop)
        asm volatile("" : "+v"(q[ks].x[0]), "+v"(q[ks].x[1]), "+v"(q[ks].x[2]), "+v"(go[ks].x[0]), "+v"(go[ks].x[1]), "+v"(go[ks].x[2]));
    asm volatile("" : "+v"(r.minus_m1), "+v"(r.minus_m2), "+v"(r.f1), "+v"(r.h1), "+v"(r.f2), "+v"(r.h2), "+v"(r.d2));
    const bool far = __builtin_amdgcn_ballot_w64(diff_far(r.minus_m1) || diff_far(r.minus_m2)) != 0;
    r.c1 = DiffScaling(a.c, diff_far(r.minus_m1)).then;
    r.c2 = DiffScaling(a.c, diff_far(r.minus_m2)).then;
    f32x16 acc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) diff_zero(acc[cb]);
    const unsigned rows0 = Lds::rows(lds_address(smem), lane), cols0 = Lds::cols(lds_address(smem), lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    for (int stage = 0; tile < p.tile_end; ++tile, stage ^= 1) {
        if (tile + 1 < p.tile_end) issue(tile + 1, stage ^ 1);
        const unsigned rows = rows0 + stage * STAGE, cols = cols0 + stage * STAGE;
        f32x16 s1, s2, dp;
        diff_zero(s1);
        diff_zero(s2);
        diff_zero(dp);
        {
            u32x4 x[2][3];
            diff_read_rows3<W, 0>(x[0], rows, 0);
            diff_landed(x[0]);
#pragma unroll
            for (int i = 0; i < 4 * KS; ++i) {  // K operands, then V operands
                if (i + 1 < 2 * KS) diff_read_rows3<W, 0>(x[(i + 1) & 1], rows, i + 1);
                else if (i + 1 < 4 * KS) diff_read_rows3<W, 3 * TILE>(x[(i + 1) & 1], rows, i + 1 - 2 * KS);
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 k[3];
                diff_rows3(x[i & 1], k);
                if (i < KS) s1 = diff_mma6(k, q[i < KS ? i : 0].x, s1);
                else if (i < 2 * KS) s2 = diff_mma6(k, q[i < 2 * KS ? i : 0].x, s2);
                else dp = diff_mma6(k, go[i < 2 * KS ? 0 : i - 2 * KS].x, dp);
                if (i + 1 < 4 * KS) diff_landed(x[(i + 1) & 1]);
            }
        }
        u32x2 v[2][6];
        diff_read_cols3<W, 0, 0>(v[0], cols, 0);
        __builtin_amdgcn_sched_barrier(0);
        if ((tile + 1) * kDiffTile > p.least) diff_hide_keys(s1, s2, tile * kDiffTile, p.limit > 0 ? p.limit : a.n_k + kDiffTile, g);
        diff_logit_grads(s1, s2, dp, r, a.c, far);
        diff_landed(v[0]);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const DiffPlanes ds1 = diff_block_planes(s1, kk), ds2 = diff_block_planes(s2, kk);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const int i = kk * CB + cb;
                if (i + 1 < CB) diff_read_cols3<W, 0, 0>(v[(i + 1) & 1], cols, i + 1);
                else if (i + 1 < 2 * CB) diff_read_cols3<W, 0, 1>(v[(i + 1) & 1], cols, i + 1 - CB);
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 x[3];
                diff_cols3(v[i & 1], x);
                acc[cb] = diff_mma6(x, cb < CB / 2 ? ds1.x : ds2.x, acc[cb]);
                if (i + 1 < 2 * CB) diff_landed(v[(i + 1) & 1]);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile, for every wavefront, and every wavefront done with this one
        lds_barrier();
    }
    diff_finish_dq<float, W>(a, acc, p.part == 0 && g == 0 ? r.d2 : 0.f, p.limit > 0, p.b, p.h, p.block, p.part, wave_lam, tid);
}

// Where a workgroup of the key pass stands: 128 keys of a kv head; the tiles of its group's heads, one head after the other, of
// which it takes a part.
struct DiffKeys {
    int part, block, b, kv, key, shift, first_query, tile_begin, n_tiles, from, to, len_q, len_k;
    __device__ bool find(const DiffArgs &a, int wave, int lane) {
        DiffItem item;
        if (!item.find(a, a.B * a.kv_heads, a.parts, false)) return false;
        part = item.part;
        block = item.block;
        const int bkv = item.bh;
        b = (unsigned)bkv / (unsigned)a.kv_heads;
        kv = bkv - b * a.kv_heads;
        const DiffLengths len(a, b);
        len_q = len.q;
        len_k = len.k;
        const int key0 = block * 128;
        key = key0 + wave * 32 + (lane & 31);
        // causal: the first query that sees key x is x - (keys - queries)
        shift = a.causal ? len_k - len_q : 0;
        first_query = a.causal ? key0 + wave * 32 - shift : 0;
        tile_begin = a.causal ? max(key0 - shift, 0) / kDiffTile : 0;
        n_tiles = key0 < len_k ? max((len_q + kDiffTile - 1) / kDiffTile - tile_begin, 0) : 0;
        diff_part(a, part, n_tiles * a.group, &from, &to);
        return true;
    }
    // Masks of a tile whose rows are queries: those behind the last one, and, causal, those that do not see the lane's key.
    __device__ bool masked(const DiffArgs &a, int tile) const { return (tile + 1) * kDiffTile > len_q || (a.causal && tile * kDiffTile < first_query + 31); }
    __device__ void hide(const DiffArgs &a, f32x16 &s1, f32x16 &s2, int tile, int g) const {
        const int from_query = a.causal ? key - shift : 0;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const int qi = tile * kDiffTile + 8 * (x / 4) + 4 * g + x % 4;
            const bool hidden = qi < from_query || qi >= len_q;
            s1[x] = hidden ? -INFINITY : s1[x];
            s2[x] = hidden ? -INFINITY : s2[x];
        }
    }
};

// dK and dV of a wavefront's keys, or its part of them: zeros behind the last key.
template <typename T, int W>
__device__ inline void diff_finish_dkv(const DiffArgs &a, const f32x16 (&dk)[W / 32], const f32x16 (&dv)[W / 32], const DiffKeys &p, int g) {
    if (p.key >= a.n_k) return;
    const bool live = p.key < p.len_k;
    T *krow = (T *)const_cast<void *>(a.dk.ptr) + p.b * a.dk.sb + p.kv * a.dk.sh + p.key * a.dk.sn;
    T *vrow = (T *)const_cast<void *>(a.dv.ptr) + p.b * a.dv.sb + p.kv * a.dv.sh + p.key * a.dv.sn;
    float *partial = a.dkv_part + (((long long)p.part * a.B * a.kv_heads + p.b * a.kv_heads + p.kv) * a.n_k + p.key) * (2 * W);
#pragma unroll
    for (int cb = 0; cb < W / 32; ++cb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int ch = 32 * cb + 8 * q4 + 4 * g;
            f32x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = live ? dk[cb][4 * q4 + e] * a.scale : 0.f;
                y[e] = live ? dv[cb][4 * q4 + e] : 0.f;
            }
            if (a.parts > 1) {
                diff_store4(partial + ch, x);
                diff_store4(partial + W + ch, y);
            } else {
                diff_store4(krow + ch, x);
                diff_store4(vrow + ch, y);
            }
        }
}

// Row x of a block: the score (which started from the stored logarithm) of both maps, dP - D1 and -lambda (D1 - D2) become the
// gradients of the logits and P1 - lambda P2.
__device__ inline void diff_weights_and_grads(f32x16 &s1, f32x16 &s2, f32x16 &dp, int x, float minus_lam_d, float c, float lam) {
    const float p1 = __builtin_amdgcn_exp2f(s1[x] * c), p2 = __builtin_amdgcn_exp2f(s2[x] * c);
    s1[x] = p1 * dp[x];
    s2[x] = p2 * fmaf(-lam, dp[x], minus_lam_d);
    dp[x] = fmaf(-lam, p2, p1);
}

// dK and dV: a wavefront keeps 32 keys of one kv head and both gradients, and walks the queries of the group's heads.  What
// lengths hide is the columns of keys behind the last, which are thrown away, and the rows of queries behind the last.
// K operands stay in registers, V in LDS (with both gradients, 4 W / 32 accumulators of 16 registers, there
// is no room for it at two wavefronts a SIMD); tiles of Q and dO and the queries' statistics come straight into two LDS stages, the
// next tile's under this one's arithmetic.  Score products start from the stored logarithms and dP from -D1, read from LDS into the
// accumulators.  LDS gives 40 + 16 KB a tile and wavefront for 4 W / 16 matrix instructions.
// Bound by issue, as the query pass: 4 x 4 096 tokens x 8 heads of 128 625 us (0.88 PFLOP/s), without loads 527, without barriers too 511, without
// the reads of statistics 501.  The offsets of the loads are worked out for every tile in rows of 128: held, two of them came from scratch memory,
// and a wait for scratch memory is one for the tile loads in flight (688 us).
template <int W>
__global__ void __launch_bounds__(256, 2) diff_attn_dkv_bf16_kernel(DiffArgs a) {
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = kDiffTile * 2 * W, STATS = 4 * kDiffTile * 4, STAGE = 2 * TILE + 1024;  // Q rows, dO rows, statistics
    static_assert(STATS <= 1024, "stages stay 1 KB aligned");
    __shared__ __align__(1024) unsigned char smem[2 * STAGE + 4 * TILE];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffKeys p;
    if (!p.find(a, wave, lane)) return;  // whole workgroup
    unsigned char *vt = smem + 2 * STAGE + wave * TILE;  // the wavefront's own values
    DiffDma<W, 4, W == 64> qload, gload;
    int next_tile = p.tile_begin, next_head = p.kv * a.group;
    if (p.n_tiles) {
        next_head += p.from / p.n_tiles;
        next_tile += p.from % p.n_tiles;
    }
    qload.start(a.q.ptr, p.b * a.q.sb + next_head * a.q.sh, a.q.sn, wave, lane);
    gload.start(a.d_o.ptr, p.b * a.d_o.sb + next_head * a.d_o.sh, a.d_o.sn, wave, lane);
    // Loads of the next tile into a stage, and on to the one after.
    auto issue = [&](int stage) {
        unsigned char *to = smem + stage * STAGE;
        const int row0 = next_tile * kDiffTile;
        qload.issue(to, row0, p.len_q, wave, lane);
        gload.issue(to + TILE, row0, p.len_q, wave, lane);
        if (wave < 2) {  // statistics 2 wave and 2 wave + 1
            const char *from = diff_uniform(a.stats + 2 * wave * diff_rows(a) + ((long long)p.b * a.heads + next_head) * a.n_q + row0);
            const long long other = diff_rows(a) * 4;
            const unsigned at = 4 * min(lane & 31, p.len_q - 1 - row0);
            __builtin_amdgcn_global_load_lds((diff_global_cvoid *)(from + (lane >> 5) * other + at), (diff_lds_void *)(to + 2 * TILE + wave * 256), 4, 0, 0);
        }
        if (++next_tile == p.tile_begin + p.n_tiles) {
            next_tile = p.tile_begin;
            ++next_head;
            qload.base += 2 * a.q.sh;
            gload.base += 2 * a.d_o.sh;
        }
    };
    u32x4 k[2 * KS];
    if (p.from < p.to) {
        DiffDma<W, 1> vload;
        const int key0 = p.block * 128 + wave * 32;
        vload.start(a.v.ptr, p.b * a.v.sb + p.kv * a.v.sh, a.v.sn, 0, lane);
        if (key0 < p.len_k) vload.issue(vt, key0, p.len_k, 0, lane);
        const bool live = p.key < p.len_k;
        const __bf16 *row = (const __bf16 *)a.k.ptr + p.b * a.k.sb + p.kv * a.k.sh + (live ? p.key : 0) * a.k.sn;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) k[ks] = as_u32x4(diff_global_frag(row, ks, g, live));
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) asm volatile("" : "+v"(k[ks]));  // (waited for here, not inside the loop)
        issue(0);
    }
    f32x16 dk[CB], dv[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        diff_zero(dk[cb]);
        diff_zero(dv[cb]);
    }
    const unsigned rows0 = Lds::rows(lds_address(smem), lane), cols0 = Lds::cols(lds_address(smem), lane), stats0 = lds_address(smem) + 2 * TILE + 16 * g;
    const unsigned vrows = Lds::rows(lds_address(vt), lane);
    float lam = 0.f;
    int tile = 0, left = 0, head = 0;  // tiles left of the present head
    if (p.n_tiles) {
        head = p.kv * a.group + p.from / p.n_tiles;
        tile = p.tile_begin + p.from % p.n_tiles;
        left = p.n_tiles - p.from % p.n_tiles;
        lam = diff_lambda<W>(a, head, lane).value;
    }
    lam = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, lam)));
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    for (int at = p.from, stage = 0; at < p.to; ++at, stage ^= 1) {
        if (at + 1 < p.to) issue(stage ^ 1);
        const unsigned rows = rows0 + stage * STAGE, cols = cols0 + stage * STAGE, stats = stats0 + stage * STAGE;
        auto read_stats = [&](u32x4 (&to)[4], auto which) {
            constexpr int at0 = decltype(which)::value * kDiffTile * 4;
            to[0] = lds_read_b128_at<at0>(stats);
            to[1] = lds_read_b128_at<at0 + 32>(stats);
            to[2] = lds_read_b128_at<at0 + 64>(stats);
            to[3] = lds_read_b128_at<at0 + 96>(stats);
        };
        f32x16 s1, s2, dp;
        {
            u32x4 i1[4], i2[4], x[KS], y[KS];
            read_stats(i1, std::integral_constant<int, 0>());
            Lds::template read_rows<0>(x, rows, 0);
            diff_landed(i1, x);
            read_stats(i2, std::integral_constant<int, 1>());
            Lds::template read_rows<0>(y, rows, KS);
            __builtin_amdgcn_sched_barrier(0);
            s1 = diff_join4(i1);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s1 = mfma32(as_bf16x8(x[ks]), as_bf16x8(k[ks]), s1);
            diff_landed(i2, y);
            s2 = diff_join4(i2);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s2 = mfma32(as_bf16x8(y[ks]), as_bf16x8(k[KS + ks]), s2);
        }
        __builtin_amdgcn_sched_barrier(0);
        {
            u32x4 i3[4], x[2], v[2];
            read_stats(i3, std::integral_constant<int, 2>());
#pragma unroll
            for (int ks = 0; ks < 2 * KS; ks += 2) {  // two operands of each at a time: more would not fit the registers
                x[0] = lds_read_b128_at<TILE>(rows ^ 32 * ks);
                x[1] = lds_read_b128_at<TILE>(rows ^ 32 * (ks + 1));
                v[0] = lds_read_b128_at<0>(vrows ^ 32 * ks);
                v[1] = lds_read_b128_at<0>(vrows ^ 32 * (ks + 1));
                if (ks == 0) {
                    diff_landed(i3, x, v);
                    dp = diff_join4(i3);
                } else {
                    diff_landed(x, v);
                }
                dp = mfma32(as_bf16x8(x[0]), as_bf16x8(v[0]), dp);
                dp = mfma32(as_bf16x8(x[1]), as_bf16x8(v[1]), dp);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        u32x4 init[4];
        read_stats(init, std::integral_constant<int, 3>());
        __builtin_amdgcn_sched_barrier(0);
        if (p.masked(a, tile)) p.hide(a, s1, s2, tile, g);
        diff_landed(init);
        {
            const f32x16 minus_lam_d = diff_join4(init);
#pragma unroll
            for (int e = 0; e < 16; ++e) diff_weights_and_grads(s1, s2, dp, e, minus_lam_d[e], a.c, lam);
        }
        bf16x8 w[2], ds1[2], ds2[2];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            w[kk] = diff_block_frag(dp, kk);
            ds1[kk] = diff_block_frag(s1, kk);
            ds2[kk] = diff_block_frag(s2, kk);
        }
        u32x2 c0[2 * CB], c1[2 * CB];
        Lds::template read_cols<TILE, 0>(c0, cols);
        diff_landed(c0);
        Lds::template read_cols<TILE, 1>(c1, cols);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) dv[cb] = mfma32(diff_join2(c0[2 * cb], c0[2 * cb + 1]), w[0], dv[cb]);
        diff_landed(c1);
        Lds::template read_cols<0, 0>(c0, cols);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) dv[cb] = mfma32(diff_join2(c1[2 * cb], c1[2 * cb + 1]), w[1], dv[cb]);
        diff_landed(c0);
        Lds::template read_cols<0, 1>(c1, cols);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) dk[cb] = mfma32(diff_join2(c0[2 * cb], c0[2 * cb + 1]), cb < CB / 2 ? ds1[0] : ds2[0], dk[cb]);
        diff_landed(c1);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) dk[cb] = mfma32(diff_join2(c1[2 * cb], c1[2 * cb + 1]), cb < CB / 2 ? ds1[1] : ds2[1], dk[cb]);
        ++tile;
        if (--left == 0 && at + 1 < p.to) {  // on to the group's next head (uniform)
            tile = p.tile_begin;
            left = p.n_tiles;
            lam = diff_lambda<W>(a, ++head, lane).value;
            lam = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, lam)));
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile, for every wavefront, and every wavefront done with this one
        lds_barrier();
    }
    diff_finish_dkv<__bf16, W>(a, dk, dv, p, g);
}

// The same for fp32 tensors, on operands of three bf16 numbers: K and V in registers, but for the last plane of V in rows of 128, which
// lies in LDS (2 x 1 024 tokens x 8 heads of 128 120 us, 0.86 PFLOP/s of bf16 products; in registers, 41 of which lay in scratch memory, 134); one
// wavefront a SIMD.  2 x 576 tokens x 12 of 64 43 us: nine tiles a wavefront, each one chain of reads, products and splits.
template <int W>
__global__ void __launch_bounds__(256, 1) diff_attn_dkv_f32_kernel(DiffArgs a) {
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = DiffTile<W>::kBytes, STATS = 6 * kDiffTile * 4, STAGE = 6 * TILE + 1024;  // Q planes, dO planes, statistics
    static_assert(STATS <= 1024, "stages stay 1 KB aligned");
    constexpr bool LAST = W == 128;  // the last plane of V in LDS
    __shared__ __align__(1024) unsigned char smem[2 * STAGE + (LAST ? 4 * TILE : 0)];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffKeys p;
    if (!p.find(a, wave, lane)) return;  // whole workgroup
    int head = p.kv * a.group, tile = p.tile_begin;
    if (p.n_tiles) {
        head += p.from / p.n_tiles;
        tile += p.from % p.n_tiles;
    }
    DiffDma3<W, 4, W == 64> qload, gload;
    int next_tile = tile, next_head = head;
    qload.start(a.planes[0], ((long long)p.b * a.heads + head) * a.n_q, wave, lane);
    gload.start(a.planes[3], ((long long)p.b * a.heads + head) * a.n_q, wave, lane);
    // Loads of the next tile into a stage, and on to the one after.
    auto issue = [&](int stage) {
        unsigned char *to = smem + stage * STAGE;
        const int row0 = next_tile * kDiffTile;
        qload.issue(to, row0, p.len_q, wave, lane);
        gload.issue(to + 3 * TILE, row0, p.len_q, wave, lane);
        if (wave < 3) {  // statistics 2 wave and 2 wave + 1
            const char *from = diff_uniform(a.stats + 2 * wave * diff_rows(a) + ((long long)p.b * a.heads + next_head) * a.n_q + row0);
            const long long other = diff_rows(a) * 4;
            int l = lane;
            if (LAST) asm volatile("" : "+v"(l));  // (worked out here: kept, it would come from scratch memory)
            const unsigned at = 4 * min(l & 31, p.len_q - 1 - row0);
            __builtin_amdgcn_global_load_lds((diff_global_cvoid *)(from + (l >> 5) * other + at), (diff_lds_void *)(to + 6 * TILE + wave * 256), 4, 0, 0);
        }
        if (++next_tile == p.tile_begin + p.n_tiles) {
            next_tile = p.tile_begin;
            ++next_head;
            qload.one.base += 6ll * W * a.n_q;
            gload.one.base += 6ll * W * a.n_q;
        }
    };
    unsigned char *vt = smem + 2 * STAGE + wave * TILE;
    const int key0 = p.block * 128 + wave * 32;
    if (p.from < p.to) {
        if (LAST && key0 < p.len_k) {
            DiffDma<W, 1> vload;
            vload.start(a.planes[2], (((long long)p.b * a.kv_heads + p.kv) * a.n_k * 3 + 2) * W, 3 * W, 0, lane);
            vload.issue(vt, key0, p.len_k, 0, lane);
        }
        issue(0);
    }
    DiffPlanes k[2 * KS], v[2 * KS];
    {
        const bool live = p.key < p.len_k;
        const long long at = (((long long)p.b * a.kv_heads + p.kv) * a.n_k + (live ? p.key : 0)) * 3 * W;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) {
            k[ks] = diff_global_planes<W>(a.planes[1] + at, ks, g, live);
            v[ks] = diff_global_planes<W>(a.planes[2] + at, ks, g, live);
        }
    }
#pragma unroll
    for (int ks = 0; ks < 2 * KS; ++ks) {  // (waited for here, not inside the loop)
        asm volatile("" : "+v"(k[ks].x[0]), "+v"(k[ks].x[1]), "+v"(k[ks].x[2]), "+v"(v[ks].x[0]), "+v"(v[ks].x[1]));
        if (!LAST) asm volatile("" : "+v"(v[ks].x[2]));
    }
    f32x16 dk[CB], dv[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        diff_zero(dk[cb]);
        diff_zero(dv[cb]);
    }
    const unsigned rows0 = Lds::rows(lds_address(smem), lane), cols0 = Lds::cols(lds_address(smem), lane), stats0 = lds_address(smem) + 6 * TILE + 16 * g, refs0 = lds_address(smem) + 6 * TILE + 4 * lane;
    const unsigned vrows = Lds::rows(lds_address(vt), lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    for (int at = p.from, stage = 0; at < p.to; ++at, stage ^= 1) {
        if (!LAST && at + 1 < p.to) issue(stage ^ 1);
        const unsigned rows = rows0 + stage * STAGE, cols = cols0 + stage * STAGE, stats = stats0 + stage * STAGE;
        f32x16 s1, s2, dp;
        bool far;  // any of the references of the tile's queries, the first two rows of statistics: all of its products are rounded then (DiffScaling)
        diff_zero(s1);
        diff_zero(s2);
        diff_zero(dp);
        {
            u32x4 x[2][3], last[2];
            unsigned ref;
            diff_read_rows3<W, 0>(x[0], rows, 0);
            asm volatile("ds_read_b32 %0, %1" : "=v"(ref) : "v"(refs0 + stage * STAGE));
            diff_landed(x[0], ref);
            far = __builtin_amdgcn_ballot_w64(diff_far(__builtin_bit_cast(float, ref))) != 0;
#pragma unroll
            for (int i = 0; i < 4 * KS; ++i) {  // Q operands, then dO operands
                const int next = (i + 1) & 1;
                if (i + 1 < 2 * KS) diff_read_rows3<W, 0>(x[next], rows, i + 1);
                else if (i + 1 < 4 * KS) {
                    diff_read_rows3<W, 3 * TILE>(x[next], rows, i + 1 - 2 * KS);
                    if (LAST) last[next] = lds_read_b128_at<0>(vrows ^ 32 * (i + 1 - 2 * KS));
                }
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 q[3];
                diff_rows3(x[i & 1], q);
                if (i < KS) s1 = diff_mma6_swapped(q, k[i < KS ? i : 0].x, s1);
                else if (i < 2 * KS) s2 = diff_mma6_swapped(q, k[i < 2 * KS ? i : 0].x, s2);
                else {
                    DiffPlanes &y = v[i < 2 * KS ? 0 : i - 2 * KS];
                    if (LAST) {
                        const bf16x8 z[3] = {y.x[0], y.x[1], as_bf16x8(last[i & 1])};
                        dp = diff_mma6(q, z, dp);
                    } else {
                        dp = diff_mma6(q, y.x, dp);
                    }
                }
                if (i + 1 < 4 * KS) {
                    if (LAST && i + 1 >= 2 * KS) diff_landed(x[next], last[next]);
                    else diff_landed(x[next]);
                }
            }
        }
        if (LAST && at + 1 < p.to) issue(stage ^ 1);  // (not in front of the products above: two operands of theirs come from scratch memory, for which they would wait for the tile too)
        if (p.masked(a, tile)) p.hide(a, s1, s2, tile, g);
        const DiffScaling scaling(a.c, far);
        if (far) {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s1[v] *= scaling.first;
                s2[v] *= scaling.first;
            }
        }
        // four rows' statistics at a time, the next four's on their way
        {
            u32x4 st[2][6];
            auto read = [&](u32x4 (&to)[6], auto q4) {
                constexpr int at0 = 32 * decltype(q4)::value, ROW = 4 * kDiffTile;
                to[0] = lds_read_b128_at<at0>(stats);
                to[1] = lds_read_b128_at<at0 + ROW>(stats);
                to[2] = lds_read_b128_at<at0 + 2 * ROW>(stats);
                to[3] = lds_read_b128_at<at0 + 3 * ROW>(stats);
                to[4] = lds_read_b128_at<at0 + 4 * ROW>(stats);
                to[5] = lds_read_b128_at<at0 + 5 * ROW>(stats);
            };
            auto landed = [](u32x4 (&x)[6]) {
                asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]));
            };
            auto work = [&](const u32x4 (&x)[6], int q4) {
                f32x4 y[6];
#pragma unroll
                for (int i = 0; i < 6; ++i) y[i] = __builtin_bit_cast(f32x4, x[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * q4 + e;
                    const float e1 = __builtin_amdgcn_exp2f(fmaf(s1[r], scaling.then, y[0][e])), e2 = __builtin_amdgcn_exp2f(fmaf(s2[r], scaling.then, y[1][e]));
                    s1[r] = e1 * fmaf(dp[r], y[2][e], y[3][e]);
                    s2[r] = e2 * fmaf(dp[r], y[4][e], y[5][e]);
                    dp[r] = fmaf(e2, y[4][e], e1 * y[2][e]);
                }
            };
            read(st[0], std::integral_constant<int, 0>());
            landed(st[0]);
            read(st[1], std::integral_constant<int, 1>());
            __builtin_amdgcn_sched_barrier(0);
            work(st[0], 0);
            landed(st[1]);
            read(st[0], std::integral_constant<int, 2>());
            __builtin_amdgcn_sched_barrier(0);
            work(st[1], 1);
            landed(st[0]);
            read(st[1], std::integral_constant<int, 3>());
            __builtin_amdgcn_sched_barrier(0);
            work(st[0], 2);
            landed(st[1]);
            work(st[1], 3);
        }
        // columns of dO for dV, then of Q for dK, 16 rows at a time
        u32x2 c[2][6];
        diff_read_cols3<W, 3 * TILE, 0>(c[0], cols, 0);
        diff_landed(c[0]);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const DiffPlanes w = diff_block_planes(dp, kk), ds1 = diff_block_planes(s1, kk), ds2 = diff_block_planes(s2, kk);
#pragma unroll
            for (int i = 0; i < 2 * CB; ++i) {
                const int cb = i % CB, j = kk * 2 * CB + i + 1;  // j: the next operand
                if (j < CB) diff_read_cols3<W, 3 * TILE, 0>(c[j & 1], cols, j);
                else if (j < 2 * CB) diff_read_cols3<W, 0, 0>(c[j & 1], cols, j - CB);
                else if (j < 3 * CB) diff_read_cols3<W, 3 * TILE, 1>(c[j & 1], cols, j - 2 * CB);
                else if (j < 4 * CB) diff_read_cols3<W, 0, 1>(c[j & 1], cols, j - 3 * CB);
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 x[3];
                diff_cols3(c[(j + 1) & 1], x);
                if (i < CB) dv[cb] = diff_mma6(x, w.x, dv[cb]);
                else dk[cb] = diff_mma6(x, cb < CB / 2 ? ds1.x : ds2.x, dk[cb]);
                if (j < 4 * CB) diff_landed(c[j & 1]);
            }
        }
        if (++tile == p.tile_begin + p.n_tiles) tile = p.tile_begin;  // on to the group's next head
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile, for every wavefront, and every wavefront done with this one
        lds_barrier();
    }
    diff_finish_dkv<float, W>(a, dk, dv, p, g);
}

// Parts of rows of `channels` fp32 numbers to be added in their order: row (x, h, n) of B x heads x n rows goes to tensor `out`, and its channels
// from W on to `out2`.  Rows behind a sequence's end hold zeros in every part.
constexpr int kDiffFinishThreads = 1024;
struct DiffSum {
    const float *part;
    int parts, heads, n, channels;
    long long rows;
    TensorArg out, out2;
    unsigned blocks;  // workgroups, 0 without parts
};
template <typename T, int W>
__device__ inline void diff_add_parts(const DiffSum &a, unsigned block) {
    const unsigned per_row = a.channels / 4;  // (divides the threads)
    const long long row = (long long)block * (kDiffFinishThreads / per_row) + threadIdx.x / per_row;
    if (row >= a.rows) return;
    const int ch = (int)(threadIdx.x % per_row) * 4;
    f32x4 sum = *(const f32x4 *)(a.part + row * a.channels + ch);
    for (int p = 1; p < a.parts; ++p) {
        const f32x4 x = *(const f32x4 *)(a.part + (p * a.rows + row) * a.channels + ch);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    const int bh = (int)((unsigned)row / (unsigned)a.n), i = (int)((unsigned)row - (unsigned)bh * a.n), b = (unsigned)bh / (unsigned)a.heads, h = bh - b * a.heads;
    const TensorArg &to = ch < W ? a.out : a.out2;
    diff_store4((T *)const_cast<void *>(to.ptr) + b * to.sb + h * to.sh + i * to.sn + (ch < W ? ch : ch - W), sum);
}

// Gradients of lambda's vectors from the sums of P2 o dP: dlambda_h is their negative sum, over the heads too where these share
// the vectors.  One workgroup, a wavefront a set; sums in 64 bits.
template <int W>
__device__ inline void diff_lambda_grads(const DiffArgs &a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = kDiffFinishThreads / 64;
    __shared__ double shared_sum[16];
    const int sets = a.l_step ? a.heads : 1;
    const int sums = a.blocks * a.parts;  // of a (batch, head)
    const long long per_image = (long long)a.heads * sums;
    for (int set = a.l_step ? wave : 0; set < sets; set += a.l_step ? waves : 1) {
        double sum = 0.0;
        if (a.l_step) {
            const long long n = (long long)a.B * sums;
            for (long long x = lane; x < n; x += 64) {
                const unsigned image = (unsigned)x / (unsigned)sums;
                sum += a.lam_part[image * per_image + (long long)set * sums + ((unsigned)x - image * sums)];
            }
        } else {
            for (long long x = threadIdx.x; x < a.B * per_image; x += kDiffFinishThreads) sum += a.lam_part[x];
        }
#pragma unroll
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        if (!a.l_step) {
            if (lane == 0) shared_sum[wave] = sum;
            __syncthreads();
            sum = 0.0;
            for (int w = 0; w < waves; ++w) sum += shared_sum[w];
            if (wave) return;
        }
        const DiffLambda l = diff_lambda<W>(a, set, lane);
        const float dl = (float)-sum;
        if (lane < W / 2) {
            const int at = set * a.l_step + lane;
            const float q1 = a.lq1[at], k1 = a.lk1[at], q2 = a.lq2[at], k2 = a.lk2[at];
            a.dlq1[at] = dl * l.e1 * k1;
            a.dlk1[at] = dl * l.e1 * q1;
            a.dlq2[at] = -dl * l.e2 * k2;
            a.dlk2[at] = -dl * l.e2 * q2;
        }
    }
}

// What is left behind both passes, in one launch: parts of dK and dV, parts of dQ, and lambda's gradients.  Three launches were 5 us each for small calls; the
// parts are bound by memory (32 768 rows of dK and dV of 128 in four parts, 134 MB, 26 us).
template <typename T, int W>
__global__ void __launch_bounds__(kDiffFinishThreads) diff_attn_finish_kernel(DiffArgs a, DiffSum keys, DiffSum queries) {
    const unsigned block = blockIdx.x;
    if (block < keys.blocks) diff_add_parts<T, W>(keys, block);
    else if (block < keys.blocks + queries.blocks) diff_add_parts<T, W>(queries, block - keys.blocks);
    else diff_lambda_grads<W>(a);
}

struct DiffBwdPlan {
    int q_blocks, k_blocks, q_parts, k_parts;
    size_t stats, lam, dq, dkv, planes;  // bytes of the workspace's pieces, in this order
};
static DiffBwdPlan diff_bwd_plan(const jv_diff_attn_desc *d) {
    DiffBwdPlan p;
    p.q_blocks = (d->n_q + 127) / 128;
    p.k_blocks = (d->n_k + 127) / 128;
    const long long group = d->heads / d->kv_heads, rows = (long long)d->batch * d->heads * d->n_q, keys = (long long)d->batch * d->kv_heads * d->n_k;
    p.q_parts = diff_bwd_parts((long long)d->batch * d->heads * p.q_blocks, (d->n_k + kDiffTile - 1) / kDiffTile, d->dtype == JV_BF16, d->causal);
    p.k_parts = diff_bwd_parts((long long)d->batch * d->kv_heads * p.k_blocks, (d->n_q + kDiffTile - 1) / kDiffTile * group, d->dtype == JV_BF16, d->causal);
    auto whole = [](long long bytes) { return ((size_t)bytes + 255) & ~(size_t)255; };
    p.stats = whole(rows * (d->dtype == JV_BF16 ? 16 : 28));
    p.planes = diff_planes_bytes(d, true);
    p.lam = whole((long long)d->batch * d->heads * p.q_blocks * p.q_parts * 4);
    p.dq = p.q_parts > 1 ? whole(rows * p.q_parts * d->head_dim * 4) : 0;
    p.dkv = p.k_parts > 1 ? whole(keys * p.k_parts * d->head_dim * 8) : 0;
    return p;
}

template <typename T, int W>
static jv_status diff_backward(DiffArgs a, const DiffBwdPlan &plan, void *planes, hipStream_t stream) {
    const long long rows = diff_rows(a), keys = (long long)a.B * a.kv_heads * a.n_k;
    constexpr int LANES = W * (int)sizeof(T) / 16;
    constexpr bool BF16 = sizeof(T) == 2;
    hipLaunchKernelGGL((diff_attn_rows_kernel<T, W>), dim3((unsigned)((rows * LANES + 255) / 256)), dim3(256), 0, stream, a);
    jv_status st = launch_status("diff_attn_rows_kernel");
    if (st != JV_OK) return st;
    if (!BF16 && (st = diff_split(a, W, planes, true, stream)) != JV_OK) return st;
    a.blocks = plan.k_blocks;
    a.parts = plan.k_parts;
    a.items = (long long)a.B * a.kv_heads * a.blocks * a.parts;
    if constexpr (BF16) hipLaunchKernelGGL((diff_attn_dkv_bf16_kernel<W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((diff_attn_dkv_f32_kernel<W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    if ((st = launch_status("diff_attn_dkv_kernel")) != JV_OK) return st;
    a.blocks = plan.q_blocks;
    a.parts = plan.q_parts;
    a.items = (long long)a.B * a.heads * a.blocks * a.parts;
    if constexpr (BF16) hipLaunchKernelGGL((diff_attn_dq_bf16_kernel<W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((diff_attn_dq_f32_kernel<W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    if ((st = launch_status("diff_attn_dq_kernel")) != JV_OK) return st;
    auto blocks = [](int parts, long long n, int channels) { return parts > 1 ? (unsigned)((n * (channels / 4) + kDiffFinishThreads - 1) / kDiffFinishThreads) : 0u; };
    const DiffSum k{a.dkv_part, plan.k_parts, a.kv_heads, a.n_k, 2 * W, keys, a.dk, a.dv, blocks(plan.k_parts, keys, 2 * W)};
    const DiffSum q{a.dq_part, plan.q_parts, a.heads, a.n_q, W, rows, a.dq, a.dq, blocks(plan.q_parts, rows, W)};
    const unsigned grid = k.blocks + q.blocks + (a.dlq1 ? 1 : 0);
    if (!grid) return JV_OK;
    hipLaunchKernelGGL((diff_attn_finish_kernel<T, W>), dim3(grid), dim3(kDiffFinishThreads), 0, stream, a, k, q);
    return launch_status("diff_attn_finish_kernel");
}

}  // namespace jv

extern "C" {

size_t jv_diff_attn_bwd_workspace_bytes(const jv_diff_attn_desc *desc) {
    jv::clear_error();
    if (jv::diff_check_desc(desc) != JV_OK) return 0;
    const jv::DiffBwdPlan plan = jv::diff_bwd_plan(desc);
    return plan.stats + plan.lam + plan.dq + plan.dkv + plan.planes;
}

jv_status jv_diff_attn_bwd(const jv_diff_attn_desc *desc, const void *q, const void *k, const void *v,
                           const jv_diff_lambda *lambda, const void *o, const void *saved, size_t saved_bytes,
                           const jv_diff_attn_grads *grads, float scale, void *workspace, size_t workspace_bytes,
                           void *hip_stream) {
    jv::clear_error();
    jv::DiffProblem p;
    jv_status st = jv::diff_problem(desc, q, k, v, const_cast<void *>(o), lambda, scale, &p);
    if (st != JV_OK) return st;
    if (!grads) return jv::fail(JV_ERR_INVALID_ARG, "grads is null");
    if (p.bf16 != p.o_bf16) return jv::fail(JV_ERR_UNSUPPORTED, "the gradient needs an output of the inputs' type");
    if (!saved || !grads->d_o || !grads->d_q || !grads->d_k || !grads->d_v)
        return jv::fail(JV_ERR_INVALID_ARG, "saved, d_o, d_q, d_k, d_v must be non-null");
    if (((uintptr_t)grads->d_o | (uintptr_t)grads->d_q | (uintptr_t)grads->d_k | (uintptr_t)grads->d_v) & 15)
        return jv::fail(JV_ERR_INVALID_ARG, "d_o, d_q, d_k, d_v must be 16-byte aligned");
    const int have = (grads->d_q1 != nullptr) + (grads->d_k1 != nullptr) + (grads->d_q2 != nullptr) + (grads->d_k2 != nullptr);
    if (have != 0 && have != 4) return jv::fail(JV_ERR_INVALID_ARG, "all four gradients of lambda's vectors, or none");
    if (((uintptr_t)grads->d_q1 | (uintptr_t)grads->d_k1 | (uintptr_t)grads->d_q2 | (uintptr_t)grads->d_k2) & 3)
        return jv::fail(JV_ERR_INVALID_ARG, "the gradients of lambda's vectors must be 4-byte aligned");
    const int B = desc->batch, H = desc->heads, G = desc->kv_heads, NQ = desc->n_q, NK = desc->n_k, W = p.W, align = p.bf16 ? 8 : 4;
    if ((st = jv::diff_check_strides("d_o", grads->d_o_strides, B, H, NQ, W, align, false)) != JV_OK) return st;
    if ((st = jv::diff_check_strides("d_q", grads->d_q_strides, B, H, NQ, W, align, true)) != JV_OK) return st;
    if ((st = jv::diff_check_strides("d_k", grads->d_k_strides, B, G, NK, W, align, true)) != JV_OK) return st;
    if ((st = jv::diff_check_strides("d_v", grads->d_v_strides, B, G, NK, W, align, true)) != JV_OK) return st;
    const int size = p.bf16 ? 2 : 4;
    struct Range { uintptr_t from, to; };
    auto range = [&](const void *ptr, const jv_strides &s, int heads, int n) {
        return Range{(uintptr_t)ptr, (uintptr_t)ptr + (uintptr_t)jv::diff_span(s, B, heads, n, W) * size};
    };
    const Range in[5] = {range(q, desc->q, H, NQ), range(k, desc->k, G, NK), range(v, desc->v, G, NK), range(o, desc->o, H, NQ), range(grads->d_o, grads->d_o_strides, H, NQ)};
    const Range out[3] = {range(grads->d_q, grads->d_q_strides, H, NQ), range(grads->d_k, grads->d_k_strides, G, NK), range(grads->d_v, grads->d_v_strides, G, NK)};
    for (const Range &x : out)
        for (const Range &y : in)
            if (x.from < y.to && y.from < x.to) return jv::fail(JV_ERR_INVALID_ARG, "d_q, d_k, d_v must not overlap what is read");
    if (((uintptr_t)saved | (uintptr_t)workspace) & 255) return jv::fail(JV_ERR_INVALID_ARG, "saved and workspace must be 256-byte aligned");
    if (!workspace) return jv::fail(JV_ERR_INVALID_ARG, "workspace must be non-null");
    if (saved_bytes < jv::diff_saved_bytes(desc))
        return jv::fail(JV_ERR_WORKSPACE_TOO_SMALL, "saved holds %zu bytes, %zu are needed", saved_bytes, jv::diff_saved_bytes(desc));
    const size_t need = jv_diff_attn_bwd_workspace_bytes(desc);
    if (workspace_bytes < need) return jv::fail(JV_ERR_WORKSPACE_TOO_SMALL, "workspace holds %zu bytes, %zu are needed", workspace_bytes, need);
    if (jv::diff_rows(p.a) * 32 > 0x7fffff00ll * 256 || (long long)B * H * (((long long)std::max(NQ, NK) + 127) / 128) > 0x7fffff0ll)
        return jv::fail(JV_ERR_UNSUPPORTED, "more than 2^31 workgroups");
    auto arg = [](const void *ptr, const jv_strides &s) { return jv::TensorArg{ptr, s.stride_b, s.stride_h, s.stride_n}; };
    p.a.d_o = arg(grads->d_o, grads->d_o_strides);
    p.a.dq = arg(grads->d_q, grads->d_q_strides);
    p.a.dk = arg(grads->d_k, grads->d_k_strides);
    p.a.dv = arg(grads->d_v, grads->d_v_strides);
    p.a.dlq1 = grads->d_q1;
    p.a.dlk1 = grads->d_k1;
    p.a.dlq2 = grads->d_q2;
    p.a.dlk2 = grads->d_k2;
    jv::diff_use_saved(&p, const_cast<void *>(saved));
    const jv::DiffBwdPlan plan = jv::diff_bwd_plan(desc);
    char *at = (char *)workspace;
    p.a.stats = (float *)at;
    p.a.lam_part = (float *)(at += plan.stats);
    p.a.dq_part = (float *)(at += plan.lam);
    p.a.dkv_part = (float *)(at += plan.dq);
    at += plan.dkv;
    return jv::diff_with_kind(p.bf16, W, [&](auto kind) {
        using K = decltype(kind);
        return jv::diff_backward<typename K::T, K::W>(p.a, plan, at, (hipStream_t)hip_stream);
    });
}

}  // extern "C"
