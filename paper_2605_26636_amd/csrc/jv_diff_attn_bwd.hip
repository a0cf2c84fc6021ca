// Gradient of differential attention (jv_diff_attn_bwd): row sums of dO against both outputs, dQ with the rows kept and the keys
// streamed, dK and dV with the keys kept and the rows streamed, and the gradients of lambda's vectors.  Scores are formed again
// in both passes, so no sum needs an atomic and the order of every sum is fixed.
#include <math.h>

#include <algorithm>

#include "jv_diff_attn.h"

namespace jv {

// D1, D2: row sums of dO o (P1 V) and dO o (P2 V), P1 V = O + lambda P2 V from the rounded rows that the forward pass left.
// A row takes as many lanes as it has 16-byte pieces.
template <typename T, int W>
__global__ void __launch_bounds__(256) diff_attn_rows_kernel(DiffArgs a) {
    constexpr int PER = 16 / (int)sizeof(T), LANES = W / PER;
    const int lane = threadIdx.x & 63;
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int ch = (threadIdx.x % LANES) * PER;
    const bool live = at < diff_rows(a);
    const long long row = live ? at : diff_rows(a) - 1;
    const int qi = (int)(row % a.n_q), bh = (int)(row / a.n_q), h = bh % a.heads, b = bh / a.heads;
    float lam = 0.f;
    // (rows of a wavefront may belong to two heads and more)
    for (int x = __builtin_amdgcn_readfirstlane(bh), last = __builtin_amdgcn_readlane(bh, 63); x <= last; ++x) {
        const float value = diff_lambda<W>(a, x % a.heads, lane).value;
        if (bh == x) lam = value;
    }
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
    if (live && ch == 0) {
        a.rows_d[row] = d1;
        a.rows_d[diff_rows(a) + row] = d2;
    }
}

// dQ, and the sums of P2 o dP (for lambda): a wavefront keeps 32 queries of one head, their dO and their dQ, and walks the keys.
// A tile takes W / 16 score products, as many of V with dO, and as many of K^T with the gradients of the logits.
template <typename T, int W>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) diff_attn_dq_kernel(DiffArgs a) {
    using Tile = DiffTile<T, W>;
    constexpr int KS = W / 16, CB = W / 32;
    __shared__ __align__(16) unsigned char smem[2][2][Tile::kBytes];
    __shared__ int wave_most[4];
    __shared__ float wave_lam[4];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, li = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long item = diff_item(a.items);
    if (item >= a.items) return;  // whole workgroup
    const int block = a.blocks - 1 - (int)(item % a.blocks), bh = (int)(item / a.blocks), b = bh / a.heads, h = bh % a.heads, kv = h / a.group;
    const DiffLengths len(a, b);
    const int qi = (block * 4 + wave) * 32 + li;
    const bool row_live = qi < a.n_q;
    const int limit = row_live ? len.limit(a, qi) : 0;
    int most = limit, least = row_live ? limit : a.n_k;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) {
        most = max(most, __shfl_xor(most, x));
        least = min(least, __shfl_xor(least, x));
    }
    if (lane == 0) wave_most[wave] = most;
    __syncthreads();
    most = __builtin_amdgcn_readfirstlane(most);
    least = __builtin_amdgcn_readfirstlane(least);
    const int wg_most = __builtin_amdgcn_readfirstlane(max(max(wave_most[0], wave_most[1]), max(wave_most[2], wave_most[3])));
    const int tile_end = (wg_most + kDiffTile - 1) / kDiffTile;
    const float lam = diff_lambda<W>(a, h, lane).value;

    DiffFrag<T> q[KS], go[KS];
    const int q_at = row_live ? qi : 0;
    {
        const T *row = (const T *)a.q.ptr + b * a.q.sb + h * a.q.sh + q_at * a.q.sn, *grow = (const T *)a.d_o.ptr + b * a.d_o.sb + h * a.d_o.sh + q_at * a.d_o.sn;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            q[ks] = diff_global_frag<T>(row, ks, g, limit > 0);
            go[ks] = diff_global_frag<T>(grow, ks, g, limit > 0);
        }
    }
    const long long at_row = (long long)bh * a.n_q + q_at;
    const float lse1 = limit > 0 ? a.lse[at_row] : INFINITY, lse2 = limit > 0 ? a.lse[diff_rows(a) + at_row] : INFINITY;
    const float d1 = limit > 0 ? a.rows_d[at_row] : 0.f, d2 = limit > 0 ? a.rows_d[diff_rows(a) + at_row] : 0.f;
    f32x16 acc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) diff_zero(acc[cb]);
    float lam_sum = 0.f;

    DiffFetch<T, W, 256> kf, vf;
    kf.start(a.k.ptr, b * a.k.sb + kv * a.k.sh, a.k.sn, tid);
    vf.start(a.v.ptr, b * a.v.sb + kv * a.v.sh, a.v.sn, tid);
    if (tile_end > 0) {
        kf.fetch(0, len.k, tid);
        vf.fetch(0, len.k, tid);
        kf.store(smem[0][0], tid);
        vf.store(smem[0][1], tid);
    }
    lds_barrier();
    int tile = 0;
    auto step = [&](auto buffer) {
        constexpr int at = decltype(buffer)::value;
        const bool more = tile + 1 < tile_end;
        if (more) {
            kf.fetch((tile + 1) * kDiffTile, len.k, tid);
            vf.fetch((tile + 1) * kDiffTile, len.k, tid);
        }
        if (tile * kDiffTile < most) {  // (uniform in the wavefront)
            const unsigned char *kt = smem[at][0], *vt = smem[at][1];
            f32x16 s1, s2, dp;
            diff_zero(s1);
            diff_zero(s2);
            diff_zero(dp);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const DiffFrag<T> k = Tile::row_frag(kt, li, ks, g);
                if (ks < KS / 2) s1 = diff_mma(k, q[ks], s1);
                else s2 = diff_mma(k, q[ks], s2);
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) dp = diff_mma(Tile::row_frag(vt, li, ks, g), go[ks], dp);
            if ((tile + 1) * kDiffTile > least) {
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const bool hidden = tile * kDiffTile + 8 * (v / 4) + 4 * g + v % 4 >= limit;
                    s1[v] = hidden ? -INFINITY : s1[v];
                    s2[v] = hidden ? -INFINITY : s2[v];
                }
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const float p1 = __builtin_amdgcn_exp2f(fmaf(s1[v], a.c, -lse1)), p2 = __builtin_amdgcn_exp2f(fmaf(s2[v], a.c, -lse2));
                lam_sum = fmaf(p2, dp[v], lam_sum);
                s1[v] = p1 * (dp[v] - d1);
                s2[v] = p2 * (dp[v] - d2) * -lam;
            }
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const DiffFrag<T> ds1 = diff_block_frag<T>(s1, kk), ds2 = diff_block_frag<T>(s2, kk);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) acc[cb] = diff_mma(Tile::col_frag(kt, kk, cb, lane), cb < CB / 2 ? ds1 : ds2, acc[cb]);
            }
        }
        if (more) {
            kf.store(smem[at ^ 1][0], tid);
            vf.store(smem[at ^ 1][1], tid);
        }
        lds_barrier();
    };
    while (tile < tile_end) {  // (one copy of the tile for each buffer)
        step(std::integral_constant<int, 0>());
        if (++tile >= tile_end) break;
        step(std::integral_constant<int, 1>());
        ++tile;
    }
    if (row_live) {
        T *dq = (T *)const_cast<void *>(a.dq.ptr) + b * a.dq.sb + h * a.dq.sh + qi * a.dq.sn;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &x = acc[cb];
                diff_store4(dq + 32 * cb + 8 * q4 + 4 * g,
                            f32x4{x[4 * q4] * a.scale, x[4 * q4 + 1] * a.scale, x[4 * q4 + 2] * a.scale, x[4 * q4 + 3] * a.scale});
            }
    }
    lam_sum = wave_sum(lam_sum);
    if (lane == 0) wave_lam[wave] = lam_sum;
    __syncthreads();
    if (tid == 0) a.lam_part[(long long)bh * a.blocks + block] = (wave_lam[0] + wave_lam[1]) + (wave_lam[2] + wave_lam[3]);
}

// dK and dV: a wavefront keeps 32 keys of one kv head, their values and both gradients, and walks the queries of the group's heads.
// Lengths mask nothing here but the rows written: a query behind the end of its sequence has weights of zero (its
// denominator is saved as infinite), and the columns of keys behind theirs are thrown away.
template <typename T, int W>
__global__ void __launch_bounds__(256, 1) diff_attn_dkv_kernel(DiffArgs a) {
    using Tile = DiffTile<T, W>;
    constexpr int KS = W / 16, CB = W / 32;
    __shared__ __align__(16) unsigned char smem[2][2][Tile::kBytes];
    __shared__ __align__(16) float stats[2][4][kDiffTile];  // of a tile's queries: both denominators, D1, D2
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, li = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const long long item = diff_item(a.items);
    if (item >= a.items) return;  // whole workgroup
    const int block = (int)(item % a.blocks), bkv = (int)(item / a.blocks), b = bkv / a.kv_heads, kv = bkv % a.kv_heads;
    const DiffLengths len(a, b);
    const int key0 = block * 128, key = key0 + wave * 32 + li;
    const bool key_live = key < len.k;

    DiffFrag<T> k[KS], v[KS];
    {
        const int at = key_live ? key : 0;
        const T *krow = (const T *)a.k.ptr + b * a.k.sb + kv * a.k.sh + at * a.k.sn, *vrow = (const T *)a.v.ptr + b * a.v.sb + kv * a.v.sh + at * a.v.sn;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            k[ks] = diff_global_frag<T>(krow, ks, g, key_live);
            v[ks] = diff_global_frag<T>(vrow, ks, g, key_live);
        }
    }
    f32x16 dk[CB], dv[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        diff_zero(dk[cb]);
        diff_zero(dv[cb]);
    }
    // causal: the first query that sees key x is x - (keys - queries)
    const int shift = a.causal ? len.k - len.q : 0;
    const int tile_begin = a.causal ? max(key0 - shift, 0) / kDiffTile : 0, tile_end = key0 < len.k ? (len.q + kDiffTile - 1) / kDiffTile : 0;
    const int n_tiles = max(tile_end - tile_begin, 0);
    const int first_query = a.causal ? key0 + wave * 32 - shift : 0;  // the wavefront's keys are seen from here on
    for (int hg = 0; hg < (n_tiles ? a.group : 0); ++hg) {
        const int h = kv * a.group + hg;
        const float lam = diff_lambda<W>(a, h, lane).value;
        const long long row0 = ((long long)b * a.heads + h) * a.n_q;
        DiffFetch<T, W, 256> qf, gf;
        qf.start(a.q.ptr, b * a.q.sb + h * a.q.sh, a.q.sn, tid);
        gf.start(a.d_o.ptr, b * a.d_o.sb + h * a.d_o.sh, a.d_o.sn, tid);
        float stat = 0.f;
        auto fetch = [&](int tile) {
            qf.fetch(tile * kDiffTile, len.q, tid);
            gf.fetch(tile * kDiffTile, len.q, tid);
            if (tid < 128) {  // statistic tid / 32 of query tid % 32
                const int qi = tile * kDiffTile + (tid & 31);
                stat = tid < 64 ? INFINITY : 0.f;
                if (qi < len.q) stat = (tid < 64 ? a.lse : a.rows_d)[(tid >> 5 & 1 ? diff_rows(a) : 0) + row0 + qi];
            }
        };
        auto store = [&](int to) {
            qf.store(smem[to][0], tid);
            gf.store(smem[to][1], tid);
            if (tid < 128) stats[to][tid >> 5][tid & 31] = stat;
        };
        fetch(tile_begin);
        store(0);
        lds_barrier();
        int tile = tile_begin;
        auto step = [&](auto buffer) {
            constexpr int at = decltype(buffer)::value;
            const bool more = tile + 1 < tile_end;
            if (more) fetch(tile + 1);
            if ((tile + 1) * kDiffTile > first_query) {  // (uniform in the wavefront)
                const unsigned char *qt = smem[at][0], *gt = smem[at][1];
                f32x16 s1, s2, dp;
                diff_zero(s1);
                diff_zero(s2);
                diff_zero(dp);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const DiffFrag<T> q = Tile::row_frag(qt, li, ks, g);
                    if (ks < KS / 2) s1 = diff_mma(q, k[ks], s1);
                    else s2 = diff_mma(q, k[ks], s2);
                }
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) dp = diff_mma(Tile::row_frag(gt, li, ks, g), v[ks], dp);
                if (a.causal && tile * kDiffTile < first_query + 31) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const bool hidden = key > tile * kDiffTile + 8 * (x / 4) + 4 * g + x % 4 + shift;
                        s1[x] = hidden ? -INFINITY : s1[x];
                        s2[x] = hidden ? -INFINITY : s2[x];
                    }
                }
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    const f32x4 lse1 = *(const f32x4 *)&stats[at][0][8 * q4 + 4 * g], lse2 = *(const f32x4 *)&stats[at][1][8 * q4 + 4 * g];
                    const f32x4 d1 = *(const f32x4 *)&stats[at][2][8 * q4 + 4 * g], d2 = *(const f32x4 *)&stats[at][3][8 * q4 + 4 * g];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int x = 4 * q4 + e;
                        const float p1 = __builtin_amdgcn_exp2f(fmaf(s1[x], a.c, -lse1[e])), p2 = -lam * __builtin_amdgcn_exp2f(fmaf(s2[x], a.c, -lse2[e]));
                        s1[x] = p1 * (dp[x] - d1[e]);
                        s2[x] = p2 * (dp[x] - d2[e]);
                        dp[x] = p1 + p2;
                    }
                }
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const DiffFrag<T> p = diff_block_frag<T>(dp, kk), ds1 = diff_block_frag<T>(s1, kk), ds2 = diff_block_frag<T>(s2, kk);
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) {
                        dv[cb] = diff_mma(Tile::col_frag(gt, kk, cb, lane), p, dv[cb]);
                        dk[cb] = diff_mma(Tile::col_frag(qt, kk, cb, lane), cb < CB / 2 ? ds1 : ds2, dk[cb]);
                    }
                }
            }
            if (more) store(at ^ 1);
            lds_barrier();
        };
        while (tile < tile_end) {  // (one copy of the tile for each buffer)
            step(std::integral_constant<int, 0>());
            if (++tile >= tile_end) break;
            step(std::integral_constant<int, 1>());
            ++tile;
        }
    }
    if (key < a.n_k) {
        T *krow = (T *)const_cast<void *>(a.dk.ptr) + b * a.dk.sb + kv * a.dk.sh + key * a.dk.sn;
        T *vrow = (T *)const_cast<void *>(a.dv.ptr) + b * a.dv.sb + kv * a.dv.sh + key * a.dv.sn;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                f32x4 x, y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = key_live ? dk[cb][4 * q4 + e] * a.scale : 0.f;
                    y[e] = key_live ? dv[cb][4 * q4 + e] : 0.f;
                }
                diff_store4(krow + 32 * cb + 8 * q4 + 4 * g, x);
                diff_store4(vrow + 32 * cb + 8 * q4 + 4 * g, y);
            }
    }
}

// Gradients of lambda's vectors from the sums of P2 o dP: dlambda_h is their negative sum, over the heads too where these share
// the vectors.  One workgroup of as many wavefronts as there are sets, 16 at most; sums in 64 bits.
template <int W>
__global__ void __launch_bounds__(1024) diff_attn_dlambda_kernel(DiffArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    __shared__ double shared_sum[16];
    const int sets = a.l_step ? a.heads : 1;
    const long long per_image = (long long)a.heads * a.blocks;
    for (int set = a.l_step ? wave : 0; set < sets; set += a.l_step ? waves : 1) {
        double sum = 0.0;
        if (a.l_step) {
            const long long n = (long long)a.B * a.blocks;
            for (long long x = lane; x < n; x += 64) sum += a.lam_part[x / a.blocks * per_image + (long long)set * a.blocks + x % a.blocks];
        } else {
            for (long long x = threadIdx.x; x < a.B * per_image; x += blockDim.x) sum += a.lam_part[x];
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

template <typename T, int W>
static jv_status diff_backward(DiffArgs a, hipStream_t stream) {
    const long long rows = diff_rows(a);
    constexpr int LANES = W * (int)sizeof(T) / 16;
    hipLaunchKernelGGL((diff_attn_rows_kernel<T, W>), dim3((unsigned)((rows * LANES + 255) / 256)), dim3(256), 0, stream, a);
    jv_status st = launch_status("diff_attn_rows_kernel");
    if (st != JV_OK) return st;
    a.blocks = (a.n_k + 127) / 128;
    a.items = (long long)a.B * a.kv_heads * a.blocks;
    hipLaunchKernelGGL((diff_attn_dkv_kernel<T, W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    if ((st = launch_status("diff_attn_dkv_kernel")) != JV_OK) return st;
    a.blocks = (a.n_q + 127) / 128;
    a.items = (long long)a.B * a.heads * a.blocks;
    hipLaunchKernelGGL((diff_attn_dq_kernel<T, W>), dim3(diff_grid(a.items)), dim3(256), 0, stream, a);
    if ((st = launch_status("diff_attn_dq_kernel")) != JV_OK) return st;
    if (!a.dlq1) return JV_OK;
    const int waves = a.l_step ? (a.heads < 16 ? a.heads : 16) : 16;
    hipLaunchKernelGGL((diff_attn_dlambda_kernel<W>), dim3(1), dim3(64 * waves), 0, stream, a);
    return launch_status("diff_attn_dlambda_kernel");
}

// Workspace: D1 and D2 of every row, then the sums for lambda of every block of 128 rows.
static size_t diff_bwd_rows_bytes(const jv_diff_attn_desc *d) { return ((size_t)d->batch * d->heads * d->n_q * 8 + 255) & ~(size_t)255; }

}  // namespace jv

extern "C" {

size_t jv_diff_attn_bwd_workspace_bytes(const jv_diff_attn_desc *desc) {
    jv::clear_error();
    if (jv::diff_check_desc(desc) != JV_OK) return 0;
    const size_t blocks = (size_t)desc->batch * desc->heads * ((desc->n_q + 127) / 128);
    return jv::diff_bwd_rows_bytes(desc) + ((blocks * 4 + 255) & ~(size_t)255);
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
    if (jv::diff_rows(p.a) * 32 > 0x7fffff00ll * 256 || (long long)B * H * (((long long)std::max(NQ, NK) + 127) / 128) > 0x7ffffff0ll)
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
    p.a.rows_d = (float *)workspace;
    p.a.lam_part = (float *)((char *)workspace + jv::diff_bwd_rows_bytes(desc));
    return jv::diff_with_kind(p.bf16, W, [&](auto kind) {
        using K = decltype(kind);
        return jv::diff_backward<typename K::T, K::W>(p.a, (hipStream_t)hip_stream);
    });
}

}  // extern "C"
