// Forward pass of differential attention, and what its entry points check on the host.
//
// A wavefront keeps 32 rows (queries) as columns and walks the keys in tiles of 32: scores of both maps, S^T = K Q^T with half
// the channels each, two running softmaxes, and O1^T, O2^T += V^T P with every V operand read once for both maps.
// The difference is formed at the end, in fp32.  24 matrix instructions of 32 x 32 x 16 a tile and wavefront (W = 128),
// against 32 exponentials a lane.  Few rows, where the keys' bytes are what counts, take one wavefront each and are cut over the keys
// (jv_plan.h); the parts are joined by a second launch.
#include <math.h>

#include <algorithm>

#include "jv_diff_attn.h"

namespace jv {

constexpr float kDiffLazySum = 256.0f;  // largest lane sum of a tile taken without a search for its maximum

// Running softmax of one map: reference m (log2 units; -inf before the first key seen), what a tile's weights are first tried
// with (-m, or +inf), this lane's half of the sum, and the unnormalised output, channels 32 cb + 8 (v / 4) + 4 g + v % 4 of the lane's row.
template <int W>
struct DiffMap {
    float m, minus_m, l;
    f32x16 acc[W / 32];
    __device__ void clear() {
        m = -INFINITY;
        minus_m = INFINITY;
        l = 0.f;
#pragma unroll
        for (int cb = 0; cb < W / 32; ++cb) diff_zero(acc[cb]);
    }
};

__device__ inline float diff_exp(f32x16 &p, const f32x16 &s, float c, float minus_m) {
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
        p[v] = __builtin_amdgcn_exp2f(fmaf(s[v], c, minus_m));
        p[v + 1] = __builtin_amdgcn_exp2f(fmaf(s[v + 1], c, minus_m));
        sum0 += p[v];
        sum1 += p[v + 1];
    }
    return sum0 + sum1;
}
// Raises the reference to the tile's maximum; returns what the tile's weights are taken against.
template <int W>
__device__ inline float diff_raise(DiffMap<W> &w, const f32x16 &s, float c) {
    const float t0 = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), t1 = fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7]));
    const float t2 = fmaxf(fmaxf(s[8], s[9]), fmaxf(s[10], s[11])), t3 = fmaxf(fmaxf(s[12], s[13]), fmaxf(s[14], s[15]));
    float lo, hi;
    pair_values(fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * c, &lo, &hi);  // this lane and lane ^ 32 share the row
    const float m_new = fmaxf(w.m, fmaxf(lo, hi));
    const float alpha = w.m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(w.m - m_new);
    w.m = m_new;
    w.l *= alpha;
    // In place, register by register, as an opaque instruction: the common path then needs no copies where the two paths meet.
    // (alpha comes from a transcendental instruction, whose result the very next one may not read; inline assembly is not padded.)
    asm volatile("s_nop 1" ::"v"(alpha));
#pragma unroll
    for (int cb = 0; cb < W / 32; ++cb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            float x = w.acc[cb][v];
            asm volatile("v_mul_f32 %0, %0, %1" : "+v"(x) : "v"(alpha));
            w.acc[cb][v] = x;
        }
    w.minus_m = fabsf(m_new) < 16777216.f ? -m_new : INFINITY;  // (diff_far: no tile is tried; NaN neither)
    return m_new == -INFINITY ? 0.f : m_new;
}
// A weight against a reference that was just raised (see DiffScaling).
__device__ inline float diff_weight(float s, float c, float ref, bool far) {
#pragma clang fp contract(off)
    const float x = s * c;
    return __builtin_amdgcn_exp2f(far ? x - ref : fmaf(s, c, -ref));
}
// Weights of a tile against the present reference, which is raised only where they come out large (numerator and denominator always
// use the same one).  Without a reference minus_m is +inf, so every tile raises until a key is seen; where all is masked (s = -inf)
// the reference stays -inf and the weights, taken against 0, are zero.
template <int W>
__device__ inline void diff_softmax(DiffMap<W> &w, f32x16 &p, const f32x16 &s, float c) {
    float sum = diff_exp(p, s, c, w.minus_m);
    if (__builtin_amdgcn_ballot_w64(!(sum <= kDiffLazySum)) != 0) {
        const float ref = diff_raise<W>(w, s, c);
        const bool far = w.minus_m == INFINITY;
        sum = 0.f;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            p[v] = diff_weight(s[v], c, ref, far);
            sum += p[v];
        }
    }
    w.l += sum;
}

// What a wavefront works on.  Rows of a (batch, kv head) are its group's heads one after the other, n_q queries each, so that a few queries of
// heads that share K and V share a tile too; 32 rows a wavefront, a lane's row in lane % 32.
struct DiffPlace {
    int split, b, kv, bkv, n_rows, first, r, qi, head, limit;
    bool row_live;
    template <int WAVES, bool SPLIT>
    __device__ bool find(const DiffArgs &a, int wave, int li) {
        DiffItem item;
        if (!item.find(a, a.B * a.kv_heads, SPLIT ? a.splits : 1, true)) return false;
        split = item.part;
        bkv = item.bh;
        // (causal: the last blocks of all heads of a group before the ones before them)
        int block = item.block;
        if (a.causal) {
            const unsigned group = a.group, per_head = (unsigned)a.blocks / group;
            if (per_head * group == (unsigned)a.blocks) block = (unsigned)block % group * per_head + (unsigned)block / group;
        }
        b = (unsigned)bkv / (unsigned)a.kv_heads;
        kv = bkv - b * a.kv_heads;
        n_rows = a.group * a.n_q;
        first = (block * WAVES + wave) * 32;
        r = first + li;
        row_live = r < n_rows;
        const int hg = row_live ? (unsigned)r / (unsigned)a.n_q : 0;
        qi = row_live ? r - hg * a.n_q : 0;
        head = kv * a.group + hg;
        return true;
    }
};

// What the backward pass needs of a row: both references and sums.  A map without a weight (no key seen, or logits of -inf alone) has m = +inf; a
// reference of +inf, and that of a row of NaN, which m does not show, are NaN.
__device__ inline float diff_saved_reference(float m, float l) {
    if (m == -INFINITY && l == 0.f) return INFINITY;
    return fabsf(m) == INFINITY ? NAN : m;
}
__device__ inline void diff_save(const DiffArgs &a, long long row, float m1, float l1, float m2, float l2) {
    const long long n = diff_rows(a);
    a.ml[row] = diff_saved_reference(m1, l1);
    a.ml[n + row] = l1;
    a.ml[2 * n + row] = diff_saved_reference(m2, l2);
    a.ml[3 * n + row] = l2;
}

// Output of a wavefront's rows, or its part of it.
template <typename T, typename TO, int W, bool SPLIT>
__device__ inline void diff_finish(const DiffArgs &a, const DiffPlace &place, const DiffMap<W> &w1, const DiffMap<W> &w2, int lane) {
    constexpr int CB = W / 32;
    const int g = lane >> 5;
    float lo, hi;
    pair_values(w1.l, &lo, &hi);
    const float l1 = lo + hi;
    pair_values(w2.l, &lo, &hi);
    const float l2 = lo + hi;
    if (SPLIT) {
        if (!place.row_live) return;
        float *part = a.part + ((long long)place.split * a.B * a.kv_heads * place.n_rows + (long long)place.bkv * place.n_rows + place.r) * (2 * W + 4);
        if (g == 0) *(f32x4 *)part = f32x4{w1.m, l1, w2.m, l2};
        if (w1.m == -INFINITY && w2.m == -INFINITY) return;  // no key of this part is seen, or all logits are -inf or NaN: not read again either
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x16 &x = w1.acc[cb], &y = w2.acc[cb];
                *(f32x4 *)(part + 4 + 32 * cb + 8 * q4 + 4 * g) = f32x4{x[4 * q4], x[4 * q4 + 1], x[4 * q4 + 2], x[4 * q4 + 3]};
                *(f32x4 *)(part + 4 + W + 32 * cb + 8 * q4 + 4 * g) = f32x4{y[4 * q4], y[4 * q4 + 1], y[4 * q4 + 2], y[4 * q4 + 3]};
            }
        return;
    }
    const int last_head = place.kv * a.group + min(place.first + 31, place.n_rows - 1) / a.n_q;
    const float lam = diff_lambda_of<W>(a, __builtin_amdgcn_readfirstlane(place.head), last_head, place.head, lane);
    if (!place.row_live) return;
    const float inv1 = l1 > 0.f ? 1.f / l1 : l1, inv2 = l2 > 0.f ? 1.f / l2 : l2;  // (0 for a map without a weight, NaN stays NaN)
    const long long row = ((long long)place.b * a.heads + place.head) * a.n_q + place.qi;
    if (a.ml && g == 0) diff_save(a, row, w1.m, l1, w2.m, l2);
    TO *o = (TO *)const_cast<void *>(a.o.ptr) + place.b * a.o.sb + place.head * a.o.sh + place.qi * a.o.sn;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int ch = 32 * cb + 8 * q4 + 4 * g;
            f32x4 x, y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y[e] = w2.acc[cb][4 * q4 + e] * inv2;
                x[e] = fmaf(-lam, y[e], w1.acc[cb][4 * q4 + e] * inv1);
            }
            diff_store4(o + ch, x);
            if (a.o2) diff_store4((T *)a.o2 + row * W + ch, y);
        }
}

// Keys that the lane's row sees (0: none), and the tiles that the workgroup walks.  A row that sees none goes along unmasked (`limit`) and is dropped at
// the end; `least`: the smallest limit of the wavefront's rows.
template <int WAVES, bool SPLIT>
__device__ inline int diff_tiles(const DiffArgs &a, const DiffPlace &place, const DiffLengths &len, int (&wave_most)[WAVES], int wave, int lane, int *limit, int *least_,
                                 int *tile, int *tile_end) {
    const int sees = place.row_live ? len.limit(a, place.qi) : 0;
    *limit = sees > 0 ? sees : a.n_k + kDiffTile;
    int most = sees, least = *limit;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) {
        most = max(most, __shfl_xor(most, x));
        least = min(least, __shfl_xor(least, x));
    }
    *least_ = __builtin_amdgcn_readfirstlane(least);
    if (WAVES > 1) {
        if (lane == 0) wave_most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < WAVES; ++x) most = max(most, wave_most[x]);
    }
    most = __builtin_amdgcn_readfirstlane(most);
    *tile = SPLIT ? place.split * a.tiles_per_split : 0;
    *tile_end = (most + kDiffTile - 1) / kDiffTile;
    if (SPLIT) *tile_end = min(*tile_end, *tile + a.tiles_per_split);
    return sees;
}

// ---------------------------------------------------------------------------------------
// bf16 tensors, WAVES x 32 rows a workgroup.  SPLIT: a workgroup takes a part of the keys and leaves (m, l) of both maps and the unnormalised
// outputs in a.part.  Tiles come from memory straight into a ring of three LDS stages, two
// tiles ahead, and LDS read in assembly with waits of its own (the compiler would wait for every load into LDS in front of
// a read, and has no registers left for tiles on their way).  A tile: first map's scores on K operands that were read at the end of
// the tile before, second map's operands meanwhile; the hand-over of the stages; V operands of 16 keys, under whose latency
// both softmaxes run; the products with V, the next 16 keys' operands and then the next tile's K operands in flight.
// Rows behind the last key are fetched as the last one, which is masked there.  Rows that see no key go along unmasked and are
// dropped at the end.
// Bound by the issue of matrix and vector instructions: 8 x 4 096 tokens x 8 heads of 128 751 us (1.10 PFLOP/s), 3 x 4 096 x 16 of 64 357 us (0.87). The same
// arithmetic on numbers that stay in LDS, without loads, barriers and LDS reads, takes 83 and 85 % of that, and its exponentials, sums and
// roundings alone, matrix instructions aside, about two thirds of it for 64 channels.  Weights formed between matrix
// instructions (a wavefront working at both at once) changed nothing for 64 channels and does not fit the registers for 128; a shader clock
// of 2.0 to 2.3 GHz under this load is part of the bound.
// ---------------------------------------------------------------------------------------
// Weights of a tile as bf16 numbers, TERMS = 1, or sums of two: rounded, and what rounding left.  One term is as much as the matrix instruction takes beside
// bf16 values: outputs in bf16 are 2.5e-3 off 64 bits (relative 2-norm), with two terms 1.7e-3, the rounding of the outputs alone.  Two terms take 8 or 16
// products more a tile, 734 / 1 113 us for 8 x 4 096 tokens x 8 heads of 128, so only rows that wait for memory anyway have them.
template <int TERMS>
struct DiffWeights {
    unsigned pk[TERMS][8];
    __device__ void set(int v, float p0, float p1) {
        pk[0][v] = pack_bf16x2(p0, p1);
        if (TERMS == 2) pk[TERMS - 1][v] = pack_bf16x2(p0 - bf16_lo(pk[0][v]), p1 - bf16_hi(pk[0][v]));
    }
    __device__ bf16x8 frag(int term, int kk) const {
        return as_bf16x8(u32x4{pk[term][4 * kk], pk[term][4 * kk + 1], pk[term][4 * kk + 2], pk[term][4 * kk + 3]});
    }
};
// Weights of a tile and the running softmax: see diff_softmax.
template <int TERMS>
__device__ inline float diff_exp_pack(DiffWeights<TERMS> &w, const f32x16 &s, float c, float minus_m) {
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[2 * v], c, minus_m)), p1 = __builtin_amdgcn_exp2f(fmaf(s[2 * v + 1], c, minus_m));
        w.set(v, p0, p1);
        sum0 += p0;
        sum1 += p1;
    }
    return sum0 + sum1;
}
template <int W, int TERMS>
__device__ inline float diff_raise_pack(DiffMap<W> &w, DiffWeights<TERMS> &p, const f32x16 &s, float c) {
    const float ref = diff_raise<W>(w, s, c);
    const bool far = w.minus_m == INFINITY;
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < 8; ++v) {
        const float p0 = diff_weight(s[2 * v], c, ref, far), p1 = diff_weight(s[2 * v + 1], c, ref, far);
        p.set(v, p0, p1);
        sum += p0 + p1;
    }
    return sum;
}
template <int W, int TERMS>
__device__ inline void diff_softmax_pack(DiffMap<W> &w, DiffWeights<TERMS> &p, const f32x16 &s, float c) {
    float sum = diff_exp_pack(p, s, c, w.minus_m);
    if (__builtin_amdgcn_ballot_w64(!(sum <= kDiffLazySum)) != 0) sum = diff_raise_pack(w, p, s, c);
    w.l += sum;
}

// BOTH (up to 16 rows, one wavefront): lanes 0 .. 15 hold the rows for the first map and lanes 16 .. 31 for the second, each with zeros for the other map's
// channels, so that a tile takes one block of scores, one softmax and half the products with V.  There is time for weights of
// two terms then.  Bound by memory: one query of 16 heads against caches of up to 16 384 keys x 8 sequences x 4 kv heads of 128 (201 MB) 37 us out of
// the last-level cache, both launches 51 from memory; one against 2 x 1 374 keys x 16 of 64 7.5 us, which is a few dependent round trips.
template <typename TO, int W, int WAVES, bool SPLIT, bool BOTH = false>
__global__ void __launch_bounds__(64 * WAVES, W == 128 && WAVES == 1 ? 1 : 2) diff_attn_fwd_bf16_kernel(DiffArgs a) {
    static_assert(!BOTH || WAVES == 1, "a wavefront holds all rows twice");
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = kDiffTile * 2 * W, STAGE = 2 * TILE, RING = 3;  // a stage: K rows, then V rows
    __shared__ __align__(1024) unsigned char smem[RING * STAGE];
    __shared__ int wave_most[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, li = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffPlace place;
    if (!place.find<WAVES, SPLIT>(a, wave, BOTH ? li & 15 : li)) return;  // whole workgroup
    const DiffLengths len(a, place.b);
    int limit, least, tile, tile_end;
    const int sees = diff_tiles<WAVES, SPLIT>(a, place, len, wave_most, wave, lane, &limit, &least, &tile, &tile_end);

    DiffDma<W, WAVES> kload, vload;
    kload.start(a.k.ptr, place.b * a.k.sb + place.kv * a.k.sh, a.k.sn, wave, lane);
    vload.start(a.v.ptr, place.b * a.v.sb + place.kv * a.v.sh, a.v.sn, wave, lane);
    auto issue = [&](int t, int to) {
        kload.issue(smem + to * STAGE, t * kDiffTile, len.k, wave, lane);
        vload.issue(smem + to * STAGE + TILE, t * kDiffTile, len.k, wave, lane);
    };
    bf16x8 q[2 * KS];
    {
        const __bf16 *row = (const __bf16 *)a.q.ptr + place.b * a.q.sb + place.head * a.q.sh + place.qi * a.q.sn;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) q[ks] = diff_global_frag(row, ks, g, sees > 0 && (!BOTH || (ks < KS) == (li < 16)));
    }
    if (tile < tile_end) issue(tile, 0);
    if (tile + 1 < tile_end) issue(tile + 1, 1);

    DiffMap<W> w1, w2;
    w1.clear();
    w2.clear();
    const unsigned kaddr = Lds::rows(lds_address(smem), lane), vaddr = Lds::cols(lds_address(smem), lane);
    u32x4 k1[KS];
    if (tile < tile_end) {
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) asm volatile("" : "+v"(q[ks]));  // (waited for here, not inside the loop)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        Lds::template read_rows<0>(k1, kaddr, 0);
        diff_landed(k1);
    }
    for (int stage = 0; tile < tile_end; ++tile) {
        const int next = stage + 1 == RING ? 0 : stage + 1, after = next + 1 == RING ? 0 : next + 1;
        const unsigned kat = kaddr + stage * STAGE, vat = vaddr + stage * STAGE;
        f32x16 s1, s2;
        diff_zero(s1);
        diff_zero(s2);
        u32x4 k2[KS];
        Lds::template read_rows<0>(k2, kat, KS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s1 = mfma32(as_bf16x8(k1[ks]), q[ks], s1);
        diff_landed(k2);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (BOTH) s1 = mfma32(as_bf16x8(k2[ks]), q[KS + ks], s1);
            else s2 = mfma32(as_bf16x8(k2[ks]), q[KS + ks], s2);
        }
        __builtin_amdgcn_sched_barrier(0);
        // the next tile has landed for every wavefront, and every wavefront has left the tile before, whose stage takes the one after
        if (tile + 1 < tile_end) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();
            if (tile + 2 < tile_end) issue(tile + 2, after);
        }
        if ((tile + 1) * kDiffTile > least) diff_hide_keys(s1, s2, tile * kDiffTile, limit, g);
        constexpr int TERMS = BOTH ? 2 : 1;
        DiffWeights<TERMS> p1, p2;
        if (BOTH) {
            float sum = diff_exp_pack(p1, s1, a.c, w1.minus_m);
            if (__builtin_amdgcn_ballot_w64(!(sum <= kDiffLazySum)) != 0) {
                // Zeros times what is not finite in a key's other half are NaN: the maps' scores apart then (and where a masked tile is tried without a reference).
                if (__builtin_amdgcn_ballot_w64(sum != sum) != 0) {
                    f32x16 t1, t2;
                    diff_zero(t1);
                    diff_zero(t2);
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        t1 = mfma32(as_bf16x8(k1[ks]), q[ks], t1);
                        t2 = mfma32(as_bf16x8(k2[ks]), q[KS + ks], t2);
                    }
#pragma unroll
                    for (int v = 0; v < 16; ++v) s1[v] = li < 16 ? t1[v] : t2[v];
                    if ((tile + 1) * kDiffTile > least) diff_hide_keys(s1, s2, tile * kDiffTile, limit, g);
                }
                sum = diff_raise_pack(w1, p1, s1, a.c);
            }
            w1.l += sum;
        } else {
            diff_softmax_pack(w1, p1, s1, a.c);
        }
        u32x2 v0[2 * CB];
        Lds::template read_cols<TILE, 0>(v0, vat);
        __builtin_amdgcn_sched_barrier(0);
        if (!BOTH) diff_softmax_pack(w2, p2, s2, a.c);
        auto products = [&](const u32x2 (&v)[2 * CB], int kk) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const bf16x8 x = diff_join2(v[2 * cb], v[2 * cb + 1]);
#pragma unroll
                for (int t = TERMS - 1; t >= 0; --t) {
                    w1.acc[cb] = mfma32(x, p1.frag(t, kk), w1.acc[cb]);
                    if (!BOTH) w2.acc[cb] = mfma32(x, p2.frag(t, kk), w2.acc[cb]);
                }
            }
        };
        diff_landed(v0);
        u32x2 v1[2 * CB];
        Lds::template read_cols<TILE, 1>(v1, vat);
        __builtin_amdgcn_sched_barrier(0);
        products(v0, 0);
        diff_landed(v1);
        // (after the last tile: of a stage that nobody needs)
        Lds::template read_rows<0>(k1, kaddr + next * STAGE, 0);
        __builtin_amdgcn_sched_barrier(0);
        products(v1, 1);
        diff_landed(k1);
        stage = next;
    }
    int l = lane;
    asm("" : "+v"(l));  // (where the rows lie is worked out again: kept across the loop it would cost registers that are missed there)
    place.find<WAVES, SPLIT>(a, wave, BOTH ? l & 15 : l & 31);
    if ((place.row_live ? len.limit(a, place.qi) : 0) == 0) {
        w1.clear();
        w2.clear();
    }
    if (BOTH) {  // the second map comes to the lanes of the first
        w2.m = __shfl_xor(w1.m, 16);
        w2.l = __shfl_xor(w1.l, 16);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
            for (int v = 0; v < 16; ++v) w2.acc[cb][v] = __shfl_xor(w1.acc[cb][v], 16);
        place.row_live = place.row_live && (l & 16) == 0;
    }
    diff_finish<__bf16, TO, W, SPLIT>(a, place, w1, w2, l);
}

// ---------------------------------------------------------------------------------------
// fp32 tensors: as above on operands of three bf16 numbers, two stages of plane tiles, the next tile on its way under this one's
// arithmetic.  A tile takes 72 (W = 64) or 144 matrix instructions and the splitting of 32 weights a lane.  A tile is a chain: the products of the scores,
// both softmaxes and their splits, the products with V.  With one wavefront a SIMD (rows of 128) nothing else is issued under the middle of it:
// 2 x 1 024 tokens x 8 heads of 128 86 us, 0.90 PFLOP/s of bf16 products, 0.61 of what a large product reaches; with few tiles a wavefront its
// start and end count too (2 x 576 x 12 of 64 in two parts 30 us, 0.60 PFLOP/s).
// ---------------------------------------------------------------------------------------
template <int W, int WAVES, bool SPLIT>
__global__ void __launch_bounds__(64 * WAVES, W == 64 && WAVES > 1 ? 2 : 1) diff_attn_fwd_f32_kernel(DiffArgs a) {
    using Lds = DiffLds<W>;
    constexpr int KS = W / 32, CB = W / 32, TILE = DiffTile<W>::kBytes, STAGE = 6 * TILE;  // a stage: three planes of K rows, three of V rows
    constexpr int STAGES = WAVES == 1 ? 1 : 2;  // (single wavefronts: three on a unit in place of one, each under the others' loads)
    __shared__ __align__(1024) unsigned char smem[STAGES * STAGE];
    __shared__ int wave_most[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, li = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    DiffPlace place;
    if (!place.find<WAVES, SPLIT>(a, wave, li)) return;  // whole workgroup
    const DiffLengths len(a, place.b);
    int limit, least, tile, tile_end;
    const int sees = diff_tiles<WAVES, SPLIT>(a, place, len, wave_most, wave, lane, &limit, &least, &tile, &tile_end);

    DiffDma3<W, WAVES> kload, vload;
    kload.start(a.planes[1], (long long)place.bkv * a.n_k, wave, lane);
    vload.start(a.planes[2], (long long)place.bkv * a.n_k, wave, lane);
    auto issue = [&](int t, int stage) {
        kload.issue(smem + stage * STAGE, t * kDiffTile, len.k, wave, lane);
        vload.issue(smem + stage * STAGE + 3 * TILE, t * kDiffTile, len.k, wave, lane);
    };
    if (tile < tile_end) issue(tile, 0);
    DiffPlanes q[2 * KS];
    {
        const __bf16 *row = a.planes[0] + (((long long)place.b * a.heads + place.head) * a.n_q + place.qi) * 3 * W;
#pragma unroll
        for (int ks = 0; ks < 2 * KS; ++ks) q[ks] = diff_global_planes<W>(row, ks, g, sees > 0);
    }
#pragma unroll
    for (int ks = 0; ks < 2 * KS; ++ks) asm volatile("" : "+v"(q[ks].x[0]), "+v"(q[ks].x[1]), "+v"(q[ks].x[2]));  // (waited for here, not inside the loop)
    DiffMap<W> w1, w2;
    w1.clear();
    w2.clear();
    const unsigned rows0 = Lds::rows(lds_address(smem), lane), cols0 = Lds::cols(lds_address(smem), lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    for (int stage = 0; tile < tile_end; ++tile, stage ^= STAGES - 1) {
        if (STAGES == 2 && tile + 1 < tile_end) issue(tile + 1, stage ^ 1);
        const unsigned rows = rows0 + stage * STAGE, cols = cols0 + stage * STAGE;
        f32x16 s1, s2, p;
        diff_zero(s1);
        diff_zero(s2);
        {
            u32x4 x[2][3];
            diff_read_rows3<W, 0>(x[0], rows, 0);
            diff_landed(x[0]);
#pragma unroll
            for (int ks = 0; ks < 2 * KS; ++ks) {
                if (ks + 1 < 2 * KS) diff_read_rows3<W, 0>(x[(ks + 1) & 1], rows, ks + 1);
                __builtin_amdgcn_sched_barrier(0);
                bf16x8 k[3];
                diff_rows3(x[ks & 1], k);
                if (ks < KS) s1 = diff_mma6(k, q[ks].x, s1);
                else s2 = diff_mma6(k, q[ks].x, s2);
                if (ks + 1 < 2 * KS) diff_landed(x[(ks + 1) & 1]);
            }
        }
        u32x2 v[2][6];
        diff_read_cols3<W, 3 * TILE, 0>(v[0], cols, 0);
        __builtin_amdgcn_sched_barrier(0);
        if ((tile + 1) * kDiffTile > least) diff_hide_keys(s1, s2, tile * kDiffTile, limit, g);
        DiffPlanes p1[2], p2[2];
        diff_softmax<W>(w1, p, s1, a.c);
        p1[0] = diff_block_planes(p, 0);
        p1[1] = diff_block_planes(p, 1);
        diff_softmax<W>(w2, p, s2, a.c);
        p2[0] = diff_block_planes(p, 0);
        p2[1] = diff_block_planes(p, 1);
        diff_landed(v[0]);
#pragma unroll
        for (int i = 0; i < 2 * CB; ++i) {
            const int kk = i / CB, cb = i % CB, next = (i + 1) % CB;
            if (i + 1 < CB) diff_read_cols3<W, 3 * TILE, 0>(v[(i + 1) & 1], cols, next);
            else if (i + 1 < 2 * CB) diff_read_cols3<W, 3 * TILE, 1>(v[(i + 1) & 1], cols, next);
            __builtin_amdgcn_sched_barrier(0);
            bf16x8 x[3];
            diff_cols3(v[i & 1], x);
            w1.acc[cb] = diff_mma6(x, p1[kk].x, w1.acc[cb]);
            w2.acc[cb] = diff_mma6(x, p2[kk].x, w2.acc[cb]);
            if (i + 1 < 2 * CB) diff_landed(v[(i + 1) & 1]);
        }
        if (STAGES == 1 && tile + 1 < tile_end) issue(tile + 1, 0);  // (its own LDS reads have landed)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile, for every wavefront, and every wavefront done with this one
        lds_barrier();
    }
    if (sees == 0) {
        w1.clear();
        w2.clear();
    }
    diff_finish<float, float, W, SPLIT>(a, place, w1, w2, lane);
}

// fp32 tensors into planes: a thread eight channels; blockIdx.y the tensor (Q, K, V, dO).  Rows behind their sequence's end are not read.  Bound by
// memory, 10 bytes a number (13 824 rows of 64 a tensor 7 us, 16 384 of 128 13).
struct DiffSplitArgs {
    TensorArg in[4];
    __bf16 *out[4];
    int heads[4], n[4];
    const int *len[4];
    long long rows[4];
};
template <int W>
__global__ void __launch_bounds__(256) diff_attn_split_kernel(DiffSplitArgs a) {
    const int t = blockIdx.y;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, row = at / (W / 8);
    if (row >= a.rows[t]) return;
    const unsigned bh = (unsigned)row / (unsigned)a.n[t], b = bh / (unsigned)a.heads[t];
    const int ch = (int)(at % (W / 8)) * 8, i = (int)((unsigned)row - bh * a.n[t]), h = (int)(bh - b * a.heads[t]);
    if (a.len[t] && i >= a.len[t][b]) return;
    const TensorArg &in = a.in[t];
    const float *from = (const float *)in.ptr + b * in.sb + h * in.sh + i * in.sn + ch;
    const f32x4 x = *(const f32x4 *)from, y = *(const f32x4 *)(from + 4);
    const float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    u32x4 planes[3];
    diff_split8(v, planes);
#pragma unroll
    for (int p = 0; p < 3; ++p) *(u32x4 *)(a.out[t] + (row * 3 + p) * W + ch) = planes[p];
}
size_t diff_planes_bytes(const jv_diff_attn_desc *d, bool with_d_o) {
    if (d->dtype != JV_F32) return 0;
    const size_t q = (size_t)d->batch * d->heads * d->n_q, k = (size_t)d->batch * d->kv_heads * d->n_k;
    auto whole = [&](size_t rows) { return (rows * 6 * d->head_dim + 255) & ~(size_t)255; };
    return whole(q) * (with_d_o ? 2 : 1) + 2 * whole(k);
}
jv_status diff_split(DiffArgs &a, int W, void *memory, bool with_d_o, hipStream_t stream) {
    DiffSplitArgs s;
    const TensorArg in[4] = {a.q, a.k, a.v, a.d_o};
    char *at = (char *)memory;
    long long most = 0;
    for (int t = 0; t < (with_d_o ? 4 : 3); ++t) {
        const bool keys = t == 1 || t == 2;
        s.in[t] = in[t];
        s.heads[t] = keys ? a.kv_heads : a.heads;
        s.n[t] = keys ? a.n_k : a.n_q;
        s.len[t] = keys ? a.k_len : a.q_len;
        s.rows[t] = (long long)a.B * s.heads[t] * s.n[t];
        s.out[t] = (__bf16 *)at;
        a.planes[t] = s.out[t];
        at += (s.rows[t] * 6 * W + 255) & ~255ll;
        most = std::max(most, s.rows[t]);
    }
    const dim3 grid((unsigned)((most * (W / 8) + 255) / 256), with_d_o ? 4 : 3);
    if (W == 128) hipLaunchKernelGGL(diff_attn_split_kernel<128>, grid, dim3(256), 0, stream, s);
    else hipLaunchKernelGGL(diff_attn_split_kernel<64>, grid, dim3(256), 0, stream, s);
    return launch_status("diff_attn_split_kernel");
}

// The parts of a row joined, in their order.  Each map asks for its own reference: a part may have weights in one of them alone (logits of -inf in the
// other), and one of -inf has a sum of 0, or of NaN, which m does not show and the total must.  Unnormalised outputs of a part where both
// references are -inf were not written: read, in bounds, and not used.
__device__ inline float diff_join_factor(float m, float top) { return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top); }
// Up to PARTS (2, 4 or 8) parts: a wavefront a row, everything it needs of all parts asked for at once (13 824 rows of 64 in two parts 8.2 us, 18 MB).
constexpr int kDiffFewParts = 8;
// Where row `at` of all (batch, kv head, row)s lies.
struct DiffRowPlace {
    int b, head, qi;
    long long row;
    __device__ DiffRowPlace(const DiffArgs &a, unsigned at) {
        const unsigned n_rows = a.group * a.n_q, bkv = at / n_rows, r = at - bkv * n_rows, hg = r / (unsigned)a.n_q;
        b = bkv / (unsigned)a.kv_heads;
        qi = r - hg * a.n_q;
        head = (bkv - b * a.kv_heads) * a.group + hg;
        row = ((long long)b * a.heads + head) * a.n_q + qi;
    }
};
template <typename T, typename TO, int W, int PARTS>
__global__ void __launch_bounds__(256) diff_attn_join_few_kernel(DiffArgs a) {
    constexpr int PER = W / 64;  // channels a lane
    const int lane = threadIdx.x & 63;
    const long long all = diff_rows(a), at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= all) return;
    const DiffRowPlace place(a, (unsigned)at);
    f32x4 ml[PARTS];
    float x1[PARTS][PER], x2[PARTS][PER];
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
        const float *part = a.part + ((long long)min(s, a.splits - 1) * all + at) * (2 * W + 4);
        ml[s] = *(const f32x4 *)part;
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            x1[s][e] = part[4 + lane * PER + e];
            x2[s][e] = part[4 + W + lane * PER + e];
        }
    }
    const float lam = diff_lambda<W>(a, place.head, lane).value;
    float m1 = -INFINITY, m2 = -INFINITY, l1 = 0.f, l2 = 0.f, y1[PER] = {}, y2[PER] = {};
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
        m1 = fmaxf(m1, ml[s][0]);
        m2 = fmaxf(m2, ml[s][2]);
    }
#pragma unroll
    for (int s = 0; s < PARTS; ++s) {
        if (s >= a.splits) continue;  // (uniform)
        const float f1 = diff_join_factor(ml[s][0], m1), f2 = diff_join_factor(ml[s][2], m2);
        l1 = fmaf(ml[s][1], f1, l1);
        l2 = fmaf(ml[s][3], f2, l2);
        if (ml[s][0] == -INFINITY && ml[s][2] == -INFINITY) continue;  // (uniform)
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            y1[e] = fmaf(x1[s][e], f1, y1[e]);
            y2[e] = fmaf(x2[s][e], f2, y2[e]);
        }
    }
    if (a.ml && lane == 0) diff_save(a, place.row, m1, l1, m2, l2);
    const float inv1 = l1 > 0.f ? 1.f / l1 : l1, inv2 = l2 > 0.f ? 1.f / l2 : l2;
    TO *o = (TO *)const_cast<void *>(a.o.ptr) + place.b * a.o.sb + place.head * a.o.sh + place.qi * a.o.sn + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const float y = y2[e] * inv2;
        o[e] = (TO)fmaf(-lam, y, y1[e] * inv1);
        if (a.o2) ((T *)a.o2)[place.row * W + lane * PER + e] = (T)y;
    }
}

// More parts, up to kDiffMostParts: a workgroup a row. A thread holds a part's references and sums; then its four wavefronts take every fourth part
// each, eight parts' loads at a time (one query against 8 192 keys x 8 heads of 128 in 64 parts, both kernels: 22.0 us with one part's
// loads after the other's, 17.9 so; alone 4 to 5 us, three dependent round trips).
template <typename T, typename TO, int W>
__global__ void __launch_bounds__(256) diff_attn_join_kernel(DiffArgs a) {
    static_assert(kDiffMostParts <= 256, "a part a thread");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long all = diff_rows(a), at = blockIdx.x;
    __shared__ float sums[4][2 * W], top[2][4], total[2][4], factor[2][256];
    const DiffRowPlace place(a, (unsigned)at);
    f32x4 ml = {-INFINITY, 0.f, -INFINITY, 0.f};
    if ((int)threadIdx.x < a.splits) ml = *(const f32x4 *)(a.part + ((long long)threadIdx.x * all + at) * (2 * W + 4));
    float m1 = ml[0], m2 = ml[2];
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        m1 = fmaxf(m1, __shfl_xor(m1, x));
        m2 = fmaxf(m2, __shfl_xor(m2, x));
    }
    if (lane == 0) {
        top[0][wave] = m1;
        top[1][wave] = m2;
    }
    __syncthreads();
    m1 = fmaxf(fmaxf(top[0][0], top[0][1]), fmaxf(top[0][2], top[0][3]));
    m2 = fmaxf(fmaxf(top[1][0], top[1][1]), fmaxf(top[1][2], top[1][3]));
    const bool written = ml[0] != -INFINITY || ml[2] != -INFINITY;
    const float f1 = diff_join_factor(ml[0], m1), f2 = diff_join_factor(ml[2], m2);
    float l1 = wave_sum(ml[1] * f1), l2 = wave_sum(ml[3] * f2);
    factor[0][threadIdx.x] = written ? f1 : -1.f;
    factor[1][threadIdx.x] = written ? f2 : -1.f;
    if (lane == 0) {
        total[0][wave] = l1;
        total[1][wave] = l2;
    }
    __syncthreads();
    l1 = (total[0][0] + total[0][1]) + (total[0][2] + total[0][3]);
    l2 = (total[1][0] + total[1][1]) + (total[1][2] + total[1][3]);
    constexpr int PER = W / 32;  // channels a lane: lanes 0 .. 31 those of the first map, 32 .. 63 of the second
    float x[PER] = {};
    const float *part = a.part + at * (2 * W + 4) + 4 + lane * PER;
    for (int first = wave; first < a.splits; first += 32) {
        float y[8][PER];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long s = min(first + 4 * i, a.splits - 1);
#pragma unroll
            for (int e = 0; e < PER; ++e) y[i][e] = part[s * all * (2 * W + 4) + e];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int s = first + 4 * i;
            const float f = s < a.splits ? factor[lane >> 5][s] : -1.f;
#pragma unroll
            for (int e = 0; e < PER; ++e) x[e] = f >= 0.f ? fmaf(y[i][e], f, x[e]) : x[e];
        }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) sums[wave][lane * PER + e] = x[e];
    const float lam = diff_lambda<W>(a, place.head, lane).value;
    __syncthreads();
    const int ch = threadIdx.x;
    if (a.ml && ch == 0) diff_save(a, place.row, m1, l1, m2, l2);
    if (ch >= W) return;
    const float inv1 = l1 > 0.f ? 1.f / l1 : l1, inv2 = l2 > 0.f ? 1.f / l2 : l2;
    const float y1 = ((sums[0][ch] + sums[1][ch]) + (sums[2][ch] + sums[3][ch])) * inv1;
    const float y2 = ((sums[0][W + ch] + sums[1][W + ch]) + (sums[2][W + ch] + sums[3][W + ch])) * inv2;
    ((TO *)const_cast<void *>(a.o.ptr) + place.b * a.o.sb + place.head * a.o.sh + place.qi * a.o.sn)[ch] = (TO)fmaf(-lam, y2, y1);
    if (a.o2) ((T *)a.o2)[place.row * W + ch] = (T)y2;
}

// ---------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------

static size_t diff_part_bytes(const DiffPlan &p, long long rows, int W) {
    return p.splits > 1 ? (size_t)p.splits * rows * (2 * W + 4) * 4 : 0;
}

jv_status diff_check_strides(const char *name, const jv_strides &s, int64_t b, int64_t h, int64_t n, int W, int64_t align, bool written) {
    const int64_t size[3] = {b, h, n}, stride[3] = {s.stride_b, s.stride_h, s.stride_n};
    int64_t reach = W;  // elements up to the end of the last row
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1) continue;  // the stride of an axis of one is not used
        if (stride[i] < 0) return fail(JV_ERR_INVALID_ARG, "%s: negative stride", name);
        if (i == 2 && stride[i] > kDiffMostTokenStride) return fail(JV_ERR_UNSUPPORTED, "%s: stride_n above 2^25", name);
        if (i == 2 && stride[i] < W) return fail(JV_ERR_INVALID_ARG, "%s: stride_n < head_dim", name);
        if (stride[i] % align) return fail(JV_ERR_INVALID_ARG, "%s: strides must keep rows 16-byte aligned", name);
        if (stride[i] > (INT64_C(1) << 56) / size[i]) return fail(JV_ERR_INVALID_ARG, "%s: strides reach beyond the address space", name);
        reach += (size[i] - 1) * stride[i];
    }
    if (reach > INT64_C(1) << 57) return fail(JV_ERR_INVALID_ARG, "%s: strides reach beyond the address space", name);
    if (written) {  // every row a place of its own: each axis steps over all that the axes of smaller strides span
        int order[3] = {0, 1, 2};
        std::sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
        int64_t span = W;
        for (int i : order) {
            if (size[i] == 1) continue;
            if (stride[i] < span) return fail(JV_ERR_INVALID_ARG, "%s: rows of a tensor that is written overlap", name);
            span += (size[i] - 1) * stride[i];
        }
    }
    return JV_OK;
}

int64_t diff_span(const jv_strides &s, int64_t b, int64_t h, int64_t n, int W) {
    return (b - 1) * s.stride_b + (h - 1) * s.stride_h + (n - 1) * s.stride_n + W;  // (an axis of one adds nothing)
}

jv_status diff_check_desc(const jv_diff_attn_desc *d) {
    if (!d) return fail(JV_ERR_INVALID_ARG, "descriptor is null");
    if (d->batch <= 0 || d->heads <= 0 || d->kv_heads <= 0 || d->n_q <= 0 || d->n_k <= 0)
        return fail(JV_ERR_INVALID_ARG, "batch, heads, kv_heads, n_q, n_k must be positive");
    if (d->heads % d->kv_heads) return fail(JV_ERR_INVALID_ARG, "heads must be a multiple of kv_heads");
    if (d->n_q > (1 << 24) || d->n_k > (1 << 24)) return fail(JV_ERR_UNSUPPORTED, "more than 2^24 queries or keys");
    if ((int64_t)d->batch * d->heads > 65535) return fail(JV_ERR_UNSUPPORTED, "batch * heads above 65535");
    if ((int64_t)d->batch * d->heads * d->n_q > 0xffff0000ll || (int64_t)d->batch * d->kv_heads * d->n_k > 0xffff0000ll)
        return fail(JV_ERR_UNSUPPORTED, "more than 2^32 - 2^16 rows of queries or keys");
    if ((int64_t)d->heads / d->kv_heads * d->n_q > (1 << 30)) return fail(JV_ERR_UNSUPPORTED, "more than 2^30 queries of a kv head");
    if (d->head_dim <= 0) return fail(JV_ERR_INVALID_ARG, "head_dim must be positive");
    if (d->head_dim != kHeadDim && d->head_dim != kHeadDimWide) return fail(JV_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if ((d->dtype != JV_F32 && d->dtype != JV_BF16) || (d->o_dtype != JV_F32 && d->o_dtype != JV_BF16))
        return fail(JV_ERR_INVALID_ARG, "unknown dtype");
    if (d->dtype == JV_F32 && d->o_dtype != JV_F32) return fail(JV_ERR_UNSUPPORTED, "fp32 inputs need an fp32 output");
    if (((uintptr_t)d->q_lengths | (uintptr_t)d->k_lengths) & 3) return fail(JV_ERR_INVALID_ARG, "lengths must be 4-byte aligned");
    const int64_t in = d->dtype == JV_BF16 ? 8 : 4, out = d->o_dtype == JV_BF16 ? 8 : 4;
    jv_status st;
    if ((st = diff_check_strides("q", d->q, d->batch, d->heads, d->n_q, d->head_dim, in, false)) != JV_OK) return st;
    if ((st = diff_check_strides("k", d->k, d->batch, d->kv_heads, d->n_k, d->head_dim, in, false)) != JV_OK) return st;
    if ((st = diff_check_strides("v", d->v, d->batch, d->kv_heads, d->n_k, d->head_dim, in, false)) != JV_OK) return st;
    return diff_check_strides("o", d->o, d->batch, d->heads, d->n_q, d->head_dim, out, true);
}

static DiffPlan diff_plan_of(const jv_diff_attn_desc *d) {
    return diff_plan(d->batch, d->kv_heads, (long long)d->heads / d->kv_heads * d->n_q, d->n_k, d->head_dim, d->dtype == JV_BF16);
}

size_t diff_saved_bytes(const jv_diff_attn_desc *d) {
    const size_t rows = (size_t)d->batch * d->heads * d->n_q;
    return ((rows * 16 + 255) & ~(size_t)255) + rows * d->head_dim * (d->dtype == JV_BF16 ? 2 : 4);
}
void diff_use_saved(DiffProblem *p, void *saved) {
    const size_t rows = (size_t)diff_rows(p->a);
    p->a.ml = (float *)saved;
    p->a.o2 = (char *)saved + ((rows * 16 + 255) & ~(size_t)255);
}

jv_status diff_problem(const jv_diff_attn_desc *d, const void *q, const void *k, const void *v, void *o,
                       const jv_diff_lambda *lambda, float scale, DiffProblem *p) {
    jv_status st = diff_check_desc(d);
    if (st != JV_OK) return st;
    if (!q || !k || !v || !o) return fail(JV_ERR_INVALID_ARG, "q, k, v, o must be non-null");
    if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) return fail(JV_ERR_INVALID_ARG, "q, k, v, o must be 16-byte aligned");
    if (!lambda) return fail(JV_ERR_INVALID_ARG, "lambda is null");
    if (!lambda->q1 || !lambda->k1 || !lambda->q2 || !lambda->k2) return fail(JV_ERR_INVALID_ARG, "lambda's vectors must be non-null");
    if (((uintptr_t)lambda->q1 | (uintptr_t)lambda->k1 | (uintptr_t)lambda->q2 | (uintptr_t)lambda->k2) & 3)
        return fail(JV_ERR_INVALID_ARG, "lambda's vectors must be 4-byte aligned");
    if (!(fabsf(lambda->init) <= 3.4028235e38f)) return fail(JV_ERR_INVALID_ARG, "lambda's init must be finite");
    if (scale > 1e30f || (scale > 0.f && scale < 1e-30f)) return fail(JV_ERR_INVALID_ARG, "a scale of its own must lie between 1e-30 and 1e30");
    *p = DiffProblem{};
    DiffArgs &a = p->a;
    a.B = d->batch;
    a.heads = d->heads;
    a.kv_heads = d->kv_heads;
    a.group = d->heads / d->kv_heads;
    a.n_q = d->n_q;
    a.n_k = d->n_k;
    a.causal = d->causal != 0;
    a.q_len = d->q_lengths;
    a.k_len = d->k_lengths;
    a.scale = scale > 0.f ? scale : (float)(1.0 / sqrt(d->head_dim / 2.0));  // (NaN fails the comparison too)
    a.c = a.scale * 1.4426950408889634f;
    a.lq1 = lambda->q1;
    a.lk1 = lambda->k1;
    a.lq2 = lambda->q2;
    a.lk2 = lambda->k2;
    a.l_init = lambda->init;
    a.l_step = lambda->per_head ? d->head_dim / 2 : 0;
    auto arg = [](const void *ptr, const jv_strides &s) { return TensorArg{ptr, s.stride_b, s.stride_h, s.stride_n}; };
    a.q = arg(q, d->q);
    a.k = arg(k, d->k);
    a.v = arg(v, d->v);
    a.o = arg(o, d->o);
    p->W = d->head_dim;
    p->bf16 = d->dtype == JV_BF16;
    p->o_bf16 = d->o_dtype == JV_BF16;
    return JV_OK;
}

template <typename T, typename TO, int W>
static jv_status diff_forward(DiffArgs a, const DiffPlan &plan, void *planes, hipStream_t stream) {
    a.blocks = plan.blocks;
    a.splits = plan.splits;
    a.tiles_per_split = plan.tiles_per_split;
    a.items = (long long)a.B * a.kv_heads * a.blocks * a.splits;
    const dim3 grid(diff_grid(a.items));
    jv_status st;
    if (sizeof(T) == 4 && (st = diff_split(a, W, planes, false, stream)) != JV_OK) return st;
    auto launch = [&](auto waves, auto split) {
        constexpr int WAVES = decltype(waves)::value;
        constexpr bool SPLIT = decltype(split)::value;
        using Out = std::conditional_t<SPLIT, float, TO>;
        if constexpr (sizeof(T) == 2 && WAVES == 1) {
            if (diff_both_maps(true, a.group * (long long)a.n_q)) {
                hipLaunchKernelGGL((diff_attn_fwd_bf16_kernel<Out, W, 1, SPLIT, true>), grid, dim3(64), 0, stream, a);
                return;
            }
        }
        if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((diff_attn_fwd_bf16_kernel<Out, W, WAVES, SPLIT>), grid, dim3(64 * WAVES), 0, stream, a);
        else hipLaunchKernelGGL((diff_attn_fwd_f32_kernel<W, WAVES, SPLIT>), grid, dim3(64 * WAVES), 0, stream, a);
    };
    if (plan.splits == 1) {
        if (plan.waves == 1) launch(std::integral_constant<int, 1>(), std::false_type());
        else launch(std::integral_constant<int, 4>(), std::false_type());
        return launch_status("diff_attn_fwd_kernel");
    }
    if (plan.waves == 1) launch(std::integral_constant<int, 1>(), std::true_type());
    else launch(std::integral_constant<int, 4>(), std::true_type());
    if ((st = launch_status("diff_attn_fwd_kernel")) != JV_OK) return st;
    const long long rows = diff_rows(a);
    const dim3 few((unsigned)((rows + 3) / 4));
    if (a.splits <= 2) hipLaunchKernelGGL((diff_attn_join_few_kernel<T, TO, W, 2>), few, dim3(256), 0, stream, a);
    else if (a.splits <= 4) hipLaunchKernelGGL((diff_attn_join_few_kernel<T, TO, W, 4>), few, dim3(256), 0, stream, a);
    else if (a.splits <= kDiffFewParts) hipLaunchKernelGGL((diff_attn_join_few_kernel<T, TO, W, kDiffFewParts>), few, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((diff_attn_join_kernel<T, TO, W>), dim3((unsigned)rows), dim3(256), 0, stream, a);
    return launch_status("diff_attn_join_kernel");
}

}  // namespace jv

extern "C" {

size_t jv_diff_attn_workspace_bytes(const jv_diff_attn_desc *desc) {
    jv::clear_error();
    if (jv::diff_check_desc(desc) != JV_OK) return 0;
    const size_t part = jv::diff_part_bytes(jv::diff_plan_of(desc), (long long)desc->batch * desc->heads * desc->n_q, desc->head_dim);
    const size_t bytes = ((part + 255) & ~(size_t)255) + jv::diff_planes_bytes(desc, false);
    return bytes > 256 ? bytes : 256;
}

size_t jv_diff_attn_saved_bytes(const jv_diff_attn_desc *desc) {
    jv::clear_error();
    return jv::diff_check_desc(desc) == JV_OK ? jv::diff_saved_bytes(desc) : 0;
}

jv_status jv_diff_attn_fwd(const jv_diff_attn_desc *desc, const void *q, const void *k, const void *v,
                           const jv_diff_lambda *lambda, void *o, float scale, void *saved, size_t saved_bytes,
                           void *workspace, size_t workspace_bytes, void *hip_stream) {
    jv::clear_error();
    jv::DiffProblem p;
    jv_status st = jv::diff_problem(desc, q, k, v, o, lambda, scale, &p);
    if (st != JV_OK) return st;
    const int in = p.bf16 ? 2 : 4, out = p.o_bf16 ? 2 : 4;
    const uintptr_t o0 = (uintptr_t)o, o1 = o0 + jv::diff_span(desc->o, desc->batch, desc->heads, desc->n_q, p.W) * out;
    auto meets = [&](const void *ptr, int64_t bytes) { return o0 < (uintptr_t)ptr + bytes && (uintptr_t)ptr < o1; };
    if (meets(q, jv::diff_span(desc->q, desc->batch, desc->heads, desc->n_q, p.W) * in) ||
        meets(k, jv::diff_span(desc->k, desc->batch, desc->kv_heads, desc->n_k, p.W) * in) ||
        meets(v, jv::diff_span(desc->v, desc->batch, desc->kv_heads, desc->n_k, p.W) * in))
        return jv::fail(JV_ERR_INVALID_ARG, "o must not overlap an input");
    if (saved) {
        if ((uintptr_t)saved & 255) return jv::fail(JV_ERR_INVALID_ARG, "saved must be 256-byte aligned");
        if (p.bf16 != p.o_bf16) return jv::fail(JV_ERR_UNSUPPORTED, "saved needs an output of the inputs' type");
        if (saved_bytes < jv::diff_saved_bytes(desc))
            return jv::fail(JV_ERR_WORKSPACE_TOO_SMALL, "saved holds %zu bytes, %zu are needed", saved_bytes, jv::diff_saved_bytes(desc));
        jv::diff_use_saved(&p, saved);
    }
    const jv::DiffPlan plan = jv::diff_plan_of(desc);
    const size_t need = jv_diff_attn_workspace_bytes(desc);
    void *planes = nullptr;
    if (need > 256) {
        if (!workspace) return jv::fail(JV_ERR_INVALID_ARG, "workspace must be non-null");
        if ((uintptr_t)workspace & 255) return jv::fail(JV_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
        if (workspace_bytes < need) return jv::fail(JV_ERR_WORKSPACE_TOO_SMALL, "workspace holds %zu bytes, %zu are needed", workspace_bytes, need);
        p.a.part = (float *)workspace;
        planes = (char *)workspace + (need - jv::diff_planes_bytes(desc, false));
    }
    if ((long long)desc->batch * desc->kv_heads * plan.blocks * plan.splits > 0x7ffffff0ll)
        return jv::fail(JV_ERR_UNSUPPORTED, "more than 2^31 workgroups");
    const hipStream_t stream = (hipStream_t)hip_stream;
    return jv::diff_with_kind(p.bf16, p.W, [&](auto kind) {
        using K = decltype(kind);
        if (p.o_bf16) {
            if constexpr (sizeof(typename K::T) == 2) return jv::diff_forward<typename K::T, __bf16, K::W>(p.a, plan, planes, stream);
        }
        return jv::diff_forward<typename K::T, float, K::W>(p.a, plan, planes, stream);
    });
}

}  // extern "C"
