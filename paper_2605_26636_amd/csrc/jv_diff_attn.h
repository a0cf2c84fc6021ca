// Differential attention (jv_diff_attn_fwd, jv_diff_attn_bwd): the problem as its kernels see it, and the tiles they share.
//
// Per (batch, head), with rows of W = head_dim channels, Q = [Q1 | Q2], K = [K1 | K2] in halves of W / 2:
//     Pm = softmax(scale Qm Km^T) over the keys a row sees,  O = P1 V - lambda P2 V.
// All products run as D = A B + C on 32 x 32 blocks whose columns are what a wavefront keeps (its queries, or its keys in
// the key pass of the gradient) and whose rows are the tokens of the tile that passes through LDS; a lane holds one
// column, so that softmax sums stay inside a lane (and the lane 32 further), and a finished block is the B
// operand of the next product as it stands.  fp32 tensors take the same steps on operands of three bf16 numbers.
#pragma once

#include <type_traits>

#include "jv_common.h"
#include "jv_mfma.h"
#include "jv_plan.h"

namespace jv {

struct DiffArgs {
    TensorArg q, k, v, o;
    int B, heads, kv_heads, group;  // group: heads that share one K and V
    int n_q, n_k, causal;
    const int *q_len, *k_len;       // [B], or null
    float scale, c;                 // c = scale log2(e)
    const float *lq1, *lk1, *lq2, *lk2;
    float l_init;
    int l_step;                     // W / 2: a set of vectors for every head; 0: one set
    float *ml;                      // saved: [4][B * heads * n_q], reference m of the first map (log2 units; +inf: no weight), sum l of
                                    // exp2(logit - m), then those of the second; or null
    void *o2;                       // saved: [B * heads * n_q][W], P2 V
    // forward pass over parts of the keys
    float *part;
    int splits, tiles_per_split;
    // gradient
    TensorArg d_o, dq, dk, dv;
    float *stats;                   // [4 or 7][B * heads * n_q]: see diff_attn_rows_kernel
    const __bf16 *planes[4];        // fp32 tensors: Q, K, V, dO split, [B * heads * n][3][W] each
    int parts;                      // of the tiles of a workgroup's rows or keys; each leaves sums of its own where there are several:
    float *dq_part, *dkv_part;      // [parts][B * heads * n_q][W]; [parts][B * kv_heads * n_k][2 W]
    float *lam_part;                // [B * heads * row blocks * parts]: sums of P2 o dP or D2
    float *dlq1, *dlk1, *dlq2, *dlk2;
    int blocks;                     // blocks of rows (or keys) a (batch, head) has
    long long items;                // workgroups with work
};

struct DiffProblem {
    DiffArgs a;
    int W;
    bool bf16, o_bf16;
};

// What a workgroup works on: a block of rows (or keys) of a (batch, head) and one of `parts` parts of it.  Without a mask, contiguous
// ranges of (batch, head)s per XCD (workgroup w runs on XCD w % 8), so that the workgroups of one share its K and V in one L2.  Sequences of different
// lengths lie on few XCDs each then, and a launch lasts as long as the longest one's: a step of 4 sequences of 854 to 1 183 tokens x 16 heads of 64
// 221 us, of four of 1 183 219, of four of their mean 187.
// Causal: the blocks with most work of all of them first (an XCD's (batch, head)s one after the other leave its last long
// blocks alone at the end: forward pass of 2 x 4 096 tokens x 16 heads of 128 channels 291 us, so 232; where their number is a multiple of
// 8 each stays on one XCD all the same).  False where a workgroup of the rounded-up grid has no work.
struct DiffItem {
    int part, block, bh;
    __device__ bool find(const DiffArgs &a, int n_bh, int parts, bool last_block_first) {
        unsigned item = blockIdx.x;  // (below 2^31; divisions of 64 bits took 130 instructions each, a microsecond of a small call)
        if (!a.causal) item = (blockIdx.x & 7) * (((unsigned)a.items + 7) / 8) + (blockIdx.x >> 3);
        if (item >= (unsigned)a.items) return false;
        if (a.causal) {
            bh = (int)(item % (unsigned)n_bh);
            item /= (unsigned)n_bh;
        }
        part = 0;
        if (parts > 1) {
            part = (int)(item % (unsigned)parts);
            item /= (unsigned)parts;
        }
        block = (int)(item % (unsigned)a.blocks);
        if (!a.causal) bh = (int)(item / (unsigned)a.blocks);
        if (last_block_first) block = a.blocks - 1 - block;
        return true;
    }
};
inline unsigned diff_grid(long long items) { return (unsigned)(8 * ((items + 7) / 8)); }

// Tokens [0, limit) of a sequence that query qi sees, by the lengths of the sequence.
struct DiffLengths {
    int q, k;
    __device__ DiffLengths(const DiffArgs &a, int b) {
        q = a.q_len ? min(max(a.q_len[b], 0), a.n_q) : a.n_q;
        k = a.k_len ? min(max(a.k_len[b], 0), a.n_k) : a.n_k;
    }
    __device__ int limit(const DiffArgs &a, int qi) const {
        if (qi >= q) return 0;
        return a.causal ? min(max(qi + 1 + k - q, 0), k) : k;
    }
};

__device__ inline void diff_zero(f32x16 &x) {
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
}
// Operands (see mfma32): lane 32 g + i holds row or column i and elements 8 g .. + 7 of 16.
// Rows 16 kk .. + 15 of a finished block as B operand: element e of lane 32 g + i is row 16 kk + 8 (e / 4) + 4 g + e % 4.  Rounded to bf16, as the operands
// beside it are: what the gradient of bf16 tensors does with P1 - lambda P2 and the gradients of the logits (2.5e-3 off 64 bits where the results'
// rounding alone is 1.7e-3; a second term would be a third more products in the query pass and half as many again in the key
// pass, which has no registers for it).
__device__ inline bf16x8 diff_block_frag(const f32x16 &s, int kk) {
    return as_bf16x8(u32x4{pack_bf16x2(s[8 * kk], s[8 * kk + 1]), pack_bf16x2(s[8 * kk + 2], s[8 * kk + 3]),
                           pack_bf16x2(s[8 * kk + 4], s[8 * kk + 5]), pack_bf16x2(s[8 * kk + 6], s[8 * kk + 7])});
}
// Channels 16 ks + 8 g .. + 7 of a row in memory.
__device__ inline bf16x8 diff_global_frag(const __bf16 *row, int ks, int g, bool live) {
    return as_bf16x8(live ? *(const u32x4 *)(row + 16 * ks + 8 * g) : u32x4{0, 0, 0, 0});
}

// 32 rows of W channels of 16 bits in LDS.  16-byte chunks are moved inside their row so that both kinds of reads spread over
// all banks: a chunk of 16 consecutive rows (row-per-lane operands) and 64 bytes of four consecutive rows (transposing reads).
template <int W>
struct DiffTile {
    static constexpr int kRowBytes = 2 * W, kBytes = kDiffTile * kRowBytes;
    __device__ static unsigned off(int row, int chunk) {
        const unsigned slot = W == 128 ? chunk ^ ((row & 3) << 2 | (row >> 2 & 3)) : chunk ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
        return row * kRowBytes + slot * 16;
    }
};

// Elements from token to token at most: a lane's place in a tile is a 32-bit offset.
constexpr long long kDiffMostTokenStride = 1 << 25;

// Keys that a query does not see weigh nothing.
__device__ inline void diff_hide_keys(f32x16 &s1, f32x16 &s2, int first, int limit, int g) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const bool hidden = first + 8 * (v / 4) + 4 * g + v % 4 >= limit;
        s1[v] = hidden ? -INFINITY : s1[v];
        s2[v] = hidden ? -INFINITY : s2[v];
    }
}
// bf16 tiles that loads bring straight into LDS, laid out as DiffTile (both kinds of reads), and read in assembly with waits of their
// own: the compiler would wait for every load into LDS that is in flight in front of a read.  All offsets of a
// lane's reads differ from its first one's by an exclusive or of small constants and by whole rows: one register holds them.
typedef __attribute__((address_space(3))) void diff_lds_void;
typedef const __attribute__((address_space(1))) void diff_global_cvoid;

__device__ inline const char *diff_uniform(const void *ptr) {
    const unsigned long long u = (unsigned long long)ptr;
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)u), hi = __builtin_amdgcn_readfirstlane((unsigned)(u >> 32));
    return (const char *)((unsigned long long)hi << 32 | lo);
}
__device__ inline void diff_landed(u32x4 (&x)[4]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
}
__device__ inline void diff_landed(u32x4 (&x)[2]) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1])); }
__device__ inline void diff_landed(u32x4 (&x)[4], u32x4 (&y)[4]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]));
}
__device__ inline void diff_landed(u32x4 (&x)[2], u32x4 (&y)[2]) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(y[0]), "+v"(y[1])); }
__device__ inline void diff_landed(u32x4 (&x)[4], u32x4 (&y)[2]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]));
}
__device__ inline void diff_landed(u32x4 (&x)[4], u32x4 (&y)[2], u32x4 (&z)[2]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(y[0]), "+v"(y[1]), "+v"(z[0]), "+v"(z[1]));
}
__device__ inline void diff_landed(u32x2 (&x)[8]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
}
__device__ inline void diff_landed(u32x2 (&x)[4]) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3])); }
__device__ inline f32x16 diff_join4(const u32x4 (&x)[4]) {
    const f32x4 a = __builtin_bit_cast(f32x4, x[0]), b = __builtin_bit_cast(f32x4, x[1]), c = __builtin_bit_cast(f32x4, x[2]), d = __builtin_bit_cast(f32x4, x[3]);
    return f32x16{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3], c[0], c[1], c[2], c[3], d[0], d[1], d[2], d[3]};
}
__device__ inline bf16x8 diff_join2(u32x2 a, u32x2 b) { return as_bf16x8(u32x4{a[0], a[1], b[0], b[1]}); }

template <int W>
struct DiffLds {
    using Tile = DiffTile<W>;
    static constexpr int kRow = 2 * W, kKS = W / 32, kCB = W / 32;  // steps of 16 channels of a map, blocks of 32 channels
    // The lane's first row-per-lane read of a tile at `tile`; operand ks is at that ^ 32 ks.
    __device__ static unsigned rows(unsigned tile, int lane) { return tile + Tile::off(lane & 31, lane >> 5); }
    // The lane's first transposing read; rows 8 further are at that ^ 32, + 8 rows; block cb at that ^ 64 cb.
    __device__ static unsigned cols(unsigned tile, int lane) {
        const int b = lane >> 4, j = lane & 15;
        return tile + Tile::off(4 * (lane >> 5) + (j >> 2), (b & 1) * 2 + ((j & 3) >> 1)) + (j & 1) * 8;
    }
    template <int OFF>
    __device__ static void read_rows(u32x4 (&x)[kKS], unsigned at, int from) {
#pragma unroll
        for (int ks = 0; ks < kKS; ++ks) x[ks] = lds_read_b128_at<OFF>(at ^ 32 * (from + ks));
    }
    // Operands of rows 16 KK .. + 15: piece 2 cb and 2 cb + 1 of block cb (join2).
    template <int OFF, int KK>
    __device__ static void read_cols(u32x2 (&x)[2 * kCB], unsigned at) {
#pragma unroll
        for (int cb = 0; cb < kCB; ++cb) {
            x[2 * cb] = lds_read_tr16_at<OFF + 16 * KK * kRow>(at ^ 64 * cb);
            x[2 * cb + 1] = lds_read_tr16_at<OFF + (16 * KK + 8) * kRow>(at ^ (64 * cb + 32));
        }
    }
};

// fp32 numbers as sums of three bf16 numbers, which together hold all 24 bits (leading 16 bits of the number, of what is left, and of
// what is left then): a product of two is six of bf16, each accumulated in fp32, without the three that lie 2^-24 below it.  Tensors are split once
// a call into planes [row][3][W]; 2.7 times the rate of the fp32 matrix instructions.
struct DiffPlanes {
    bf16x8 x[3];
};
__device__ inline f32x16 diff_mma6(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16 c) {
    c = mfma32(a[2], b[0], c);
    c = mfma32(a[0], b[2], c);
    c = mfma32(a[1], b[1], c);
    c = mfma32(a[1], b[0], c);
    c = mfma32(a[0], b[1], c);
    return mfma32(a[0], b[0], c);
}
// The bits of diff_mma6(b, a, c)'s transpose.
__device__ inline f32x16 diff_mma6_swapped(const bf16x8 (&a)[3], const bf16x8 (&b)[3], f32x16 c) {
    c = mfma32(a[0], b[2], c);
    c = mfma32(a[2], b[0], c);
    c = mfma32(a[1], b[1], c);
    c = mfma32(a[0], b[1], c);
    c = mfma32(a[1], b[0], c);
    return mfma32(a[0], b[0], c);
}
// Leading parts of two numbers packed, and what is left of them.
__device__ inline unsigned diff_take_pair(float &x, float &y) {
    const unsigned u = __builtin_bit_cast(unsigned, x), v = __builtin_bit_cast(unsigned, y);
    x -= __builtin_bit_cast(float, u & 0xffff0000u);
    y -= __builtin_bit_cast(float, v & 0xffff0000u);
    return __builtin_amdgcn_perm(v, u, 0x07060302);
}
__device__ inline void diff_split8(const float (&v)[8], u32x4 (&planes)[3]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x = v[2 * e], y = v[2 * e + 1];
#pragma unroll
        for (int p = 0; p < 3; ++p) planes[p][e] = diff_take_pair(x, y);
    }
}
// diff_block_frag in three planes.
__device__ inline DiffPlanes diff_block_planes(const f32x16 &s, int kk) {
    float v[8];
    u32x4 x[3];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = s[8 * kk + e];
    diff_split8(v, x);
    return {{as_bf16x8(x[0]), as_bf16x8(x[1]), as_bf16x8(x[2])}};
}
template <int W>
__device__ inline DiffPlanes diff_global_planes(const __bf16 *row, int ks, int g, bool live) {
    return {{diff_global_frag(row, ks, g, live), diff_global_frag(row + W, ks, g, live), diff_global_frag(row + 2 * W, ks, g, live)}};
}
__device__ inline void diff_landed(u32x4 (&x)[3]) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2])); }
__device__ inline void diff_landed(u32x4 (&x)[3], u32x4 &y) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(y)); }
__device__ inline void diff_landed(u32x4 (&x)[3], unsigned &y) { asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(y)); }
__device__ inline void diff_landed(u32x2 (&x)[6]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]));
}
__device__ inline void diff_rows3(const u32x4 (&x)[3], bf16x8 (&to)[3]) {
#pragma unroll
    for (int p = 0; p < 3; ++p) to[p] = as_bf16x8(x[p]);
}
__device__ inline void diff_cols3(const u32x2 (&x)[6], bf16x8 (&to)[3]) {
#pragma unroll
    for (int p = 0; p < 3; ++p) to[p] = diff_join2(x[2 * p], x[2 * p + 1]);
}
// Operands of three plane tiles, one behind the other from OFF bytes on: rows (step ks of 16 channels) and columns (rows 16 KK .. + 15, block cb).
template <int W, int OFF>
__device__ inline void diff_read_rows3(u32x4 (&x)[3], unsigned rows, int ks) {
    constexpr int TILE = DiffTile<W>::kBytes;
    x[0] = lds_read_b128_at<OFF>(rows ^ 32 * ks);
    x[1] = lds_read_b128_at<OFF + TILE>(rows ^ 32 * ks);
    x[2] = lds_read_b128_at<OFF + 2 * TILE>(rows ^ 32 * ks);
}
template <int W, int OFF, int KK>
__device__ inline void diff_read_cols3(u32x2 (&x)[6], unsigned cols, int cb) {
    constexpr int TILE = DiffTile<W>::kBytes, AT = OFF + 16 * KK * 2 * W, EIGHT = 8 * 2 * W;
    x[0] = lds_read_tr16_at<AT>(cols ^ 64 * cb);
    x[1] = lds_read_tr16_at<AT + EIGHT>(cols ^ (64 * cb + 32));
    x[2] = lds_read_tr16_at<AT + TILE>(cols ^ 64 * cb);
    x[3] = lds_read_tr16_at<AT + TILE + EIGHT>(cols ^ (64 * cb + 32));
    x[4] = lds_read_tr16_at<AT + 2 * TILE>(cols ^ 64 * cb);
    x[5] = lds_read_tr16_at<AT + 2 * TILE + EIGHT>(cols ^ (64 * cb + 32));
}

// Loads of tiles into LDS by WAVES wavefronts, 1 KB an instruction: a lane fetches the chunk that belongs in its slot.  Rows at
// `limit` and beyond are fetched as the one before it (the kernels mask them).  HELD: a lane's offsets are kept in registers, or worked
// out at every load (a dozen instructions a tile, where registers are short).
template <int W, int WAVES, bool HELD = true>
struct DiffDma {
    using Tile = DiffTile<W>;
    static constexpr int kLoads = kDiffTile * W / (512 * WAVES), kRows = 512 / W, kChunks = W / 8;
    const char *base;
    long long step;
    unsigned off[HELD ? kLoads : 1];
    __device__ static unsigned chunk(int row, int slot) { return (Tile::off(row, slot) - row * 2 * W) / 16; }  // (its own inverse)
    __device__ unsigned offset(int i, int wave, int lane) const {
        return (unsigned)(lane / kChunks) * (unsigned)step + 16 * chunk((wave * kLoads + i) * kRows + lane / kChunks, lane % kChunks);
    }
    __device__ void start(const void *tensor, long long offset_, long long sn, int wave, int lane) {
        base = diff_uniform((const __bf16 *)tensor + offset_);
        step = 2 * sn;
        if (HELD)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) off[HELD ? i : 0] = offset(i, wave, lane);
    }
    __device__ void issue(unsigned char *tile, int row0, int limit, int wave, int lane) const {
        const char *from = base + row0 * step;
        if (row0 + kDiffTile <= limit) {  // (uniform)
            if (!HELD) asm volatile("" : "+v"(lane));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int first = (wave * kLoads + i) * kRows;
                __builtin_amdgcn_global_load_lds((diff_global_cvoid *)(from + first * step + (HELD ? off[HELD ? i : 0] : offset(i, wave, lane))),
                                                 (diff_lds_void *)(tile + first * 2 * W), 16, 0, 0);
            }
        } else {
            asm volatile("" : "+v"(lane));
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int first = (wave * kLoads + i) * kRows, row = first + lane / kChunks;
                const unsigned at = (unsigned)min(row, limit - 1 - row0);
                __builtin_amdgcn_global_load_lds((diff_global_cvoid *)(from + (at * (unsigned)step + 16 * chunk(row, lane % kChunks))), (diff_lds_void *)(tile + first * 2 * W), 16, 0, 0);
            }
        }
    }
};

// The same for the three planes of split fp32 rows.
template <int W, int WAVES, bool HELD = true>
struct DiffDma3 {
    DiffDma<W, WAVES, HELD> one;
    __device__ void start(const __bf16 *planes, long long row, int wave, int lane) { one.start(planes, row * 3 * W, 3 * W, wave, lane); }
    __device__ void issue(unsigned char *tiles, int row0, int limit, int wave, int lane) const {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            DiffDma<W, WAVES, HELD> plane = one;
            plane.base += p * 2 * W;
            plane.issue(tiles + p * DiffTile<W>::kBytes, row0, limit, wave, lane);
        }
    }
};

// lambda of head h: exp(lq1 . lk1) - exp(lq2 . lk2) + init, and its two exponentials, in every lane of the wavefront.
struct DiffLambda {
    float e1, e2, value;
};
template <int W>
__device__ inline DiffLambda diff_lambda(const DiffArgs &a, int h, int lane) {
    const int at = h * a.l_step + lane;
    float x1 = 0.f, x2 = 0.f;
    if (lane < W / 2) {
        x1 = a.lq1[at] * a.lk1[at];
        x2 = a.lq2[at] * a.lk2[at];
    }
    DiffLambda l;
    l.e1 = expf(wave_sum(x1));
    l.e2 = expf(wave_sum(x2));
    l.value = l.e1 - l.e2 + a.l_init;
    return l;
}
// lambda of the lane's head `mine`, one of first .. last, which the wavefront's rows belong to (numbers modulo the heads).  More than two: eight at a
// time, whose loads and sums go on together (one query of 32 heads against 100 keys of one kv head x 1 024 sequences, a set a head: 53 us one after the
// other, 44 so).
template <int W>
__device__ inline float diff_lambda_of(const DiffArgs &a, int first, int last, int mine, int lane) {
    if (!a.l_step) return diff_lambda<W>(a, 0, lane).value;
    float lam = 0.f;
    if (last - first < 2) {
        for (int x = first; x <= last; ++x) {
            const float value = diff_lambda<W>(a, x % a.heads, lane).value;
            if (mine == x) lam = value;
        }
        return lam;
    }
    for (int from = first; from <= last; from += 8) {
        float x1[8], x2[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int at = min(from + u, last) % a.heads * a.l_step + min(lane, W / 2 - 1);
            x1[u] = a.lq1[at] * a.lk1[at];
            x2[u] = a.lq2[at] * a.lk2[at];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float value = expf(wave_sum(lane < W / 2 ? x1[u] : 0.f)) - expf(wave_sum(lane < W / 2 ? x2[u] : 0.f)) + a.l_init;
            if (mine == from + u) lam = value;
        }
    }
    return lam;
}

// A weight of a score s is 2^(s c - m), the product exact and the reference m rounded, in every tile and in both passes: what the rounding costs is one factor
// of a row's weights and of their sum.  It is up to 2^(|m| 2^-24): from |m| = 2^24 on products are rounded as the reference was.  Both by the same
// instruction, (s first) then - m: (s c) 1 - m there, (s 1) c - m below.
__device__ inline bool diff_far(float m) { return fabsf(m) >= 16777216.f && fabsf(m) < INFINITY; }
struct DiffScaling {
    float first, then;
    __device__ DiffScaling(float c, bool far) : first(far ? c : 1.f), then(far ? 1.f : c) {}
};

// Four consecutive channels of an output row.
__device__ inline void diff_store4(float *p, f32x4 x) { *(f32x4 *)p = x; }
__device__ inline void diff_store4(__bf16 *p, f32x4 x) { *(u32x2 *)p = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])}; }

// Query rows of all sequences and heads.
__host__ __device__ inline long long diff_rows(const DiffArgs &a) { return (long long)a.B * a.heads * a.n_q; }

// Validates the descriptor, and with it the base pointers of q, k, v, o.
jv_status diff_problem(const jv_diff_attn_desc *desc, const void *q, const void *k, const void *v, void *o,
                       const jv_diff_lambda *lambda, float scale, DiffProblem *out);
jv_status diff_check_desc(const jv_diff_attn_desc *desc);
// fp32 tensors: bytes of their planes in a workspace (with_d_o: of dO too), and the launch that fills them.
size_t diff_planes_bytes(const jv_diff_attn_desc *desc, bool with_d_o);
jv_status diff_split(DiffArgs &a, int W, void *memory, bool with_d_o, hipStream_t stream);
// Strides of a [b, h, n, W] tensor; a written one must have a place of its own for every row.
jv_status diff_check_strides(const char *name, const jv_strides &s, int64_t b, int64_t h, int64_t n, int W, int64_t align, bool written);
int64_t diff_span(const jv_strides &s, int64_t b, int64_t h, int64_t n, int W);  // elements up to the end of the last row
size_t diff_saved_bytes(const jv_diff_attn_desc *desc);
void diff_use_saved(DiffProblem *p, void *saved);

// Kernels are built for two types and two widths: f(DiffKind of the call).
template <typename ELEM, int WIDTH>
struct DiffKind {
    using T = ELEM;
    static constexpr int W = WIDTH;
};
template <typename F>
jv_status diff_with_kind(bool bf16, int W, F f) {
    if (bf16) return W == 128 ? f(DiffKind<__bf16, 128>()) : f(DiffKind<__bf16, 64>());
    return W == 128 ? f(DiffKind<float, 128>()) : f(DiffKind<float, 64>());
}

}  // namespace jv
