// Gradient of LayerNorm (jv_layernorm_bwd).  With xh = (x - mean) rstd and g = dy gamma, per row
//     dx = rstd (g - mean(g) - xh mean(g xh)) + residual,
// and dgamma = sum dy xh, dbeta = sum dy over the rows.  One pass over x and dy: a row lies in the registers of LANES lanes, which
// take every so many-th row and keep the column sums of theirs; a second launch adds the workgroups' sums in their order.
// Bound by memory where rows are many.
#include "jv_common.h"
#include "jv_mfma.h"
#include "jv_plan.h"

#include <type_traits>

namespace jv {

struct NormGradArgs {
    const void *x, *dy, *residual;
    const float *gamma;
    void *dx;
    float *part;  // [workgroups][2][cols]: sums of dy xh, then of dy; or null
    long long rows;
    int cols;
    float eps;
};

// Eight columns from an element on.
template <bool BF16>
__device__ inline void norm_load8(const void *x, size_t at, float (&v)[8]) {
    if (BF16) {
        const u32x4 raw = *(const u32x4 *)((const __bf16 *)x + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = bf16_lo(raw[e]);
            v[2 * e + 1] = bf16_hi(raw[e]);
        }
    } else {
        const f32x4 a = *(const f32x4 *)((const float *)x + at), b = *(const f32x4 *)((const float *)x + at + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
    }
}
template <bool BF16>
__device__ inline void norm_store8(void *x, size_t at, const float (&v)[8]) {
    if (BF16) {
        *(u32x4 *)((__bf16 *)x + at) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    } else {
        *(f32x4 *)((float *)x + at) = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4 *)((float *)x + at + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
}

template <int CTRL>
__device__ inline float norm_add_dpp(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
// Sum over groups of LANES neighbouring lanes (8 to 64), in every lane, by exchanges of registers: with the neighbour, the other
// pair of a quad, then mirrored halves of 8 and 16 lanes (equal inside the halves by then), 16 and 32 lanes across.
template <int LANES>
__device__ inline float norm_sum(float x) {
    x = norm_add_dpp<0xb1>(x);
    x = norm_add_dpp<0x4e>(x);
    x = norm_add_dpp<0x141>(x);
    if (LANES >= 16) x = norm_add_dpp<0x140>(x);
    if (LANES >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
    }
    if (LANES >= 64) {
        float lo, hi;
        pair_values(x, &lo, &hi);
        x = lo + hi;
    }
    return x;
}

// LANES lanes a row, NV pieces of eight columns a lane: piece p of lane l is columns 8 (l + LANES p) .. + 7.  At most two pieces, so
// that two workgroups share a unit: rows of more than 1 024 columns lie in two to eight wavefronts, which join their sums through LDS (three or four pieces
// in one wavefront, or in four with half the wavefronts a unit: 20 000 x 1280 in bf16 61 us, 16 000 x 2560 113, so 35 and 53).
// Reads and writes a row once: 32 768 x 1024 in bf16 with a residual (268 MB) 45 us out of the caches, both launches 55 from memory (4.8 TB/s);
// 262 144 x 128 without (201 MB) 37 and 44.  Few rows: 200 x 1024 5.3 us, a chain of two row sums.
template <bool X_BF16, bool DY_BF16, int LANES, int NV>
__global__ void __launch_bounds__(kNormGradThreads) layernorm_bwd_kernel(NormGradArgs a) {
    constexpr int THREADS = kNormGradThreads, ROWS = THREADS / LANES;  // rows of a workgroup at a time
    constexpr int ROW_WAVES = LANES > 64 ? LANES / 64 : 1, GROUPS = LANES > 64 ? ROWS : THREADS / 64;  // wavefronts of a row; column sums of a workgroup
    const int tid = threadIdx.x, lane = tid % LANES, wave = tid >> 6;
    __shared__ float across[2][2][THREADS / 64];
    __shared__ __align__(16) float column[GROUPS * 8 * LANES];
    const float inv_cols = 1.0f / (float)a.cols;
    int turn = 0;
    // both sums over the lanes of a row
    auto sums = [&](float &x, float &y) {
        x = norm_sum<(LANES < 64 ? LANES : 64)>(x);
        y = norm_sum<(LANES < 64 ? LANES : 64)>(y);
        if constexpr (ROW_WAVES > 1) {
            if ((tid & 63) == 0) {
                across[turn][0][wave] = x;
                across[turn][1][wave] = y;
            }
            __syncthreads();
            x = y = 0.f;
#pragma unroll
            for (int w = 0; w < ROW_WAVES; ++w) {
                x += across[turn][0][wave / ROW_WAVES * ROW_WAVES + w];
                y += across[turn][1][wave / ROW_WAVES * ROW_WAVES + w];
            }
            turn ^= 1;  // (the next sums are written elsewhere: one barrier each suffices)
        }
    };
    float gamma[NV][8], dgamma[NV][8], dbeta[NV][8];
#pragma unroll
    for (int p = 0; p < NV; ++p) {
        const int c = 8 * (lane + LANES * p);
        if (c < a.cols) norm_load8<false>(a.gamma, c, gamma[p]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (c >= a.cols) gamma[p][e] = 0.f;
            dgamma[p][e] = dbeta[p][e] = 0.f;
        }
    }
    // (the loop runs alike for all lanes of a workgroup: rows past the end are read as zeros and not written)
    for (long long first = (long long)blockIdx.x * ROWS; first < a.rows; first += (long long)gridDim.x * ROWS) {
        const long long row = first + tid / LANES;
        const bool live = row < a.rows;
        float x[NV][8], dy[NV][8], sum = 0.f, sum_g = 0.f;
#pragma unroll
        for (int p = 0; p < NV; ++p) {
            const int c = 8 * (lane + LANES * p);
            if (live && c < a.cols) {
                norm_load8<X_BF16>(a.x, (size_t)row * a.cols + c, x[p]);
                norm_load8<DY_BF16>(a.dy, (size_t)row * a.cols + c, dy[p]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[p][e] = dy[p][e] = 0.f;
            }
        }
#pragma unroll
        for (int p = 0; p < NV; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum += x[p][e];
                sum_g = fmaf(dy[p][e], gamma[p][e], sum_g);
            }
        sums(sum, sum_g);
        const float mean = sum * inv_cols, mean_g = sum_g * inv_cols;
        float sq = 0.f, sum_gx = 0.f;
#pragma unroll
        for (int p = 0; p < NV; ++p) {
            if (8 * (lane + LANES * p) < a.cols) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[p][e] -= mean;
                    sq = fmaf(x[p][e], x[p][e], sq);
                    sum_gx = fmaf(dy[p][e] * gamma[p][e], x[p][e], sum_gx);
                }
            }
        }
        sums(sq, sum_gx);
        const float rstd = 1.0f / sqrtf(sq * inv_cols + a.eps), mean_gx = sum_gx * rstd * inv_cols;
#pragma unroll
        for (int p = 0; p < NV; ++p) {
            const int c = 8 * (lane + LANES * p);
            if (!live || c >= a.cols) continue;
            const size_t at = (size_t)row * a.cols + c;
            float add[8] = {}, out[8];
            if (a.residual) norm_load8<X_BF16>(a.residual, at, add);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = x[p][e] * rstd;
                out[e] = fmaf(rstd, fmaf(-xh, mean_gx, fmaf(dy[p][e], gamma[p][e], -mean_g)), add[e]);
                dgamma[p][e] = fmaf(dy[p][e], xh, dgamma[p][e]);
                dbeta[p][e] += dy[p][e];
            }
            norm_store8<X_BF16>(a.dx, at, out);
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int p = 0; p < NV; ++p) {
            float(&v)[8] = which ? dbeta[p] : dgamma[p];
            // rows of a wavefront (every LANES-th lane), then those of the workgroup
#pragma unroll
            for (int x = LANES; x < 64; x *= 2)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += __shfl_xor(v[e], x);
            __syncthreads();
            if (LANES >= 64 || (tid & 63) < LANES) {
#pragma unroll
                for (int e = 0; e < 8; ++e) column[((LANES > 64 ? tid / LANES : wave) * 8 + e) * LANES + lane] = v[e];
            }
            __syncthreads();
            for (int y = tid; y < 8 * LANES; y += THREADS) {
                const int e = y / LANES, l = y % LANES, to = 8 * (l + LANES * p) + e;
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < GROUPS; ++w) s += column[(w * 8 + e) * LANES + l];
                if (to < a.cols) part[(size_t)which * a.cols + to] = s;
            }
        }
}

// Column sums of the workgroups' sums: 64 of the 2 * cols columns a workgroup, 16 wavefronts that take every 16th part (2.4 us of 25 parts of 1 024 columns,
// 4.7 of 512; 3.1 MB of 768).
__global__ void __launch_bounds__(1024) layernorm_bwd_columns_kernel(const float *__restrict__ part, int n, int cols, float *__restrict__ dgamma,
                                                                     float *__restrict__ dbeta) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    __shared__ float sums[16][64];
    float sum = 0.f;
    const float *column = part + min(c, 2 * cols - 1);
    for (int p0 = wave; p0 < n; p0 += 256) {  // sixteen loads at a time, also where fewer are left (of the last part again, not added)
        float x[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) x[u] = column[(size_t)min(p0 + 16 * u, n - 1) * 2 * cols];
#pragma unroll
        for (int u = 0; u < 16; ++u) sum += p0 + 16 * u < n ? x[u] : 0.f;
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || c >= 2 * cols) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) sum += sums[w][lane];
    if (c < cols) dgamma[c] = sum;
    else dbeta[c - cols] = sum;
}

// f(integral_constant LANES, integral_constant NV) for rows of `cols`.
template <typename F>
static void norm_with_row(int cols, F f) {
    auto lanes = [&](auto l) {
        if (norm_grad_pieces(cols) == 1) f(l, std::integral_constant<int, 1>());
        else f(l, std::integral_constant<int, 2>());
    };
    switch (norm_grad_lanes(cols)) {
        case 8: return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
        case 16: return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
        case 32: return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
        case 64: return lanes(std::integral_constant<int, 64>());
        case 128: return f(std::integral_constant<int, 128>(), std::integral_constant<int, 2>());
        case 256: return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
        default: return f(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
    }
}

static jv_status norm_check_sizes(int64_t rows, int32_t cols) {
    if (rows <= 0 || cols <= 0) return fail(JV_ERR_INVALID_ARG, "rows and cols must be positive");
    if (cols % 8) return fail(JV_ERR_UNSUPPORTED, "cols must be a multiple of 8");
    if (cols > 8192) return fail(JV_ERR_UNSUPPORTED, "cols above 8192");
    if (rows > (1ll << 31)) return fail(JV_ERR_UNSUPPORTED, "rows above 2^31");
    return JV_OK;
}

}  // namespace jv

extern "C" {

size_t jv_layernorm_bwd_workspace_bytes(int64_t rows, int32_t cols) {
    jv::clear_error();
    if (jv::norm_check_sizes(rows, cols) != JV_OK) return 0;
    return ((size_t)jv::norm_grad_groups(rows, cols) * 2 * cols * 4 + 255) & ~(size_t)255;
}

jv_status jv_layernorm_bwd(const void *x, const float *gamma, const void *dy, const void *residual, void *dx,
                           float *dgamma, float *dbeta, int64_t rows, int32_t cols, float eps, jv_dtype x_dtype,
                           jv_dtype dy_dtype, void *workspace, size_t workspace_bytes, void *hip_stream) {
    jv::clear_error();
    if (!x || !gamma || !dy || !dx) return jv::fail(JV_ERR_INVALID_ARG, "null pointer");
    if (!dgamma != !dbeta) return jv::fail(JV_ERR_INVALID_ARG, "dgamma and dbeta: both, or none");
    jv_status st = jv::norm_check_sizes(rows, cols);
    if (st != JV_OK) return st;
    if (!(eps >= 0.f)) return jv::fail(JV_ERR_INVALID_ARG, "eps must be >= 0");
    if ((x_dtype != JV_F32 && x_dtype != JV_BF16) || (dy_dtype != JV_F32 && dy_dtype != JV_BF16))
        return jv::fail(JV_ERR_INVALID_ARG, "unknown dtype");
    if (((uintptr_t)x | (uintptr_t)gamma | (uintptr_t)dy | (uintptr_t)residual | (uintptr_t)dx | (uintptr_t)dgamma | (uintptr_t)dbeta) & 15)
        return jv::fail(JV_ERR_INVALID_ARG, "pointers must be 16-byte aligned");
    const size_t n = (size_t)rows * cols, x_bytes = n * (x_dtype == JV_BF16 ? 2 : 4), dy_bytes = n * (dy_dtype == JV_BF16 ? 2 : 4);
    auto meet = [](const void *p, size_t p_bytes, const void *q, size_t q_bytes) {
        return (uintptr_t)p < (uintptr_t)q + q_bytes && (uintptr_t)q < (uintptr_t)p + p_bytes;
    };
    if (meet(dx, x_bytes, x, x_bytes) || meet(dx, x_bytes, dy, dy_bytes) || (residual && residual != dx && meet(dx, x_bytes, residual, x_bytes)))
        return jv::fail(JV_ERR_INVALID_ARG, "dx must not overlap an input (residual: only as the same tensor)");
    const size_t need = jv_layernorm_bwd_workspace_bytes(rows, cols);
    if (dgamma) {
        if (!workspace) return jv::fail(JV_ERR_INVALID_ARG, "workspace must be non-null");
        if ((uintptr_t)workspace & 255) return jv::fail(JV_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
        if (workspace_bytes < need) return jv::fail(JV_ERR_WORKSPACE_TOO_SMALL, "workspace holds %zu bytes, %zu are needed", workspace_bytes, need);
    }
    const jv::NormGradArgs a{x, dy, residual, gamma, dx, dgamma ? (float *)workspace : nullptr, rows, cols, eps};
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int groups = (int)jv::norm_grad_groups(rows, cols);
    jv::norm_with_row(cols, [&](auto lanes, auto nv) {
        constexpr int L = decltype(lanes)::value, NV = decltype(nv)::value;
        auto kernel = x_dtype == JV_BF16 ? (dy_dtype == JV_BF16 ? jv::layernorm_bwd_kernel<true, true, L, NV> : jv::layernorm_bwd_kernel<true, false, L, NV>)
                                         : (dy_dtype == JV_BF16 ? jv::layernorm_bwd_kernel<false, true, L, NV> : jv::layernorm_bwd_kernel<false, false, L, NV>);
        hipLaunchKernelGGL(kernel, dim3(groups), dim3(jv::kNormGradThreads), 0, stream, a);
    });
    if ((st = jv::launch_status("layernorm_bwd_kernel")) != JV_OK || !dgamma) return st;
    hipLaunchKernelGGL(jv::layernorm_bwd_columns_kernel, dim3((2 * cols + 63) / 64), dim3(1024), 0, stream, (const float *)workspace, groups, cols, dgamma, dbeta);
    return jv::launch_status("layernorm_bwd_columns_kernel");
}

}  // extern "C"
