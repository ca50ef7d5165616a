// Rows in 4 or 8 bits times weights in microscaled 4 bits.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sbn_mx.h"
#include "sbn_ops.h"

namespace sbn {
namespace {

typedef int i8v __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

// ---- layout ------------------------------------------------------------------------------------

// Row-major codes and scales into tiles (back = false), or tiles into row-major ones.  One lane of the layout per thread.
__global__ __launch_bounds__(256) void layout_codes_kernel(uint8_t* rows, uint8_t* tiles, long long lanes, int steps, int blocks, int c_out, int c_in, bool back)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= lanes) return;
    const int lane = (int)(i & 63);
    const long long tile = i >> 6;
    const long long row = tile / steps * 16 + (lane & 15);
    const int block = (int)(tile % steps) * 4 + (lane >> 4);
    const bool in = row < c_out && block < blocks;
    u4* const t = (u4*)tiles + i;
    u4* const r = (u4*)rows + row * blocks + block;
    if (back) {
        if (in) *r = *t;
        return;
    }
    u4 v = {};
    if (in) {
        v = *r;
        const int left = c_in - block * 32;                               // codes past c_in are no weights
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int n = left - 8 * w;
            if (n < 8) v[w] = n <= 0 ? 0u : v[w] & ((1u << 4 * n) - 1u);
        }
    }
    *t = v;
}
__global__ __launch_bounds__(256) void layout_scales_kernel(uint8_t* rows, uint8_t* tiles, long long bytes, int quads, int blocks, int c_out, bool back)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= bytes) return;
    const int lane = (int)(i >> 2 & 63);
    const long long q = i >> 8;
    const long long row = q / quads * 16 + (lane & 15);
    const int block = ((int)(q % quads) * 4 + (int)(i & 3)) * 4 + (lane >> 4);
    const bool in = row < c_out && block < blocks;
    if (back) {
        if (in) rows[row * blocks + block] = tiles[i];
    } else {
        const int s = in ? rows[row * blocks + block] : 0;
        tiles[i] = (uint8_t)(s > 252 ? 255 : s);
    }
}

// ---- the product -------------------------------------------------------------------------------

struct LinearArgs {
    const uint8_t *w, *ws;                  // tiles
    const float* bias;
    const uint8_t* x;                       // codes [rows][blocks * 16 or 32]
    const uint8_t* xs;                      // scales [rows][blocks], or float [rows]
    void* y;
    long long rows, ldy;
    int c_out, blocks, steps, quads, tile_rows, act;
};

// The scale a byte stands for, as the conversions take it: 255 is NaN.
__device__ inline float mx_scale(unsigned byte)
{
    return __builtin_bit_cast(float, byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}
// Eight E2M1 codes / E4M3 codes times their scale as bfloat16, which holds them exactly (4 significant bits at most).
__device__ inline b8 wide4(unsigned c, float scale)
{
    const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 1);
    const b2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, 3);
    return (b8){a.x, a.y, b.x, b.y, d.x, d.y, e.x, e.y};
}
__device__ inline b8 wide8(unsigned lo, unsigned hi, float scale)
{
    const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const b2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return (b8){a.x, a.y, b.x, b.y, d.x, d.y, e.x, e.y};
}

// Four consecutive output channels of a row.
template <class T>
__device__ inline void put4(T* y, int n, f4 v)
{
    if (n >= 4) {
        if constexpr (sizeof(T) == 4) {
            ((Any16*)y)->v = __builtin_bit_cast(u4, v);
        } else {
            T t[4] = {Elem<T>::put(v[0]), Elem<T>::put(v[1]), Elem<T>::put(v[2]), Elem<T>::put(v[3])};
            ((Any8*)y)->v = __builtin_bit_cast(u2, t);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) y[i] = Elem<T>::put(v[i]);
    }
}
template <int FMT, class T>
__device__ inline void finish4(const LinearArgs& a, long long row, int n, f4 v)
{
    if (row >= a.rows || n >= a.c_out) return;
    if constexpr (FMT == SBN_FP8_ROW) v *= ((const float*)a.xs)[row];
    v += *(const f4*)(a.bias + n);
    if (a.act == SBN_ACT_RELU)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = v[i] > 0.0f ? v[i] : 0.0f;
    put4((T*)a.y + row * a.ldy + n, a.c_out - n, v);
}

// 16 rows x 16 NT output channels to a workgroup, whose four waves take every fourth quad of steps (512 input channels) and join
// their sums in LDS.
template <int FMT, class T, int NT>
__global__ __launch_bounds__(256) void rows_kernel(const LinearArgs a)
{
    __shared__ f4 sums[3][NT][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
    const int tile0 = blockIdx.x * NT;
    const long long row = (long long)blockIdx.y * 16 + (lane & 15);
    const bool live = row < a.rows;
    const uint8_t* const x = a.x + (live ? row : 0) * a.blocks * (FMT == SBN_MXFP4 ? 16 : 32);
    const uint8_t* const xs = a.xs + (live ? row : 0) * a.blocks;
    f4 acc[NT] = {};
    for (int q = wave; q < a.quads; q += 4) {
        unsigned ws[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int tile = min(tile0 + t, a.tile_rows - 1);
            ws[t] = ((const unsigned*)a.ws)[((long long)tile * a.quads + q) * 64 + lane];
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int step = q * 4 + s;
            if (step >= a.steps) break;
            u4 w[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int tile = min(tile0 + t, a.tile_rows - 1);
                w[t] = ((const u4*)a.w)[((long long)tile * a.steps + step) * 64 + lane];
            }
            const int block = step * 4 + g;
            const bool in = live && block < a.blocks;
            if constexpr (FMT == SBN_MXFP4) {
                const u4 c = in ? ((const u4*)x)[block] : (u4){};
                const int sx = in ? xs[block] : 0;
                const i8v B = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const i8v A = {(int)w[t].x, (int)w[t].y, (int)w[t].z, (int)w[t].w, 0, 0, 0, 0};
                    acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc[t], 4, 4, 0, (int)(ws[t] >> 8 * s & 255u), 0, sx);
                }
            } else {
                u4 c[2] = {};
                float sx = 1.0f;
                if (in) {
                    c[0] = ((const u4*)x)[block * 2], c[1] = ((const u4*)x)[block * 2 + 1];
                    if constexpr (FMT == SBN_MXFP8) sx = mx_scale(xs[block]);
                }
                b8 B[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) B[i] = wide8(c[i >> 1][(i & 1) * 2], c[i >> 1][(i & 1) * 2 + 1], sx);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const float sw = mx_scale(ws[t] >> 8 * s & 255u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide4(w[t][i], sw), B[i], acc[t], 0, 0, 0);
                }
            }
        }
    }
    if (wave)
#pragma unroll
        for (int t = 0; t < NT; ++t) sums[wave - 1][t][lane] = acc[t];
    __syncthreads();
    if (wave == 0)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (tile0 + t < a.tile_rows) finish4<FMT, T>(a, row, (tile0 + t) * 16 + g * 4, acc[t] + sums[0][t][lane] + sums[1][t][lane] + sums[2][t][lane]);
}

template <int FMT, class T>
int run_linear(LinearArgs a, hipStream_t stream)
{
    const long long all = a.rows, most = 65535ll * 16;
    for (long long r0 = 0; r0 < all; r0 += most) {
        LinearArgs b = a;
        b.rows = std::min(most, all - r0);
        b.x = a.x + r0 * a.blocks * (FMT == SBN_MXFP4 ? 16 : 32);
        b.xs = a.xs + r0 * (FMT == SBN_FP8_ROW ? 4 : a.blocks);
        b.y = (T*)a.y + r0 * a.ldy;
        const dim3 grid((unsigned)a.tile_rows, (unsigned)((b.rows + 15) / 16));
        rows_kernel<FMT, T, 1><<<grid, 256, 0, stream>>>(b);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return fail(SBN_EHIP, "sbn_linear_mx: %s", hipGetErrorString(e));
    }
    return SBN_OK;
}
template <int FMT>
int run_linear(const LinearArgs& a, int y_type, hipStream_t stream)
{
    return y_type == SBN_F32 ? run_linear<FMT, float>(a, stream) : y_type == SBN_BF16 ? run_linear<FMT, __bf16>(a, stream)
                                                                                     : run_linear<FMT, _Float16>(a, stream);
}

}  // namespace

int launch_mx_layout(const sbn_mx* p, const uint8_t* codes, const uint8_t* scales, bool back, uint8_t* codes_out, uint8_t* scales_out)
{
    const long long lanes = (long long)p->tile_rows * p->steps * 64, bytes = (long long)p->tile_rows * p->quads * 256;
    uint8_t* const c = back ? codes_out : const_cast<uint8_t*>(codes);
    uint8_t* const s = back ? scales_out : const_cast<uint8_t*>(scales);
    layout_codes_kernel<<<(unsigned)((lanes + 255) / 256), 256>>>(c, p->d_codes, lanes, p->steps, p->blocks, p->c_out, p->c_in, back);
    layout_scales_kernel<<<(unsigned)((bytes + 255) / 256), 256>>>(s, p->d_scales, bytes, p->quads, p->blocks, p->c_out, back);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return fail(SBN_EHIP, "sbn_mx layout: %s", hipGetErrorString(e));
    return SBN_OK;
}

size_t linear_mx_workspace(const sbn_mx*, int, long long) { return 0; }

int launch_linear_mx(const sbn_mx* p, const void* codes, const void* scales, int format, long long rows, void* y, int y_type, long long ldy, void*, void* stream)
{
    LinearArgs a = {};
    a.w = p->d_codes, a.ws = p->d_scales, a.bias = p->d_bias, a.x = (const uint8_t*)codes, a.xs = (const uint8_t*)scales;
    a.y = y, a.rows = rows, a.ldy = ldy, a.c_out = p->c_out, a.blocks = p->blocks, a.steps = p->steps, a.quads = p->quads;
    a.tile_rows = p->tile_rows, a.act = p->act;
    const hipStream_t s = (hipStream_t)stream;
    return format == SBN_MXFP4 ? run_linear<SBN_MXFP4>(a, y_type, s) : format == SBN_MXFP8 ? run_linear<SBN_MXFP8>(a, y_type, s)
                                                                                         : run_linear<SBN_FP8_ROW>(a, y_type, s);
}

}  // namespace sbn
