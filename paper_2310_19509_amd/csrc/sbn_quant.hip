// Rows into 4- and 8-bit formats and back, and the root-mean-square norm with the residual's addition in front.
//
// All of it is bound by memory: every kernel reads its inputs once with 16-byte loads (32-bit rows: two), eight columns
// to a lane -- a "unit" -- so that four neighbouring lanes hold a block of 32 and its largest magnitude takes two lane swaps.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "sbn_mx.h"
#include "sbn_ops.h"

namespace sbn {
namespace {

// Units of a row: its blocks of 32 columns, four each.
__host__ __device__ inline long long units_of(long long cols) { return (cols + 31) / 32 * 4; }

template <int FMT>
__device__ inline void put_block_codes(const float (&v)[8], void* codes, uint8_t* scales, long long at)
{
    const unsigned top = quad_max(top_bits(v));
    const int byte = scale_byte<FMT == SBN_MXFP4 ? kEmax4 : kEmax8>(top);
    const float scale = scale_of(byte == 255 ? 0 : byte);
    if constexpr (FMT == SBN_MXFP4)
        ((unsigned*)codes)[at] = codes4(v, scale);
    else
        ((u2*)codes)[at] = codes8(v, scale);
    if ((at & 3) == 0) scales[at >> 2] = (uint8_t)byte;
}

// Blocks.  A thread takes kItems units of the launch's rows, a workgroup apart.
constexpr int kItems = 4;
template <class T, int FMT, bool ONCE>
__global__ __launch_bounds__(256) void quantize_kernel(const T* __restrict__ x, long long ldx, unsigned units, unsigned total,
                                                       long long cols, void* __restrict__ codes, uint8_t* __restrict__ scales)
{
    const unsigned first = blockIdx.x * (256u * kItems) + threadIdx.x;
    Raw<T> raw[kItems];
    const T* row[kItems];
    unsigned unit[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const unsigned u = min(first + 256u * i, total - 1u);
        row[i] = x + (long long)(u / units) * ldx;
        unit[i] = u % units;
        raw[i] = fetch_unit<ONCE>(row[i], unit[i], cols);
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const unsigned u = first + 256u * i;
        float v[8];
        expand_unit(raw[i], row[i], unit[i], cols, v, 0.0f);
        if (u < total) put_block_codes<FMT>(v, codes, scales, u);      // (blocks are whole: four lanes agree)
    }
}

template <class T, int FMT>
__global__ __launch_bounds__(256) void dequantize_kernel(const void* __restrict__ codes, const void* __restrict__ scales, T* __restrict__ y, long long ldy,
                                                         unsigned units, unsigned total, long long cols)
{
    const unsigned first = blockIdx.x * (256u * kItems) + threadIdx.x;
    u2 c[kItems];
    float s[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const unsigned u = min(first + 256u * i, total - 1u);
        if constexpr (FMT == SBN_MXFP4)
            c[i].x = ((const unsigned*)codes)[u];
        else
            c[i] = ((const u2*)codes)[u];
        if constexpr (FMT == SBN_FP8_ROW) {
            s[i] = ((const float*)scales)[u / units];
        } else {
            const int byte = ((const uint8_t*)scales)[u >> 2];
            s[i] = byte == 255 ? __builtin_nanf("") : scale_of(byte);
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const unsigned u = first + 256u * i;
        if (u >= total) return;
        f2 f[4];
        if constexpr (FMT == SBN_MXFP4) {
            f[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, 1.0f, 0);
            f[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, 1.0f, 1);
            f[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, 1.0f, 2);
            f[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i].x, 1.0f, 3);
        } else {
            f[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i].x, false);
            f[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i].x, true);
            f[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i].y, false);
            f[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i].y, true);
        }
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = f[j >> 1][j & 1] * s[i];
        const unsigned unit = u % units;
        if ((long long)unit * 8 < cols) store_unit(y + (long long)(u / units) * ldy, unit, cols, v);
    }
}

// What the row kernel needs.  `norm` 0: y = x (the row format of plain rows).
struct RowArgs {
    long long rows, cols, ldx, ldr, ldt, ldy;
    const void* x;
    const void* residual;
    void* total;
    const float* weight;
    void* y;
    void* codes;
    void* scales;
    float eps;
    int norm, format;
};

struct Root {                              // 1 / sqrt(mean + eps) as a sum of two floats
    float hi, lo;
};
__device__ inline Root inverse_root(float sum, long long cols, float eps)
{
    const float s = sum / (float)cols + eps;
    Root r;
    r.hi = rsqrtf(s);
    // one Newton step kept apart: the residue 1 - s r^2 with the product's own rounding in it
    const float t = s * r.hi, te = __builtin_fmaf(s, r.hi, -t);
    const float e = __builtin_fmaf(-t, r.hi, 1.0f) - te * r.hi;
    r.lo = s > 0.0f && s < __builtin_inff() ? 0.5f * r.hi * e : 0.0f;
    return r;
}
// h * w / rms with one rounding: codes that lie near a tie go where the exact value goes, up to the sum's own error.
__device__ inline float normed(float h, float w, const Root& r)
{
    const float p = h * w, e = __builtin_fmaf(h, w, -p);
    return __builtin_fmaf(p, r.hi, __builtin_fmaf(p, r.lo, e * r.hi));
}

// Sum / largest over a row's threads, the same on all of them.
template <int THREADS>
__device__ inline float row_sum(float v, float* lds)
{
    v = wave_sum(v);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) v += lds[i];
    }
    return v;
}
template <int THREADS>
__device__ inline unsigned row_max(unsigned v, unsigned* lds)
{
    v = wave_max(v);
    if constexpr (THREADS > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) v = max(v, lds[i]);
    }
    return v;
}

template <class XT>
__device__ inline void put_row_outputs(const RowArgs& a, long long row, long long unit, const float (&v)[8], float inverse)
{
    const long long at = row * units_of(a.cols) + unit;
    if (a.y && unit * 8 < a.cols) store_unit((XT*)a.y + row * a.ldy, unit, a.cols, v);
    if (a.format == SBN_MXFP4) {
        put_block_codes<SBN_MXFP4>(v, a.codes, (uint8_t*)a.scales, at);
    } else if (a.format == SBN_MXFP8) {
        put_block_codes<SBN_MXFP8>(v, a.codes, (uint8_t*)a.scales, at);
    } else if (a.format == SBN_FP8_ROW) {
        float q[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = v[j] * inverse;
        ((u2*)a.codes)[at] = codes8(q, 1.0f);
    }
}

// scale and 448 (1 / a) of a row from the bits of its largest magnitude
__device__ inline float row_scale(unsigned top, float& inverse)
{
    const float t = __builtin_bit_cast(float, top);
    inverse = 0.0f;
    if (top >= 0x7F800000u) return __builtin_nanf("");
    if (t < kLeastRow) return 0.0f;
    inverse = kTop8 * (1.0f / t);
    return t / kTop8;
}

// One row to THREADS threads, held in registers: ITEMS units each.  RT: the residual's type, or void.
template <class XT, class RT, int THREADS, int ITEMS, bool ONCE = false>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void row_kernel(const RowArgs a)
{
    __shared__ float lds_sum[16];
    __shared__ unsigned lds_max[16];
    constexpr bool ADD = !std::is_same<RT, void>::value;
    using R = typename std::conditional<ADD, RT, XT>::type;
    const int t = threadIdx.x % THREADS;
    const long long row = THREADS < 256 ? (long long)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS : (long long)blockIdx.x;
    if (THREADS < 256 && row >= a.rows) return;
    const long long cols = a.cols;
    const int units = (int)units_of(cols);
    const XT* const x = (const XT*)a.x + row * a.ldx;
    const R* const res = ADD ? (const R*)a.residual + row * a.ldr : nullptr;

    Raw<XT> rx[ITEMS];
    Raw<R> rr[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        rx[i] = fetch_unit<ONCE>(x, i * THREADS + t, cols);
        if constexpr (ADD) rr[i] = fetch_unit<ONCE>(res, i * THREADS + t, cols);
    }
    // Few rows wait for memory: their weights are asked for together with the rows.
    constexpr bool EARLY = ITEMS == 1;
    Raw<float> rw = {};
    if (EARLY && a.weight) rw = fetch_unit(a.weight, t, cols);
    float v[ITEMS][8];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int unit = i * THREADS + t;
        expand_unit(rx[i], x, unit, cols, v[i], 0.0f);
        if constexpr (ADD) {
            float b[8];
            expand_unit(rr[i], res, unit, cols, b, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] += b[j];
            if (a.total && (long long)unit * 8 < cols) store_unit((R*)a.total + row * a.ldt, unit, cols, v[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(v[i][j], v[i][j], sum);
    }
    if (a.norm) {
        const Root root = inverse_root(row_sum<THREADS>(sum, lds_sum), cols, a.eps);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int unit = i * THREADS + t;
            float w[8];
            if (a.weight) {
                expand_unit(EARLY ? rw : fetch_unit(a.weight, unit, cols), a.weight, unit, cols, w, 0.0f);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.0f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = normed(v[i][j], w[j], root);
        }
    }
    float inverse = 0.0f;
    if (a.format == SBN_FP8_ROW) {
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) top = max(top, top_bits(v[i]));
        const float scale = row_scale(row_max<THREADS>(top, lds_max), inverse);
        if (t == 0) ((float*)a.scales)[row] = scale;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int unit = i * THREADS + t;
        if (unit < units) put_row_outputs<XT>(a, row, unit, v[i], inverse);
    }
}

// Rows that no workgroup's registers hold: read again for every step.  The sums x + residual are written in the last step
// only, each by the lane that reads the same places, so that they may take their inputs' place.
template <class XT, class RT>
__global__ __launch_bounds__(1024) void long_row_kernel(const RowArgs a)
{
    __shared__ float lds_sum[16];
    __shared__ unsigned lds_max[16];
    constexpr bool ADD = !std::is_same<RT, void>::value;
    using R = typename std::conditional<ADD, RT, XT>::type;
    const long long row = blockIdx.x, cols = a.cols, units = units_of(cols);
    const XT* const x = (const XT*)a.x + row * a.ldx;
    const R* const res = ADD ? (const R*)a.residual + row * a.ldr : nullptr;
    auto get = [&](long long unit, float (&v)[8]) {
        expand_unit(fetch_unit(x, unit, cols), x, unit, cols, v, 0.0f);
        if constexpr (ADD) {
            float b[8];
            expand_unit(fetch_unit(res, unit, cols), res, unit, cols, b, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += b[j];
        }
    };
    Root root = {1.0f, 0.0f};
    if (a.norm) {
        float sum = 0.0f;
        for (long long u = threadIdx.x; u < units; u += 1024) {
            float v[8], part = 0.0f;
            get(u, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) part = __builtin_fmaf(v[j], v[j], part);
            sum += part;
        }
        root = inverse_root(row_sum<1024>(sum, lds_sum), cols, a.eps);
    }
    auto finish = [&](long long unit, float (&v)[8]) {
        if (!a.norm) return;
        float w[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
        if (a.weight) expand_unit(fetch_unit(a.weight, unit, cols), a.weight, unit, cols, w, 0.0f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = normed(v[j], w[j], root);
    };
    float inverse = 0.0f;
    if (a.format == SBN_FP8_ROW) {
        unsigned top = 0;
        for (long long u = threadIdx.x; u < units; u += 1024) {
            float v[8];
            get(u, v);
            finish(u, v);
            top = max(top, top_bits(v));
        }
        const float scale = row_scale(row_max<1024>(top, lds_max), inverse);
        if (threadIdx.x == 0) ((float*)a.scales)[row] = scale;
    }
    for (long long u = threadIdx.x; u < units; u += 1024) {
        float v[8];
        get(u, v);
        if constexpr (ADD)
            if (a.total && u * 8 < cols) store_unit((R*)a.total + row * a.ldt, u, cols, v);
        finish(u, v);
        put_row_outputs<XT>(a, row, u, v, inverse);
    }
}

template <class XT, class RT>
int launch_rows(RowArgs a, hipStream_t stream)
{
    const long long units = units_of(a.cols);
    constexpr long long kMost = 1ll << 21;                    // rows a launch (below 2^32 work items of 1024 threads)
    for (long long r0 = 0; r0 < a.rows; r0 += kMost) {
        RowArgs b = a;
        b.rows = std::min(kMost, a.rows - r0);
        const int fmt = a.format;
        const long long per = units * (fmt == SBN_MXFP4 ? 4 : 8);
        b.x = (const XT*)a.x + r0 * a.ldx;
        if constexpr (!std::is_same<RT, void>::value) {
            b.residual = (const RT*)a.residual + r0 * a.ldr;
            if (a.total) b.total = (RT*)a.total + r0 * a.ldt;
        }
        if (a.y) b.y = (XT*)a.y + r0 * a.ldy;
        if (fmt) b.codes = (char*)a.codes + r0 * per, b.scales = (char*)a.scales + r0 * (fmt == SBN_FP8_ROW ? 4 : units / 4);
        const unsigned rows = (unsigned)b.rows;
        constexpr bool MAY = sizeof(XT) == 2;
        const bool once = read_once<XT>(a.rows, a.cols);
        if (units <= 256 && rows >= 1024)
            (once ? row_kernel<XT, RT, 64, 4, MAY> : row_kernel<XT, RT, 64, 4>)<<<(rows + 3) / 4, 256, 0, stream>>>(b);
        else if (units <= 512)
            (once ? row_kernel<XT, RT, 256, 2, MAY> : row_kernel<XT, RT, 256, 2>)<<<rows, 256, 0, stream>>>(b);
        else if (units <= 1024 && rows >= 512)
            (once ? row_kernel<XT, RT, 256, 4, MAY> : row_kernel<XT, RT, 256, 4>)<<<rows, 256, 0, stream>>>(b);
        else if (units <= 1024)
            row_kernel<XT, RT, 1024, 1><<<rows, 1024, 0, stream>>>(b);
        else if (units <= 4096)
            (once ? row_kernel<XT, RT, 1024, 4, MAY> : row_kernel<XT, RT, 1024, 4>)<<<rows, 1024, 0, stream>>>(b);
        else
            long_row_kernel<XT, RT><<<rows, 1024, 0, stream>>>(b);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return fail(SBN_EHIP, "row kernel: %s", hipGetErrorString(e));
    }
    return SBN_OK;
}

// Calls f(rows of the launch, first row) so that no launch has more than 2^31 units.
template <class F>
int by_rows(long long rows, long long units, const char* who, F&& f)
{
    const long long most = std::max(1ll, (1ll << 30) / units);
    for (long long r0 = 0; r0 < rows; r0 += most) {
        f(std::min(most, rows - r0), r0);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return fail(SBN_EHIP, "%s: %s", who, hipGetErrorString(e));
    }
    return SBN_OK;
}
inline unsigned groups_of(long long total) { return (unsigned)((total + 256 * kItems - 1) / (256 * kItems)); }

template <class T>
int quantize_blocks(const T* x, long long rows, long long cols, long long ldx, int format, char* codes, char* scales, hipStream_t stream)
{
    const long long units = units_of(cols);
    return by_rows(rows, units, "sbn_quantize", [&](long long n, long long r0) {
        const unsigned total = (unsigned)(n * units);
        uint8_t* const s = (uint8_t*)scales + r0 * (units / 4);
        char* const c = codes + r0 * units * (format == SBN_MXFP4 ? 4 : 8);
        constexpr bool MAY = sizeof(T) == 2;
        const bool once = read_once<T>(rows, cols);
        auto* const kernel = format == SBN_MXFP4 ? (once ? quantize_kernel<T, SBN_MXFP4, MAY> : quantize_kernel<T, SBN_MXFP4, false>)
                                                 : (once ? quantize_kernel<T, SBN_MXFP8, MAY> : quantize_kernel<T, SBN_MXFP8, false>);
        kernel<<<groups_of(total), 256, 0, stream>>>(x + r0 * ldx, ldx, (unsigned)units, total, cols, c, s);
    });
}

template <class T>
int dequantize_all(const char* codes, const char* scales, int format, long long rows, long long cols, T* y, long long ldy, hipStream_t stream)
{
    const long long units = units_of(cols);
    return by_rows(rows, units, "sbn_dequantize", [&](long long n, long long r0) {
        const unsigned total = (unsigned)(n * units), u = (unsigned)units;
        T* const to = y + r0 * ldy;
        if (format == SBN_MXFP4)
            dequantize_kernel<T, SBN_MXFP4><<<groups_of(total), 256, 0, stream>>>(codes + r0 * units * 4, scales + r0 * (units / 4), to, ldy, u, total, cols);
        else if (format == SBN_MXFP8)
            dequantize_kernel<T, SBN_MXFP8><<<groups_of(total), 256, 0, stream>>>(codes + r0 * units * 8, scales + r0 * (units / 4), to, ldy, u, total, cols);
        else
            dequantize_kernel<T, SBN_FP8_ROW><<<groups_of(total), 256, 0, stream>>>(codes + r0 * units * 8, scales + r0 * 4, to, ldy, u, total, cols);
    });
}

}  // namespace

int launch_add_rmsnorm(const sbn_rmsnorm_t& n, bool norm, void* stream)
{
    RowArgs a = {};
    a.rows = n.rows, a.cols = n.cols, a.ldx = n.ldx, a.ldr = n.ldr, a.ldt = n.ldt, a.ldy = n.ldy;
    a.x = n.x, a.residual = n.residual, a.total = n.total, a.weight = n.weight, a.y = n.y, a.codes = n.codes, a.scales = n.scales;
    a.eps = n.eps, a.norm = norm, a.format = n.format;
    const hipStream_t s = (hipStream_t)stream;
    auto typed = [&](auto* t) -> int {
        using T = typename std::remove_pointer<decltype(t)>::type;
        if (!n.residual) return launch_rows<T, void>(a, s);
        if (n.r_type == n.x_type) return launch_rows<T, T>(a, s);
        return launch_rows<T, float>(a, s);
    };
    return n.x_type == SBN_F32 ? typed((float*)nullptr) : n.x_type == SBN_BF16 ? typed((__bf16*)nullptr) : typed((_Float16*)nullptr);
}

int launch_quantize(const void* x, int x_type, long long rows, long long cols, long long ldx, int format, void* codes, void* scales, void* stream)
{
    if (format == SBN_FP8_ROW) {
        sbn_rmsnorm_t n = {};
        n.rows = rows, n.cols = cols, n.x = x, n.x_type = x_type, n.ldx = ldx, n.format = format, n.codes = codes, n.scales = scales;
        return launch_add_rmsnorm(n, false, stream);
    }
    const hipStream_t s = (hipStream_t)stream;
    char *const c = (char*)codes, *const q = (char*)scales;
    return x_type == SBN_F32 ? quantize_blocks((const float*)x, rows, cols, ldx, format, c, q, s)
         : x_type == SBN_BF16 ? quantize_blocks((const __bf16*)x, rows, cols, ldx, format, c, q, s)
                              : quantize_blocks((const _Float16*)x, rows, cols, ldx, format, c, q, s);
}

int launch_dequantize(const void* codes, const void* scales, int format, long long rows, long long cols, void* y, int y_type, long long ldy, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    const char *const c = (const char*)codes, *const q = (const char*)scales;
    return y_type == SBN_F32 ? dequantize_all(c, q, format, rows, cols, (float*)y, ldy, s)
         : y_type == SBN_BF16 ? dequantize_all(c, q, format, rows, cols, (__bf16*)y, ldy, s)
                              : dequantize_all(c, q, format, rows, cols, (_Float16*)y, ldy, s);
}

}  // namespace sbn
