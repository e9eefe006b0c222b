// Block-scaled numbers that are only streamed (tern.h: tern_mx_quantize, tern_mx_values, tern_mx_gate,
// tern_mx_gate_grad): every value is read once and every result written once, and memory bounds them.
//
// A lane takes eight neighbouring values, a block of 32 is four lanes of a quad, and the block's largest magnitude
// crosses them by two lane permutations.  Measured: 16384 x 4096 bf16 to 4 bits 34 us (5.0 TB/s) and back 26 (6.6); the gate of
// 8192 x 8192 bf16 with its halves saved 90 to 101 us (5.4 to 6.0), the gradient at 8001 x 8190 (rows at any multiple of
// four bytes) 121 to 128 (4.7 to 4.9).
#include "tern_mx_common.h"
#include "tern_division.h"

#include <type_traits>

namespace tern {
namespace {

constexpr int kThreads = 256;

// ---- 4-bit records: 32 rows x 256 columns a workgroup ------------------------------------------------------------
// Eight lanes take 64 columns of a row (whole lines where rows are aligned), a workgroup 32 rows, four times; a record's
// 4 KB leave in runs of 64 bytes.
// SAVE: in 8 bits as well, row by row.
template <typename T, bool SAVE>
__global__ __launch_bounds__(kThreads) void quantize_f4_kernel(const T* x, int64_t rows, int64_t cols, int64_t ld, Divisor groups,
                                                               uint8_t* codes, uint8_t* scales, uint8_t* codes8, uint8_t* scales8,
                                                               int64_t blocks8)
{
    const int r = quotient((int)blockIdx.x, groups), g = (int)blockIdx.x - r * groups.d;
    const int j = threadIdx.x >> 3, h = (threadIdx.x >> 2) & 1, quarter = threadIdx.x & 3;
    const int64_t row = (int64_t)r * 32 + j, record = blockIdx.x;
    const int64_t col0 = (int64_t)g * 256 + h * 32 + quarter * 8;
    float v[4][8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t left = row < rows ? cols - (col0 + 64 * q) : 0;
        load_eight(v[q], x + row * ld + col0 + 64 * q, left < 8 ? (left < 0 ? 0 : (int)left) : 8);
    }
    uint32_t packed = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t most = block_most(v[q]), byte = scale_byte<TERN_MX_F4>(most);
        packed |= byte << (8 * q);
        *reinterpret_cast<uint32_t*>(codes + record * kMxRecord + q * 1024 + h * 512 + j * 16 + quarter * 4) = f4_codes(v[q], byte);
        if constexpr (SAVE) {
            const int64_t block = (col0 + 64 * q) >> 5;
            if (row < rows && block < blocks8) {
                const uint32_t byte8 = scale_byte<TERN_MX_I8>(most);
                *reinterpret_cast<mx_u32x2*>(codes8 + (row * blocks8 + block) * 32 + quarter * 8) = i8_codes(v[q], byte8);
                if (quarter == 0) scales8[row * blocks8 + block] = (uint8_t)byte8;
            }
        }
    }
    if (quarter == 0) *reinterpret_cast<uint32_t*>(scales + record * kMxScaleRecord + h * 128 + j * 4) = packed;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void values_f4_kernel(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols,
                                                             Divisor groups, T* out, int64_t ld)
{
    const int r = quotient((int)blockIdx.x, groups), g = (int)blockIdx.x - r * groups.d;
    const int j = threadIdx.x >> 3, h = (threadIdx.x >> 2) & 1, quarter = threadIdx.x & 3;
    const int64_t row = (int64_t)r * 32 + j, record = blockIdx.x;
    const int64_t col0 = (int64_t)g * 256 + h * 32 + quarter * 8;
    const uint32_t packed = *reinterpret_cast<const uint32_t*>(scales + record * kMxScaleRecord + h * 128 + j * 4);
    uint32_t c[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        c[q] = *reinterpret_cast<const uint32_t*>(codes + record * kMxRecord + q * 1024 + h * 512 + j * 16 + quarter * 4);
    if (row >= rows) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int64_t left = cols - (col0 + 64 * q);
        if (left <= 0) return;
        float v[8];
        f4_values(v, c[q], (packed >> (8 * q)) & 255u);
        store_eight(out + row * ld + col0 + 64 * q, v, left < 8 ? (int)left : 8);
    }
}

// ---- row by row ---------------------------------------------------------------------------------------------------
// Chunk e of eight values: row e / chunks, chunk e % chunks; chunks = 4 blocks a row, so that a quad never straddles rows
// (the last block's lanes past the end hold zeros).
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_i8_kernel(const T* x, int64_t cols, int64_t ld, int total, Divisor chunks,
                                                               uint8_t* codes, uint8_t* scales)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int row = quotient((int)e, chunks), at = ((int)e - row * chunks.d) * 8;
    float v[8];
    load_eight(v, x + row * ld + at, (int)min((int64_t)8, max((int64_t)0, cols - at)));
    const uint32_t byte = scale_byte<TERN_MX_I8>(block_most(v));
    *reinterpret_cast<mx_u32x2*>(codes + e * 8) = i8_codes(v, byte);
    if ((e & 3) == 0) scales[e >> 2] = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void values_i8_kernel(const uint8_t* codes, const uint8_t* scales, int64_t cols, int total,
                                                             Divisor chunks, T* out, int64_t ld)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int row = quotient((int)e, chunks), at = ((int)e - row * chunks.d) * 8;
    float v[8];
    i8_values(v, *reinterpret_cast<const mx_u32x2*>(codes + e * 8), scales[e >> 2]);
    const int64_t left = cols - at;
    if (left > 0) store_eight(out + row * ld + at, v, left < 8 ? (int)left : 8);
}

// e = exp(-|g|) as 2^n m, n <= 0 and m in (1/2, 1], and r = 1 / (1 + e): the sigmoid of g is r for g >= 0 and e r below, and one less
// it the other.  n is taken off -|g| log2(e) by fused operations with both halves of the constant, so that what exp2 gets is right
// to 2^-24 whatever |g| is (rounded as a product it was |g| 2^-23 off: 1.0e-6 of e at |g| = 20, 3.8e-6 at 80); exp2 and the
// reciprocal as the device has them (right to their last bit).  e itself may have no leading bit or be zero: n and m hold it.
struct Decay {
    float m, r;
    int n;
};
__device__ __forceinline__ Decay decay(float g)
{
    Decay d;
    const float a = fabsf(g), n = fmaxf(__builtin_ceilf(a * -1.442695021629333f), -400.0f);     // (beyond: every product is zero)
    d.n = (int)n;
    d.m = __builtin_amdgcn_exp2f(__builtin_fmaf(a, -1.925963033500e-8f, __builtin_fmaf(a, -1.442695021629333f, -n)));
    d.r = __builtin_amdgcn_rcpf(1.0f + __builtin_ldexpf(d.m, d.n));
    return d;
}
// v e p q, |p| less than 2^9: part of 2^n on v and the rest behind the products, so that none of them leaves a float's range where
// the result does not (for |v q| up to 2^150).
__device__ __forceinline__ float decayed(const Decay& d, float v, float p, float q = 1.0f)
{
    const int first = max(d.n, -32);
    return __builtin_ldexpf(p * (__builtin_ldexpf(v, first) * d.m) * q, d.n - first);
}
// Down to here e is a factor like any other.
constexpr float kDeep = -40.0f;
__device__ __forceinline__ float least(const float (&v)[8])
{
    float m = v[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fminf(m, v[i]);
    return m;
}

template <typename T, bool SAVE>
__global__ __launch_bounds__(kThreads) void gate_kernel(const T* gu, int64_t rows, int64_t c, int64_t ld, int total, Divisor chunks,
                                                        T* h, int64_t ldh, uint8_t* codes, uint8_t* scales)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int row = quotient((int)e, chunks), at = ((int)e - row * chunks.d) * 8;
    const int n = (int)min((int64_t)8, max((int64_t)0, c - at));
    float g[8], u[8], y[8];
    load_eight(g, gu + row * ld + at, n);
    load_eight(u, gu + row * ld + c + at, n);
    if (least(g) < kDeep) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Decay d = decay(g[i]);
            const float a = g[i] * d.r;
            y[i] = g[i] < 0.0f ? decayed(d, u[i], a) : a * u[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Decay d = decay(g[i]);
            y[i] = g[i] * d.r * (u[i] * (g[i] < 0.0f ? __builtin_ldexpf(d.m, d.n) : 1.0f));
        }
    }
    store_eight(h + row * ldh + at, y, n);
    if constexpr (SAVE) {
        const int64_t half = rows * (int64_t)chunks.d + e;      // the same chunk of u, `rows` rows further down
        const uint32_t bg = scale_byte<TERN_MX_I8>(block_most(g)), bu = scale_byte<TERN_MX_I8>(block_most(u));
        *reinterpret_cast<mx_u32x2*>(codes + e * 8) = i8_codes(g, bg);
        *reinterpret_cast<mx_u32x2*>(codes + half * 8) = i8_codes(u, bu);
        if ((e & 3) == 0) {
            scales[e >> 2] = (uint8_t)bg;
            scales[half >> 2] = (uint8_t)bu;
        }
    }
}

template <typename T, bool HIDDEN>
__global__ __launch_bounds__(kThreads) void gate_grad_kernel(const T* dh, int64_t rows, int64_t c, int64_t ldh, int total,
                                                             Divisor chunks, const uint8_t* codes, const uint8_t* scales, T* dgu,
                                                             int64_t ld, uint8_t* hcodes, uint8_t* hscales)
{
    const int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (e >= total) return;
    const int row = quotient((int)e, chunks), at = ((int)e - row * chunks.d) * 8;
    const int n = (int)min((int64_t)8, max((int64_t)0, c - at));
    const int64_t half = rows * (int64_t)chunks.d + e;
    float d[8], g[8], u[8], y[8];
    load_eight(d, dh + row * ldh + at, n);
    i8_values(g, *reinterpret_cast<const mx_u32x2*>(codes + e * 8), scales[e >> 2]);
    i8_values(u, *reinterpret_cast<const mx_u32x2*>(codes + half * 8), scales[half >> 2]);
    if (least(g) < kDeep) {             // (few chunks hold any; if all went this way: 2 % of the time, and 1 % of the gate's)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Decay k = decay(g[i]);
            const float a = g[i] * k.r;
            if (g[i] < 0.0f) {          // s = e r and 1 - s = r: e last, s by itself may have no bits left
                y[i] = decayed(k, u[i], a);
                g[i] = decayed(k, u[i], k.r * (1.0f + a), d[i]);
                u[i] = decayed(k, d[i], a);
            } else {
                y[i] = a * u[i];
                g[i] = d[i] * u[i] * (k.r + a * (__builtin_ldexpf(k.m, k.n) * k.r));
                u[i] = d[i] * a;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Decay k = decay(g[i]);
            const float small = __builtin_ldexpf(k.m, k.n) * k.r, s = g[i] < 0.0f ? small : k.r, less = g[i] < 0.0f ? k.r : small, a = g[i] * s;
            y[i] = a * u[i];
            g[i] = d[i] * u[i] * (s + a * less);
            u[i] = d[i] * a;
        }
    }
    store_eight(dgu + row * ld + at, g, n);
    store_eight(dgu + row * ld + c + at, u, n);
    if constexpr (HIDDEN) {
        const uint32_t byte = scale_byte<TERN_MX_I8>(block_most(y));
        *reinterpret_cast<mx_u32x2*>(hcodes + e * 8) = i8_codes(y, byte);
        if ((e & 3) == 0) hscales[e >> 2] = (uint8_t)byte;
    }
}

// Chunks of eight values over all rows (mx_shape's limit keeps them, and records, below 2^31), and workgroups for them.
struct Chunks {
    int total;
    Divisor per_row;
    dim3 grid;
};
Chunks chunks_of(int64_t rows, const MxShape& s)
{
    Chunks c;
    c.total = (int)(rows * s.blocks * 4);
    c.per_row = divisor((int)(s.blocks * 4));
    c.grid = dim3((unsigned)((c.total + (int64_t)kThreads - 1) / kThreads));
    return c;
}

// f on a null pointer of the type's own.
template <typename F>
int by_type(int type, F f)
{
    if (type == TERN_F32) f((float*)nullptr);
    else if (type == TERN_BF16) f((__bf16*)nullptr);
    else f((_Float16*)nullptr);
    TERN_HIP_CHECK(hipGetLastError());
    return TERN_OK;
}

}  // namespace

int launch_mx_quantize(const void* x, int type, int64_t rows, int64_t cols, int64_t ld, int kind, void* dst, hipStream_t stream)
{
    MxShape s;
    mx_shape(rows, cols, kind, &s);
    auto *codes = (uint8_t*)dst, *scales = codes + s.code_bytes;
    const Chunks c = chunks_of(rows, s);
    return by_type(type, [&](auto* t) {
        const auto* p = (decltype(t))x;
        if (kind == TERN_MX_F4)
            quantize_f4_kernel<std::remove_pointer_t<decltype(t)>, false><<<dim3((unsigned)(s.row_blocks * s.groups)), kThreads, 0, stream>>>(
                p, rows, cols, ld, divisor((int)s.groups), codes, scales, nullptr, nullptr, 0);
        else
            quantize_i8_kernel<<<c.grid, kThreads, 0, stream>>>(p, cols, ld, c.total, c.per_row, codes, scales);
    });
}

int launch_mx_quantize_both(const void* x, int type, int64_t rows, int64_t cols, int64_t ld, void* f4, void* i8, hipStream_t stream)
{
    MxShape s, s8;
    mx_shape(rows, cols, TERN_MX_F4, &s);
    mx_shape(rows, cols, TERN_MX_I8, &s8);
    auto *codes = (uint8_t*)f4, *codes8 = (uint8_t*)i8;
    return by_type(type, [&](auto* t) {
        quantize_f4_kernel<std::remove_pointer_t<decltype(t)>, true><<<dim3((unsigned)(s.row_blocks * s.groups)), kThreads, 0, stream>>>(
            (decltype(t))x, rows, cols, ld, divisor((int)s.groups), codes, codes + s.code_bytes, codes8, codes8 + s8.code_bytes, s8.blocks);
    });
}

int launch_mx_values(const void* src, int kind, int64_t rows, int64_t cols, int type, void* out, int64_t ld, hipStream_t stream)
{
    MxShape s;
    mx_shape(rows, cols, kind, &s);
    const auto *codes = (const uint8_t*)src, *scales = codes + s.code_bytes;
    const Chunks c = chunks_of(rows, s);
    return by_type(type, [&](auto* t) {
        auto* p = (decltype(t))out;
        if (kind == TERN_MX_F4)
            values_f4_kernel<<<dim3((unsigned)(s.row_blocks * s.groups)), kThreads, 0, stream>>>(codes, scales, rows, cols,
                                                                                                 divisor((int)s.groups), p, ld);
        else
            values_i8_kernel<<<c.grid, kThreads, 0, stream>>>(codes, scales, cols, c.total, c.per_row, p, ld);
    });
}

int launch_mx_gate(const void* gu, int type, int64_t rows, int64_t ld, int64_t c, void* h, int64_t ldh, void* saved, hipStream_t stream)
{
    MxShape s;
    mx_shape(2 * rows, c, TERN_MX_I8, &s);
    auto *codes = (uint8_t*)saved, *scales = codes + s.code_bytes;
    const Chunks k = chunks_of(rows, s);
    return by_type(type, [&](auto* t) {
        const auto* p = (decltype(t))gu;
        auto* q = (decltype(t))h;
        if (saved) gate_kernel<std::remove_pointer_t<decltype(t)>, true><<<k.grid, kThreads, 0, stream>>>(p, rows, c, ld, k.total, k.per_row, q, ldh, codes, scales);
        else gate_kernel<std::remove_pointer_t<decltype(t)>, false><<<k.grid, kThreads, 0, stream>>>(p, rows, c, ld, k.total, k.per_row, q, ldh, nullptr, nullptr);
    });
}

int launch_mx_gate_grad(const void* dh, int type, int64_t rows, int64_t ldh, const void* saved, int64_t c, void* dgu, int64_t ld,
                        void* hidden, hipStream_t stream)
{
    MxShape s, sh;
    mx_shape(2 * rows, c, TERN_MX_I8, &s);
    mx_shape(rows, c, TERN_MX_I8, &sh);
    const auto *codes = (const uint8_t*)saved, *scales = codes + s.code_bytes;
    auto *hc = (uint8_t*)hidden, *hs = hc + sh.code_bytes;
    const Chunks k = chunks_of(rows, s);
    return by_type(type, [&](auto* t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        const auto* p = (const T*)dh;
        auto* q = (T*)dgu;
        if (hidden) gate_grad_kernel<T, true><<<k.grid, kThreads, 0, stream>>>(p, rows, c, ldh, k.total, k.per_row, codes, scales, q, ld, hc, hs);
        else gate_grad_kernel<T, false><<<k.grid, kThreads, 0, stream>>>(p, rows, c, ldh, k.total, k.per_row, codes, scales, q, ld, nullptr, nullptr);
    });
}

}  // namespace tern
