// Root-mean-square normalization with the residual's addition for gfx950: forward (results in the element type or in 8 bits
// with a scale per row), backward, and the C ABI of include/mtfm_rms.h.
//
// Bound by HBM: an element is read once and written once.  A row belongs to a fixed set of lanes -- 8 to 64 of a wave for up
// to 1024 features, 256 (a workgroup) beyond -- which keep it in registers between the sum of its squares and its result, and
// since every row is multiplied by the same weights, a lane holds its features' weights, and in the backward pass its share of
// their gradients, in registers for all the rows that come by.  Narrow rows lie side by side in a wave.  The next row's loads
// are in flight while the current one is worked on.
//
// 215 871 rows of 512, bf16, with a residual: forward 169 us, backward 161, 5.2 and 5.5 TB/s of the rows that come and go: the rate of a copy (4.9) or a little
// above, since part of what was written last is still in the memory-side cache.  20 011 rows of 1001, float32, by single elements: 31.7 and 46.1 us, 5.1 and
// 5.2 TB/s.  17 rows: 3.1 us, a launch and two trips to memory.
#include "../../include/mtfm_rms.h"
#include "hta_common.h"
#include "hta_mfma.h"

#include <hip/hip_runtime.h>

namespace rms {

constexpr int MAX_WIDTH = 8192;
constexpr int FWD_THREADS = 256, FWD_BLOCKS = 2048;
constexpr int MAX_SHARES = 512;  // workgroups of a backward launch, each with a share of dweight
constexpr int REDUCE_THREADS = 512, REDUCE_COLS = 32, REDUCE_SLICES = REDUCE_THREADS / (REDUCE_COLS / 4);

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

enum Out { PLAIN = -1, INT8 = MTFM_RMS_INT8, E4M3 = MTFM_RMS_E4M3 };

struct Args {
    const void *x, *residual, *dy, *dh;  // backward: x is h
    int64_t ldx, ldr, ldy, ldh;
    const float *weight, *rstd_in;
    void *h, *y;   // y: the result of any type; backward: dx
    float *rstd, *scale, *partials;
    int64_t n;
    int32_t d, out;
    float eps;
};

// V elements that a lane moves at once, as they lie in memory
template <typename T, int V>
struct Raw {
    typedef T type __attribute__((ext_vector_type(V)));
    type v;
    __device__ void load(const T* p) { v = __builtin_nontemporal_load((const type*)p); }
    __device__ float get(int j) const { return (float)v[j]; }
};
template <typename T>
struct Raw<T, 1> {
    T v;
    __device__ void load(const T* p) { v = *p; }
    __device__ float get(int) const { return (float)v; }
};

template <typename T, int V>
__device__ inline void store(T* p, const float* f) {
    if constexpr (V == 1) {
        *p = (T)f[0];  // (bf16: round to nearest even)
    } else {
        typename Raw<T, V>::type v;
#pragma unroll
        for (int j = 0; j < V; j++) v[j] = (T)f[j];
        __builtin_nontemporal_store(v, (typename Raw<T, V>::type*)p);
    }
}

// Sum over the L lanes of a row that lie in one wave, the same value in all of them, in a fixed order
template <int L>
__device__ inline float lanes_sum(float v) {
    v = hta::sum_lanes<(L < 32 ? L : 32)>(v);
    return L > 32 ? v + hta::other_half(v) : v;
}
// Largest magnitude, as the bits of a float without its sign: ordered like the values, with NaN above infinity
template <int L>
__device__ inline uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int m = 1; m < (L < 64 ? L : 64); m *= 2) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}
// of a row of 256 lanes: the four waves' values through LDS.  `buf` has a half for odd and even turns, so one barrier per turn does.
template <int TPR, typename U, typename F>
__device__ inline U across_waves(U v, U* buf, int turn, F join) {
    if constexpr (TPR <= 64) return v;
    U* b = buf + (turn & 1) * 4;
    if ((threadIdx.x & 63) == 0) b[threadIdx.x >> 6] = v;
    __syncthreads();
    return join(join(b[0], b[1]), join(b[2], b[3]));
}

template <typename T, int V, int TPR, int NG>
struct Row {  // a lane's NG groups of V features of a row: group g at feature (g TPR + lane) V
    Raw<T, V> g[NG];
    __device__ void load(const T* row, int fl, int d) {
#pragma unroll
        for (int i = 0; i < NG; i++)
            if ((i * TPR + fl) * V < d) g[i].load(row + (i * TPR + fl) * V);
    }
};

// TPR lanes hold a row, FWD_THREADS / TPR rows lie in a workgroup side by side.  In 8 bits 2176 rows of 512 take 6.8 us: 7.8 MB, of which the launch and the
// trips to memory are most.
template <typename T, int V, int TPR, int NG>
__global__ __launch_bounds__(FWD_THREADS) void fwd_kernel(const Args a) {
    constexpr int RPB = FWD_THREADS / TPR;
    __shared__ float sums_s[8];
    __shared__ uint32_t tops_s[8];
    const int fl = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = a.d;
    const float inv_d = 1.f / (float)d;
    const T* xg = (const T*)a.x;
    const T* rg = (const T*)a.residual;
    Row<T, V, TPR, NG> xr, rr;
    const auto fetch = [&](int64_t t) {
        if (t >= a.n) return;
        xr.load(xg + t * a.ldx, fl, d);
        if (rg) rr.load(rg + t * a.ldr, fl, d);
    };
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t base = (int64_t)blockIdx.x * RPB;
    fetch(base + sub);
    float w[NG][V];
#pragma unroll
    for (int i = 0; i < NG; i++)
#pragma unroll
        for (int j = 0; j < V; j++) w[i][j] = (i * TPR + fl) * V < d ? a.weight[(i * TPR + fl) * V + j] : 0.f;
    for (int turn = 0; base < a.n; base += stride, turn++) {
        const int64_t t = base + sub;
        const bool there = TPR == 256 || t < a.n;
        float h[NG][V], s = 0.f;
#pragma unroll
        for (int i = 0; i < NG; i++) {
            const bool in = there && (i * TPR + fl) * V < d;
#pragma unroll
            for (int j = 0; j < V; j++) {
                float f = xr.g[i].get(j);
                if (rg) f = (float)(T)(f + rr.g[i].get(j));  // rounded to the stored type: what a later pass reads is what is normalized
                h[i][j] = in ? f : 0.f;
                s += h[i][j] * h[i][j];
            }
            if (rg && in) store<T, V>((T*)a.h + t * d + (i * TPR + fl) * V, h[i]);
        }
        if (base + stride < a.n) fetch(t + stride);
        s = across_waves<TPR>(lanes_sum<TPR>(s), sums_s, turn, [](float p, float q) { return p + q; });
        const float rstd = 1.f / sqrtf(s * inv_d + a.eps);
        if (a.out == PLAIN) {
#pragma unroll
            for (int i = 0; i < NG; i++) {
                if (there && (i * TPR + fl) * V < d) {
                    float y[V];
#pragma unroll
                    for (int j = 0; j < V; j++) y[j] = h[i][j] * rstd * w[i][j];
                    store<T, V>((T*)a.y + t * d + (i * TPR + fl) * V, y);
                }
            }
            if (there && fl == 0 && a.rstd) a.rstd[t] = rstd;
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < NG; i++)
#pragma unroll
                for (int j = 0; j < V; j++) {
                    h[i][j] = h[i][j] * rstd * w[i][j];  // (features that are not there: 0)
                    top = max(top, __builtin_bit_cast(uint32_t, h[i][j]) & 0x7FFFFFFFu);
                }
            top = across_waves<TPR>(lanes_max<TPR>(top), tops_s, turn, [](uint32_t p, uint32_t q) { return max(p, q); });
            const bool whole = a.out == INT8;
            const float limit = whole ? 127.f : 448.f;
            const float scale = __builtin_bit_cast(float, top) / limit;
            const float by = scale == 0.f ? 1.f : scale;
#pragma unroll
            for (int i = 0; i < NG; i++) {
                if (there && (i * TPR + fl) * V < d) {
                    uint32_t packed[(V + 3) / 4];
#pragma unroll
                    for (int j = 0; j < (V + 3) / 4; j++) packed[j] = 0;
                    float q[V];
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        q[j] = h[i][j] / by;  // (a quotient: the reciprocal of a scale near the smallest float is infinite)
                        q[j] = q[j] > limit ? limit : q[j] < -limit ? -limit : q[j];
                    }
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < V; j++)
                            packed[j / 4] |= (uint32_t)((q[j] == q[j] ? (int)rintf(q[j]) : 0) & 0xFF) << (8 * (j % 4));
                    } else {
#pragma unroll
                        for (int j = 0; j < V; j += 2) {
                            const float b = q[V > 1 ? j + 1 : j];
                            if (j % 4 == 0) packed[j / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(q[j], b, packed[j / 4], false);
                            else packed[j / 4] = __builtin_amdgcn_cvt_pk_fp8_f32(q[j], b, packed[j / 4], true);
                        }
                    }
                    uint8_t* p = (uint8_t*)a.y + t * d + (i * TPR + fl) * V;
                    if constexpr (V == 8) *(uint64_t*)p = packed[0] | (uint64_t)packed[1] << 32;
                    else if constexpr (V == 4) *(uint32_t*)p = packed[0];
                    else *p = (uint8_t)packed[0];
                }
            }
            if (there && fl == 0) a.scale[t] = scale;
        }
    }
}

// dx, and the workgroup's share of dweight: few workgroups (512, all on the chip at once) with many rows each, since a share is written and read again.
// 215 871 rows of 512: 161 us, and 4.5 for the sum of the shares.
constexpr int bwd_threads(int TPR) { return TPR == 256 ? 256 : 512; }

template <typename T, int V, int TPR, int NG>
__global__ __launch_bounds__(bwd_threads(TPR)) void bwd_kernel(const Args a) {
    constexpr int NTHR = bwd_threads(TPR), RPB = NTHR / TPR, NW = NTHR / 64, COLS = TPR * NG * V;
    __shared__ float sums_s[8];
    __shared__ float part_s[TPR == 256 ? 1 : NW / 2 * COLS];
    const int fl = threadIdx.x % TPR, sub = threadIdx.x / TPR, wave = threadIdx.x >> 6, d = a.d;
    const float inv_d = 1.f / (float)d;
    const T* yg = (const T*)a.dy;
    const T* xg = (const T*)a.x;
    const T* hg = (const T*)a.dh;
    Row<T, V, TPR, NG> yr, xr, hr;
    float rstd_next = 0.f;
    const auto fetch = [&](int64_t t) {
        if (t >= a.n) return;
        yr.load(yg + t * a.ldy, fl, d);
        xr.load(xg + t * a.ldx, fl, d);
        if (hg) hr.load(hg + t * a.ldh, fl, d);
        rstd_next = a.rstd_in[t];
    };
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t base = (int64_t)blockIdx.x * RPB;
    fetch(base + sub);
    float w[NG][V], dw[NG][V];
#pragma unroll
    for (int i = 0; i < NG; i++)
#pragma unroll
        for (int j = 0; j < V; j++) {
            w[i][j] = (i * TPR + fl) * V < d ? a.weight[(i * TPR + fl) * V + j] : 0.f;
            dw[i][j] = 0.f;
        }
    for (int turn = 0; base < a.n; base += stride, turn++) {
        const int64_t t = base + sub;
        const bool there = TPR == 256 || t < a.n;
        const float rstd = rstd_next;
        const Row<T, V, TPR, NG> y = yr, x = xr, h = hr;
        if (base + stride < a.n) fetch(t + stride);
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NG; i++)
            if (there && (i * TPR + fl) * V < d) {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const float yx = y.g[i].get(j) * (x.g[i].get(j) * rstd);
                    s += w[i][j] * yx;
                    dw[i][j] += yx;
                }
            }
        s = across_waves<TPR>(lanes_sum<TPR>(s), sums_s, turn, [](float p, float q) { return p + q; }) * inv_d;
#pragma unroll
        for (int i = 0; i < NG; i++)
            if (there && (i * TPR + fl) * V < d) {
                float o[V];
#pragma unroll
                for (int j = 0; j < V; j++) {
                    o[j] = rstd * (w[i][j] * y.g[i].get(j) - x.g[i].get(j) * rstd * s);
                    if (hg) o[j] += h.g[i].get(j);
                }
                store<T, V>((T*)a.y + t * d + (i * TPR + fl) * V, o);
            }
    }
    // the workgroup's share: rows side by side in a wave, then the waves by halves
    float* share = a.partials + (size_t)blockIdx.x * ((d + 3) & ~3);
    if constexpr (TPR < 64) {
#pragma unroll
        for (int m = TPR; m < 64; m *= 2)
#pragma unroll
            for (int i = 0; i < NG; i++)
#pragma unroll
                for (int j = 0; j < V; j++) dw[i][j] += __shfl_xor(dw[i][j], m);
    }
    if constexpr (TPR <= 64) {
        const bool lead = (threadIdx.x & 63) < TPR;
#pragma unroll
        for (int half = NW / 2; half > 0; half /= 2) {
            if (lead && wave >= half && wave < 2 * half) {
#pragma unroll
                for (int i = 0; i < NG; i++)
#pragma unroll
                    for (int j = 0; j < V; j++) part_s[(wave - half) * COLS + (i * V + j) * TPR + fl] = dw[i][j];
            }
            __syncthreads();
            if (lead && wave < half) {
#pragma unroll
                for (int i = 0; i < NG; i++)
#pragma unroll
                    for (int j = 0; j < V; j++) dw[i][j] += part_s[wave * COLS + (i * V + j) * TPR + fl];
            }
            __syncthreads();
        }
        if (!lead || wave > 0) return;
    }
#pragma unroll
    for (int i = 0; i < NG; i++)
#pragma unroll
        for (int j = 0; j < V; j++)
            if ((i * TPR + fl) * V + j < d) share[(i * TPR + fl) * V + j] = dw[i][j];
}

// dweight = the sum of the workgroups' shares in a fixed order: a lane takes four columns of every 64th share, the eight lanes of a column in a
// wave add up, then the eight waves
__global__ __launch_bounds__(REDUCE_THREADS) void reduce_kernel(const float* partials, int n_shares, int d, float* dweight) {
    __shared__ floatx4 part[REDUCE_THREADS / 64][REDUCE_COLS / 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quad = lane % (REDUCE_COLS / 4);
    const int pitch = (d + 3) & ~3, slice = (int)threadIdx.x / (REDUCE_COLS / 4);
    const float* col4 = partials + min((int)blockIdx.x * REDUCE_COLS + 4 * quad, pitch - 4);
    constexpr int PER = MAX_SHARES / REDUCE_SLICES;
    floatx4 v[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) v[i] = *(const floatx4*)(col4 + (size_t)max(0, min(i * REDUCE_SLICES + slice, n_shares - 1)) * pitch);
    floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PER; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) s[j] += i * REDUCE_SLICES + slice < n_shares ? v[i][j] : 0.f;
#pragma unroll
    for (int m = REDUCE_COLS / 4; m < 64; m *= 2)
#pragma unroll
        for (int j = 0; j < 4; j++) s[j] += __shfl_xor(s[j], m);
    if (lane < REDUCE_COLS / 4) part[wave][quad] = s;
    __syncthreads();
    const int col = blockIdx.x * REDUCE_COLS + (int)threadIdx.x;
    if (threadIdx.x < REDUCE_COLS && col < d) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < REDUCE_THREADS / 64; w++) total += part[w][threadIdx.x / 4][threadIdx.x % 4];
        dweight[col] = total;
    }
}

int grid_for(int64_t n, int per_block, int most) {
    const int64_t blocks = (n + per_block - 1) / per_block;
    return (int)(blocks < most ? blocks : most);
}

template <typename T, int V, int TPR, int CPL>
hipError_t launch_as(Args& a, float* dweight, int* shares, hipStream_t s) {
    constexpr int NG = 8 * CPL / V;
    if (!shares) {
        const int grid = grid_for(a.n, FWD_THREADS / TPR, FWD_BLOCKS);
        hipLaunchKernelGGL((fwd_kernel<T, V, TPR, NG>), dim3(grid), dim3(FWD_THREADS), 0, s, a);
        return hipGetLastError();
    }
    constexpr int NTHR = bwd_threads(TPR);
    // up to four turns of one workgroup: its share is the sum, and a second launch costs as much
    *shares = a.n <= 4 * (NTHR / TPR) ? 1 : grid_for(a.n, NTHR / TPR, MAX_SHARES);
    if (*shares == 1) a.partials = dweight;
    hipLaunchKernelGGL((bwd_kernel<T, V, TPR, NG>), dim3(*shares), dim3(NTHR), 0, s, a);
    return hipGetLastError();
}

template <typename T, int V>
hipError_t dispatch_width(Args& a, float* dweight, int* shares, hipStream_t s) {
    if (a.d <= 64) return launch_as<T, V, 8, 1>(a, dweight, shares, s);
    if (a.d <= 128) return launch_as<T, V, 16, 1>(a, dweight, shares, s);
    if (a.d <= 256) return launch_as<T, V, 32, 1>(a, dweight, shares, s);
    if (a.d <= 512) return launch_as<T, V, 64, 1>(a, dweight, shares, s);
    if (a.d <= 1024) return launch_as<T, V, 64, 2>(a, dweight, shares, s);
    if (a.d <= 2048) return launch_as<T, V, 256, 1>(a, dweight, shares, s);
    if (a.d <= 4096) return launch_as<T, V, 256, 2>(a, dweight, shares, s);
    return launch_as<T, V, 256, 4>(a, dweight, shares, s);
}

bool misaligned(const void* p, unsigned a) { return ((uintptr_t)p & (a - 1)) != 0; }

// dweight, shares: null for the forward pass
hipError_t dispatch(int dtype, Args& a, float* dweight, int* shares, hipStream_t s) {
    const int v = dtype == MTFM_HTA_BF16 ? 8 : 4;
    const void* all[] = {a.x, a.residual, a.dy, a.dh, a.weight, a.h, a.y};
    bool words = a.d % v == 0 && a.ldx % v == 0 && a.ldr % v == 0 && a.ldy % v == 0 && a.ldh % v == 0;
    for (const void* p : all) words = words && !misaligned(p, 16);
    if (dtype == MTFM_HTA_BF16) return words ? dispatch_width<__bf16, 8>(a, dweight, shares, s) : dispatch_width<__bf16, 1>(a, dweight, shares, s);
    return words ? dispatch_width<float, 4>(a, dweight, shares, s) : dispatch_width<float, 1>(a, dweight, shares, s);
}

int check_shape(int64_t n, int32_t d, int dtype) {
    if (dtype != MTFM_HTA_BF16 && dtype != MTFM_HTA_FP32)
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "dtype must be MTFM_HTA_BF16 or MTFM_HTA_FP32, got %d", dtype);
    if (n < 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "negative n_rows");
    if (d <= 0) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "width must be positive, got %d", d);
    if (d > MAX_WIDTH) return hta::report_error(MTFM_HTA_ERR_UNSUPPORTED, "width %d exceeds %d", d, MAX_WIDTH);
    return MTFM_HTA_OK;
}

int check_strides(int64_t n, int32_t d, std::initializer_list<std::pair<const void*, int64_t>> rows) {
    for (const auto& r : rows) {
        if (r.first && r.second < d)
            return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "a row stride of %lld is less than the width %d", (long long)r.second, d);
        if (r.first && n > 0 && r.second > ((int64_t)1 << 46) / n)
            return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "a row stride of %lld reaches beyond any memory", (long long)r.second);
    }
    return MTFM_HTA_OK;
}

int forward(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight, void* h, void* y,
            float* rstd, float* scale, int64_t n_rows, int32_t width, float eps, int dtype, int out, void* stream) {
    if (int rc = check_shape(n_rows, width, dtype)) return rc;
    if (!(eps >= 0.f)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "eps must be >= 0");
    if (n_rows == 0) return MTFM_HTA_OK;
    if (!x || !weight || !y || (out != PLAIN && !scale)) return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    if ((residual == nullptr) != (h == nullptr))
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "residual and h must both be given or both be NULL");
    if (int rc = check_strides(n_rows, width, {{x, x_stride}, {residual, residual_stride}})) return rc;
    const unsigned size = dtype == MTFM_HTA_BF16 ? 2 : 4;
    if (misaligned(x, size) || misaligned(residual, size) || misaligned(h, size) || (out == PLAIN && misaligned(y, size)) ||
        misaligned(weight, 4) || misaligned(rstd, 4) || misaligned(scale, 4))
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "arrays must be aligned to their elements");
    Args a = {};
    a.x = x, a.residual = residual, a.weight = weight, a.h = h, a.y = y, a.rstd = rstd, a.scale = scale;
    a.ldx = x_stride, a.ldr = residual ? residual_stride : 0;
    a.n = n_rows, a.d = width, a.out = out, a.eps = eps;
    hipStream_t s = (hipStream_t)stream;
    hta::timing_begin(MTFM_RMS_KERNEL_FWD, s);
    const hipError_t e = dispatch(dtype, a, nullptr, nullptr, s);
    hta::timing_end(MTFM_RMS_KERNEL_FWD, s);
    if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "rms forward launch: %s", hipGetErrorString(e));
    return MTFM_HTA_OK;
}

}  // namespace rms

extern "C" {

int mtfm_rms_fwd(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight, void* h,
                 void* y, float* rstd, int64_t n_rows, int32_t width, float eps, int dtype, void* stream) {
    return rms::forward(x, x_stride, residual, residual_stride, weight, h, y, rstd, nullptr, n_rows, width, eps, dtype, rms::PLAIN, stream);
}

int mtfm_rms_fwd_q8(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, const float* weight, void* h,
                    void* q, float* scale, int64_t n_rows, int32_t width, float eps, int dtype, int kind, void* stream) {
    if (kind != MTFM_RMS_INT8 && kind != MTFM_RMS_E4M3)
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "kind must be MTFM_RMS_INT8 or MTFM_RMS_E4M3, got %d", kind);
    return rms::forward(x, x_stride, residual, residual_stride, weight, h, q, nullptr, scale, n_rows, width, eps, dtype, kind, stream);
}

size_t mtfm_rms_bwd_workspace_bytes(int32_t width) {
    if (rms::check_shape(0, width, MTFM_HTA_BF16) != MTFM_HTA_OK) return 0;
    return (size_t)rms::MAX_SHARES * ((width + 3) & ~3) * sizeof(float);
}

int mtfm_rms_bwd(const void* dy, int64_t dy_stride, const void* h, int64_t h_stride, const float* weight, const float* rstd,
                 const void* dh, int64_t dh_stride, void* dx, float* dweight, int64_t n_rows, int32_t width, int dtype,
                 void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = rms::check_shape(n_rows, width, dtype)) return rc;
    if (!dweight || (n_rows > 0 && (!dy || !h || !weight || !rstd || !dx)))
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "null pointer argument");
    if (n_rows > 0)
        if (int rc = rms::check_strides(n_rows, width, {{dy, dy_stride}, {h, h_stride}, {dh, dh_stride}})) return rc;
    const unsigned size = dtype == MTFM_HTA_BF16 ? 2 : 4;
    if (rms::misaligned(dy, size) || rms::misaligned(h, size) || rms::misaligned(dh, size) || rms::misaligned(dx, size) ||
        rms::misaligned(weight, 4) || rms::misaligned(rstd, 4) || rms::misaligned(dweight, 4))
        return hta::report_error(MTFM_HTA_ERR_INVALID_ARG, "arrays must be aligned to their elements");
    const size_t need = mtfm_rms_bwd_workspace_bytes(width);
    if (!workspace || workspace_bytes < need)
        return hta::report_error(MTFM_HTA_ERR_WORKSPACE, "this call needs %zu bytes of workspace, got %zu", need,
                                 workspace ? workspace_bytes : (size_t)0);
    if (rms::misaligned(workspace, 256)) return hta::report_error(MTFM_HTA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    rms::Args a = {};
    a.dy = dy, a.x = h, a.dh = dh, a.weight = weight, a.rstd_in = rstd, a.y = dx, a.partials = (float*)workspace;
    a.ldy = dy_stride, a.ldx = h_stride, a.ldh = dh ? dh_stride : 0;
    a.n = n_rows, a.d = width, a.out = rms::PLAIN;
    hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    int shares = 0;
    if (n_rows > 0) {
        hta::timing_begin(MTFM_RMS_KERNEL_BWD, s);
        e = rms::dispatch(dtype, a, dweight, &shares, s);
        hta::timing_end(MTFM_RMS_KERNEL_BWD, s);
        if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "rms backward launch: %s", hipGetErrorString(e));
        if (shares == 1) return MTFM_HTA_OK;
    }
    hta::timing_begin(MTFM_RMS_KERNEL_BWD_REDUCE, s);
    hipLaunchKernelGGL(rms::reduce_kernel, dim3((width + rms::REDUCE_COLS - 1) / rms::REDUCE_COLS), dim3(rms::REDUCE_THREADS), 0, s,
                       (const float*)workspace, shares, width, dweight);
    e = hipGetLastError();
    hta::timing_end(MTFM_RMS_KERNEL_BWD_REDUCE, s);
    if (e != hipSuccess) return hta::report_error(MTFM_HTA_ERR_LAUNCH, "rms reduce launch: %s", hipGetErrorString(e));
    return MTFM_HTA_OK;
}

}  // extern "C"
