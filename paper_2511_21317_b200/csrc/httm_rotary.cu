// Rows of queries and keys in front of the attention: per-head norm, rotation by position, their gradients, and the same rows on their
// way into the pages of a cache.
//
// A row is the head_dim channels of one head of one token.  With x its values:
//   mean = 0 (rms) or the mean of x (layer),  r = 1 / sqrt(mean((x - mean)^2) + eps),  xh = (x - mean) r,  z = xh w + b,
// and every rotated pair (a, b) of channels becomes (z_a c - z_b s, z_a s + z_b c) with (c, s) of the token's position.  Backwards, with dy the
// gradient of the output: g = dy rotated back, dw = sum g xh, db = sum g over all rows, u = g w, dx = r (u - [mean u] - xh mean(u xh)).
//
// Both directions are bound by memory (a row is read and written once, 2 operations per byte).  A row belongs to head_dim / 8 lanes, and a lane holds
// the four channels a .. a + 3 and the four it pairs them with, so that the rotation needs no exchange between lanes and each lane
// fetches the cos and sin of its own four pairs only; the sums of the norm are butterflies over the row's lanes.  The price is two
// 8-byte loads per row and lane instead of one of 16, at the same sectors.  A thread keeps to one chunk of heads, so that weights stay in
// registers, and walks the tokens; the rows of a chunk are loaded before the first is used.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "httm_cache.h"
#include "httm_internal.h"
#include "httm_launch.cuh"

namespace httm {

namespace {

constexpr int kThreads = 256;
constexpr int kHeadsPerChunk = 4;       // rows a lane has in flight
constexpr int kGradHeadsPerChunk = 2;   // (two tensors are read)

template <typename T>
struct Pair2;
template <>
struct Pair2<__nv_bfloat16> {
    static __device__ __forceinline__ float2 load(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
    static __device__ __forceinline__ uint32_t store(float a, float b) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};
template <>
struct Pair2<__half> {
    static __device__ __forceinline__ float2 load(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t store(float a, float b) {
        const __half2 v = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
};

__device__ __forceinline__ uint2 ld_row(const void* p) {   // behind depend_wait, and the row is read once
    uint2 v;
    asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
template <typename T>
__device__ __forceinline__ void unpack4(uint2 w, float* v) {
    const float2 a = Pair2<T>::load(w.x), b = Pair2<T>::load(w.y);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
template <typename T>
__device__ __forceinline__ uint2 pack4(const float* v) {
    return make_uint2(Pair2<T>::store(v[0], v[1]), Pair2<T>::store(v[2], v[3]));
}

// The channels of lane `l` of a row: v[0..3] are channels a .. a + 3, v[4..7] channels b .. b + 3.  Halves: pair i is (v[i], v[4 + i]); interleaved: the
// pairs are (v[0], v[1]), (v[2], v[3]), (v[4], v[5]), (v[6], v[7]).
struct LaneChannels {
    int a, b, axis, first;   // first of the four frequencies
    bool rotates;
    __device__ __forceinline__ LaneChannels(const RotationTable& t, int l) {
        rotates = 8 * l < t.rotated_dim;
        axis = first = 0;
        a = 8 * l;
        b = a + 4;
        if (rotates) {
            axis = 4 * l / t.half;
            first = 4 * l - axis * t.half;
            if (!t.interleaved) {
                a = axis * 2 * t.half + first;
                b = a + t.half;
            }
        }
    }
};
struct Turn {   // cos and sin of the lane's four pairs
    float c[4], s[4];
};
__device__ __forceinline__ Turn load_turn(const RotationTable& t, const LaneChannels& ch, const int32_t* positions, int64_t token, int32_t* status) {
    Turn r;
    const int32_t p = ld_global(positions + token * t.axes + ch.axis);
    if ((uint32_t)p >= (uint32_t)t.n_positions) {   // no such row of the table
        atomicCAS(status, kDevOk, kDevBadIndex);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.c[i] = r.s[i] = __int_as_float(0x7fc00000);
        return r;
    }
    const float4* at = reinterpret_cast<const float4*>(t.cos_sin + (int64_t)p * t.half + ch.first);
    const float4 u = __ldg(at), v = __ldg(at + 1);
    r.c[0] = u.x, r.s[0] = u.y, r.c[1] = u.z, r.s[1] = u.w;
    r.c[2] = v.x, r.s[2] = v.y, r.c[3] = v.z, r.s[3] = v.w;
    return r;
}
template <bool BACK>
__device__ __forceinline__ void turn(float (&v)[8], const Turn& t, bool interleaved) {
    auto one = [](float& a, float& b, float c, float s) {
        const float u = BACK ? fmaf(a, c, b * s) : fmaf(a, c, -(b * s));
        b = BACK ? fmaf(b, c, -(a * s)) : fmaf(a, s, b * c);
        a = u;
    };
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) one(v[2 * i], v[2 * i + 1], t.c[i], t.s[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) one(v[i], v[4 + i], t.c[i], t.s[i]);
    }
}
template <int LANES>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 1; o < LANES; o *= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// x -> xh in place; returns r.  The mean is taken off before the squares are added up: a row far from zero keeps its digits.
template <int LANES>
__device__ __forceinline__ float normalise(float (&x)[8], int norm, float eps) {
    constexpr float kInv = 1.0f / (8 * LANES);
    if (norm == HTTM_NORM_LAYER) {
        const float mean = row_sum<LANES>(((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]))) * kInv;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= mean;
    }
    float q0 = x[0] * x[0], q1 = x[1] * x[1];
#pragma unroll
    for (int i = 2; i < 8; i += 2) q0 = fmaf(x[i], x[i], q0), q1 = fmaf(x[i + 1], x[i + 1], q1);
    const float r = rsqrtf(fmaf(row_sum<LANES>(q0 + q1), kInv, eps));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= r;
    return r;
}
__device__ __forceinline__ void load_channels(const float* p, const LaneChannels& ch, float (&v)[8], float without) {
    if (p) {
        const float4 a = make_float4(p[ch.a], p[ch.a + 1], p[ch.a + 2], p[ch.a + 3]);
        const float4 b = make_float4(p[ch.b], p[ch.b + 1], p[ch.b + 2], p[ch.b + 3]);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = without;
    }
}

template <typename T, int LANES, bool PAGED>
__global__ void __launch_bounds__(kThreads) rows_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int GROUPS = kThreads / LANES;
    const bool second = (int)blockIdx.y >= a.t[0].chunks;
    const RowsTensor& t = a.t[second ? 1 : 0];
    const int h0 = ((int)blockIdx.y - (second ? a.t[0].chunks : 0)) * kHeadsPerChunk;
    const int lane = threadIdx.x % LANES;
    RotationTable table = a.table;
    if (!t.rotate) table.rotated_dim = 0;
    const LaneChannels ch(table, lane);
    const int rows = min(kHeadsPerChunk, t.heads - h0);
    depend_wait();
    dependents_launch();
    float w[8], b[8];
    load_channels(t.weight, ch, w, 1.f);
    load_channels(t.bias, ch, b, -0.f);   // (x + -0 is x, a zero's sign included)
    const T* in = static_cast<const T*>(t.in) + h0 * t.in_head;
    T* out = static_cast<T*>(t.out) + h0 * t.out_head;
    // (all lanes of a warp go through the loop together: the sums over a row exchange between lanes)
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < a.n_tokens; first += (int64_t)gridDim.x * GROUPS) {
        const int64_t token = first + threadIdx.x / LANES;
        const bool here = token < a.n_tokens;
        uint2 raw[kHeadsPerChunk][2];
        const T* src = in + token * t.in_token;
#pragma unroll
        for (int i = 0; i < kHeadsPerChunk; ++i) {
            if (here && i < rows) {
                raw[i][0] = ld_row(src + i * t.in_head + ch.a);
                raw[i][1] = ld_row(src + i * t.in_head + ch.b);
            } else {
                raw[i][0] = raw[i][1] = make_uint2(0u, 0u);
            }
        }
        Turn cs;
        if (here && ch.rotates) cs = load_turn(table, ch, a.positions, token, a.status);
        T* dst = out;
        if (here) {
            if (PAGED) {
                const int32_t slot = ld_global(a.slots + token);
                dst += (int64_t)(slot >> a.page_shift) * t.out_page + (int64_t)(slot & ((1 << a.page_shift) - 1)) * t.out_token;
            } else {
                dst += token * t.out_token;
            }
        }
#pragma unroll
        for (int i = 0; i < kHeadsPerChunk; ++i) {
            float x[8];
            unpack4<T>(raw[i][0], x);
            unpack4<T>(raw[i][1], x + 4);
            if (t.norm != HTTM_NORM_NONE) {
                normalise<LANES>(x, t.norm, a.eps);
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) x[c] = fmaf(x[c], w[c], b[c]);
            if (ch.rotates) turn<false>(x, cs, table.interleaved != 0);
            if (here && i < rows) {
                *reinterpret_cast<uint2*>(dst + i * t.out_head + ch.a) = pack4<T>(x);
                *reinterpret_cast<uint2*>(dst + i * t.out_head + ch.b) = pack4<T>(x + 4);
            }
        }
    }
}

// Gradients.  A CTA keeps to one tensor; its threads add up what they see of dw and db in registers, the CTA adds those up in shared memory, and the
// CTA of a tensor that arrives last adds the CTAs' sums, in the order of their numbers: the same sizes give the same bits.
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads) rows_grad_kernel(const __grid_constant__ RowsGradArgs a) {
    constexpr int GROUPS = kThreads / LANES, D = 8 * LANES;
    __shared__ float sums[2][GROUPS][D];
    __shared__ bool last;
    const int which = blockIdx.y;
    const RowsGradTensor& t = a.t[which];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const LaneChannels ch(a.table, lane);
    depend_wait();
    dependents_launch();
    float w[8], dw[8], db[8];
    load_channels(t.weight, ch, w, 1.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] = db[i] = 0.f;
    const T *xs = static_cast<const T*>(t.x), *dys = static_cast<const T*>(t.dy);
    T* dxs = static_cast<T*>(t.dx);
    const int64_t units = a.n_tokens * t.chunks;   // (token, chunk of heads)
    for (int64_t first = (int64_t)blockIdx.x * GROUPS; first < units; first += (int64_t)gridDim.x * GROUPS) {
        const int64_t unit = first + group;
        const bool here = unit < units;
        const int64_t token = here ? unit / t.chunks : 0;
        const int h0 = here ? (int)(unit - token * t.chunks) * kGradHeadsPerChunk : 0;
        const int rows = here ? min(kGradHeadsPerChunk, t.heads - h0) : 0;
        uint2 rx[kGradHeadsPerChunk][2], rg[kGradHeadsPerChunk][2];
#pragma unroll
        for (int i = 0; i < kGradHeadsPerChunk; ++i) {
            const T* x = xs + (h0 + i) * t.x_head + token * t.x_token;
            const T* dy = dys + (h0 + i) * t.dy_head + token * t.dy_token;
            if (i < rows) {
                rx[i][0] = ld_row(x + ch.a), rx[i][1] = ld_row(x + ch.b);
                rg[i][0] = ld_row(dy + ch.a), rg[i][1] = ld_row(dy + ch.b);
            } else {
                rx[i][0] = rx[i][1] = rg[i][0] = rg[i][1] = make_uint2(0u, 0u);
            }
        }
        Turn cs;
        if (here && ch.rotates) cs = load_turn(a.table, ch, a.positions, token, a.status);
#pragma unroll
        for (int i = 0; i < kGradHeadsPerChunk; ++i) {
            float x[8], g[8];
            unpack4<T>(rx[i][0], x);
            unpack4<T>(rx[i][1], x + 4);
            unpack4<T>(rg[i][0], g);
            unpack4<T>(rg[i][1], g + 4);
            if (ch.rotates) turn<true>(g, cs, a.table.interleaved != 0);
            float r = 1.f;
            if (a.norm != HTTM_NORM_NONE) r = normalise<LANES>(x, a.norm, a.eps);
            if (i < rows) {
#pragma unroll
                for (int c = 0; c < 8; ++c) dw[c] = fmaf(g[c], x[c], dw[c]), db[c] += g[c];
            }
#pragma unroll
            for (int c = 0; c < 8; ++c) g[c] *= w[c];
            if (a.norm != HTTM_NORM_NONE) {
                float su = 0.f, sux = 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) su += g[c], sux = fmaf(g[c], x[c], sux);
                sux = row_sum<LANES>(sux) * (1.0f / D);
                su = a.norm == HTTM_NORM_LAYER ? row_sum<LANES>(su) * (1.0f / D) : 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) g[c] = r * (g[c] - su - x[c] * sux);
            }
            if (i < rows) {
                T* dx = dxs + (h0 + i) * t.dx_head + token * t.dx_token;
                *reinterpret_cast<uint2*>(dx + ch.a) = pack4<T>(g);
                *reinterpret_cast<uint2*>(dx + ch.b) = pack4<T>(g + 4);
            }
        }
    }
    if (!t.dweight && !t.dbias) return;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        sums[0][group][ch.a + c] = dw[c], sums[0][group][ch.b + c] = dw[4 + c];
        sums[1][group][ch.a + c] = db[c], sums[1][group][ch.b + c] = db[4 + c];
    }
    __syncthreads();
    float* mine = a.partial + ((int64_t)which * gridDim.x + blockIdx.x) * 2 * D;
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll 8
        for (int g = 0; g < GROUPS; ++g) v += sums[i / D][g][i % D];
        __stcg(mine + i, v);
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.arrived + which, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    const float* all = a.partial + (int64_t)which * gridDim.x * 2 * D;
    // each of `parts` threads per sum takes every parts-th CTA
    constexpr int PARTS = 2 * D >= kThreads ? 1 : kThreads / (2 * D);
    float* flat = &sums[0][0][0];
    for (int i = threadIdx.x; i < 2 * D * PARTS; i += kThreads) {
        const int at = i % (2 * D);
        float v = 0.f;
#pragma unroll 16
        for (int c = i / (2 * D); c < (int)gridDim.x; c += PARTS) v += __ldcg(all + (int64_t)c * 2 * D + at);
        flat[i] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) v += flat[p * 2 * D + i];
        float* to = i < D ? t.dweight : t.dbias;
        if (to) to[i % D] = v;
    }
    if (threadIdx.x == 0) a.arrived[which] = 0;
}

__global__ void table_kernel(float2* table, const double* frequencies, int64_t n, int half) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= n) return;
    double s, c;
    sincos((double)(i / half) * frequencies[i % half], &s, &c);
    table[i] = make_float2((float)c, (float)s);
}

template <typename T, bool PAGED>
cudaError_t launch_rows_of(const RowsArgs& a, int head_dim, dim3 grid, cudaStream_t stream) {
    switch (head_dim) {
        case 32: return launch_kernel(rows_kernel<T, 4, PAGED>, grid, kThreads, 0, stream, a);
        case 64: return launch_kernel(rows_kernel<T, 8, PAGED>, grid, kThreads, 0, stream, a);
        case 128: return launch_kernel(rows_kernel<T, 16, PAGED>, grid, kThreads, 0, stream, a);
        case 256: return launch_kernel(rows_kernel<T, 32, PAGED>, grid, kThreads, 0, stream, a);
    }
    return cudaErrorInvalidValue;
}
template <typename T>
cudaError_t launch_rows_grad_of(const RowsGradArgs& a, int head_dim, dim3 grid, cudaStream_t stream) {
    switch (head_dim) {
        case 32: return launch_kernel(rows_grad_kernel<T, 4>, grid, kThreads, 0, stream, a);
        case 64: return launch_kernel(rows_grad_kernel<T, 8>, grid, kThreads, 0, stream, a);
        case 128: return launch_kernel(rows_grad_kernel<T, 16>, grid, kThreads, 0, stream, a);
        case 256: return launch_kernel(rows_grad_kernel<T, 32>, grid, kThreads, 0, stream, a);
    }
    return cudaErrorInvalidValue;
}
int grad_ctas(int sm_count) { return 2 * sm_count; }   // of each tensor

}  // namespace

cudaError_t launch_rows(const RowsArgs& args, int head_dim, int dtype, int sm_count, cudaStream_t stream) {
    RowsArgs a = args;
    int chunks = 0;
    for (RowsTensor& t : a.t) chunks += t.chunks = (t.heads + kHeadsPerChunk - 1) / kHeadsPerChunk;
    const int groups = kThreads / (head_dim / 8);
    const int64_t all = (a.n_tokens + groups - 1) / groups, most = ((int64_t)sm_count * 8 + chunks - 1) / chunks;
    const dim3 grid((unsigned)(all < most ? all : most), (unsigned)chunks);
    if (dtype == HTTM_BF16)
        return a.slots ? launch_rows_of<__nv_bfloat16, true>(a, head_dim, grid, stream) : launch_rows_of<__nv_bfloat16, false>(a, head_dim, grid, stream);
    return a.slots ? launch_rows_of<__half, true>(a, head_dim, grid, stream) : launch_rows_of<__half, false>(a, head_dim, grid, stream);
}

size_t rows_grad_partial_floats(int head_dim, int sm_count) { return (size_t)2 * grad_ctas(sm_count) * 2 * head_dim; }

cudaError_t launch_rows_grad(const RowsGradArgs& args, int head_dim, int dtype, int sm_count, cudaStream_t stream) {
    RowsGradArgs a = args;
    int64_t units = 1;
    int tensors = 0;
    for (RowsGradTensor& t : a.t) {
        t.chunks = (t.heads + kGradHeadsPerChunk - 1) / kGradHeadsPerChunk;
        units = units > a.n_tokens * t.chunks ? units : a.n_tokens * t.chunks;
        tensors += t.heads > 0 ? 1 : 0;
    }
    const int groups = kThreads / (head_dim / 8);
    const int64_t all = (units + groups - 1) / groups;
    const int most = grad_ctas(sm_count);
    const dim3 grid((unsigned)(all < most ? all : most), (unsigned)tensors);
    return dtype == HTTM_BF16 ? launch_rows_grad_of<__nv_bfloat16>(a, head_dim, grid, stream) : launch_rows_grad_of<__half>(a, head_dim, grid, stream);
}

int global_fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try {
        set_global_error(buf);
    } catch (...) {   // no memory for the text; the code still says what happened
    }
    return code;
}

int check_rows_layout(const httm_tensor& t, int64_t heads, int64_t tokens, int dim, bool written, const char* name) {
    if (!t.ptr) return global_fail(HTTM_ERR_INVALID_ARG, "%s: null pointer", name);
    if (((uintptr_t)t.ptr & 15u) != 0) return global_fail(HTTM_ERR_ALIGNMENT, "%s: pointer is not 16-byte aligned", name);
    if ((heads > 1 && t.stride_head % 8 != 0) || (tokens > 1 && t.stride_token % 8 != 0))
        return global_fail(HTTM_ERR_ALIGNMENT, "%s: strides must be multiples of 8 elements", name);
    const int64_t least = written ? dim : 0;   // (inputs may be broadcast)
    if ((heads > 1 && t.stride_head < least) || (tokens > 1 && t.stride_token < least))
        return global_fail(HTTM_ERR_INVALID_ARG, written ? "%s: strides must be >= head_dim" : "%s: strides must not be negative", name);
    if (written && heads > 1 && tokens > 1) {   // rows of one head must not reach into those of another
        const int64_t lo = t.stride_head < t.stride_token ? t.stride_head : t.stride_token, hi = t.stride_head + t.stride_token - lo;
        const int64_t n_lo = t.stride_head < t.stride_token ? heads : tokens;
        if (hi < (n_lo - 1) * lo + dim) return global_fail(HTTM_ERR_INVALID_ARG, "%s: rows overlap one another", name);
    }
    return HTTM_OK;
}

bool rows_conflict(const httm_tensor& x, int64_t x_heads, const httm_tensor& y, int64_t y_heads, int64_t tokens, int dim) {
    if (x.ptr == y.ptr && (x_heads <= 1 || x.stride_head == y.stride_head) && (tokens <= 1 || x.stride_token == y.stride_token)) return false;
    auto bytes = [&](const httm_tensor& t, int64_t heads) { return (((heads - 1) * t.stride_head) + (tokens - 1) * t.stride_token + dim) * 2; };
    const uintptr_t x0 = (uintptr_t)x.ptr, y0 = (uintptr_t)y.ptr;
    return x0 < y0 + (uintptr_t)bytes(y, y_heads) && y0 < x0 + (uintptr_t)bytes(x, x_heads);
}

}  // namespace httm

using namespace httm;

struct httm_rotary {
    httm_rotary_config cfg{};
    int32_t sm_count = 148;
    float2* table = nullptr;
    float* partial = nullptr;
    int32_t* words = nullptr;   // status, arrivals of the gradients' sums [2]
    RotationTable view() const {
        return RotationTable{table, cfg.n_positions, cfg.axes, cfg.rotated_dim / cfg.axes / 2, cfg.rotated_dim, cfg.interleaved};
    }
    ~httm_rotary() {
        for (void* p : {(void*)table, (void*)partial, (void*)words})
            if (p) cudaFree(p);
    }
};

namespace httm {
bool rotary_view(const httm_rotary* r, RotaryView* out) {
    if (!r) return false;
    *out = RotaryView{r->view(), r->cfg.device, r->cfg.head_dim, r->cfg.norm, (float)r->cfg.eps};
    return true;
}
}  // namespace httm

namespace {

int check_dtype(int32_t dtype, const char* what) {
    return dtype == HTTM_BF16 || dtype == HTTM_FP16 ? HTTM_OK : global_fail(HTTM_ERR_INVALID_ARG, "%s: dtype must be HTTM_BF16 or HTTM_FP16", what);
}
int cuda_result(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return HTTM_OK;
    cudaGetLastError();
    return global_fail(HTTM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

template <typename T>
int alloc(T** p, size_t count, const char* what) {
    const cudaError_t e = cudaMalloc(reinterpret_cast<void**>(p), count * sizeof(T));
    if (e == cudaSuccess) return HTTM_OK;
    *p = nullptr;
    cudaGetLastError();
    return global_fail(e == cudaErrorMemoryAllocation ? HTTM_ERR_NOMEM : HTTM_ERR_CUDA, "%s: cudaMalloc(%zu bytes): %s", what, count * sizeof(T),
                       cudaGetErrorString(e));
}

int check_call(httm_rotary* r, int32_t dtype, int64_t n_tokens, const int32_t* positions, const char* what) {
    if (!r) return global_fail(HTTM_ERR_INVALID_ARG, "%s: null handle", what);
    if (int rc = check_dtype(dtype, what)) return rc;
    if (n_tokens < 0 || n_tokens > (1ll << 31) - 1) return global_fail(HTTM_ERR_INVALID_ARG, "%s: number of tokens out of range", what);
    if (n_tokens > 0 && r->cfg.rotated_dim > 0 && (!positions || ((uintptr_t)positions & 3u) != 0))
        return global_fail(HTTM_ERR_INVALID_ARG, "%s: positions are missing or not aligned", what);
    return HTTM_OK;
}
int check_heads(int32_t heads, const char* name) {
    return heads >= 1 && heads <= 65535 ? HTTM_OK : global_fail(HTTM_ERR_INVALID_ARG, "%s: number of heads out of range", name);
}
int check_vector(const float* p, const char* name) {
    return ((uintptr_t)p & 3u) == 0 ? HTTM_OK : global_fail(HTTM_ERR_ALIGNMENT, "%s: not aligned", name);
}

}  // namespace

extern "C" {

int httm_rotary_create(const httm_rotary_config* config, httm_rotary** out) {
    if (out) *out = nullptr;
    if (!config || !out) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: null argument");
    const httm_rotary_config& c = *config;
    if (c.head_dim != 32 && c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256)
        return global_fail(HTTM_ERR_UNSUPPORTED, "rotary: head_dim must be 32, 64, 128 or 256");
    if (c.norm < HTTM_NORM_NONE || c.norm > HTTM_NORM_LAYER) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: unknown norm");
    if (c.axes != 1 && c.axes != 2) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: axes must be 1 or 2");
    if (c.interleaved != 0 && c.interleaved != 1) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: interleaved must be 0 or 1");
    if (c.rotated_dim < 0 || c.rotated_dim > c.head_dim || c.rotated_dim % (8 * c.axes) != 0)
        return global_fail(HTTM_ERR_INVALID_ARG, "rotary: rotated_dim must be a multiple of 8 * axes, at most head_dim");
    if (!(c.eps >= 0.0) || !std::isfinite(c.eps)) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: eps must be finite and not negative");
    const int half = c.rotated_dim / c.axes / 2;
    if (half > 0 && c.n_positions < 1) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: n_positions must be positive");
    if (half > 0 && !c.frequencies && (!(c.base > 0.0) || !std::isfinite(c.base)))
        return global_fail(HTTM_ERR_INVALID_ARG, "rotary: base must be positive");
    int devices = 0;
    if (cudaGetDeviceCount(&devices) != cudaSuccess) cudaGetLastError(), devices = 0;
    if (c.device < 0 || c.device >= devices) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: no such device");
    OnDevice guard(c.device);
    if (!guard.ok) return global_fail(HTTM_ERR_CUDA, "rotary: cudaSetDevice failed");
    try {
        std::vector<double> f((size_t)half);
        for (int i = 0; i < half; ++i) f[i] = c.frequencies ? c.frequencies[i] : std::pow(c.base, -(double)i / half);
        httm_rotary* r = new httm_rotary;
        r->cfg = c;
        r->cfg.frequencies = nullptr;
        cudaDeviceGetAttribute(&r->sm_count, cudaDevAttrMultiProcessorCount, c.device);
        double* d_f = nullptr;
        const int64_t n = (int64_t)(half > 0 ? c.n_positions : 0) * half;
        int rc = alloc(&r->words, 4, "rotary");
        if (!rc) rc = alloc(&r->partial, rows_grad_partial_floats(c.head_dim, r->sm_count), "rotary");
        if (!rc && n > 0) rc = alloc(&r->table, (size_t)n, "rotary");
        if (!rc) rc = cuda_result(cudaMemset(r->words, 0, 4 * sizeof(int32_t)), "rotary");
        if (!rc && n > 0) {
            rc = alloc(&d_f, (size_t)half, "rotary");
            if (!rc) rc = cuda_result(cudaMemcpy(d_f, f.data(), half * sizeof(double), cudaMemcpyHostToDevice), "rotary");
            if (!rc) {
                table_kernel<<<(unsigned)((n + 255) / 256), 256>>>(r->table, d_f, n, half);
                rc = cuda_result(cudaGetLastError(), "rotary table");
            }
        }
        if (!rc) rc = cuda_result(cudaDeviceSynchronize(), "rotary");
        if (d_f) cudaFree(d_f);
        if (rc) {
            delete r;
            return rc;
        }
        *out = r;
        return HTTM_OK;
    } catch (const std::bad_alloc&) {
        return global_fail(HTTM_ERR_NOMEM, "rotary: out of host memory");
    }
}

int httm_rotary_destroy(httm_rotary* r) {
    if (!r) return HTTM_OK;
    OnDevice guard(r->cfg.device);
    delete r;
    return HTTM_OK;
}

int httm_rotary_status(httm_rotary* r, int64_t* status) {
    if (!r || !status) return global_fail(HTTM_ERR_INVALID_ARG, "rotary: null argument");
    OnDevice guard(r->cfg.device);
    if (!guard.ok) return global_fail(HTTM_ERR_CUDA, "rotary: cudaSetDevice failed");
    int32_t s = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&s, r->words, sizeof s, cudaMemcpyDeviceToHost);
    if (int rc = cuda_result(e, "rotary status")) return rc;
    *status = s;
    return s == kDevOk ? HTTM_OK : global_fail(HTTM_ERR_CUDA, "a position was outside the rotation's table");
}

int httm_norm_rotate(httm_rotary* r, int32_t dtype, int64_t n_tokens, const int32_t* positions, const httm_rows* q, const httm_rows* k, void* stream) {
    if (int rc = check_call(r, dtype, n_tokens, positions, "norm_rotate")) return rc;
    if (!q && !k) return global_fail(HTTM_ERR_INVALID_ARG, "norm_rotate: neither q nor k");
    const httm_rows* in[2] = {q, k};
    const char* names[2] = {"norm_rotate: q", "norm_rotate: k"};
    RowsArgs a{};
    int n = 0;
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        const httm_rows& t = *in[i];
        int rc = check_heads(t.heads, names[i]);
        if (!rc && r->cfg.norm == HTTM_NORM_NONE && (t.weight || t.bias))
            rc = global_fail(HTTM_ERR_INVALID_ARG, "%s: a weight or bias without a norm", names[i]);
        if (!rc) rc = check_vector(t.weight, names[i]);
        if (!rc) rc = check_vector(t.bias, names[i]);
        if (!rc && n_tokens > 0) rc = check_rows_layout(t.x, t.heads, n_tokens, r->cfg.head_dim, false, names[i]);
        if (!rc && n_tokens > 0) rc = check_rows_layout(t.y, t.heads, n_tokens, r->cfg.head_dim, true, names[i]);
        if (!rc && n_tokens > 0 && rows_conflict(t.x, t.heads, t.y, t.heads, n_tokens, r->cfg.head_dim))
            rc = global_fail(HTTM_ERR_INVALID_ARG, "%s: the output overlaps the input", names[i]);
        if (rc) return rc;
        a.t[n++] = RowsTensor{t.x.ptr, t.y.ptr, t.x.stride_head, t.x.stride_token, t.y.stride_head, t.y.stride_token, 0, t.weight, t.bias, t.heads, 0,
                              r->cfg.norm, r->cfg.rotated_dim > 0};
    }
    if (n_tokens == 0) return HTTM_OK;
    OnDevice guard(r->cfg.device);
    if (!guard.ok) return global_fail(HTTM_ERR_CUDA, "norm_rotate: cudaSetDevice failed");
    a.table = r->view();
    a.positions = positions;
    a.n_tokens = n_tokens;
    a.eps = (float)r->cfg.eps;
    a.status = r->words;
    return cuda_result(launch_rows(a, r->cfg.head_dim, dtype, r->sm_count, static_cast<cudaStream_t>(stream)), "norm_rotate launch");
}

int httm_norm_rotate_backward(httm_rotary* r, int32_t dtype, int64_t n_tokens, const int32_t* positions, const httm_rows_grad* q,
                              const httm_rows_grad* k, void* stream) {
    if (int rc = check_call(r, dtype, n_tokens, positions, "norm_rotate_backward")) return rc;
    if (!q && !k) return global_fail(HTTM_ERR_INVALID_ARG, "norm_rotate_backward: neither q nor k");
    const httm_rows_grad* in[2] = {q, k};
    const char* names[2] = {"norm_rotate_backward: q", "norm_rotate_backward: k"};
    const int dim = r->cfg.head_dim;
    RowsGradArgs a{};
    int n = 0;
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        const httm_rows_grad& t = *in[i];
        int rc = check_heads(t.heads, names[i]);
        if (!rc && r->cfg.norm == HTTM_NORM_NONE && (t.weight || t.dweight || t.dbias))
            rc = global_fail(HTTM_ERR_INVALID_ARG, "%s: a weight or bias without a norm", names[i]);
        for (const float* v : {t.weight, (const float*)t.dweight, (const float*)t.dbias})
            if (!rc) rc = check_vector(v, names[i]);
        if (n_tokens > 0) {
            if (!rc) rc = check_rows_layout(t.x, t.heads, n_tokens, dim, false, names[i]);
            if (!rc) rc = check_rows_layout(t.dy, t.heads, n_tokens, dim, false, names[i]);
            if (!rc) rc = check_rows_layout(t.dx, t.heads, n_tokens, dim, true, names[i]);
            if (!rc && (rows_conflict(t.x, t.heads, t.dx, t.heads, n_tokens, dim) || rows_conflict(t.dy, t.heads, t.dx, t.heads, n_tokens, dim)))
                rc = global_fail(HTTM_ERR_INVALID_ARG, "%s: the output overlaps an input", names[i]);
        }
        if (rc) return rc;
        a.t[n++] = RowsGradTensor{t.x.ptr, t.dy.ptr, t.dx.ptr, t.x.stride_head, t.x.stride_token, t.dy.stride_head, t.dy.stride_token, t.dx.stride_head,
                                  t.dx.stride_token, t.weight, t.dweight, t.dbias, t.heads, 0};
    }
    OnDevice guard(r->cfg.device);
    if (!guard.ok) return global_fail(HTTM_ERR_CUDA, "norm_rotate_backward: cudaSetDevice failed");
    a.table = r->view();
    a.positions = positions;
    a.n_tokens = n_tokens;
    a.eps = (float)r->cfg.eps;
    a.norm = r->cfg.norm;
    a.partial = r->partial;
    a.arrived = r->words + 1;
    a.status = r->words;
    return cuda_result(launch_rows_grad(a, dim, dtype, r->sm_count, static_cast<cudaStream_t>(stream)), "norm_rotate_backward launch");
}

}  // extern "C"
