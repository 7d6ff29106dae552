// Attention over a paged cache for row tiles of at most 64 rows (single tokens, drafts), and the sum of partial results.
//
// A row tile has the query rows (token, head of the group) that share a key head, up to 64 of them, and walks the keys in tiles of 64:
//   s = scale q K^T,  m' = max(m, max s),  p = 2^(s - m'),  l = l 2^(m - m') + sum p,  O = O 2^(m - m') + p V   (scores in units of log2 e)
// Few rows leave nothing to compute per byte (at 4 rows 4 operations a byte), so the kernel is a stream of K and V through shared memory: 16-byte
// asynchronous copies three tiles deep, two CTAs per SM.  The products are done by warp-level matrix instructions of 16 rows; four warps share
// a tile of 16 rows by keys (16 keys each), one of 32 rows two by two, one of 64 by rows, and keep their own maxima and sums until the
// job ends.  The weights p are rounded to the values' type for the product with V, as they enter the matrix instruction; the sum l takes them before.
#include <type_traits>

#include "httm_cache.h"
#include "httm_internal.h"
#include "httm_launch.cuh"

namespace httm {

namespace {

constexpr int kThreads = 128;
constexpr int kStages = 3;

template <int D>
constexpr int kStageBytes = 2 * kNarrowKeys * D * 2;   // K and V of a key tile

__device__ __forceinline__ uint32_t smem_of(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;   // (0: sixteen zeros, nothing is read)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(at)
                 : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t ld_global_u32(const void* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// Byte of 16-byte piece `piece` of row `row` in a tile of rows of D values: pieces are exchanged within a row so that the eight rows a matrix
// load takes at once lie in distinct banks.
template <int D>
__device__ __forceinline__ uint32_t tile_at(int row, int piece) {
    return (uint32_t)(row * (D * 2) + ((piece ^ (row & 7)) << 4));
}

struct KeyTile {   // one tile of 64 keys
    const int32_t* pages;
    int key0, keys;      // its first key in the prefix / in the sequence, how many the tile has
    bool own;
};
__device__ __forceinline__ KeyTile key_tile(const CacheArgs& a, const CacheSeg& seg, int tile) {
    const int n_prefix = (seg.prefix_keys + kNarrowKeys - 1) / kNarrowKeys;
    KeyTile t;
    t.own = tile >= n_prefix;
    t.key0 = (t.own ? tile - n_prefix : tile) * kNarrowKeys;
    t.keys = min(kNarrowKeys, (t.own ? seg.own_keys : seg.prefix_keys) - t.key0);
    t.pages = a.table + (t.own ? seg.own_table : 0);
    return t;
}

template <typename T, int D>
__device__ __forceinline__ void fetch(const CacheArgs& a, const KeyTile& t, int head, uint32_t stage, int tid) {
    constexpr int PIECES = D / 8, ROWS = kThreads / PIECES;   // rows that the CTA fetches at once
    const int piece = tid % PIECES;
    const T* k = static_cast<const T*>(a.k) + head * a.k_head + piece * 8;
    const T* v = static_cast<const T*>(a.v) + head * a.v_head + piece * 8;
    const int mask = (1 << a.page_shift) - 1;
#pragma unroll
    for (int i = 0; i < kNarrowKeys / ROWS; ++i) {
        const int row = tid / PIECES + i * ROWS;
        const bool valid = row < t.keys;
        const int key = t.key0 + (valid ? row : 0);
        const int64_t page = ld_global(t.pages + (key >> a.page_shift));
        const uint32_t at = stage + tile_at<D>(row, piece);
        copy16(at, k + page * a.k_page + (key & mask) * a.k_slot, valid);
        copy16(at + kNarrowKeys * D * 2, v + page * a.v_page + (key & mask) * a.v_slot, valid);
    }
}

// One job with a tile of 16 MT rows.  Warp w has rows 16 (w mod MT) .. and of every key tile the keys 16 MT (w / MT) .. .
template <typename T, int D, int MT>
__device__ __forceinline__ void narrow_job(const CacheArgs& a, const CacheSeg& seg, const CacheJob& job, unsigned char* smem) {
    constexpr int KG = 4 / MT, NB = 2 * MT;   // warps that share a row by keys; blocks of eight keys of a warp
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row0 = (warp % MT) * 16 + (lane >> 2), key_base = (warp / MT) * 16 * MT;
    const int n_rows = seg.tokens * a.group;
    const uint32_t base = smem_of(smem);
    const int n = job.tile1 - job.tile0;

    for (int i = 0; i < kStages - 1; ++i) {
        if (i < n) fetch<T, D>(a, key_tile(a, seg, job.tile0 + i), job.head, base + i * kStageBytes<D>, tid);
        copies_commit();
    }
    // rows as operands of the matrix instruction: this thread has rows row0 and row0 + 8
    uint32_t qf[D / 16][4];
    int seen[2];   // own keys that the two rows see
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + 8 * r;
        const bool valid = row < n_rows;
        const int token = valid ? row / a.group : 0;
        seen[r] = min(seg.own_keys, seg.seen0 + token * seg.seen_step);
        const T* q = static_cast<const T*>(a.q) + (int64_t)(seg.token0 + token) * a.q_token + (int64_t)(job.head * a.group + (valid ? row % a.group : 0)) * a.q_head +
                     2 * (lane & 3);
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            qf[c][r] = valid ? ld_global_u32(q + 16 * c) : 0u;
            qf[c][2 + r] = valid ? ld_global_u32(q + 16 * c + 8) : 0u;
        }
    }
    float o[D / 8][4];
#pragma unroll
    for (int c = 0; c < D / 8; ++c) o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int i = 0; i < n; ++i) {
        copies_wait<kStages - 2>();
        __syncthreads();   // tile i is there for everybody, and everybody is done with tile i - 1
        const int next = i + kStages - 1;
        if (next < n) fetch<T, D>(a, key_tile(a, seg, job.tile0 + next), job.head, base + (next % kStages) * kStageBytes<D>, tid);
        copies_commit();
        const KeyTile t = key_tile(a, seg, job.tile0 + i);
        const uint32_t ks = base + (i % kStages) * kStageBytes<D>, vs = ks + kNarrowKeys * D * 2;
        float s[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b][0] = s[b][1] = s[b][2] = s[b][3] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
#pragma unroll
            for (int b = 0; b < MT; ++b) {   // sixteen keys
                uint32_t kf[4];
                ldmatrix4(kf, ks + tile_at<D>(key_base + 16 * b + (lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)));
                mma<T>(s[2 * b], qf[c], kf[0], kf[1]);
                mma<T>(s[2 * b + 1], qf[c], kf[2], kf[3]);
            }
        }
        float top[2] = {-INFINITY, -INFINITY};
        int limit[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) limit[r] = t.own ? min(t.keys, seen[r] - t.key0) : t.keys;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int key = key_base + 8 * b + 2 * (lane & 3) + (e & 1);
                s[b][e] = key < limit[e >> 1] ? s[b][e] * a.scale_log2 : -INFINITY;
                top[e >> 1] = fmaxf(top[e >> 1], s[b][e]);
            }
        float from[2];   // what is taken off the scores: the maximum so far; 0 as long as a row has seen no key
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
            const float to = fmaxf(m[r], top[r]);
            from[r] = to == -INFINITY ? 0.f : to;
            top[r] = exp2_fast(m[r] - from[r]);   // what earlier sums shrink by
            m[r] = to;
        }
        if (__any_sync(0xffffffffu, top[0] != 1.f || top[1] != 1.f)) {
#pragma unroll
            for (int c = 0; c < D / 8; ++c) o[c][0] *= top[0], o[c][1] *= top[0], o[c][2] *= top[1], o[c][3] *= top[1];
            l[0] *= top[0], l[1] *= top[1];
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[b][e] = exp2_fast(s[b][e] - from[e >> 1]);
                l[e >> 1] += s[b][e];
            }
#pragma unroll
        for (int b = 0; b < MT; ++b) {
            const uint32_t pf[4] = {pack2<T>(s[2 * b][0], s[2 * b][1]), pack2<T>(s[2 * b][2], s[2 * b][3]), pack2<T>(s[2 * b + 1][0], s[2 * b + 1][1]),
                                    pack2<T>(s[2 * b + 1][2], s[2 * b + 1][3])};
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t vf[4];
                ldmatrix4_t(vf, vs + tile_at<D>(key_base + 16 * b + (lane & 15), 2 * c + (lane >> 4)));
                mma<T>(o[2 * c], pf, vf[0], vf[1]);
                mma<T>(o[2 * c + 1], pf, vf[2], vf[3]);
            }
        }
    }
    // the warps that share rows, added up in the order of their keys
    copies_wait<0>();
    __syncthreads();
    float* all = reinterpret_cast<float*>(smem);                    // [warp][16][D]
    float2* stats = reinterpret_cast<float2*>(smem + 4 * 16 * D * 4);   // [warp][16]
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        const int at = warp * 16 + (lane >> 2) + 8 * r;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) *reinterpret_cast<float2*>(all + at * D + 8 * c + 2 * (lane & 3)) = make_float2(o[c][2 * r], o[c][2 * r + 1]);
        if ((lane & 3) == 0) stats[at] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    constexpr int QUADS = D / 4;
    for (int i = tid; i < n_rows * QUADS; i += kThreads) {
        const int row = i / QUADS, c = i % QUADS;
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < KG; ++g) top = fmaxf(top, stats[(g * MT + row / 16) * 16 + row % 16].x);
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        float total = 0.f;
#pragma unroll
        for (int g = 0; g < KG; ++g) {
            const int at = (g * MT + row / 16) * 16 + row % 16;
            const float2 st = stats[at];
            const float f = st.x == -INFINITY ? 0.f : exp2_fast(st.x - top);
            const float4 v = *reinterpret_cast<const float4*>(all + at * D + 4 * c);
            sum.x = fmaf(v.x, f, sum.x), sum.y = fmaf(v.y, f, sum.y), sum.z = fmaf(v.z, f, sum.z), sum.w = fmaf(v.w, f, sum.w);
            total = fmaf(st.y, f, total);
        }
        if (job.part < 0) {
            const float inv = top == -INFINITY ? 0.f : 1.f / total;
            T* out = static_cast<T*>(a.out) + (int64_t)(seg.token0 + row / a.group) * a.out_token + (int64_t)(job.head * a.group + row % a.group) * a.out_head + 4 * c;
            *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(sum.x * inv, sum.y * inv), pack2<T>(sum.z * inv, sum.w * inv));
        } else {
            float* to = a.partial + (int64_t)job.part * (kPartUnit * (D + 2));
            __stcg(reinterpret_cast<float4*>(to + row * D + 4 * c), sum);
            if (c == 0) __stcg(reinterpret_cast<float2*>(to + 16 * MT * D + 2 * row), make_float2(top, total));
        }
    }
    __syncthreads();   // the next job's copies go over what has been read here
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) cache_narrow_kernel(const __grid_constant__ CacheArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    depend_wait();
    dependents_launch();
    const int last = ld_global(a.job_start + blockIdx.x + 1);
    for (int j = ld_global(a.job_start + blockIdx.x); j < last; ++j) {
        const CacheJob job = a.jobs[j];
        const CacheSeg seg = a.segs[job.seg];
        if (seg.tile_rows == 16)
            narrow_job<T, D, 1>(a, seg, job, smem);
        else if (seg.tile_rows == 32)
            narrow_job<T, D, 2>(a, seg, job, smem);
        else
            narrow_job<T, D, 4>(a, seg, job, smem);
    }
}

// The partial results of rows whose keys were shared out, added up in the order of the keys: out = sum O_i 2^(m_i - m) / sum l_i 2^(m_i - m).  A CTA takes a few
// rows; with fewer rows than warps the parts of a row are dealt to several warps, since a row of single tokens behind a long prefix has some
// twenty parts and the time is that of the loads behind one another.  A row without parts gets zeros.
constexpr int kCombineWarps = 8;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kCombineWarps) cache_combine_kernel(const __grid_constant__ CacheArgs a) {
    constexpr int V = D / 32;   // channels of a lane
    __shared__ float4 shared_sum[kCombineWarps][32];
    __shared__ float2 shared_stat[kCombineWarps];
    depend_wait();
    dependents_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const CombineTask task = a.combine_tasks[blockIdx.x];
    const int rows = task.tokens * a.group;
    int ways = 1;   // warps that share a row's parts
    while (2 * ways * rows <= kCombineWarps) ways *= 2;
    const int way = warp % ways;
    // the parts of a tile lie one behind the other: n, the tile's rows, its first row of this task
    int n0 = 0, n1 = 0, rows0 = 0, rows1 = 0, first0 = 0, first1 = 0;
    const float *base0 = nullptr, *base1 = nullptr;
    auto find = [&](int seg, int& n, int& tile_rows, int& first, const float*& base) {
        if (seg < 0) return;
        const int2 part = a.parts[(int64_t)seg * a.kv_heads + task.head];
        const int4 s = *reinterpret_cast<const int4*>(a.segs + seg);   // token0, tokens, tile_rows
        n = part.y;
        tile_rows = s.z;
        first = (task.token0 - s.x) * a.group;
        base = a.partial + (int64_t)part.x * (kPartUnit * (D + 2));
    };
    find(task.prefix_seg, n0, rows0, first0, base0);
    find(task.own_seg, n1, rows1, first1, base1);
    const int n = n0 + n1;
    for (int r0 = 0; r0 < rows; r0 += kCombineWarps / ways) {
        const int row = r0 + warp / ways;
        const bool here = row < rows;
        // part p of the row: its values and its (maximum, sum)
        auto values = [&](int p) {
            return p < n0 ? base0 + (int64_t)p * rows0 * (D + 2) + (first0 + row) * D : base1 + (int64_t)(p - n0) * rows1 * (D + 2) + (first1 + row) * D;
        };
        auto stat = [&](int p) {
            return p < n0 ? base0 + (int64_t)p * rows0 * (D + 2) + rows0 * D + 2 * (first0 + row)
                          : base1 + (int64_t)(p - n0) * rows1 * (D + 2) + rows1 * D + 2 * (first1 + row);
        };
        float top = -INFINITY, total = 0.f, sum[V];
#pragma unroll
        for (int c = 0; c < V; ++c) sum[c] = 0.f;
        if (here) {
            for (int p0 = way; p0 < n; p0 += 32 * ways) {   // 32 parts at a time, one per lane
                const int mine = p0 + lane * ways;
                float2 st = make_float2(-INFINITY, 0.f);
                if (mine < n) st = __ldcg(reinterpret_cast<const float2*>(stat(mine)));
                float high = st.x;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
                const float to = fmaxf(top, high), shrink = top == -INFINITY ? 0.f : exp2_fast(top - to);
                const float f = st.x == -INFINITY ? 0.f : exp2_fast(st.x - to);
                top = to;
                total = fmaf(st.y, f, total * shrink);   // (a lane's share; added up below)
#pragma unroll
                for (int c = 0; c < V; ++c) sum[c] *= shrink;
                const int m = min(32, (n - p0 + ways - 1) / ways);
#pragma unroll 8
                for (int i = 0; i < m; ++i) {
                    const float w = __shfl_sync(0xffffffffu, f, i);
                    const float* at = values(p0 + i * ways) + lane * V;
                    if constexpr (V == 4) {
                        const float4 v = __ldcg(reinterpret_cast<const float4*>(at));
                        sum[0] = fmaf(v.x, w, sum[0]), sum[1] = fmaf(v.y, w, sum[1]), sum[2] = fmaf(v.z, w, sum[2]), sum[3] = fmaf(v.w, w, sum[3]);
                    } else {
                        const float2 v = __ldcg(reinterpret_cast<const float2*>(at));
                        sum[0] = fmaf(v.x, w, sum[0]), sum[1] = fmaf(v.y, w, sum[1]);
                    }
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        }
        if (ways > 1) {   // (one round of rows: rows * ways <= warps)
            if constexpr (V == 4)
                shared_sum[warp][lane] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            else
                shared_sum[warp][lane] = make_float4(sum[0], sum[1], 0.f, 0.f);
            if (lane == 0) shared_stat[warp] = make_float2(top, total);
            __syncthreads();
            if (way == 0) {
                float high = top;
                for (int i = 1; i < ways; ++i) high = fmaxf(high, shared_stat[warp + i].x);
                const float own = top == -INFINITY ? 0.f : exp2_fast(top - high);
                total *= own;
#pragma unroll
                for (int c = 0; c < V; ++c) sum[c] *= own;
                for (int i = 1; i < ways; ++i) {
                    const float2 st = shared_stat[warp + i];
                    const float4 v = shared_sum[warp + i][lane];
                    const float f = st.x == -INFINITY ? 0.f : exp2_fast(st.x - high);
                    total = fmaf(st.y, f, total);
                    sum[0] = fmaf(v.x, f, sum[0]), sum[1] = fmaf(v.y, f, sum[1]);
                    if constexpr (V == 4) sum[2] = fmaf(v.z, f, sum[2]), sum[3] = fmaf(v.w, f, sum[3]);
                }
                top = high;
            }
        }
        if (here && way == 0) {
            const float inv = top == -INFINITY ? 0.f : 1.f / total;
            const int token = task.token0 + row / a.group, head = task.head * a.group + row % a.group;
            T* out = static_cast<T*>(a.out) + (int64_t)token * a.out_token + (int64_t)head * a.out_head + lane * V;
            if constexpr (V == 4)
                *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(sum[0] * inv, sum[1] * inv), pack2<T>(sum[2] * inv, sum[3] * inv));
            else
                *reinterpret_cast<uint32_t*>(out) = pack2<T>(sum[0] * inv, sum[1] * inv);
        }
    }
}

template <typename F>
cudaError_t allow_smem(F kernel, int bytes) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
template <typename T, int D>
cudaError_t narrow_of(const CacheArgs& a, int ctas, cudaStream_t stream) {
    return launch_kernel(cache_narrow_kernel<T, D>, ctas, kThreads, kStages * kStageBytes<D>, stream, a);
}
template <typename T, int D>
cudaError_t combine_of(const CacheArgs& a, int tasks, cudaStream_t stream) {
    return launch_kernel(cache_combine_kernel<T, D>, tasks, 32 * kCombineWarps, 0, stream, a);
}

}  // namespace

cudaError_t configure_cache_attention() {
    cudaError_t e = allow_smem(cache_narrow_kernel<__nv_bfloat16, 64>, kStages * kStageBytes<64>);
    if (e == cudaSuccess) e = allow_smem(cache_narrow_kernel<__nv_bfloat16, 128>, kStages * kStageBytes<128>);
    if (e == cudaSuccess) e = allow_smem(cache_narrow_kernel<__half, 64>, kStages * kStageBytes<64>);
    if (e == cudaSuccess) e = allow_smem(cache_narrow_kernel<__half, 128>, kStages * kStageBytes<128>);
    return e;
}

cudaError_t launch_cache_narrow(const CacheArgs& a, int head_dim, int dtype, int ctas, cudaStream_t stream) {
    if (dtype == HTTM_BF16) return head_dim == 64 ? narrow_of<__nv_bfloat16, 64>(a, ctas, stream) : narrow_of<__nv_bfloat16, 128>(a, ctas, stream);
    return head_dim == 64 ? narrow_of<__half, 64>(a, ctas, stream) : narrow_of<__half, 128>(a, ctas, stream);
}
cudaError_t launch_cache_combine(const CacheArgs& a, int head_dim, int dtype, int tasks, cudaStream_t stream) {
    if (dtype == HTTM_BF16) return head_dim == 64 ? combine_of<__nv_bfloat16, 64>(a, tasks, stream) : combine_of<__nv_bfloat16, 128>(a, tasks, stream);
    return head_dim == 64 ? combine_of<__half, 64>(a, tasks, stream) : combine_of<__half, 128>(a, tasks, stream);
}

}  // namespace httm
