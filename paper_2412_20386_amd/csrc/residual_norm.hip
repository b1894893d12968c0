// Norms after and before a block, with the block's gate and the residual stream between them:
//   q = norm(h) * w_post (or h),  r = scale * residual + gate * q,  y = norm(r) * w,  norm(v) = v / sqrt(mean(v^2) + eps)
// h is a block's output, r the residual stream behind it, y the next block's input.  Backward, for the gradients dy of y and
// dr of r, with n = norm(r), m = norm(h) and the two means computed again from r and h:
//   e = dr + (dy w - n mean(dy w n)) / rms(r),  dresidual = scale e,  dgate = sum e q,  f = gate e,
//   dh = (f w_post - m mean(f w_post m)) / rms(h)  (or f),  dw = sum dy n,  dw_post = sum f m.
//
// Bound by memory.  A row is held in registers by the 2^n lanes of a wavefront that share it (V = 8 or 6 elements to a lane and
// load, up to two loads; 6 where that leaves fewer lanes idle: 192, 384 and 768 columns are 32, 64 and 2 x 64 of them), or by 4, 8 or 16
// wavefronts where it is wider than that: every matrix is read once and written once, the next row in flight under this one.  Sums
// are fp32.  Groups of lanes stride over the rows, so the parameters stay in registers, and so do the gradients of the
// parameters, which leave as one partial sum per workgroup.  Forward, 50432 x 768 in fp16 with an fp32 stream: 84 us, 5.5 TB/s
// (part of it from the memory-side cache); backward, 50240 x 384 in bf16, both norms and a gate an image: 58 us, 4.0 TB/s.
// Wide rows, both norms, 49 million elements in fp16 with an fp32 stream, forward / backward: 4096 columns 125 / 337 us, 8192 138 / 343, 16384
// 190 / 1229.  From 4097 columns on the backward pass, and from 8193 the forward pass too, keeps part of a row in scratch: 64 to 100 bytes a lane in
// 8 wavefronts, 44 to 72 forward and about 660 backward in 16, whose lanes have 128 registers for two loads of 8 elements of every matrix.
// A gate for each few rows leaves slots of the backward pass idle, since a workgroup's rows share one: 30000 x 64 with a gate for 3 rows
// takes 75 us, without gates 16.
#include <type_traits>

#include "token_ops.hpp"

namespace {

using namespace ptq4vm;

template <typename T, typename R>
struct NormArgs {
    const T *h;
    const R *residual;
    const float *w, *gate, *w_post;
    T *y;
    R *r;  // in in the backward pass
    const T *dy;
    const R *dr;
    T *dh;
    R *dresidual;
    float *partial, *gate_partial;
    float scale, eps;
    int K;
    uint32_t M, gate_rows, parts, part_rows;  // rows of one gate, parts they are cut into (backward), rows of a part
    int lanes_log2;                // lanes that share a row where one wavefront holds it
    int64_t ldh, ldres, ldy, ldr, lddy, lddr, lddh, lddres;
};

// Sum over the lanes that hold a row
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, int lanes, float *red) {
    v = group_sum(v, lanes);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int i = 1; i < WAVES; i++) v += red[i];
        __syncthreads();
    }
    return v;
}

template <typename T, int CHUNKS, int V>
__device__ __forceinline__ void load_row(const T *p, const int (&k)[CHUNKS], const int (&n)[CHUNKS], T (&v)[CHUNKS][V]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) load_first<V>(p + k[c], n[c], v[c]);
}

// Which columns a lane holds, and which of the workgroup's row slots it belongs to
template <int V, int CHUNKS, int WAVES, bool FULL>
struct Lane {
    int k[CHUNKS], n[CHUNKS], lanes, slot, slots;
    __device__ __forceinline__ Lane(int K, int lanes_log2) {
        lanes = WAVES > 1 ? 64 : 1 << lanes_log2;
        const int across = WAVES > 1 ? WAVES * 64 : lanes, in_row = threadIdx.x & (across - 1);
        slot = WAVES > 1 ? 0 : threadIdx.x >> lanes_log2;
        slots = WAVES > 1 ? 1 : 256 >> lanes_log2;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            k[c] = (in_row + c * across) * V;
            n[c] = FULL ? V : max(0, min(V, K - k[c]));  // (known to the compiler where all lanes are full)
            if (!FULL && n[c] == 0) k[c] = 0;
        }
    }
};

template <typename T, typename R, int V, int CHUNKS, int WAVES, bool FULL>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void residual_norm_rows(NormArgs<T, R> p) {
    __shared__ float red[WAVES];
    const Lane<V, CHUNKS, WAVES, FULL> at(p.K, p.lanes_log2);
    const float per_k = 1.0f / p.K;
    float w[CHUNKS][V], w_post[CHUNKS][V];
    load_row<float, CHUNKS, V>(p.w, at.k, at.n, w);
    if (p.w_post) load_row<float, CHUNKS, V>(p.w_post, at.k, at.n, w_post);
    // whole workgroups stay together: rows beyond the last are computed as it and not written
    T next_h[CHUNKS][V];
    R next_res[CHUNKS][V];
    const auto fetch = [&](uint64_t first) {
        const int64_t row = min(first + at.slot, (uint64_t)p.M - 1);
        load_row<T, CHUNKS, V>(p.h + row * p.ldh, at.k, at.n, next_h);
        if (p.residual) load_row<R, CHUNKS, V>(p.residual + row * p.ldres, at.k, at.n, next_res);
    };
    const uint64_t step = (uint64_t)gridDim.x * at.slots;
    fetch((uint64_t)blockIdx.x * at.slots);
    for (uint64_t first = (uint64_t)blockIdx.x * at.slots; first < p.M; first += step) {
        const bool own = first + at.slot < p.M;
        const uint32_t row = own ? (uint32_t)(first + at.slot) : p.M - 1;
        T h[CHUNKS][V];
        R res[CHUNKS][V];
        float gate[CHUNKS][V], v[CHUNKS][V];
        __builtin_memcpy(h, next_h, sizeof(h));
        if (p.residual) __builtin_memcpy(res, next_res, sizeof(res));
        if (first + step < p.M) fetch(first + step);
        if (p.gate) load_row<float, CHUNKS, V>(p.gate + (int64_t)(row / p.gate_rows) * p.K, at.k, at.n, gate);
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
#pragma unroll
            for (int i = 0; i < V; i++) v[c][i] = (float)h[c][i];
        if (p.w_post) {
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) sum = fmaf(v[c][i], v[c][i], sum);
            const float f = rsqrtf(row_sum<WAVES>(sum, at.lanes, red) * per_k + p.eps);
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) v[c][i] = v[c][i] * f * w_post[c][i];
        }
        if (p.gate)
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) v[c][i] *= gate[c][i];
        if (p.residual)
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) v[c][i] = fmaf(p.scale, (float)res[c][i], v[c][i]);
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
#pragma unroll
            for (int i = 0; i < V; i++) sum = i < at.n[c] ? fmaf(v[c][i], v[c][i], sum) : sum;  // (a gate of NaN times the zeros behind a row)
        const float f = rsqrtf(row_sum<WAVES>(sum, at.lanes, red) * per_k + p.eps);
        if (!own) continue;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++) {
            if (at.n[c] == 0) continue;
            store_first<V>(p.r + row * p.ldr + at.k[c], at.n[c], v[c]);
            float y[V];
#pragma unroll
            for (int i = 0; i < V; i++) y[i] = v[c][i] * f * w[c][i];
            store_first<V>(p.y + row * p.ldy + at.k[c], at.n[c], y);
        }
    }
}

// Sum of v over the row slots of a workgroup, to out[k] (its row of partial sums)
template <int V, int CHUNKS, int WAVES, bool FULL>
__device__ __forceinline__ void sum_slots(const float (&v)[CHUNKS][V], const Lane<V, CHUNKS, WAVES, FULL> &at, float *out, float (*red)[V + 1]) {
    if (WAVES > 1 || at.slots == 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
            if (at.n[c]) store_first<V>(out + at.k[c], at.n[c], v[c]);
        return;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; c++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; i++) red[threadIdx.x][i] = v[c][i];
        __syncthreads();
        if (at.slot == 0 && at.n[c]) {
            float sum[V];
#pragma unroll
            for (int i = 0; i < V; i++) sum[i] = v[c][i];
            for (int s = 1; s < at.slots; s++)
#pragma unroll
                for (int i = 0; i < V; i++) sum[i] += red[s * at.lanes + threadIdx.x][i];
            store_first<V>(out + at.k[c], at.n[c], sum);
        }
    }
}

// A part is a run of rows under one gate; a workgroup takes every gridDim-th part.  partial[workgroup] is [K | K] (dw,
// dw_post), gate_partial[part] is [K]; where every row has a gate of its own, its gradient is written to gate_partial[row].
template <typename T, typename R, int V, int CHUNKS, int WAVES, bool FULL>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void residual_norm_backward_rows(NormArgs<T, R> p, int64_t all_parts) {
    __shared__ float red[WAVES], cols[WAVES == 1 ? 256 : 1][V + 1];
    const Lane<V, CHUNKS, WAVES, FULL> at(p.K, p.lanes_log2);
    const float per_k = 1.0f / p.K;
    const bool row_gates = p.gate && p.gate_rows == 1;
    float w[CHUNKS][V], w_post[CHUNKS][V], dw[CHUNKS][V] = {}, dw_post[CHUNKS][V] = {}, dgate[CHUNKS][V];
    load_row<float, CHUNKS, V>(p.w, at.k, at.n, w);
    if (p.w_post) load_row<float, CHUNKS, V>(p.w_post, at.k, at.n, w_post);
    for (int64_t part = blockIdx.x; part < all_parts; part += gridDim.x) {
        const uint32_t rows_together = row_gates ? p.M : p.gate_rows;
        const uint32_t group = (uint32_t)(part / p.parts), begin = (uint32_t)(part - (int64_t)group * p.parts) * p.part_rows;
        const uint64_t first = (uint64_t)group * rows_together + begin;
        const uint32_t count = begin < rows_together ? min(p.part_rows, rows_together - begin) : 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; c++)
#pragma unroll
            for (int i = 0; i < V; i++) dgate[c][i] = 0.0f;
        float gate[CHUNKS][V];
        if (p.gate && !row_gates) load_row<float, CHUNKS, V>(p.gate + (int64_t)group * p.K, at.k, at.n, gate);
        T next_h[CHUNKS][V], next_dy[CHUNKS][V];
        R next_r[CHUNKS][V], next_dr[CHUNKS][V];
        const auto fetch = [&](uint32_t i0) {
            const int64_t row = first + min(i0 + at.slot, count - 1);
            load_row<T, CHUNKS, V>(p.h + row * p.ldh, at.k, at.n, next_h);
            load_row<T, CHUNKS, V>(p.dy + row * p.lddy, at.k, at.n, next_dy);
            load_row<R, CHUNKS, V>(p.r + row * p.ldr, at.k, at.n, next_r);
            if (p.dr) load_row<R, CHUNKS, V>(p.dr + row * p.lddr, at.k, at.n, next_dr);
        };
        if (count > 0) fetch(0);
        for (uint32_t i0 = 0; i0 < count; i0 += at.slots) {
            const bool own = i0 + at.slot < count;
            const int64_t row = first + (own ? i0 + at.slot : count - 1);
            T raw_h[CHUNKS][V], raw_dy[CHUNKS][V];
            R raw_r[CHUNKS][V], raw_dr[CHUNKS][V];
            __builtin_memcpy(raw_h, next_h, sizeof(raw_h));
            __builtin_memcpy(raw_dy, next_dy, sizeof(raw_dy));
            __builtin_memcpy(raw_r, next_r, sizeof(raw_r));
            if (p.dr) __builtin_memcpy(raw_dr, next_dr, sizeof(raw_dr));
            if (i0 + at.slots < count) fetch(i0 + at.slots);
            if (row_gates) load_row<float, CHUNKS, V>(p.gate + row * p.K, at.k, at.n, gate);
            float rr = 0.0f, tr = 0.0f, hh = 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float r = (float)raw_r[c][i], h = (float)raw_h[c][i];
                    rr = fmaf(r, r, rr);
                    tr = fmaf((float)raw_dy[c][i] * w[c][i], r, tr);
                    hh = fmaf(h, h, hh);
                }
            const float fr = rsqrtf(row_sum<WAVES>(rr, at.lanes, red) * per_k + p.eps);
            const float mean_tn = row_sum<WAVES>(tr, at.lanes, red) * per_k * fr;
            float fh = 1.0f;
            if (p.w_post) fh = rsqrtf(row_sum<WAVES>(hh, at.lanes, red) * per_k + p.eps);
            float e[CHUNKS][V], f[CHUNKS][V], fm = 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; c++)
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float dy = (float)raw_dy[c][i], n = (float)raw_r[c][i] * fr;
                    e[c][i] = fr * (dy * w[c][i] - n * mean_tn) + (p.dr ? (float)raw_dr[c][i] : 0.0f);
                    if (own) dw[c][i] = fmaf(dy, n, dw[c][i]);
                    f[c][i] = p.gate ? gate[c][i] * e[c][i] : e[c][i];
                    if (p.w_post) {
                        const float m = (float)raw_h[c][i] * fh;
                        if (own) dw_post[c][i] = fmaf(f[c][i], m, dw_post[c][i]);
                        f[c][i] *= w_post[c][i];
                        fm = i < at.n[c] ? fmaf(f[c][i], m, fm) : fm;
                    }
                }
            float mean_fm = 0.0f;
            if (p.w_post) mean_fm = row_sum<WAVES>(fm, at.lanes, red) * per_k;
            if (!own) continue;
#pragma unroll
            for (int c = 0; c < CHUNKS; c++) {
                if (at.n[c] == 0) continue;
                float dh[V], dres[V], dg[V];
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float m = (float)raw_h[c][i] * fh;
                    dh[i] = p.w_post ? fh * (f[c][i] - m * mean_fm) : f[c][i];
                    dres[i] = p.scale * e[c][i];
                    dg[i] = e[c][i] * (p.w_post ? m * w_post[c][i] : m);
                    dgate[c][i] += dg[i];
                }
                store_first<V>(p.dh + row * p.lddh + at.k[c], at.n[c], dh);
                if (p.dresidual) store_first<V>(p.dresidual + row * p.lddres + at.k[c], at.n[c], dres);
                if (row_gates) store_first<V>(p.gate_partial + row * p.K + at.k[c], at.n[c], dg);
            }
        }
        if (p.gate && !row_gates) sum_slots<V, CHUNKS, WAVES, FULL>(dgate, at, p.gate_partial + part * p.K, cols);
    }
    sum_slots<V, CHUNKS, WAVES, FULL>(dw, at, p.partial + (int64_t)blockIdx.x * 2 * p.K, cols);
    if (p.w_post) sum_slots<V, CHUNKS, WAVES, FULL>(dw_post, at, p.partial + (int64_t)blockIdx.x * 2 * p.K + p.K, cols);
}

// Sums over the parts of each gate's rows (the first gate_blocks workgroups) and over the workgroups' partial sums of dw and dw_post
__global__ __launch_bounds__(kSumThreads) void sum_norm_partials(const float *__restrict__ gate_partial, float *__restrict__ dgate, int64_t gates, int K, uint32_t parts,
                                                                uint32_t gate_blocks, const float *__restrict__ partial, int64_t rows, int64_t stride, int64_t cols,
                                                                SumOut out) {
    if (blockIdx.x >= gate_blocks) return sum_columns(partial, rows, stride, cols, out, blockIdx.x - gate_blocks);
    for (int64_t i = (int64_t)blockIdx.x * kSumThreads + threadIdx.x; i < gates; i += (int64_t)gate_blocks * kSumThreads) {
        const int64_t g = i / K;
        const float *from = gate_partial + g * parts * K + (i - g * K);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        uint32_t s = 0;
        for (; s + 4 <= parts; s += 4)
#pragma unroll
            for (int j = 0; j < 4; j++) sum[j] += from[(int64_t)(s + j) * K];
        for (; s < parts; s++) sum[0] += from[(int64_t)s * K];
        dgate[i] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
}

// How a row is held: chunks loads of vec elements by 2^n lanes, or by 4, 8 or 16 wavefronts
struct Shape {
    int vec, chunks, waves, lanes_log2;
};
Shape shape_of(int64_t K) {
    Shape best{8, 0, 0, 6};
    for (const int vec : {8, 6}) {
        const int64_t loads = ceil_div(K, vec);
        if (loads > 128) continue;
        int lanes_log2 = 0;
        while (lanes_log2 < 6 && ((int64_t)1 << lanes_log2) < loads) lanes_log2++;
        const int chunks = (int)ceil_div(loads, 1 << lanes_log2);
        if (!best.waves || (chunks * vec) << lanes_log2 < (best.chunks * best.vec) << best.lanes_log2) best = {vec, chunks, 1, lanes_log2};
    }
    if (best.waves) return best;
    const int waves = K <= 4 * 64 * 8 * 2 ? 4 : K <= 8 * 64 * 8 * 2 ? 8 : 16;
    return {8, (int)ceil_div(ceil_div(K, 8), waves * 64), waves, 6};
}

// f(vec, chunks, waves, whether all lanes are full: a row of one wavefront has a variant without bounds for it)
template <typename F>
int for_shape(const Shape &s, int64_t K, F &&f) {
    using std::bool_constant;
    using std::integral_constant;
    constexpr integral_constant<int, 8> eight{};
    constexpr integral_constant<int, 1> one{};
    constexpr integral_constant<int, 2> two{};
    constexpr bool_constant<false> bounds{};
    constexpr bool_constant<true> full{};
    if (s.waves == 16) return f(eight, two, integral_constant<int, 16>{}, bounds);  // (more than 8 wavefronts' two loads)
    if (s.waves == 8) return f(eight, two, integral_constant<int, 8>{}, bounds);
    if (s.waves == 4) return s.chunks == 1 ? f(eight, one, integral_constant<int, 4>{}, bounds) : f(eight, two, integral_constant<int, 4>{}, bounds);
    const auto with = [&](auto vec, auto chunks) { return (s.vec * s.chunks) << s.lanes_log2 == K ? f(vec, chunks, one, full) : f(vec, chunks, one, bounds); };
    if (s.vec == 8) return s.chunks == 1 ? with(eight, one) : with(eight, two);
    return s.chunks == 1 ? with(integral_constant<int, 6>{}, one) : with(integral_constant<int, 6>{}, two);
}

template <typename F>
int for_types(int dtype, int stream_dtype, F &&f) {
    return for_dtype(dtype, [&](auto t) {
        if (stream_dtype == dtype) return f(t, t);
        return f(t, float{});
    });
}

int check_norm(int dtype, int stream_dtype, const void *h, const float *w, const float *gate, const float *w_post, int64_t M, int64_t K, int64_t G) {
    if (!valid_dtype(dtype) || (stream_dtype != dtype && stream_dtype != PTQ4VM_F32)) return PTQ4VM_ERR_SHAPE;
    if (!w || (M != 0 && !h)) return PTQ4VM_ERR_NULL;  // (a matrix of no rows has no address)
    if (M < 0 || M > kMaxTokenRows || K <= 0 || K > PTQ4VM_MAX_NORM_K) return PTQ4VM_ERR_SHAPE;
    if (gate && (G <= 0 || M % G != 0)) return PTQ4VM_ERR_SHAPE;
    if (!aligned_to(h, dtype_bytes(dtype)) || !aligned_to(w, 4) || !aligned_to(gate, 4) || !aligned_to(w_post, 4)) return PTQ4VM_ERR_ALIGN;
    return PTQ4VM_OK;
}

// How the rows of a backward pass are cut
struct Cut {
    Shape shape;
    uint32_t gate_rows, parts, part_rows;
    int64_t all_parts, blocks;
};
Cut cut_rows(int64_t M, int64_t K, int64_t G) {
    Cut c{shape_of(K), 0, 0, 0, 0, 0};
    c.gate_rows = (uint32_t)(G > 0 ? M / G : M);
    const bool row_gates = G > 0 && c.gate_rows == 1;
    const int64_t groups = G > 0 && !row_gates ? G : 1, together = groups == 1 ? M : c.gate_rows;
    const int64_t slots = c.shape.waves == 1 ? 256 >> c.shape.lanes_log2 : 1;
    // about 1024 workgroups, of 4 rows to a slot at least: a workgroup's partial sums cost a row or two of traffic
    int64_t parts = ceil_div(1024, groups);
    const int64_t most = ceil_div(together, 4 * slots);
    if (parts > most) parts = most;
    c.part_rows = (uint32_t)ceil_div(together, parts);
    c.parts = (uint32_t)ceil_div(together, c.part_rows);
    c.all_parts = groups * c.parts;
    c.blocks = c.all_parts < 1024 ? c.all_parts : 1024;
    return c;
}
// Whether the parts' sums go through the workspace (else a part is a gate's rows, and its sum the gradient)
bool gate_in_parts(const Cut &c, int64_t G) { return G > 0 && c.gate_rows > 1 && c.parts > 1; }

}  // namespace

extern "C" {

int ptq4vm_residual_norm(int dtype, int stream_dtype, const void *h, const void *residual, const float *w, const float *gate, const float *w_post, void *y, void *r,
                         float scale, float eps, int64_t M, int64_t K, int64_t G, int64_t ldh, int64_t ldres, int64_t ldy, int64_t ldr, void *stream) {
    const int rc = check_norm(dtype, stream_dtype, h, w, gate, w_post, M, K, G);
    if (rc != PTQ4VM_OK) return rc;
    if (M != 0 && (!y || !r)) return PTQ4VM_ERR_NULL;
    if (ldh < K || (residual && ldres < K) || ldy < K || ldr < K) return PTQ4VM_ERR_STRIDE;
    const uintptr_t er = dtype_bytes(stream_dtype);
    if (!aligned_to(residual, er) || !aligned_to(r, er) || !aligned_to(y, dtype_bytes(dtype))) return PTQ4VM_ERR_ALIGN;
    if (M == 0) return PTQ4VM_OK;
    return for_types(dtype, stream_dtype, [&](auto t, auto s) {
        using T = decltype(t);
        using R = decltype(s);
        const Shape shape = shape_of(K);
        NormArgs<T, R> a{};
        a.h = static_cast<const T *>(h), a.residual = static_cast<const R *>(residual), a.w = w, a.gate = gate, a.w_post = w_post;
        a.y = static_cast<T *>(y), a.r = static_cast<R *>(r), a.scale = scale, a.eps = eps, a.K = (int)K, a.M = (uint32_t)M;
        a.gate_rows = gate ? (uint32_t)(M / G) : 1, a.lanes_log2 = shape.lanes_log2;
        a.ldh = ldh, a.ldres = ldres, a.ldy = ldy, a.ldr = ldr;
        int64_t blocks = ceil_div(M, shape.waves == 1 ? 256 >> shape.lanes_log2 : 1);
        if (blocks > 8192) blocks = 8192;  // (50432 x 768: 85 us, 1024 or 2048 workgroups 91 and 90)
        return for_shape(shape, K, [&](auto vec, auto chunks, auto waves, auto full) {
            residual_norm_rows<T, R, vec(), chunks(), waves(), full()><<<dim3((unsigned)blocks), dim3(waves() > 4 ? waves() * 64 : 256), 0, static_cast<hipStream_t>(stream)>>>(a);
            return check_launch("residual_norm_rows");
        });
    });
}

int64_t ptq4vm_residual_norm_backward_workspace(int64_t M, int64_t K, int64_t G) {
    if (M <= 0 || M > kMaxTokenRows || K <= 0 || K > PTQ4VM_MAX_NORM_K || G < 0 || (G > 0 && M % G != 0)) return 0;
    const Cut c = cut_rows(M, K, G);
    return 4 * K * (2 * c.blocks + (gate_in_parts(c, G) ? c.all_parts : 0));
}

int ptq4vm_residual_norm_backward(int dtype, int stream_dtype, const void *dy, const void *dr, const void *h, const void *r, const float *w, const float *gate,
                                  const float *w_post, void *dh, void *dresidual, float *dw, float *dgate, float *dw_post, void *workspace, int64_t workspace_bytes,
                                  float scale, float eps, int64_t M, int64_t K, int64_t G, int64_t lddy, int64_t lddr, int64_t ldh, int64_t ldr, int64_t lddh,
                                  int64_t lddres, void *stream_) {
    int rc = check_norm(dtype, stream_dtype, h, w, gate, w_post, M, K, G);
    if (rc != PTQ4VM_OK) return rc;
    if (!dw || (gate && !dgate) || (w_post && !dw_post) || (M != 0 && (!dy || !r || !dh || !workspace))) return PTQ4VM_ERR_NULL;
    if (lddy < K || (dr && lddr < K) || ldh < K || ldr < K || lddh < K || (dresidual && lddres < K)) return PTQ4VM_ERR_STRIDE;
    const int64_t gates = gate ? G : 0;
    if (workspace_bytes < ptq4vm_residual_norm_backward_workspace(M, K, gates)) return PTQ4VM_ERR_SHAPE;
    const uintptr_t e = dtype_bytes(dtype), er = dtype_bytes(stream_dtype);
    if (!aligned_to(dy, e) || !aligned_to(dh, e) || !aligned_to(dr, er) || !aligned_to(r, er) || !aligned_to(dresidual, er) || !aligned_to(dw, 4) ||
        !aligned_to(dgate, 4) || !aligned_to(dw_post, 4) || !aligned_to(workspace, 16))
        return PTQ4VM_ERR_ALIGN;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    Cut c{};
    float *const partial = static_cast<float *>(workspace);
    float *gate_partial = nullptr;
    if (M > 0) {
        c = cut_rows(M, K, gates);
        gate_partial = gate_in_parts(c, gates) ? partial + 2 * K * c.blocks : dgate;
        rc = for_types(dtype, stream_dtype, [&](auto t, auto s) {
            using T = decltype(t);
            using R = decltype(s);
            NormArgs<T, R> a{};
            a.h = static_cast<const T *>(h), a.w = w, a.gate = gate, a.w_post = w_post, a.r = static_cast<R *>(const_cast<void *>(r));
            a.dy = static_cast<const T *>(dy), a.dr = static_cast<const R *>(dr), a.dh = static_cast<T *>(dh), a.dresidual = static_cast<R *>(dresidual);
            a.partial = partial, a.gate_partial = gate_partial, a.scale = scale, a.eps = eps, a.K = (int)K, a.M = (uint32_t)M;
            a.gate_rows = c.gate_rows, a.parts = c.parts, a.part_rows = c.part_rows, a.lanes_log2 = c.shape.lanes_log2;
            a.ldh = ldh, a.ldr = ldr, a.lddy = lddy, a.lddr = lddr, a.lddh = lddh, a.lddres = lddres;
            return for_shape(c.shape, K, [&](auto vec, auto chunks, auto waves, auto full) {
                residual_norm_backward_rows<T, R, vec(), chunks(), waves(), full()><<<dim3((unsigned)c.blocks), dim3(waves() > 4 ? waves() * 64 : 256), 0, stream>>>(a, c.all_parts);
                return check_launch("residual_norm_backward_rows");
            });
        });
        if (rc != PTQ4VM_OK) return rc;
    }
    const bool parts = gate && (M == 0 || gate_in_parts(c, gates));
    const int64_t gate_blocks = !parts ? 0 : G * K < (int64_t)1 << 30 ? ceil_div(G * K, kSumThreads) : 1 << 20, cols = w_post ? 2 * K : K;
    sum_norm_partials<<<dim3((unsigned)(gate_blocks + ceil_div(cols, kSumCols))), dim3(kSumThreads), 0, stream>>>(
        gate_partial, dgate, G * K, (int)K, c.parts, (uint32_t)gate_blocks, partial, c.blocks, 2 * K, cols, {dw, dw_post, nullptr, K, K});
    return check_launch("sum_norm_partials");
}

}  // extern "C"
