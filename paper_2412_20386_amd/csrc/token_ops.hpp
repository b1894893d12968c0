// Shared by the operators between a block's linears (gated_scan, token_conv, residual_norm): element types, vectors of
// elements at any alignment, the activations, and the sum over the partial results of workgroups.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.hpp"

namespace ptq4vm {

constexpr int64_t kMaxTokenRows = 0x7fffffff;  // rows and widths are 32-bit in the kernels, offsets 64-bit
// Whether a grid of one dimension can be launched: it holds fewer than 2^32 threads
inline bool grid_fits(int64_t blocks, int threads) { return blocks * threads < ((int64_t)1 << 32); }

inline bool valid_dtype(int dtype) { return dtype == PTQ4VM_F16 || dtype == PTQ4VM_BF16 || dtype == PTQ4VM_F32; }
inline uintptr_t dtype_bytes(int dtype) { return dtype == PTQ4VM_F32 ? 4 : 2; }

// f(zero of the element type) for a dtype that valid_dtype() took
template <typename F>
int for_dtype(int dtype, F &&f) {
    if (dtype == PTQ4VM_F16) return f(_Float16{});
    if (dtype == PTQ4VM_BF16) return f(__bf16{});
    return f(float{});
}

// Tokens of a sequence in the order of time: row b * L + t, or b * L + (L - 1 - t) where time runs backwards.
template <typename T>
struct Tokens {
    T *data;         // token 0 of sequence 0
    int64_t token;   // elements to the next token
    int64_t sequence;
    __host__ __device__ __forceinline__ T *at(int b, int64_t t) const { return data + b * sequence + t * token; }
};
template <typename T>
inline Tokens<T> tokens(const void *p, int64_t L, int64_t ld, bool reverse) {
    T *data = static_cast<T *>(const_cast<void *>(p));
    if (!p) return {nullptr, 0, 0};
    return {reverse ? data + (L - 1) * ld : data, reverse ? -ld : ld, L * ld};
}

// Whether two matrices of rows x `width` elements of `size` bytes, which both are aligned to, share one.  With the same pitch (halves of one
// matrix, say) this is exact: the second begins q pitches and r elements behind the first, and its rows meet those q further, and if r + width >
// pitch those q + 1 further.  With different pitches it is whether their ranges meet.
inline bool overlap(const void *a, int64_t pitch_a, const void *b, int64_t pitch_b, int64_t rows, int64_t width, int64_t size) {
    const int64_t apart = ((int64_t)reinterpret_cast<uintptr_t>(b) - (int64_t)reinterpret_cast<uintptr_t>(a)) / size;
    if (pitch_a != pitch_b) return apart < (__int128)(rows - 1) * pitch_a + width && -apart < (__int128)(rows - 1) * pitch_b + width;
    const int64_t q = apart / pitch_a - (apart % pitch_a < 0), r = apart - q * pitch_a;
    return (r < width && q > -rows && q < rows) || (width > pitch_a - r && q + 1 > -rows && q + 1 < rows);
}
inline bool overlap(const void *a, const void *b, int64_t bytes) { return a && b && overlap(a, bytes, b, bytes, 1, bytes, 1); }

// Workgroups go to the 8 XCDs in turn, and each XCD has an L2 of its own: work that shares lines or operands gets
// consecutive numbers, and an XCD a consecutive range of them.  Some numbers are beyond `total`: the caller leaves.
__device__ __forceinline__ uint32_t xcd_contiguous(uint32_t block, uint32_t total) {
    return (block & 7) * ((total + 7) >> 3) + (block >> 3);
}
inline uint32_t xcd_grid(int64_t total) { return (uint32_t)((total + 7) & ~(int64_t)7); }

// V elements from p, aligned to an element only (gfx950 loads and stores 16 bytes at any alignment of 2 or 4)
template <int V, typename T>
__device__ __forceinline__ void load_whole(const T *p, T (&v)[V]) {
    __builtin_memcpy(v, p, sizeof(v));
}
// The first n of V elements, zero behind them: nothing beyond a row's width is read
template <int V, typename T>
__device__ __forceinline__ void load_first(const T *p, int n, T (&v)[V]) {
    if (n >= V) return load_whole<V>(p, v);
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = i < n ? p[i] : (T)0.0f;
}
template <int V, typename T>
__device__ __forceinline__ void store_first(T *p, int n, const float (&v)[V]) {
    T out[V];
#pragma unroll
    for (int i = 0; i < V; i++) out[i] = (T)v[i];  // to nearest even, once
    if (n >= V) {
        __builtin_memcpy(p, out, sizeof(out));
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++)
        if (i < n) p[i] = out[i];
}

// e^v with the hardware's 2^v (1 ulp); the product's rounding is relative to v: |v| <= 16 costs 2^-20 of the result
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896340736f); }
// 1 / (1 + e^-v): 0 and 1 at the infinities, NaN for a NaN
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-v)); }

// ln(1 + e^v) = max(v, 0) + ln(1 + e), e = e^-|v| in [0, 1].  The sum w = 1 + e loses up to 2^-24 of e; what it lost, e - (w - 1),
// is exact, and added to ln w to first order (its factor 1 / w matters only where ln w is large): small results (a step size
// of 0.001 is an input of -7) keep all their digits, where ln w alone would keep 14 bits.
__device__ __forceinline__ float softplus_of(float v) {
    const float e = exp_of(-fabsf(v)), w = 1.0f + e;
    return fmaxf(v, 0.0f) + fmaf(__builtin_amdgcn_logf(w), 0.69314718055994530942f, e - (w - 1.0f));
}

// v + v of another lane of the row of 16, a VALU instruction
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum over the 4 lanes of a quad, in every lane of it
__device__ __forceinline__ float quad_sum(float v) { return add_dpp<0x4E>(add_dpp<0xB1>(v)); }
// Sums over the lanes of a quad of C values each: in lane q that of value q modulo C
template <int C>
__device__ __forceinline__ float quad_sums(const float (&v)[C], int q) {
    static_assert(C == 1 || C == 2, "one value or two");
    if constexpr (C == 1) return quad_sum(v[0]);
    const float mine = q & 1 ? v[C - 1] : v[0], other = q & 1 ? v[0] : v[C - 1];
    return add_dpp<0x4E>(mine + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, other), 0xB1, 0xf, 0xf, true)));
}
// Two values of each lane summed over pairs of lanes, one to a lane: lanes 0-31 get a's sums over lanes l and l + 32, lanes 32-63
// b's; or rows of 16 lanes, the even rows a's over rows r and r + 1, the odd rows b's.  A swap and an addition for two sums.
__device__ __forceinline__ float sum_halves(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_rows(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
// Sum over the four lanes of a row of 16 that have the same place in their quads
__device__ __forceinline__ float sum_quads(float v) { return add_dpp<0x128>(add_dpp<0x124>(v)); }  // row_ror 4, 8
// Sum over an aligned group of `lanes` = 2^n lanes, in every lane of it
__device__ __forceinline__ float group_sum(float v, int lanes) {
    if (lanes >= 2) v = add_dpp<0xB1>(v);    // quad_perm 1,0,3,2
    if (lanes >= 4) v = add_dpp<0x4E>(v);    // quad_perm 2,3,0,1
    if (lanes >= 8) v = add_dpp<0x141>(v);   // row_half_mirror: quads of 8 lanes
    if (lanes >= 16) v = add_dpp<0x140>(v);  // row_mirror: halves of 16 lanes
    if (lanes >= 32) v = sum_rows(v, v);
    if (lanes >= 64) v = sum_halves(v, v);
    return v;
}

// Column sums of partial[rows][cols] in a fixed order: the gradients of parameters, which every workgroup adds to.  The
// first `first` columns go to `out0`, the next `second` to out1, the rest to out2.  No rows: zeros.
struct SumOut {
    float *out0, *out1, *out2;
    int64_t first, second;
};
constexpr int kSumThreads = 1024, kSumCols = 32;  // (32 rows at a time: sums of 1024 rows take 32 round trips to memory)
namespace {
__device__ __forceinline__ void sum_columns(const float *__restrict__ partial, int64_t rows, int64_t stride, int64_t cols, const SumOut &out, uint32_t block) {
    constexpr int kSlots = kSumThreads / kSumCols;
    __shared__ float red[kSlots][kSumCols];
    const int slot = threadIdx.x / kSumCols, c = threadIdx.x % kSumCols;
    const int64_t col = (int64_t)block * kSumCols + c;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < cols) {
        int64_t r = slot;
        for (; r + 3 * kSlots < rows; r += 4 * kSlots)
#pragma unroll
            for (int i = 0; i < 4; i++) sum[i] += partial[(r + i * kSlots) * stride + col];
        for (; r < rows; r += kSlots) sum[0] += partial[r * stride + col];
    }
    red[slot][c] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    __syncthreads();
    if (slot == 0 && col < cols) {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < kSlots; i++) v += red[i][c];
        float *const to = col < out.first ? out.out0 : col < out.first + out.second ? out.out1 : out.out2;
        const int64_t at = col < out.first ? col : col < out.first + out.second ? col - out.first : col - out.first - out.second;
        if (to) to[at] = v;
    }
}
__global__ __launch_bounds__(kSumThreads) void sum_partials(const float *__restrict__ partial, int64_t rows, int64_t cols, SumOut out) {
    for (uint32_t block = blockIdx.x; (int64_t)block * kSumCols < cols; block += gridDim.x) {
        sum_columns(partial, rows, cols, cols, out, block);
        __syncthreads();  // (the next columns go through the same LDS)
    }
}
constexpr int64_t kSumBlocks = (int64_t)1 << 21;  // 2^31 threads: a grid holds fewer than 2^32
inline int launch_sum_partials(const float *partial, int64_t rows, int64_t cols, const SumOut &out, hipStream_t stream) {
    const int64_t blocks = ceil_div(cols, kSumCols);
    sum_partials<<<dim3((unsigned)(blocks < kSumBlocks ? blocks : kSumBlocks)), dim3(kSumThreads), 0, stream>>>(partial, rows, cols, out);
    return check_launch("sum_partials");
}
}  // namespace

}  // namespace ptq4vm
