// Short convolution over the tokens of a sequence, one filter per channel (between in_proj and x_proj of a block):
//   p[t,k] = bias[k] + sum_j w[k,j] x[t - W + 1 + j, k],  y = p / (1 + e^-p) or p,  x before token 0 from the state or 0.
// Backward, with dp = dy * (derivative of the activation at p, computed again):
//   dx[t,k] = sum_j w[k,j] dp[t + W - 1 - j, k],  dw[k,j] = sum_t dp[t,k] x[t - W + 1 + j, k],  dbias[k] = sum_t dp[t,k].
//
// Bound by memory (2 - 12 flops a byte).  A lane owns 8 adjacent channels (16 bytes of 16-bit elements) and walks over a run of tokens with
// the window of W - 1 earlier ones in registers, so that a token is read once by its run; the next run reads the last W - 1
// again (from the L2: neighbouring runs are neighbours in a workgroup).  Sums are fp32.  Forward, 128 x 197 x 768 in fp16: 21 us,
// 3.7 TB/s (one round of wavefronts, whose first loads nothing hides); backward, 64 x 197 x 1536 in bf16: 37 us, 3.2 TB/s, 4.8 of
// them the sums of the filters' gradients.
#include <type_traits>

#include "token_ops.hpp"

namespace {

using namespace ptq4vm;

constexpr int kThreads = 256, kUnroll = 4;
constexpr int kVec = 8, kVecBackward = 4;  // channels of a lane: the backward pass holds three windows and the filters' gradients

template <typename T>
struct ConvArgs {
    Tokens<T> x, y, dy;  // (y: dx in the backward pass)
    const float *w, *bias;
    const T *state;  // may be the buffer of state_out for one token
    T *state_out;
    float *partial;
    int K, B, silu;
    int64_t L;
    int run;          // tokens of a run
    int64_t runs;     // runs of a sequence
    int lanes_log2;   // lanes side by side in a row; the other lanes of the workgroup take other runs
    int column_blocks;
};

// Where a lane works: its channels, and its first run
struct Place {
    int k, n, slot, slots;
};
template <int V>
__device__ __forceinline__ Place place(int lanes_log2, int column_block, int K) {
    const int lanes = 1 << lanes_log2;
    const int k = (column_block * lanes + (threadIdx.x & (lanes - 1))) * V;
    return {k, max(0, min(V, K - k)), (int)threadIdx.x >> lanes_log2, kThreads >> lanes_log2};
}

// WHOLE: every lane that has a channel has all V
template <int V, bool WHOLE, typename T>
__device__ __forceinline__ void load_channels(const T *p, const Place &at, T (&v)[V]) {
    if constexpr (WHOLE)
        load_whole<V>(p + at.k, v);
    else
        load_first<V>(p + at.k, at.n, v);
}
template <int V, bool WHOLE, typename T>
__device__ __forceinline__ void store_channels(T *p, const Place &at, const float (&v)[V]) {
    store_first<V>(p + at.k, WHOLE ? V : at.n, v);
}

template <typename T, int W, int V, bool WHOLE>
__device__ __forceinline__ void filters(const ConvArgs<T> &p, const Place &at, float (&w)[V][W], float (&bias)[V]) {
    float flat[V * W];
    if constexpr (WHOLE)
        load_whole<V * W>(p.w + (int64_t)at.k * W, flat);
    else
        load_first<V * W>(p.w + (int64_t)at.k * W, at.n * W, flat);
#pragma unroll
    for (int i = 0; i < V * W; i++) w[i / W][i % W] = flat[i];
#pragma unroll
    for (int i = 0; i < V; i++) bias[i] = 0.0f;
    if (p.bias) load_channels<V, WHOLE>(p.bias, at, bias);
}

// x of the W - 1 tokens before token t
template <typename T, int W, int V, bool WHOLE>
__device__ __forceinline__ void window_before(const ConvArgs<T> &p, const Place &at, int b, int64_t t, float (&win)[W - 1][V]) {
#pragma unroll
    for (int j = 0; j < W - 1; j++) {
        const int64_t s = t - (W - 1) + j;
        T raw[V];
        if (s >= 0)
            load_channels<V, WHOLE>(p.x.at(b, s), at, raw);
        else if (p.state)
            load_channels<V, WHOLE>(p.state + ((int64_t)b * (W - 1) + s + (W - 1)) * p.K, at, raw);
        else
#pragma unroll
            for (int i = 0; i < V; i++) raw[i] = (T)0.0f;
#pragma unroll
        for (int i = 0; i < V; i++) win[j][i] = (float)raw[i];
    }
}

template <int W, int V>
__device__ __forceinline__ void shift_in(float (&win)[W - 1][V], const float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int j = 0; j + 1 < W - 1; j++) win[j][i] = win[j + 1][i];
        win[W - 2][i] = x[i];
    }
}

template <int W, int V>
__device__ __forceinline__ float convolve(const float (&w)[V][W], const float (&bias)[V], const float (&win)[W - 1][V], const float (&x)[V], int i) {
    float v = fmaf(w[i][W - 1], x[i], bias[i]);
#pragma unroll
    for (int j = 0; j < W - 1; j++) v = fmaf(w[i][j], win[j][i], v);
    return v;
}

template <typename T, int W, bool WHOLE>
__global__ __launch_bounds__(kThreads) void token_conv_runs(ConvArgs<T> p) {
    constexpr int V = kVec;
    const int column_block = blockIdx.x % p.column_blocks;
    const Place at = place<V>(p.lanes_log2, column_block, p.K);
    const int64_t item = (int64_t)(blockIdx.x / p.column_blocks) * at.slots + at.slot;
    if (item >= p.runs * p.B || at.n == 0) return;
    const int b = (int)(item / p.runs);
    const int64_t t0 = (item - b * p.runs) * p.run, t1 = min(p.L, t0 + p.run);
    T next[kUnroll][V];
    // (behind the run's last token the lane loads that one again)
    const auto fetch = [&](int64_t t) {
#pragma unroll
        for (int s = 0; s < kUnroll; s++) load_channels<V, WHOLE>(p.x.at(b, min(t + s, t1 - 1)), at, next[s]);
    };
    fetch(t0);
    float win[W - 1][V], w[V][W], bias[V];
    window_before<T, W, V, WHOLE>(p, at, b, t0, win);
    filters<T, W, V, WHOLE>(p, at, w, bias);
    for (int64_t t = t0; t < t1; t += kUnroll) {
        T raw[kUnroll][V];
#pragma unroll
        for (int s = 0; s < kUnroll; s++)
#pragma unroll
            for (int i = 0; i < V; i++) raw[s][i] = next[s][i];
        if (t + kUnroll < t1) fetch(t + kUnroll);
#pragma unroll
        for (int s = 0; s < kUnroll; s++) {
            if (t + s >= t1) break;
            float x[V], y[V];
#pragma unroll
            for (int i = 0; i < V; i++) x[i] = (float)raw[s][i];
#pragma unroll
            for (int i = 0; i < V; i++) y[i] = convolve<W, V>(w, bias, win, x, i);
            if (p.silu)
#pragma unroll
                for (int i = 0; i < V; i++) y[i] *= sigmoid_of(y[i]);
            store_channels<V, WHOLE>(p.y.at(b, t + s), at, y);
            shift_in<W, V>(win, x);
        }
    }
    if (p.state_out && t1 == p.L)  // the window as it is now: the last W - 1 tokens, older ones from the state
#pragma unroll
        for (int j = 0; j < W - 1; j++) store_channels<V, WHOLE>(p.state_out + ((int64_t)b * (W - 1) + j) * p.K, at, win[j]);
}

// A workgroup takes every gridDim-th group of runs and adds the filters' gradients up in registers; partial[workgroup row]
// is [K * W | K].
template <typename T, int W, bool WHOLE>
__global__ __launch_bounds__(kThreads) void token_conv_backward_runs(ConvArgs<T> p, int groups) {
    constexpr int V = kVecBackward;
    const int column_block = blockIdx.x % p.column_blocks, group = blockIdx.x / p.column_blocks;
    const Place at = place<V>(p.lanes_log2, column_block, p.K);
    float w[V][W] = {}, bias[V] = {}, dw[W + 1][V] = {};
    if (at.n > 0) filters<T, W, V, WHOLE>(p, at, w, bias);
    for (int64_t item = (int64_t)group * at.slots + at.slot; item < p.runs * p.B && at.n > 0; item += (int64_t)groups * at.slots) {
        const int b = (int)(item / p.runs);
        const int64_t t0 = (item - b * p.runs) * p.run, t1 = min(p.L, t0 + p.run);
        // dp of the run, and of the W - 1 tokens behind it, which the run's last tokens take part in
        const int64_t t_read = min(p.L, t1 + W - 1);
        T next_x[kUnroll][V], next_dy[kUnroll][V];
        const auto fetch = [&](int64_t t) {
#pragma unroll
            for (int s = 0; s < kUnroll; s++) {
                load_channels<V, WHOLE>(p.x.at(b, min(t + s, t_read - 1)), at, next_x[s]);
                load_channels<V, WHOLE>(p.dy.at(b, min(t + s, t_read - 1)), at, next_dy[s]);
            }
        };
        fetch(t0);
        float win[W - 1][V], late[W - 1][V] = {};  // the last tokens' x and dp
        window_before<T, W, V, WHOLE>(p, at, b, t0, win);
        for (int64_t t = t0; t < t1 + W - 1; t += kUnroll) {
            T rx[kUnroll][V], rdy[kUnroll][V];
#pragma unroll
            for (int s = 0; s < kUnroll; s++)
#pragma unroll
                for (int i = 0; i < V; i++) rx[s][i] = next_x[s][i], rdy[s][i] = next_dy[s][i];
            if (t + kUnroll < t_read) fetch(t + kUnroll);
#pragma unroll
            for (int s = 0; s < kUnroll; s++) {
                if (t + s >= t1 + W - 1) break;
                float x[V], dp[V], dx[V];
#pragma unroll
                for (int i = 0; i < V; i++) x[i] = (float)rx[s][i], dp[i] = (float)rdy[s][i];
                if (p.silu)
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float v = convolve<W, V>(w, bias, win, x, i), g = sigmoid_of(v);
                        dp[i] *= g * fmaf(v, 1.0f - g, 1.0f);
                    }
                if (t + s >= p.L)
#pragma unroll
                    for (int i = 0; i < V; i++) dp[i] = 0.0f;
#pragma unroll
                for (int i = 0; i < V; i++) {
                    float v = w[i][0] * dp[i];
#pragma unroll
                    for (int j = 1; j < W; j++) v = fmaf(w[i][j], late[W - 1 - j][i], v);
                    dx[i] = v;
                }
                if (t + s - (W - 1) >= t0) store_channels<V, WHOLE>(p.y.at(b, t + s - (W - 1)), at, dx);
                if (t + s < t1)
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        dw[W - 1][i] = fmaf(dp[i], x[i], dw[W - 1][i]);
#pragma unroll
                        for (int j = 0; j < W - 1; j++) dw[j][i] = fmaf(dp[i], win[j][i], dw[j][i]);
                        dw[W][i] += dp[i];
                    }
                shift_in<W, V>(win, x);
                shift_in<W, V>(late, dp);
            }
        }
    }
    __shared__ float red[kThreads][V + 1];
    float *const row = p.partial + (int64_t)group * p.K * (W + 1);
    const int lanes = 1 << p.lanes_log2;
#pragma unroll
    for (int j = 0; j <= W; j++) {
#pragma unroll
        for (int i = 0; i < V; i++) red[threadIdx.x][i] = dw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < lanes * V; c += kThreads) {
            float sum = 0.0f;
            for (int s = 0; s < at.slots; s++) sum += red[s * lanes + c / V][c % V];
            const int64_t k = (int64_t)column_block * lanes * V + c;
            if (k < p.K) row[j < W ? k * W + j : (int64_t)p.K * W + k] = sum;
        }
        __syncthreads();
    }
}

// Lanes side by side over K, and the workgroups that K takes: 64 lanes, fewer where that leaves fewer of them idle (768 channels
// of 8 to a lane are 3 x 32)
template <typename T>
void columns(ConvArgs<T> &a, int64_t K, int vec) {
    const int64_t chunks = ceil_div(K, vec);
    a.lanes_log2 = 6;
    for (int lanes_log2 = 5; lanes_log2 >= 0; lanes_log2--)
        if (ceil_div(chunks, 1 << lanes_log2) << lanes_log2 < ceil_div(chunks, 1 << a.lanes_log2) << a.lanes_log2 && (lanes_log2 >= 3 || chunks <= 4)) a.lanes_log2 = lanes_log2;
    a.column_blocks = (int)ceil_div(chunks, 1 << a.lanes_log2);
}

int check_conv(int dtype, const void *x, const float *w, const float *bias, const void *state, int64_t B, int64_t L, int64_t K, int64_t W) {
    if (!valid_dtype(dtype)) return PTQ4VM_ERR_SHAPE;
    if (!w || (B != 0 && !x)) return PTQ4VM_ERR_NULL;  // (a matrix of no rows has no address)
    if (B < 0 || L <= 0 || K <= 0 || W < 2 || W > 4) return PTQ4VM_ERR_SHAPE;
    if (L > kMaxTokenRows || K > kMaxTokenRows / 16 || (B > 0 && B > kMaxTokenRows / L)) return PTQ4VM_ERR_SHAPE;
    const uintptr_t e = dtype_bytes(dtype);
    if (!aligned_to(x, e) || !aligned_to(state, e) || !aligned_to(w, 4) || !aligned_to(bias, 4)) return PTQ4VM_ERR_ALIGN;
    return PTQ4VM_OK;
}

// Whether the lanes of one run would write what those of another read: an output's elements among an input's.  A sequence of one token is
// read by the lanes that write it, so there the two may be the same.
bool run_overlap(int dtype, const void *out, int64_t ld_out, const void *in, int64_t ld_in, int64_t B, int64_t L, int64_t K) {
    if (L == 1 && out == in && (B == 1 || ld_out == ld_in)) return false;
    return overlap(out, ld_out, in, ld_in, B * L, K, (int64_t)dtype_bytes(dtype));
}

// f(W, WHOLE)
template <typename F>
int for_filter(int64_t W, bool whole, F &&f) {
    using std::bool_constant;
    using std::integral_constant;
    const auto with = [&](auto taps) { return whole ? f(taps, bool_constant<true>{}) : f(taps, bool_constant<false>{}); };
    return W == 2 ? with(integral_constant<int, 2>{}) : W == 3 ? with(integral_constant<int, 3>{}) : with(integral_constant<int, 4>{});
}

int conv(int dtype, const void *x, const float *w, const float *bias, const void *state, void *y, void *state_out, int silu, int reverse, int64_t B, int64_t L,
         int64_t K, int64_t W, int64_t ldx, int64_t ldy, void *stream) {
    if (B == 0) return PTQ4VM_OK;
    return for_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        ConvArgs<T> a{tokens<T>(x, L, ldx, reverse), tokens<T>(y, L, ldy, reverse), {}, w, bias, static_cast<const T *>(state), static_cast<T *>(state_out), nullptr,
                      (int)K, (int)B, silu, L, 0, 0, 0, 0};
        columns(a, K, kVec);
        // A run of 16 tokens reads 3 of its neighbour's again; shorter ones where there would be fewer than 8 wavefronts a CU
        const int64_t per_token = B * ceil_div(K, kVec);
        a.run = 16;
        while (a.run > 4 && per_token * ceil_div(L, a.run) < 8 * 256 * 64) a.run /= 2;
        a.runs = ceil_div(L, a.run);
        const int64_t blocks = ceil_div(a.runs * B, kThreads >> a.lanes_log2) * a.column_blocks;
        if (!grid_fits(blocks, kThreads)) return (int)PTQ4VM_ERR_SHAPE;
        return for_filter(W, K % kVec == 0, [&](auto taps, auto whole) {
            token_conv_runs<T, taps(), whole()><<<dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(stream)>>>(a);
            return check_launch("token_conv_runs");
        });
    });
}

// Rows of the backward pass's partial sums: workgroups over the runs, up to 2048 with all column blocks
struct BackwardPlan {
    int run;
    int64_t runs, groups;
};
template <typename T>
BackwardPlan backward_plan(const ConvArgs<T> &a, int64_t B, int64_t L, int64_t K) {
    BackwardPlan plan{32, 0, 0};
    while (plan.run > 8 && B * ceil_div(K, kVecBackward) * ceil_div(L, plan.run) < 8 * 256 * 64) plan.run /= 2;
    plan.runs = ceil_div(L, plan.run);
    const int64_t most = 2048 / a.column_blocks > 1 ? 2048 / a.column_blocks : 1;
    plan.groups = ceil_div(plan.runs * B, kThreads >> a.lanes_log2);
    if (plan.groups > most) plan.groups = most;
    return plan;
}

}  // namespace

extern "C" {

int ptq4vm_token_conv(int dtype, const void *x, const float *w, const float *bias, const void *state, void *y, void *state_out, int silu, int reverse, int64_t B,
                      int64_t L, int64_t K, int64_t W, int64_t ldx, int64_t ldy, void *stream) {
    const int rc = check_conv(dtype, x, w, bias, state, B, L, K, W);
    if (rc != PTQ4VM_OK) return rc;
    if (B != 0 && !y) return PTQ4VM_ERR_NULL;
    if (ldx < K || ldy < K) return PTQ4VM_ERR_STRIDE;
    if (!aligned_to(y, dtype_bytes(dtype)) || !aligned_to(state_out, dtype_bytes(dtype))) return PTQ4VM_ERR_ALIGN;
    if (B > 0 && (run_overlap(dtype, y, ldy, x, ldx, B, L, K) || overlap(state, state_out, B * (W - 1) * K * (int64_t)dtype_bytes(dtype)))) return PTQ4VM_ERR_OVERLAP;
    return conv(dtype, x, w, bias, state, y, state_out, silu, reverse, B, L, K, W, ldx, ldy, stream);
}

int ptq4vm_token_conv_step(int dtype, const void *x, const float *w, const float *bias, const void *state, void *y, void *state_out, int silu, int64_t B, int64_t K,
                           int64_t W, int64_t ldx, int64_t ldy, void *stream) {
    const int rc = check_conv(dtype, x, w, bias, state, B, 1, K, W);
    if (rc != PTQ4VM_OK) return rc;
    if (B != 0 && (!state || !y || !state_out)) return PTQ4VM_ERR_NULL;
    if (ldx < K || ldy < K) return PTQ4VM_ERR_STRIDE;
    if (!aligned_to(y, dtype_bytes(dtype)) || !aligned_to(state_out, dtype_bytes(dtype))) return PTQ4VM_ERR_ALIGN;
    if (B > 0 && (run_overlap(dtype, y, ldy, x, ldx, B, 1, K) || (state != state_out && overlap(state, state_out, B * (W - 1) * K * (int64_t)dtype_bytes(dtype)))))
        return PTQ4VM_ERR_OVERLAP;
    return conv(dtype, x, w, bias, state, y, state_out, silu, 0, B, 1, K, W, ldx, ldy, stream);
}

int64_t ptq4vm_token_conv_backward_workspace(int64_t B, int64_t L, int64_t K, int64_t W) {
    if (B <= 0 || L <= 0 || K <= 0 || W < 2 || W > 4 || L > kMaxTokenRows || K > kMaxTokenRows / 16 || B > kMaxTokenRows / L) return 0;
    ConvArgs<float> a{};
    columns(a, K, kVecBackward);
    return backward_plan(a, B, L, K).groups * K * (W + 1) * 4;
}

int ptq4vm_token_conv_backward(int dtype, const void *dy, const void *x, const float *w, const float *bias, const void *state, void *dx, float *dw, float *dbias,
                               void *workspace, int64_t workspace_bytes, int silu, int reverse, int64_t B, int64_t L, int64_t K, int64_t W, int64_t lddy, int64_t ldx,
                               int64_t lddx, void *stream_) {
    int rc = check_conv(dtype, x, w, bias, state, B, L, K, W);
    if (rc != PTQ4VM_OK) return rc;
    if (!dw || (B != 0 && (!dy || !dx || !workspace))) return PTQ4VM_ERR_NULL;
    if (ldx < K || lddy < K || lddx < K) return PTQ4VM_ERR_STRIDE;
    if (workspace_bytes < ptq4vm_token_conv_backward_workspace(B, L, K, W)) return PTQ4VM_ERR_SHAPE;
    const uintptr_t e = dtype_bytes(dtype);
    if (!aligned_to(dy, e) || !aligned_to(dx, e) || !aligned_to(dw, 4) || !aligned_to(dbias, 4) || !aligned_to(workspace, 16)) return PTQ4VM_ERR_ALIGN;
    if (B > 0 && (run_overlap(dtype, dx, lddx, x, ldx, B, L, K) || run_overlap(dtype, dx, lddx, dy, lddy, B, L, K))) return PTQ4VM_ERR_OVERLAP;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    int64_t groups = 0;
    if (B > 0) {
        rc = for_dtype(dtype, [&](auto zero) {
            using T = decltype(zero);
            ConvArgs<T> a{tokens<T>(x, L, ldx, reverse), tokens<T>(dx, L, lddx, reverse), tokens<T>(dy, L, lddy, reverse), w, bias, static_cast<const T *>(state), nullptr,
                          static_cast<float *>(workspace), (int)K, (int)B, silu, L, 0, 0, 0, 0};
            columns(a, K, kVecBackward);
            const BackwardPlan plan = backward_plan(a, B, L, K);
            a.run = plan.run, a.runs = plan.runs, groups = plan.groups;
            return for_filter(W, K % kVecBackward == 0, [&](auto taps, auto whole) {
                token_conv_backward_runs<T, taps(), whole()><<<dim3((unsigned)(groups * a.column_blocks)), dim3(kThreads), 0, stream>>>(a, (int)groups);
                return check_launch("token_conv_backward_runs");
            });
        });
        if (rc != PTQ4VM_OK) return rc;
    }
    return launch_sum_partials(static_cast<const float *>(workspace), groups, K * (W + 1), {dw, dbias, nullptr, K * W, K}, stream);
}

}  // extern "C"
