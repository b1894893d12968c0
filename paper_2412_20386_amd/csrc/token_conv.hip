// Short convolution over the tokens of a sequence, one filter per channel (between in_proj and x_proj of a block):
//   p[t,k] = bias[k] + sum_j w[k,j] x[t - W + 1 + j, k],  y = p / (1 + e^-p) or p,  x before token 0 from the state or 0.
// Backward, with dp = dy * (derivative of the activation at p, computed again):
//   dx[t,k] = sum_j w[k,j] dp[t + W - 1 - j, k],  dw[k,j] = sum_t dp[t,k] x[t - W + 1 + j, k],  dbias[k] = sum_t dp[t,k].
//
// Bound by memory (2 - 12 flops a byte).  A lane owns 8 adjacent channels (16 bytes of 16-bit elements) and walks over a run of tokens with
// the window of W - 1 earlier ones in registers, so that a token is read once by its run; the next run reads the last W - 1
// again (from the L2: neighbouring runs are neighbours in a workgroup).  Sums are fp32.
#include "token_ops.hpp"

namespace {

using namespace ptq4vm;

constexpr int kThreads = 256, kVec = 8, kUnroll = 4;

template <typename T>
struct ConvArgs {
    Tokens<T> x, y, dy;  // (y: dx in the backward pass)
    const float *w, *bias;
    const T *state;  // may be the buffer of state_out where one run spans the sequence
    T *state_out;
    float *partial;
    int K, B;
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
__device__ __forceinline__ Place place(int lanes_log2, int column_block, int K) {
    const int lanes = 1 << lanes_log2;
    const int k = (column_block * lanes + (threadIdx.x & (lanes - 1))) * kVec;
    return {k, max(0, min(kVec, K - k)), (int)threadIdx.x >> lanes_log2, kThreads >> lanes_log2};
}

template <typename T, int W>
__device__ __forceinline__ void filters(const ConvArgs<T> &p, const Place &at, float (&w)[W][kVec], float (&bias)[kVec]) {
#pragma unroll
    for (int i = 0; i < kVec; i++) {
        bias[i] = i < at.n && p.bias ? p.bias[at.k + i] : 0.0f;
#pragma unroll
        for (int j = 0; j < W; j++) w[j][i] = i < at.n ? p.w[(int64_t)(at.k + i) * W + j] : 0.0f;
    }
}

// x of the W - 1 tokens before token t
template <typename T, int W>
__device__ __forceinline__ void window_before(const ConvArgs<T> &p, const Place &at, int b, int64_t t, float (&win)[W - 1][kVec]) {
#pragma unroll
    for (int j = 0; j < W - 1; j++) {
        const int64_t s = t - (W - 1) + j;
        T raw[kVec];
        if (s >= 0)
            load_first<kVec>(p.x.at(b, s) + at.k, at.n, raw);
        else if (p.state)
            load_first<kVec>(p.state + ((int64_t)b * (W - 1) + s + (W - 1)) * p.K + at.k, at.n, raw);
        else
#pragma unroll
            for (int i = 0; i < kVec; i++) raw[i] = (T)0.0f;
#pragma unroll
        for (int i = 0; i < kVec; i++) win[j][i] = (float)raw[i];
    }
}

template <int W>
__device__ __forceinline__ void shift_in(float (&win)[W - 1][kVec], const float (&x)[kVec]) {
#pragma unroll
    for (int i = 0; i < kVec; i++) {
#pragma unroll
        for (int j = 0; j + 1 < W - 1; j++) win[j][i] = win[j + 1][i];
        win[W - 2][i] = x[i];
    }
}

template <typename T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void token_conv_runs(ConvArgs<T> p) {
    const int column_block = blockIdx.x % p.column_blocks;
    const Place at = place(p.lanes_log2, column_block, p.K);
    const int64_t item = (int64_t)(blockIdx.x / p.column_blocks) * at.slots + at.slot;
    if (item >= p.runs * p.B || at.n == 0) return;
    const int b = (int)(item / p.runs);
    const int64_t t0 = (item - b * p.runs) * p.run, t1 = min(p.L, t0 + p.run);
    float win[W - 1][kVec], w[W][kVec], bias[kVec];
    window_before<T, W>(p, at, b, t0, win);
    filters<T, W>(p, at, w, bias);
    for (int64_t t = t0; t < t1; t += kUnroll) {
        T raw[kUnroll][kVec];
#pragma unroll
        for (int s = 0; s < kUnroll; s++)
            if (t + s < t1) load_first<kVec>(p.x.at(b, t + s) + at.k, at.n, raw[s]);
#pragma unroll
        for (int s = 0; s < kUnroll; s++) {
            if (t + s >= t1) break;
            float x[kVec], y[kVec];
#pragma unroll
            for (int i = 0; i < kVec; i++) {
                x[i] = (float)raw[s][i];
                float v = fmaf(w[W - 1][i], x[i], bias[i]);
#pragma unroll
                for (int j = 0; j < W - 1; j++) v = fmaf(w[j][i], win[j][i], v);
                y[i] = SILU ? v * sigmoid_of(v) : v;
            }
            store_first<kVec>(p.y.at(b, t + s) + at.k, at.n, y);
            shift_in<W>(win, x);
        }
    }
    if (p.state_out && t1 == p.L)  // the window as it is now: the last W - 1 tokens, older ones from the state
#pragma unroll
        for (int j = 0; j < W - 1; j++) store_first<kVec>(p.state_out + ((int64_t)b * (W - 1) + j) * p.K + at.k, at.n, win[j]);
}

// A workgroup takes every gridDim-th group of runs and adds the filters' gradients up in registers; partial[workgroup row]
// is [K * W | K].
template <typename T, int W, bool SILU>
__global__ __launch_bounds__(kThreads) void token_conv_backward_runs(ConvArgs<T> p, int groups) {
    const int column_block = blockIdx.x % p.column_blocks, group = blockIdx.x / p.column_blocks;
    const Place at = place(p.lanes_log2, column_block, p.K);
    float w[W][kVec], bias[kVec], dw[W + 1][kVec];
    filters<T, W>(p, at, w, bias);
#pragma unroll
    for (int j = 0; j <= W; j++)
#pragma unroll
        for (int i = 0; i < kVec; i++) dw[j][i] = 0.0f;
    for (int64_t item = (int64_t)group * at.slots + at.slot; item < p.runs * p.B && at.n > 0; item += (int64_t)groups * at.slots) {
        const int b = (int)(item / p.runs);
        const int64_t t0 = (item - b * p.runs) * p.run, t1 = min(p.L, t0 + p.run);
        float win[W - 1][kVec], late[W - 1][kVec] = {};  // the last tokens' x and dp
        window_before<T, W>(p, at, b, t0, win);
        // dp of the run, and of the W - 1 tokens behind it, which the run's last tokens take part in
        for (int64_t t = t0; t < t1 + W - 1; t += kUnroll) {
            T rx[kUnroll][kVec], rdy[kUnroll][kVec];
#pragma unroll
            for (int s = 0; s < kUnroll; s++)
                if (t + s < min(p.L, t1 + W - 1)) {
                    load_first<kVec>(p.x.at(b, t + s) + at.k, at.n, rx[s]);
                    load_first<kVec>(p.dy.at(b, t + s) + at.k, at.n, rdy[s]);
                }
#pragma unroll
            for (int s = 0; s < kUnroll; s++) {
                if (t + s >= t1 + W - 1) break;
                float x[kVec], dp[kVec], dx[kVec];
#pragma unroll
                for (int i = 0; i < kVec; i++) x[i] = dp[i] = 0.0f;
                if (t + s < p.L)
#pragma unroll
                    for (int i = 0; i < kVec; i++) {
                        x[i] = (float)rx[s][i];
                        dp[i] = (float)rdy[s][i];
                        if constexpr (SILU) {
                            float v = fmaf(w[W - 1][i], x[i], bias[i]);
#pragma unroll
                            for (int j = 0; j < W - 1; j++) v = fmaf(w[j][i], win[j][i], v);
                            const float g = sigmoid_of(v);
                            dp[i] *= g * fmaf(v, 1.0f - g, 1.0f);
                        }
                    }
#pragma unroll
                for (int i = 0; i < kVec; i++) {
                    float v = w[0][i] * dp[i];
#pragma unroll
                    for (int j = 1; j < W; j++) v = fmaf(w[j][i], late[W - 1 - j][i], v);
                    dx[i] = v;
                }
                if (t + s - (W - 1) >= t0) store_first<kVec>(p.y.at(b, t + s - (W - 1)) + at.k, at.n, dx);
                if (t + s < t1)
#pragma unroll
                    for (int i = 0; i < kVec; i++) {
                        dw[W - 1][i] = fmaf(dp[i], x[i], dw[W - 1][i]);
#pragma unroll
                        for (int j = 0; j < W - 1; j++) dw[j][i] = fmaf(dp[i], win[j][i], dw[j][i]);
                        dw[W][i] += dp[i];
                    }
                shift_in<W>(win, x);
                shift_in<W>(late, dp);
            }
        }
    }
    __shared__ float red[kThreads][kVec + 1];
    float *const row = p.partial + (int64_t)group * p.K * (W + 1);
    const int lanes = 1 << p.lanes_log2;
#pragma unroll
    for (int j = 0; j <= W; j++) {
#pragma unroll
        for (int i = 0; i < kVec; i++) red[threadIdx.x][i] = dw[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < lanes * kVec; c += kThreads) {
            float sum = 0.0f;
            for (int s = 0; s < at.slots; s++) sum += red[s * lanes + c / kVec][c % kVec];
            const int64_t k = (int64_t)column_block * lanes * kVec + c;
            if (k < p.K) row[j < W ? k * W + j : (int64_t)p.K * W + k] = sum;
        }
        __syncthreads();
    }
}

// Lanes side by side over K, and the workgroups that K takes
template <typename T>
void columns(ConvArgs<T> &a, int64_t K) {
    const int64_t chunks = ceil_div(K, kVec);
    a.lanes_log2 = 0;
    while ((1 << a.lanes_log2) < chunks && a.lanes_log2 < 6) a.lanes_log2++;
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

template <typename T, bool SILU>
int launch_conv(const ConvArgs<T> &a, int W, dim3 grid, hipStream_t stream) {
    switch (W) {
        case 2: token_conv_runs<T, 2, SILU><<<grid, dim3(kThreads), 0, stream>>>(a); break;
        case 3: token_conv_runs<T, 3, SILU><<<grid, dim3(kThreads), 0, stream>>>(a); break;
        default: token_conv_runs<T, 4, SILU><<<grid, dim3(kThreads), 0, stream>>>(a); break;
    }
    return check_launch("token_conv_runs");
}

int conv(int dtype, const void *x, const float *w, const float *bias, const void *state, void *y, void *state_out, int silu, int reverse, int64_t B, int64_t L,
         int64_t K, int64_t W, int64_t ldx, int64_t ldy, void *stream) {
    if (B == 0) return PTQ4VM_OK;
    return for_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        ConvArgs<T> a{tokens<T>(x, L, ldx, reverse), tokens<T>(y, L, ldy, reverse), {}, w, bias, static_cast<const T *>(state), static_cast<T *>(state_out), nullptr,
                      (int)K, (int)B, L, 0, 0, 0, 0};
        columns(a, K);
        // A run of 16 tokens reads 3 of its neighbour's again; shorter ones where there would be fewer than 8 wavefronts a CU
        const int64_t per_token = B * ceil_div(K, kVec);
        a.run = 16;
        while (a.run > 4 && per_token * ceil_div(L, a.run) < 8 * 256 * 64) a.run /= 2;
        a.runs = ceil_div(L, a.run);
        const int64_t blocks = ceil_div(a.runs * B, kThreads >> a.lanes_log2) * a.column_blocks;
        if (blocks > kMaxTokenRows) return (int)PTQ4VM_ERR_SHAPE;
        const dim3 grid((unsigned)blocks);
        return silu ? launch_conv<T, true>(a, (int)W, grid, static_cast<hipStream_t>(stream)) : launch_conv<T, false>(a, (int)W, grid, static_cast<hipStream_t>(stream));
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
    while (plan.run > 8 && B * ceil_div(K, kVec) * ceil_div(L, plan.run) < 8 * 256 * 64) plan.run /= 2;
    plan.runs = ceil_div(L, plan.run);
    const int64_t most = 2048 / a.column_blocks > 1 ? 2048 / a.column_blocks : 1;
    plan.groups = ceil_div(plan.runs * B, kThreads >> a.lanes_log2);
    if (plan.groups > most) plan.groups = most;
    return plan;
}

template <typename T, bool SILU>
int launch_conv_backward(const ConvArgs<T> &a, int W, int64_t groups, hipStream_t stream) {
    const dim3 grid((unsigned)(groups * a.column_blocks));
    switch (W) {
        case 2: token_conv_backward_runs<T, 2, SILU><<<grid, dim3(kThreads), 0, stream>>>(a, (int)groups); break;
        case 3: token_conv_backward_runs<T, 3, SILU><<<grid, dim3(kThreads), 0, stream>>>(a, (int)groups); break;
        default: token_conv_backward_runs<T, 4, SILU><<<grid, dim3(kThreads), 0, stream>>>(a, (int)groups); break;
    }
    return check_launch("token_conv_backward_runs");
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
    return conv(dtype, x, w, bias, state, y, state_out, silu, reverse, B, L, K, W, ldx, ldy, stream);
}

int ptq4vm_token_conv_step(int dtype, const void *x, const float *w, const float *bias, const void *state, void *y, void *state_out, int silu, int64_t B, int64_t K,
                           int64_t W, int64_t ldx, int64_t ldy, void *stream) {
    const int rc = check_conv(dtype, x, w, bias, state, B, 1, K, W);
    if (rc != PTQ4VM_OK) return rc;
    if (B != 0 && (!state || !y || !state_out)) return PTQ4VM_ERR_NULL;
    if (ldx < K || ldy < K) return PTQ4VM_ERR_STRIDE;
    if (!aligned_to(y, dtype_bytes(dtype)) || !aligned_to(state_out, dtype_bytes(dtype))) return PTQ4VM_ERR_ALIGN;
    return conv(dtype, x, w, bias, state, y, state_out, silu, 0, B, 1, K, W, ldx, ldy, stream);
}

int64_t ptq4vm_token_conv_backward_workspace(int64_t B, int64_t L, int64_t K, int64_t W) {
    if (B <= 0 || L <= 0 || K <= 0 || W < 2 || W > 4 || L > kMaxTokenRows || K > kMaxTokenRows / 16 || B > kMaxTokenRows / L) return 0;
    ConvArgs<float> a{};
    columns(a, K);
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
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    int64_t groups = 0;
    if (B > 0) {
        rc = for_dtype(dtype, [&](auto zero) {
            using T = decltype(zero);
            ConvArgs<T> a{tokens<T>(x, L, ldx, reverse), tokens<T>(dx, L, lddx, reverse), tokens<T>(dy, L, lddy, reverse), w, bias, static_cast<const T *>(state), nullptr,
                          static_cast<float *>(workspace), (int)K, (int)B, L, 0, 0, 0, 0};
            columns(a, K);
            const BackwardPlan plan = backward_plan(a, B, L, K);
            a.run = plan.run, a.runs = plan.runs, groups = plan.groups;
            return silu ? launch_conv_backward<T, true>(a, (int)W, groups, stream) : launch_conv_backward<T, false>(a, (int)W, groups, stream);
        });
        if (rc != PTQ4VM_OK) return rc;
    }
    return launch_sum_partials(static_cast<const float *>(workspace), groups, K * (W + 1), {dw, dbias, nullptr, K * W, K}, stream);
}

}  // extern "C"
