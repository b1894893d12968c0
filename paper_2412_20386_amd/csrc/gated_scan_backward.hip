// Backward pass of the gated linear recurrence (gated_scan.hpp has the forward formulas and the layout).  With
// G = dy z / (1 + e^-z) and g_t the gradient of h_t:
//   g_t = c_t G_t + e^{D a} (at t + 1) g_{t+1},  w_t = g_t e^{D a} h_{t-1},
//   dc_t = sum_k G h_t,  db_t = sum_k g D u,  da = sum_{b,t} w D,  dd = sum G u,  dz = dy s (derivative of the gate),
//   du = d G + D sum_n g b,  dD = u sum_n g b + sum_n w a,  ddt = dD / (1 + e^-(dt + dt_bias)),  ddt_bias = sum ddt.
// A wavefront takes its tiles of kTile tokens from the last to the first: the states of a tile are computed again from its
// mark into registers, then the tile is run through backwards.  Sums over channels (db, dc) leave a wavefront as one row of
// 2 N partial sums a token, sums over tokens (da, dd, ddt_bias) as one row for each sequence and chunk; both are summed up
// in a fixed order by kernels of their own.
#include "gated_scan.hpp"

namespace {

using namespace ptq4vm;

constexpr float kLn2 = 0.69314718055994530942f;

// CARRY_ONLY: from a zero gradient behind the chunk, without outputs; leaves e^{D a} g at the chunk's first token and the sum
// of D, from which the chunks before it know the gradient that comes in.
template <typename T, int NS, int C, bool PADDED, bool CARRY_ONLY>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(2))) void gated_scan_backward_tokens(ScanArgs<T> p) {
    using S = ScanLane<NS, C>;
    static_assert(S::kPasses == 1, "a lane loads one token of a tile");
    constexpr int kSub = NS * C >= 16 ? 8 : 16;  // tokens whose states are in registers: 128 of them
    __shared__ float2 steps[kTile][S::kChannels];  // D and D u; then sum g b and sum w a log2(e)
    __shared__ float grad[kTile][S::kChannels];    // G; then s without d u
    __shared__ float sb[kTile][S::kStates], sc[kTile][S::kStates];
    __shared__ float bc[CARRY_ONLY ? 1 : kTile][4][2][S::kStates];  // db and dc of each row of 16 lanes
    const uint32_t block = xcd_contiguous(blockIdx.x, p.blocks);
    if (block >= p.blocks) return;
    const int cb = block % p.column_blocks, from = block / p.column_blocks, b = from % p.B;
    const uint32_t chunk = from / p.B + (CARRY_ONLY ? 1 : 0);  // (nobody asks for the first chunk's)
    const int lane = threadIdx.x, q = lane & 3, cl = lane >> 2, n0 = q * NS;
    const int64_t t_begin = chunk * p.chunk_tokens, t_end = min(p.L, t_begin + p.chunk_tokens);

    float a2[C][NS], carry[C][NS], da[C][NS], sum_d[C];
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int k = cb * S::kChannels + cl * C + c, n = k < p.K ? p.N : 0;
        load_channel<NS>(p.a + (int64_t)(n ? k : 0) * p.N, n0, n, a2[c]);
        sum_d[c] = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; i++) a2[c][i] *= kLog2e, carry[c][i] = da[c][i] = 0.0f;
        if constexpr (!CARRY_ONLY)
            for (uint32_t i = p.chunks - 1; i > chunk; i--) {
                const int64_t at = n ? ((int64_t)i * p.B + b) * p.K + k : 0;
                float end[NS];
                load_channel<NS>(p.chunk_state + at * p.N, n0, n, end);
                const float D = n ? p.chunk_dt[at] : 0.0f;
#pragma unroll
                for (int j = 0; j < NS; j++) carry[c][j] = fmaf(__builtin_amdgcn_exp2f(a2[c][j] * D), carry[c][j], end[j]);
            }
    }

    const int vt = lane / S::kAcross, vk = (lane % S::kAcross) * S::kVec, k = cb * S::kChannels + vk, nk = max(0, min(S::kVec, p.K - k));
    float bias[S::kVec], skip[S::kVec], dd[S::kVec], dbias[S::kVec];
#pragma unroll
    for (int i = 0; i < S::kVec; i++) {
        bias[i] = p.dt_bias && i < nk ? p.dt_bias[k + i] : 0.0f;
        skip[i] = p.d && i < nk ? p.d[k + i] : 0.0f;
        dd[i] = dbias[i] = 0.0f;
    }
    T ru[S::kVec], rdt[S::kVec], rz[S::kVec], rdy[S::kVec], rb[NS], rc[NS];
    float h0[C][NS];
    const auto fetch = [&](int64_t t0) {
        const int n = t0 + vt < t_end ? nk : 0;
        const int64_t t = n ? t0 + vt : 0;
        load_first<S::kVec>(p.dt.at(b, t) + k, n, rdt);
        load_first<S::kVec>(p.dy.at(b, t) + k, n, rdy);
        if (p.z.data) load_first<S::kVec>(p.z.at(b, t) + k, n, rz);
        load_states<NS>(p.c, b, t0, t_end, p.N, rc);
        if constexpr (!CARRY_ONLY) {
            load_first<S::kVec>(p.u.at(b, t) + k, n, ru);
            load_states<NS>(p.b, b, t0, t_end, p.N, rb);
#pragma unroll
            for (int c = 0; c < C; c++) {
                const int kc = cb * S::kChannels + cl * C + c;
                load_channel<NS>(p.marks + (((t0 / kTile) * p.B + b) * p.K + (kc < p.K ? kc : 0)) * p.N, n0, kc < p.K ? p.N : 0, h0[c]);
            }
        }
    };
    int64_t t0 = t_begin + (t_end - t_begin - 1) / kTile * kTile;
    fetch(t0);
    for (; t0 >= t_begin; t0 -= kTile) {
        const bool there = t0 + vt < t_end;  // tokens behind the last change nothing: D, D u, G, b and c are 0
        float u[S::kVec], D[S::kVec], G[S::kVec], z[S::kVec], dy[S::kVec], slope[S::kVec];
#pragma unroll
        for (int i = 0; i < S::kVec; i++) {
            const float x = (float)rdt[i] + bias[i];
            D[i] = there ? softplus_of(x) : 0.0f;
            slope[i] = sigmoid_of(x);
            dy[i] = (float)rdy[i];
            G[i] = dy[i];
            if (p.z.data) {
                z[i] = (float)rz[i];
                G[i] *= z[i] * sigmoid_of(z[i]);
            }
            G[i] = there ? G[i] : 0.0f;
            u[i] = CARRY_ONLY ? 0.0f : (float)ru[i];
            steps[vt][vk + i] = {D[i], there ? D[i] * u[i] : 0.0f};
            grad[vt][vk + i] = G[i];
        }
        keep_states<NS>(rc, sc);
        if constexpr (!CARRY_ONLY) keep_states<NS>(rb, sb);
        __syncthreads();
        float start[C][NS];
#pragma unroll
        for (int c = 0; c < C; c++)
#pragma unroll
            for (int i = 0; i < NS; i++) start[c][i] = CARRY_ONLY ? 0.0f : h0[c][i];
        if (t0 > t_begin) fetch(t0 - kTile);
        if constexpr (CARRY_ONLY) {
            for (int t = kTile - 1; t >= 0; t--)
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const float D_t = steps[t][cl * C + c].x, G_t = grad[t][cl * C + c];
                    sum_d[c] += D_t;
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        carry[c][i] = __builtin_amdgcn_exp2f(a2[c][i] * D_t) * fmaf(sc[t][n0 + i], G_t, carry[c][i]);
                        if (PADDED) carry[c][i] = n0 + i < p.N ? carry[c][i] : 0.0f;
                    }
                }
            __syncthreads();
            continue;
        }
        for (int sub = kTile - kSub; sub >= 0; sub -= kSub) {
            float h[kSub + 1][C][NS];
            const auto advance = [&](int t, const float (&before)[C][NS], float (&after)[C][NS]) {
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const float2 D_t = steps[t][cl * C + c];
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        after[c][i] = fmaf(__builtin_amdgcn_exp2f(a2[c][i] * D_t.x), before[c][i], D_t.y * sb[t][n0 + i]);
                        if (PADDED) after[c][i] = n0 + i < p.N ? after[c][i] : 0.0f;
                    }
                }
            };
#pragma unroll
            for (int c = 0; c < C; c++)
#pragma unroll
                for (int i = 0; i < NS; i++) h[0][c][i] = start[c][i];
            for (int t = 0; t < sub; t++) advance(t, h[0], h[0]);
#pragma unroll
            for (int s = 0; s < kSub; s++) advance(sub + s, h[s], h[s + 1]);
#pragma unroll
            for (int s = kSub - 1; s >= 0; s--) {
                const int t = sub + s;
                float gb[C], wa[C], v[C], db[NS], dc[NS];
#pragma unroll
                for (int i = 0; i < NS; i++) db[i] = dc[i] = 0.0f;
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const float2 D_t = steps[t][cl * C + c];
                    const float G_t = grad[t][cl * C + c];
                    gb[c] = wa[c] = v[c] = 0.0f;
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        const float g = fmaf(sc[t][n0 + i], G_t, carry[c][i]);
                        v[c] = fmaf(sc[t][n0 + i], h[s + 1][c][i], v[c]);
                        dc[i] = fmaf(h[s + 1][c][i], G_t, dc[i]);
                        db[i] = fmaf(g, D_t.y, db[i]);
                        gb[c] = fmaf(g, sb[t][n0 + i], gb[c]);
                        carry[c][i] = g * __builtin_amdgcn_exp2f(a2[c][i] * D_t.x);
                        if (PADDED) carry[c][i] = n0 + i < p.N ? carry[c][i] : 0.0f;
                        const float w = carry[c][i] * h[s][c][i];
                        wa[c] = fmaf(w, a2[c][i], wa[c]);
                        da[c][i] = fmaf(w, D_t.x, da[c][i]);
                    }
                    gb[c] = quad_sum(gb[c]);
                    wa[c] = quad_sum(wa[c]);
                    v[c] = quad_sum(v[c]);
                }
                // (a lane's own reads of this token are done, and so are its quad's: one wavefront, LDS in order)
                if (q < C) {
                    const bool second = C == 2 && q == 1;
                    steps[t][cl * C + q] = {second ? gb[C - 1] : gb[0], second ? wa[C - 1] : wa[0]};
                    grad[t][cl * C + q] = second ? v[C - 1] : v[0];
                }
#pragma unroll
                for (int i = 0; i < NS; i++) {  // over the four quads of a row of 16 lanes
                    db[i] = add_dpp<0x128>(add_dpp<0x124>(db[i]));
                    dc[i] = add_dpp<0x128>(add_dpp<0x124>(dc[i]));
                    if ((lane & 12) == 0) bc[t][lane >> 4][0][n0 + i] = db[i], bc[t][lane >> 4][1][n0 + i] = dc[i];
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kTile * 2 * S::kStates / 64; j++) {
            const int at = j * 64 + lane, t = at / (2 * S::kStates), which = at / S::kStates % 2, n = at % S::kStates;
            const float v = (bc[t][0][which][n] + bc[t][1][which][n]) + (bc[t][2][which][n] + bc[t][3][which][n]);
            if (t0 + t < t_end && n < p.N) p.partial_bc[((((int64_t)cb * p.B + b) * p.L + t0 + t) * 2 + which) * p.N + n] = v;
        }
        float du[S::kVec], ddt[S::kVec], dz[S::kVec];
#pragma unroll
        for (int i = 0; i < S::kVec; i++) {
            const float2 sums = steps[vt][vk + i];
            du[i] = fmaf(skip[i], G[i], D[i] * sums.x);
            ddt[i] = fmaf(u[i], sums.x, sums.y * kLn2) * slope[i];
            if (p.z.data) {
                const float g = sigmoid_of(z[i]);
                dz[i] = dy[i] * fmaf(skip[i], u[i], grad[vt][vk + i]) * (g * fmaf(z[i], 1.0f - g, 1.0f));
            }
            if (there && i < nk) dd[i] = fmaf(G[i], u[i], dd[i]), dbias[i] += ddt[i];
        }
        if (there && nk) {
            store_first<S::kVec>(p.du.at(b, t0 + vt) + k, nk, du);
            store_first<S::kVec>(p.ddt.at(b, t0 + vt) + k, nk, ddt);
            if (p.z.data) store_first<S::kVec>(p.dz.at(b, t0 + vt) + k, nk, dz);
        }
        __syncthreads();
    }
    const int64_t rows = (int64_t)chunk * p.B + b;
    float *const sums = CARRY_ONLY ? nullptr : p.partial_a + rows * p.K * (p.N + 2);
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int kc = cb * S::kChannels + cl * C + c;
        if (kc >= p.K) continue;
        if constexpr (CARRY_ONLY) {
            store_channel<NS>(p.chunk_state + (rows * p.K + kc) * p.N, n0, p.N, carry[c]);
            if (q == 0) p.chunk_dt[rows * p.K + kc] = sum_d[c];
        } else {
            store_channel<NS>(sums + (int64_t)kc * p.N, n0, p.N, da[c]);
        }
    }
    if constexpr (!CARRY_ONLY) {
        static_assert(S::kAcross == 4, "lanes of the same remainder by 4 hold the same channels");
#pragma unroll
        for (int i = 0; i < S::kVec; i++) {
            dd[i] = add_dpp<0x128>(add_dpp<0x124>(dd[i]));
            dd[i] += __shfl_xor(dd[i], 16, 64);
            dd[i] += __shfl_xor(dd[i], 32, 64);
            dbias[i] = add_dpp<0x128>(add_dpp<0x124>(dbias[i]));
            dbias[i] += __shfl_xor(dbias[i], 16, 64);
            dbias[i] += __shfl_xor(dbias[i], 32, 64);
        }
        if (lane < 4 && nk) {
            store_first<S::kVec>(sums + (int64_t)p.K * p.N + k, nk, dd);
            store_first<S::kVec>(sums + (int64_t)p.K * (p.N + 1) + k, nk, dbias);
        }
    }
}

// db and dc from the column blocks' rows of partial sums
template <typename T>
__global__ __launch_bounds__(256) void sum_column_blocks(const float *__restrict__ partial, int column_blocks, int64_t L, int64_t values, int N, Tokens<T> db,
                                                         Tokens<T> dc) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= values) return;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    int s = 0;
    for (; s + 4 <= column_blocks; s += 4)
#pragma unroll
        for (int j = 0; j < 4; j++) sum[j] += partial[(s + j) * values + i];
    for (; s < column_blocks; s++) sum[0] += partial[s * values + i];
    const float v = (sum[0] + sum[1]) + (sum[2] + sum[3]);
    const int64_t row = i / (2 * N);
    const int at = (int)(i - row * 2 * N);
    const int b = (int)(row / L);
    const int64_t t = row - b * L;
    if (at < N)
        db.at(b, t)[at] = (T)v;
    else
        dc.at(b, t)[at - N] = (T)v;
}

struct BackwardSizes {
    int64_t bc, a, chunk;  // floats
};
BackwardSizes backward_sizes(const ScanPlan &plan, int64_t B, int64_t L, int64_t K, int64_t N) {
    return {ceil_div(plan.column_blocks * B * L * 2 * N, 4) * 4, ceil_div(plan.chunks * B * K * (N + 2), 4) * 4, plan.chunks > 1 ? plan.chunks * B * K * (N + 1) : 0};
}

}  // namespace

extern "C" {

int64_t ptq4vm_gated_scan_backward_workspace(int64_t B, int64_t L, int64_t K, int64_t N) {
    if (!scan_sizes(B, L, K, N) || B == 0) return 0;
    const BackwardSizes s = backward_sizes(scan_plan(B, L, K, N), B, L, K, N);
    return (s.bc + s.a + s.chunk) * 4;
}

int ptq4vm_gated_scan_backward(int dtype, const void *dy, const void *u, const void *dt, const float *a, const void *b, const void *c, const float *d, const void *z,
                               const float *dt_bias, const float *marks, void *du, void *ddt, float *da, void *db, void *dc, float *dd, void *dz, float *ddt_bias,
                               void *workspace, int64_t workspace_bytes, int reverse, int64_t B, int64_t L, int64_t K, int64_t N, int64_t lddy, int64_t ldu,
                               int64_t lddt, int64_t ldb, int64_t ldc, int64_t ldz, int64_t lddu, int64_t ldddt, int64_t lddb, int64_t lddc, int64_t lddz,
                               void *stream_) {
    if (!valid_dtype(dtype)) return PTQ4VM_ERR_SHAPE;
    if (!a || !da || (d && !dd) || (dt_bias && !ddt_bias)) return PTQ4VM_ERR_NULL;
    if (B != 0 && (!dy || !u || !dt || !b || !c || !marks || !du || !ddt || !db || !dc || (z && !dz))) return PTQ4VM_ERR_NULL;
    if (!scan_sizes(B, L, K, N)) return PTQ4VM_ERR_SHAPE;
    if (lddy < K || ldu < K || lddt < K || ldb < N || ldc < N || (z && (ldz < K || lddz < K)) || lddu < K || ldddt < K || lddb < N || lddc < N)
        return PTQ4VM_ERR_STRIDE;
    const int64_t need = ptq4vm_gated_scan_backward_workspace(B, L, K, N);
    if (need > 0 && !workspace) return PTQ4VM_ERR_NULL;
    if (workspace_bytes < need) return PTQ4VM_ERR_SHAPE;
    const uintptr_t e = dtype_bytes(dtype);
    for (const void *ptr : {dy, u, dt, b, c, z, (const void *)du, (const void *)ddt, (const void *)db, (const void *)dc, (const void *)dz})
        if (!aligned_to(ptr, e)) return PTQ4VM_ERR_ALIGN;
    for (const void *ptr : {(const void *)a, (const void *)d, (const void *)dt_bias, (const void *)marks, (const void *)da, (const void *)dd, (const void *)ddt_bias})
        if (!aligned_to(ptr, 4)) return PTQ4VM_ERR_ALIGN;
    if (need > 0 && !aligned_to(workspace, 16)) return PTQ4VM_ERR_ALIGN;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    const SumOut parameters{da, dd, ddt_bias, K * N, K};
    if (B == 0) return launch_sum_partials(nullptr, 0, K * (N + 2), parameters, stream);
    const ScanPlan plan = scan_plan(B, L, K, N);
    const BackwardSizes sizes = backward_sizes(plan, B, L, K, N);
    float *const ws = static_cast<float *>(workspace);
    const int64_t values = B * L * 2 * N;
    if (ceil_div(values, 256) > kMaxTokenRows) return PTQ4VM_ERR_SHAPE;
    const int rc = for_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        ScanArgs<T> s{};
        s.u = tokens<T>(u, L, ldu, reverse), s.dt = tokens<T>(dt, L, lddt, reverse), s.b = tokens<T>(b, L, ldb, reverse), s.c = tokens<T>(c, L, ldc, reverse);
        s.z = tokens<T>(z, L, ldz, reverse), s.dy = tokens<T>(dy, L, lddy, reverse);
        s.du = tokens<T>(du, L, lddu, reverse), s.ddt = tokens<T>(ddt, L, ldddt, reverse), s.dz = tokens<T>(dz, L, lddz, reverse);
        s.a = a, s.d = d, s.dt_bias = dt_bias, s.marks = const_cast<float *>(marks);
        s.partial_bc = ws, s.partial_a = ws + sizes.bc, s.chunk_state = s.partial_a + sizes.a, s.chunk_dt = s.chunk_state + (sizes.chunk ? plan.chunks * B * K * N : 0);
        s.B = (int)B, s.K = (int)K, s.N = (int)N, s.column_blocks = (int)plan.column_blocks, s.L = L, s.chunk_tokens = plan.chunk_tokens;
        s.chunks = (uint32_t)plan.chunks;
        const int e2 = for_layout(plan, N, [&](auto ns, auto ch, auto padded) {
            const auto go = [&](auto carry_only, int64_t chunks) {
                s.blocks = (uint32_t)(chunks * B * plan.column_blocks);
                gated_scan_backward_tokens<T, ns(), ch(), padded(), carry_only()><<<dim3(xcd_grid(s.blocks)), dim3(64), 0, stream>>>(s);
                return check_launch("gated_scan_backward_tokens");
            };
            if (plan.chunks > 1)
                if (const int e3 = go(std::true_type{}, plan.chunks - 1)) return e3;
            return go(std::false_type{}, plan.chunks);
        });
        if (e2) return e2;
        sum_column_blocks<T><<<dim3((unsigned)ceil_div(values, 256)), dim3(256), 0, stream>>>(
            ws, (int)plan.column_blocks, L, values, (int)N, tokens<T>(db, L, lddb, reverse), tokens<T>(dc, L, lddc, reverse));
        return check_launch("sum_column_blocks");
    });
    if (rc != PTQ4VM_OK) return rc;
    return launch_sum_partials(ws + sizes.bc, plan.chunks * B, K * (N + 2), parameters, stream);
}

}  // extern "C"
