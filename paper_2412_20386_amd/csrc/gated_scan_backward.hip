// Backward pass of the gated linear recurrence (gated_scan.hpp has the forward formulas and the layout).  With
// G = dy z / (1 + e^-z) and g_t the gradient of h_t:
//   g_t = c_t G_t + e^{D a} (at t + 1) g_{t+1},  w_t = g_t e^{D a} h_{t-1},
//   dc_t = sum_k G h_t,  db_t = sum_k g D u,  da = sum_{b,t} w D,  dd = sum G u,  dz = dy s (derivative of the gate),
//   du = d G + D sum_n g b,  dD = u sum_n g b + sum_n w a,  ddt = dD / (1 + e^-(dt + dt_bias)),  ddt_bias = sum ddt.
// A wavefront takes its tiles of kMark tokens from the last to the first: the states of a tile are computed again from its
// mark into registers, then the tile is run through backwards.  Sums over channels (db, dc) leave a wavefront as one row of
// 2 N partial sums a token, sums over tokens (da, dd, ddt_bias) as one row for each sequence and chunk; both are summed up
// in a fixed order by kernels of their own.
// Bound by the vector ALU (79 % busy): 128 x 197 x 768 x 16 takes 262 us, and 19 for the sums; two channels to a lane take 251
// registers, two wavefronts to a SIMD, so that 3/2 rounds of them run.
#include "gated_scan.hpp"

namespace {

using namespace ptq4vm;

constexpr int kTile = kMark;  // tokens that are staged together, and whose states are in registers
constexpr int64_t kFull = 2048;  // wavefronts from which two channels to a lane are faster: 2 to a SIMD (at 3 to a SIMD 275 us against 295)
constexpr int64_t kHeld = 6144;  // wavefronts that sequences are cut for: three rounds of them (20000 x 1536, one round: 786 us, one and a half: 587, three: 543)
constexpr float kLn2 = 0.69314718055994530942f;

// CARRY_ONLY: from a zero gradient behind the chunk, without outputs; leaves e^{D a} g at the chunk's first token and the sum
// of D, from which the chunks before it know the gradient that comes in.
template <typename T, int NS, int C, bool RAGGED, bool CARRY_ONLY>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(NS * C > 8 ? 1 : CARRY_ONLY ? 4 : NS * C > 4 || (C == 2 && NS > 1) ? 2 : 3))) void gated_scan_backward_tokens(ScanArgs<T> p) {
    using S = ScanLane<NS, C, kTile>;
    constexpr int V = S::kVec;
    alignas(16) __shared__ float2 steps[kTile][S::kChannels];  // D and D u, then sum g b
    alignas(16) __shared__ float grad[kTile][S::kChannels];    // G, then sum w a log2(e)
    alignas(16) __shared__ float sb[kTile][S::kStates], sc[kTile][S::kStates];
    alignas(16) __shared__ float out_sums[CARRY_ONLY ? 1 : kTile][S::kChannels];  // s without d u
    alignas(16) __shared__ float bc[CARRY_ONLY ? 1 : kTile][2][S::kStates];       // the wavefront's db and dc
    alignas(16) __shared__ float bias[S::kChannels], skip[S::kChannels];
    const uint32_t block = xcd_contiguous(blockIdx.x, p.blocks);
    if (block >= p.blocks) return;
    const int cb = block % p.column_blocks, from = block / p.column_blocks, b = from % p.B;
    const uint32_t chunk = from / p.B + (CARRY_ONLY ? 1 : 0);  // (nobody asks for the first chunk's)
    const int lane = threadIdx.x, q = lane & 3, cl = lane >> 2, n0 = q * NS;
    const int64_t t_begin = chunk * p.chunk_tokens, t_end = min(p.L, t_begin + p.chunk_tokens);

    float a2[C][NS], carry[C][NS], da[C][NS], sum_d[C];
    const int kc = cb * S::kChannels + cl * C;  // the quad's first channel
#pragma unroll
    for (int c = 0; c < C; c++) {
        const bool mine = !RAGGED || kc + c < p.K;
        load_channel<NS, RAGGED>(p.a, kc + c, n0, p.N, mine, a2[c]);
        sum_d[c] = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; i++) a2[c][i] = rate_of(a2[c][i]), carry[c][i] = da[c][i] = 0.0f;
        if constexpr (!CARRY_ONLY) {
            if (p.joined) {
                if (chunk + 1 < p.chunks) load_channel<NS, RAGGED>(p.chunk_state, ((int64_t)(chunk + 1) * p.B + b) * p.K + kc + c, n0, p.N, mine, carry[c]);
            } else if (chunk + 1 < p.chunks) {
                float end[kJoin - 2][NS], D[kJoin - 2];
#pragma unroll
                for (int s = 0; s < kJoin - 2; s++) {  // from the last chunk on
                    const int64_t channel = ((int64_t)max((int)p.chunks - 1 - s, (int)chunk + 1) * p.B + b) * p.K + (mine ? kc + c : 0);
                    load_channel<NS, RAGGED>(p.chunk_state, channel, n0, p.N, mine, end[s]);
                    D[s] = p.chunk_dt[channel];
                }
#pragma unroll
                for (int s = 0; s < kJoin - 2; s++)
                    if ((int)p.chunks - 1 - s > (int)chunk)
#pragma unroll
                        for (int j = 0; j < NS; j++) carry[c][j] = decayed(carry[c][j], a2[c][j] * D[s], end[s][j]);
            }
        }
    }

    // what this lane loads: V channels of a token
    const int vt = lane / S::kAcross, vk = (lane % S::kAcross) * V, k = cb * S::kChannels + vk, nk = max(0, min(V, p.K - k));
    if (lane < S::kChannels) {
        const int at = cb * S::kChannels + lane;
        bias[lane] = p.dt_bias && at < p.K ? p.dt_bias[at] : 0.0f;
        skip[lane] = p.d && at < p.K ? p.d[at] : 0.0f;
    }
    __syncthreads();
    float dd[V], dbias[V];
#pragma unroll
    for (int i = 0; i < V; i++) dd[i] = dbias[i] = 0.0f;
    T ru[V], rdt[V], rz[V], rdy[V], rb[S::kStateVec], rc[S::kStateVec];
    float mark[C][NS];
    const auto fetch = [&](int64_t t0) {
        const int last = (int)min((int64_t)kTile, t_end - t0) - 1;
        load_token<V, RAGGED>(p.dt, b, t0, vt, last, k, nk, rdt);
        load_token<V, RAGGED>(p.dy, b, t0, vt, last, k, nk, rdy);
        if (p.z.data) load_token<V, RAGGED>(p.z, b, t0, vt, last, k, nk, rz);
        load_states<S, RAGGED>(p.c, b, t0, last, p.N, rc);
        if constexpr (!CARRY_ONLY) {
            load_token<V, RAGGED>(p.u, b, t0, vt, last, k, nk, ru);
            load_states<S, RAGGED>(p.b, b, t0, last, p.N, rb);
#pragma unroll
            for (int c = 0; c < C; c++)
                load_channel<NS, RAGGED>(p.marks, ((t0 / kMark) * p.B + b) * p.K + kc + c, n0, p.N, kc + c < p.K, mark[c]);
        }
    };
    int64_t t0 = t_begin + (t_end - t_begin - 1) / kTile * kTile;
    fetch(t0);
    for (; t0 >= t_begin; t0 -= kTile) {
        const bool there = t0 + vt < t_end;  // tokens behind the last change nothing: D, D u, G, b and c are 0
        T u[V], dt[V], z[V], dy[V];
        float h[kTile + 1][C][NS];
#pragma unroll
        for (int i = 0; i < V; i++) {
            dt[i] = rdt[i], dy[i] = rdy[i], z[i] = rz[i];
            if constexpr (!CARRY_ONLY) u[i] = ru[i];
        }
        if constexpr (!CARRY_ONLY)
#pragma unroll
            for (int c = 0; c < C; c++)
#pragma unroll
                for (int i = 0; i < NS; i++) h[0][c][i] = mark[c][i];
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float D = softplus_of((float)dt[i] + bias[vk + i]);
            steps[vt][vk + i] = {D, CARRY_ONLY ? 0.0f : D * (float)u[i]};
            grad[vt][vk + i] = (float)dy[i];
        }
        if (p.z.data)
#pragma unroll
            for (int i = 0; i < V; i++) grad[vt][vk + i] = (float)dy[i] * ((float)z[i] * sigmoid_of((float)z[i]));
        if (!there)
#pragma unroll
            for (int i = 0; i < V; i++) steps[vt][vk + i] = {0.0f, 0.0f}, grad[vt][vk + i] = 0.0f;
        keep_states<S>(rc, sc);
        if constexpr (!CARRY_ONLY) keep_states<S>(rb, sb);
        __syncthreads();
        if (t0 > t_begin) fetch(t0 - kTile);  // in flight under this tile's steps
        if constexpr (CARRY_ONLY) {
            for (int t = kTile - 1; t >= 0; t--)
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const float D_t = steps[t][cl * C + c].x, G_t = grad[t][cl * C + c];
                    sum_d[c] += D_t;
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        carry[c][i] = __builtin_amdgcn_exp2f(a2[c][i] * D_t) * fmaf(sc[t][n0 + i], G_t, carry[c][i]);
                        if (RAGGED) carry[c][i] = n0 + i < p.N ? carry[c][i] : 0.0f;
                    }
                }
            __syncthreads();
            continue;
        }
        struct Token {
            float b[NS], c[NS], G[C];
            float2 D[C];
        };
        const auto token_at = [&](int t, int n0, int ch) {
            Token v;
#pragma unroll
            for (int i = 0; i < NS; i++) v.b[i] = sb[t][n0 + i], v.c[i] = sc[t][n0 + i];
#pragma unroll
            for (int c = 0; c < C; c++) v.D[c] = steps[t][ch + c], v.G[c] = grad[t][ch + c];
            return v;
        };
        // The same places behind the compiler's back: values and exponentials that it knew from the pass forwards it would keep
        // through the pass backwards, and they do not fit the registers
        int q_again = q, cl_again = cl;
        asm("" : "+v"(q_again), "+v"(cl_again));
        const auto token = [&](int t) { return token_at(t, n0, cl * C); };
        const auto token_again = [&](int t) { return token_at(t, q_again * NS, cl_again * C); };
        // the next token's values are read under this one's arithmetic, and no earlier: more would not fit the registers
        Token next = token(0);
#pragma unroll
        for (int t = 0; t < kTile; t++) {
            const Token v = next;
            next = t + 1 < kTile ? token(t + 1) : token_again(kTile - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < C; c++)
#pragma unroll
                for (int i = 0; i < NS; i++) {
                    h[t + 1][c][i] = fmaf(__builtin_amdgcn_exp2f(a2[c][i] * v.D[c].x), h[t][c][i], v.D[c].y * v.b[i]);
                    if (RAGGED) h[t + 1][c][i] = n0 + i < p.N ? h[t + 1][c][i] : 0.0f;
                }
        }
#pragma unroll
        for (int t = kTile - 1; t >= 0; t--) {
            const Token v = next;
            if (t > 0) next = token_again(t - 1);
            __builtin_amdgcn_sched_barrier(0);
            float gb[C], wa[C], out[C], db[NS], dc[NS];
#pragma unroll
            for (int i = 0; i < NS; i++) db[i] = dc[i] = 0.0f;
#pragma unroll
            for (int c = 0; c < C; c++) {
                gb[c] = wa[c] = out[c] = 0.0f;
#pragma unroll
                for (int i = 0; i < NS; i++) {
                    const float g = fmaf(v.c[i], v.G[c], carry[c][i]);
                    out[c] = fmaf(v.c[i], h[t + 1][c][i], out[c]);
                    dc[i] = fmaf(h[t + 1][c][i], v.G[c], dc[i]);
                    db[i] = fmaf(g, v.D[c].y, db[i]);
                    gb[c] = fmaf(g, v.b[i], gb[c]);
                    carry[c][i] = g * __builtin_amdgcn_exp2f(a2[c][i] * v.D[c].x);
                    if (RAGGED) carry[c][i] = n0 + i < p.N ? carry[c][i] : 0.0f;
                    const float w = carry[c][i] * h[t][c][i];
                    wa[c] = fmaf(w, a2[c][i], wa[c]);
                    da[c][i] = fmaf(w, v.D[c].x, da[c][i]);
                }
            }
            // a lane's own reads of this token are done, and so are its quad's: one wavefront, LDS in order (and lanes of the same
            // place write the same values)
            steps[t][cl * C + q % C].y = quad_sums<C>(gb, q);
            grad[t][cl * C + q % C] = quad_sums<C>(wa, q);
            out_sums[t][cl * C + q % C] = quad_sums<C>(out, q);
            // db and dc over the wavefront's channels: halves, rows, then the quads of a row
            float half[NS];
#pragma unroll
            for (int i = 0; i < NS; i++) half[i] = sum_halves(db[i], dc[i]);
            if constexpr (NS == 1)
                bc[t][lane >> 5][n0] = sum_quads(sum_rows(half[0], half[0]));
            else
#pragma unroll
                for (int i = 0; i < NS; i += 2) bc[t][lane >> 5][n0 + i + (lane >> 4 & 1)] = sum_quads(sum_rows(half[i], half[i + 1]));
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kTile * 2 * S::kStates / 64; j++) {
            const int at = j * 64 + lane, t = at / (2 * S::kStates), which = at / S::kStates % 2, n = at % S::kStates;
            if (t0 + t < t_end && (!RAGGED || n < p.N))
                p.partial_bc[((((int64_t)cb * p.B + b) * p.L + t0 + t) * 2 + which) * (RAGGED ? p.N : S::kStates) + n] = bc[t][which][n];
        }
        if (there) {
            float G[V], out[V];
#pragma unroll
            for (int i = 0; i < V; i++) G[i] = (float)dy[i];
            if (p.z.data) {
#pragma unroll
                for (int i = 0; i < V; i++) {
                    const float g = sigmoid_of((float)z[i]), zg = (float)z[i] * g;
                    out[i] = G[i] * fmaf(skip[vk + i], (float)u[i], out_sums[vt][vk + i]) * fmaf(zg, 1.0f - g, g);
                    G[i] *= zg;
                }
                store_token<V, RAGGED>(p.dz, b, t0, vt, k, nk, out);
            }
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float2 sums = steps[vt][vk + i];
                out[i] = fmaf(skip[vk + i], G[i], sums.x * sums.y);
                dd[i] = fmaf(G[i], (float)u[i], dd[i]);
            }
            store_token<V, RAGGED>(p.du, b, t0, vt, k, nk, out);
#pragma unroll
            for (int i = 0; i < V; i++) {
                out[i] = fmaf((float)u[i], steps[vt][vk + i].y, grad[vt][vk + i] * kLn2) * sigmoid_of((float)dt[i] + bias[vk + i]);
                dbias[i] += out[i];
            }
            store_token<V, RAGGED>(p.ddt, b, t0, vt, k, nk, out);
        }
        __syncthreads();
    }
    const int64_t rows = (int64_t)chunk * p.B + b;
    float *const sums = CARRY_ONLY ? nullptr : p.partial_a + rows * p.K * (p.N + 2);
#pragma unroll
    for (int c = 0; c < C; c++) {
        if constexpr (CARRY_ONLY) {
            store_channel<NS, RAGGED>(p.chunk_state, rows * p.K + kc + c, n0, p.N, kc + c < p.K, carry[c]);
            if (q == 0 && kc + c < p.K) p.chunk_dt[rows * p.K + kc + c] = sum_d[c];
        } else {
            store_channel<NS, RAGGED>(sums, kc + c, n0, p.N, kc + c < p.K, da[c]);
        }
    }
    if constexpr (!CARRY_ONLY) {
        static_assert(S::kAcross == 8, "lanes of the same remainder by 8 hold the same channels");
#pragma unroll
        for (int i = 0; i < V; i++) {
            const float half = sum_halves(add_dpp<0x128>(dd[i]), add_dpp<0x128>(dbias[i]));  // lanes 0 - 31: dd, 32 - 63: ddt_bias
            dd[i] = sum_rows(half, half);
        }
        if ((lane & 24) == 0 && nk) store_first<V>(sums + (int64_t)p.K * (p.N + (lane >> 5)) + k, nk, dd);
    }
}

// db and dc from the column blocks' rows of partial sums
template <typename T>
__global__ __launch_bounds__(256) void sum_column_blocks(const float *__restrict__ partial, int column_blocks, int64_t L, int64_t values, int N, Tokens<T> db,
                                                         Tokens<T> dc) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < values; i += (int64_t)gridDim.x * 256) {
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
}

// (24 x 197 x 768 in chunks and two channels to a lane 91 us, whole and one 114)
ScanPlan backward_plan(int64_t B, int64_t L, int64_t K, int64_t N) { return scan_plan(B, L, K, N, kFull, kHeld, kTile, false); }

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
    const BackwardSizes s = backward_sizes(backward_plan(B, L, K, N), B, L, K, N);
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
    for (const int64_t ld : {lddy, ldu, lddt, ldb, ldc, z ? ldz : 0, lddu, ldddt, lddb, lddc, z ? lddz : 0})
        if (ld >= kMaxPitch) return PTQ4VM_ERR_STRIDE;
    const int64_t need = ptq4vm_gated_scan_backward_workspace(B, L, K, N);
    if (need > 0 && !workspace) return PTQ4VM_ERR_NULL;
    if (workspace_bytes < need) return PTQ4VM_ERR_SHAPE;
    const uintptr_t e = dtype_bytes(dtype);
    for (const void *ptr : {dy, u, dt, b, c, z, (const void *)du, (const void *)ddt, (const void *)db, (const void *)dc, (const void *)dz})
        if (!aligned_to(ptr, e)) return PTQ4VM_ERR_ALIGN;
    for (const void *ptr : {(const void *)a, (const void *)d, (const void *)dt_bias, (const void *)marks, (const void *)da, (const void *)dd, (const void *)ddt_bias})
        if (!aligned_to(ptr, 4)) return PTQ4VM_ERR_ALIGN;
    if (!aligned_to(workspace, 16)) return PTQ4VM_ERR_ALIGN;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    const SumOut parameters{da, dd, ddt_bias, K * N, K};
    if (B == 0) return launch_sum_partials(nullptr, 0, K * (N + 2), parameters, stream);
    const ScanPlan plan = backward_plan(B, L, K, N);
    const BackwardSizes sizes = backward_sizes(plan, B, L, K, N);
    float *const ws = static_cast<float *>(workspace);
    const int64_t values = B * L * 2 * N;
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
        const int e2 = for_layout(plan, K, N, [&](auto ns, auto ch, auto ragged) {
            const auto go = [&](auto carry_only, int64_t chunks) {
                s.blocks = (uint32_t)(chunks * B * plan.column_blocks);
                gated_scan_backward_tokens<T, ns(), ch(), ragged(), carry_only()><<<dim3(xcd_grid(s.blocks)), dim3(64), 0, stream>>>(s);
                return check_launch("gated_scan_backward_tokens");
            };
            if (plan.chunks > 1)
                if (const int e3 = go(std::true_type{}, plan.chunks - 1)) return e3;
            s.joined = plan.chunks >= kJoin;
            if (s.joined)
                if (const int e3 = launch_join_chunks<true>(s, stream)) return e3;
            return go(std::false_type{}, plan.chunks);
        });
        if (e2) return e2;
        sum_column_blocks<T><<<dim3((unsigned)(values < (int64_t)1 << 30 ? ceil_div(values, 256) : 1 << 22)), dim3(256), 0, stream>>>(
            ws, (int)plan.column_blocks, L, values, (int)N, tokens<T>(db, L, lddb, reverse), tokens<T>(dc, L, lddc, reverse));
        return check_launch("sum_column_blocks");
    });
    if (rc != PTQ4VM_OK) return rc;
    return launch_sum_partials(ws + sizes.bc, plan.chunks * B, K * (N + 2), parameters, stream);
}

}  // extern "C"
