// Forward pass of the gated linear recurrence (gated_scan.hpp has the formulas and the layout), and its form for one token.
#include "gated_scan.hpp"

namespace {

using namespace ptq4vm;

constexpr int kTile = 16;           // tokens that are staged together
constexpr int64_t kFull = 4096;     // wavefronts from which two channels to a lane are faster: 4 to a SIMD (at 3 to a SIMD 112 us against 102)
constexpr int64_t kFullWide = 4096; // wavefronts from which a channel to a lane is faster: 4 to a SIMD (at 1.5 to a SIMD 128 us against 102)
constexpr int64_t kHeld = 6144;     // wavefronts that sequences are cut for (16384 x 768: 2048 134 us, 4096 110, 5120 103, 6144 99)

// One wavefront: 16 C channels of one sequence through the tokens of one chunk.
// STATES_ONLY: from a zero state, without outputs; leaves the chunk's end state and its sum of D, from which the chunks behind
// it know their first state: h_in(i + 1) = exp(a sum D(i)) h_in(i) + h_end(i).
// RAGGED: K or N leave lanes without a channel or a state; the states behind N are kept at zero.
// 128 sequences of 197 tokens x 768 x 16 with marks: 101 us, vector ALU 72 % busy.  1 x 16384 x 768 x 16 in chunks: 37 us for the
// end states, 9 for the join, 53 for the outputs.
template <typename T, int NS, int C, bool RAGGED, bool STATES_ONLY>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(NS * C > 8 ? 2 : 4))) void gated_scan_tokens(ScanArgs<T> p) {
    using S = ScanLane<NS, C, kTile>;
    alignas(16) __shared__ float2 steps[kTile][S::kChannels];  // D and D u
    alignas(16) __shared__ float sums[kTile][S::kChannels];    // s without its d u
    alignas(16) __shared__ float sb[kTile][S::kStates], sc[kTile][S::kStates];
    const uint32_t block = xcd_contiguous(blockIdx.x, p.blocks);
    if (block >= p.blocks) return;
    const int cb = block % p.column_blocks, bc = block / p.column_blocks, b = bc % p.B;
    const uint32_t chunk = bc / p.B;
    const int lane = threadIdx.x, q = lane & 3, cl = lane >> 2, n0 = q * NS;
    const int64_t t_begin = chunk * p.chunk_tokens, t_end = min(p.L, t_begin + p.chunk_tokens);

    float a2[C][NS], h[C][NS], sum_d[C];
    const int kc = cb * S::kChannels + cl * C;  // the quad's first channel
#pragma unroll
    for (int c = 0; c < C; c++) {
        const bool mine = !RAGGED || kc + c < p.K;
        load_channel<NS, RAGGED>(p.a, kc + c, n0, p.N, mine, a2[c]);
        sum_d[c] = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; i++) a2[c][i] = rate_of(a2[c][i]), h[c][i] = 0.0f;
        if constexpr (!STATES_ONLY) {
            if (p.joined && chunk > 0)
                load_channel<NS, RAGGED>(p.chunk_state, ((int64_t)(chunk - 1) * p.B + b) * p.K + kc + c, n0, p.N, mine, h[c]);
            else if (p.state)
                load_channel<NS, RAGGED>(p.state, (int64_t)b * p.K + kc + c, n0, p.N, mine, h[c]);
            if (!p.joined && chunk > 0) {
                float end[kJoin - 2][NS], D[kJoin - 2];
#pragma unroll
                for (int s = 0; s < kJoin - 2; s++) {
                    const int64_t channel = ((int64_t)min((uint32_t)s, chunk - 1) * p.B + b) * p.K + (mine ? kc + c : 0);
                    load_channel<NS, RAGGED>(p.chunk_state, channel, n0, p.N, mine, end[s]);
                    D[s] = p.chunk_dt[channel];
                }
#pragma unroll
                for (int s = 0; s < kJoin - 2; s++)
                    if ((uint32_t)s < chunk)
#pragma unroll
                        for (int j = 0; j < NS; j++) h[c][j] = decayed(h[c][j], a2[c][j] * D[s], end[s][j]);
            }
        }
    }

    // what this lane loads: kVec channels of a token
    const int vt = lane / S::kAcross, vk = (lane % S::kAcross) * S::kVec, k = cb * S::kChannels + vk, nk = max(0, min(S::kVec, p.K - k));
    alignas(16) __shared__ float bias[S::kChannels], skip[S::kChannels];
    if (lane < S::kChannels) {
        const int at = cb * S::kChannels + lane;
        bias[lane] = p.dt_bias && at < p.K ? p.dt_bias[at] : 0.0f;
        skip[lane] = p.d && at < p.K ? p.d[at] : 0.0f;
    }
    __syncthreads();
    T ru[S::kVec], rdt[S::kVec], rz[S::kVec], rb[S::kStateVec], rc[S::kStateVec];
    const auto fetch = [&](int64_t t0) {
        const int last = (int)min((int64_t)kTile, t_end - t0) - 1;
        load_token<S::kVec, RAGGED>(p.u, b, t0, vt, last, k, nk, ru);
        load_token<S::kVec, RAGGED>(p.dt, b, t0, vt, last, k, nk, rdt);
        if (!STATES_ONLY && p.z.data) load_token<S::kVec, RAGGED>(p.z, b, t0, vt, last, k, nk, rz);
        load_states<S, RAGGED>(p.b, b, t0, last, p.N, rb);
        if constexpr (!STATES_ONLY) load_states<S, RAGGED>(p.c, b, t0, last, p.N, rc);
    };
    fetch(t_begin);
    for (int64_t t0 = t_begin; t0 < t_end; t0 += kTile) {
        T u[S::kVec], z[S::kVec];
        const bool there = t0 + vt < t_end;  // (tokens behind the last change nothing: D = 0)
#pragma unroll
        for (int i = 0; i < S::kVec; i++) {
            u[i] = ru[i];
            if (!STATES_ONLY) z[i] = rz[i];
            const float D = softplus_of((float)rdt[i] + bias[vk + i]);
            steps[vt][vk + i] = {D, D * (float)ru[i]};
        }
        if (!there)
#pragma unroll
            for (int i = 0; i < S::kVec; i++) steps[vt][vk + i] = {0.0f, 0.0f};
        keep_states<S>(rb, sb);
        if constexpr (!STATES_ONLY) keep_states<S>(rc, sc);
        __syncthreads();
        if (t0 + kTile < t_end) fetch(t0 + kTile);  // in flight under this tile's steps
        const int groups = (int)((min((int64_t)kTile, t_end - t0) + 3) / 4);
        for (int g = 0; g < groups; g++) {
            static_assert(kMark == 8 && kTile == 16, "a mark before every other group of four tokens");
            if (!STATES_ONLY && p.marks && g % 2 == 0)
#pragma unroll
                for (int c = 0; c < C; c++)
                    store_channel<NS, RAGGED>(p.marks, ((t0 / kMark + g / 2) * p.B + b) * p.K + kc + c, n0, p.N, kc + c < p.K, h[c]);
#pragma unroll
            for (int s = 0; s < 4; s++) {
                const int t = 4 * g + s;
                float B[NS], CC[NS], v[C];
#pragma unroll
                for (int i = 0; i < NS; i++) {
                    B[i] = sb[t][n0 + i];
                    if (!STATES_ONLY) CC[i] = sc[t][n0 + i];
                }
#pragma unroll
                for (int c = 0; c < C; c++) {
                    const float2 D = steps[t][cl * C + c];
                    v[c] = 0.0f;
                    if (STATES_ONLY) sum_d[c] += D.x;
#pragma unroll
                    for (int i = 0; i < NS; i++) {
                        h[c][i] = fmaf(__builtin_amdgcn_exp2f(a2[c][i] * D.x), h[c][i], D.y * B[i]);
                        if (RAGGED) h[c][i] = n0 + i < p.N ? h[c][i] : 0.0f;
                        if (!STATES_ONLY) v[c] = fmaf(h[c][i], CC[i], v[c]);
                    }
                }
                if constexpr (!STATES_ONLY) sums[t][cl * C + q % C] = quad_sums<C>(v, q);  // (lanes of the same place write the same value)
            }
        }
        __syncthreads();
        if constexpr (!STATES_ONLY) {
            float y[S::kVec];
#pragma unroll
            for (int i = 0; i < S::kVec; i++) y[i] = fmaf(skip[vk + i], (float)u[i], sums[vt][vk + i]);
            if (p.z.data)
#pragma unroll
                for (int i = 0; i < S::kVec; i++) y[i] *= (float)z[i] * sigmoid_of((float)z[i]);
            if (there) store_token<S::kVec, RAGGED>(p.y, b, t0, vt, k, nk, y);
        }
    }
    float *const out = STATES_ONLY ? p.chunk_state + (int64_t)chunk * p.B * p.K * p.N : t_end == p.L ? p.state_out : nullptr;
    if (out)
#pragma unroll
        for (int c = 0; c < C; c++) {
            store_channel<NS, RAGGED>(out, (int64_t)b * p.K + kc + c, n0, p.N, kc + c < p.K, h[c]);
            if (STATES_ONLY && q == 0 && kc + c < p.K) p.chunk_dt[((int64_t)chunk * p.B + b) * p.K + kc + c] = sum_d[c];
        }
}

// The same with a channel's 16 states in one lane, 64 channels to a wavefront: no sums over lanes, and the products D u b of a
// token, an outer product of 4 channels and 4 states for every quad of lanes, come with the addition to e^{D a} h from the matrix
// pipe (v_mfma_f32_4x4x1: 16 products for an instruction of a lane's 4, and the vector ALU is what bounds this kernel).  An exponential and three
// instructions a state and a quarter, against an exponential, four and the sums' seven eighths: 256 x 197 x 1536 takes 274 us, with
// two channels to a lane 287.  (118 registers, four wavefronts to a SIMD; squeezed into five or six it spills: 377 and 415 us.)
constexpr int kWideTile = 8;  // tokens that are staged together
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T, bool RAGGED>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(RAGGED && sizeof(T) == 4 ? 3 : 4))) void gated_scan_wide(ScanArgs<T> p) {
    using S = ScanLane<4, 4, kWideTile>;
    constexpr int V = S::kVec;
    static_assert(S::kChannels == 64 && S::kStates == 16, "a lane to a channel");
    alignas(16) __shared__ float steps[kWideTile][64];  // D; then s without its d u
    alignas(16) __shared__ float inputs[kWideTile][64];  // D u
    alignas(16) __shared__ float sb[kWideTile][4][4];    // state n at [n % 4][n / 4]: what lane n % 4 of a quad gives to the products
    alignas(16) __shared__ float sc[kWideTile][16];
    alignas(16) __shared__ float bias[64], skip[64];
    const uint32_t block = xcd_contiguous(blockIdx.x, p.blocks);
    if (block >= p.blocks) return;
    const int cb = block % p.column_blocks, b = block / p.column_blocks, lane = threadIdx.x, kc = cb * 64 + lane;
    const bool mine = !RAGGED || kc < p.K;

    f32x4 a2[4], h[4];
    const auto load_states_of = [&](const float *from, int64_t channel, f32x4 (&to)[4]) {
        float v[16];
        load_channel<16, true>(from, channel, 0, RAGGED ? p.N : 16, mine, v);
#pragma unroll
        for (int i = 0; i < 16; i++) to[i / 4][i % 4] = v[i];
    };
    const auto store_states_of = [&](float *to, int64_t channel) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; i++) v[i] = h[i / 4][i % 4];
        store_channel<16, true>(to, channel, 0, RAGGED ? p.N : 16, mine, v);
    };
    load_states_of(p.a, kc, a2);
#pragma unroll
    for (int m = 0; m < 4; m++) {
#pragma unroll
        for (int i = 0; i < 4; i++) a2[m][i] = rate_of(a2[m][i]);
        h[m] = 0.0f;
    }
    if (p.state) load_states_of(p.state, (int64_t)b * p.K + kc, h);
    const int vt = lane / S::kAcross, vk = (lane % S::kAcross) * V, k = cb * 64 + vk, nk = max(0, min(V, p.K - k));
    bias[lane] = p.dt_bias && kc < p.K ? p.dt_bias[kc] : 0.0f;
    skip[lane] = p.d && kc < p.K ? p.d[kc] : 0.0f;
    __syncthreads();
    T ru[V], rdt[V], rz[V], rb[S::kStateVec], rc[S::kStateVec];
    const auto fetch = [&](int64_t t0) {
        const int last = (int)min((int64_t)kWideTile, p.L - t0) - 1;
        load_token<V, RAGGED>(p.u, b, t0, vt, last, k, nk, ru);
        load_token<V, RAGGED>(p.dt, b, t0, vt, last, k, nk, rdt);
        if (p.z.data) load_token<V, RAGGED>(p.z, b, t0, vt, last, k, nk, rz);
        load_states<S, RAGGED>(p.b, b, t0, last, p.N, rb);
        load_states<S, RAGGED>(p.c, b, t0, last, p.N, rc);
    };
    fetch(0);
    for (int64_t t0 = 0; t0 < p.L; t0 += kWideTile) {
        T u[V], z[V];
        const bool there = t0 + vt < p.L;  // (tokens behind the last change nothing: D = 0)
#pragma unroll
        for (int i = 0; i < V; i++) {
            u[i] = ru[i];
            z[i] = rz[i];
            const float D = softplus_of((float)rdt[i] + bias[vk + i]);
            steps[vt][vk + i] = D, inputs[vt][vk + i] = D * (float)ru[i];
        }
        if (!there)
#pragma unroll
            for (int i = 0; i < V; i++) steps[vt][vk + i] = inputs[vt][vk + i] = 0.0f;
#pragma unroll
        for (int i = 0; i < S::kStateVec; i++) {
            const int n = lane % 8 * S::kStateVec + i;
            sb[lane / 8][n % 4][n / 4] = (float)rb[i];
            sc[lane / 8][n] = (float)rc[i];
        }
        __syncthreads();
        if (t0 + kWideTile < p.L) fetch(t0 + kWideTile);  // in flight under this tile's steps
        static_assert(kWideTile == kMark, "a mark before every tile");
        if (p.marks) store_states_of(p.marks, ((t0 / kMark) * p.B + b) * p.K + kc);
#pragma unroll
        for (int t = 0; t < kWideTile; t++) {
            const float D = steps[t][lane], Du = inputs[t][lane];
            f32x4 v = 0.0f;
#pragma unroll
            for (int m = 0; m < 4; m++) {
                f32x4 e;
#pragma unroll
                for (int i = 0; i < 4; i++) e[i] = __builtin_amdgcn_exp2f(a2[m][i] * D) * h[m][i];
                h[m] = __builtin_amdgcn_mfma_f32_4x4x1f32(sb[t][lane & 3][m], Du, e, 0, 0, 0);
                if (RAGGED)
#pragma unroll
                    for (int i = 0; i < 4; i++) h[m][i] = m * 4 + i < p.N ? h[m][i] : 0.0f;
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = fmaf(h[m][i], sc[t][m * 4 + i], v[i]);
            }
            steps[t][lane] = (v[0] + v[1]) + (v[2] + v[3]);
        }
        __syncthreads();
        float y[V];
#pragma unroll
        for (int i = 0; i < V; i++) y[i] = fmaf(skip[vk + i], (float)u[i], steps[vt][vk + i]);
        if (p.z.data)
#pragma unroll
            for (int i = 0; i < V; i++) y[i] *= (float)z[i] * sigmoid_of((float)z[i]);
        if (there) store_token<V, RAGGED>(p.y, b, t0, vt, k, nk, y);
        __syncthreads();
    }
    if (p.state_out) store_states_of(p.state_out, (int64_t)b * p.K + kc);
}

// Few short sequences of few channels, up to 16 states: a lane takes one state, a wavefront 4 channels of one tile of tokens, a
// workgroup all tiles of a sequence.  The tiles run side by side from a zero state, tell each other through LDS what they leave and
// their sums of D, and run again from their true first states on what is staged already: one launch, and of the tokens'
// latencies those of two tiles, on four times the compute units that quads of lanes would fill (sums over 16 lanes cost four
// additions a token for it).  One image, 197 tokens x 384 channels x 16 states: 12 us in chunks (two launches), 10.8 us with quads of
// lanes here, and 6.0 us so.
constexpr int kShortTiles = 16, kShortStates = 16, kShortChannels = 4;
template <typename T, bool RAGGED>
__global__ __launch_bounds__(kShortTiles * 64) void gated_scan_short(ScanArgs<T> p) {
    struct Tile {
        float2 steps[kTile][kShortChannels];  // D and D u; then s without its d u in D's place
        float b[kTile][kShortStates], c[kTile][kShortStates];
        float end[kShortChannels][kShortStates], sum_d[kShortChannels];
    };
    alignas(16) __shared__ Tile tiles[kShortTiles];
    const uint32_t block = xcd_contiguous(blockIdx.x, p.blocks);
    if (block >= p.blocks) return;
    const int cb = block % p.column_blocks, b = block / p.column_blocks, lane = threadIdx.x & 63;
    Tile &tile = tiles[threadIdx.x >> 6];
    const int64_t t0 = (int64_t)(threadIdx.x >> 6) * kTile;
    const int last = (int)min((int64_t)kTile, p.L - t0) - 1;
    // what the lane loads: one channel of a token, four states of a token's b and c
    const int vt = lane >> 2, vc = lane & 3, k = cb * kShortChannels + vc, from = min(vt, last);
    const bool column = !RAGGED || k < p.K;
    const float x = column ? (float)*in_tile(p.dt, b, t0, from, k) : 0.0f, u = column ? (float)*in_tile(p.u, b, t0, from, k) : 0.0f;
    const float z = column && p.z.data ? (float)*in_tile(p.z, b, t0, from, k) : 0.0f;
    T rb[4], rc[4];
    const int n_load = RAGGED ? max(0, min(4, p.N - vc * 4)) : 4;
    load_first<4>(in_tile(p.b, b, t0, from, vc * 4), n_load, rb);
    load_first<4>(in_tile(p.c, b, t0, from, vc * 4), n_load, rc);
    const float bias = column && p.dt_bias ? p.dt_bias[k] : 0.0f, skip = column && p.d ? p.d[k] : 0.0f;
    // what it runs: one state
    const int n = lane & 15, cl = lane >> 4, kc = cb * kShortChannels + cl;
    const bool mine = !RAGGED || (kc < p.K && n < p.N);
    const int64_t state = (int64_t)kc * p.N + n;
    const float a2 = mine ? rate_of(p.a[state]) : 0.0f;
    const float start = mine && p.state ? p.state[(int64_t)b * p.K * p.N + state] : 0.0f;

    const float D_in = softplus_of(x + bias);
    tile.steps[vt][vc] = {vt <= last ? D_in : 0.0f, vt <= last ? D_in * u : 0.0f};  // (tokens behind the last change nothing)
#pragma unroll
    for (int i = 0; i < 4; i++) tile.b[vt][vc * 4 + i] = vt <= last ? (float)rb[i] : 0.0f, tile.c[vt][vc * 4 + i] = (float)rc[i];
    __syncthreads();
    float h = 0.0f, sum = 0.0f;
    const auto advance = [&](int t) {
        const float2 D = tile.steps[t][cl];
        h = fmaf(__builtin_amdgcn_exp2f(a2 * D.x), h, D.y * tile.b[t][n]);
        if (RAGGED) h = mine ? h : 0.0f;
        return D.x;
    };
#pragma unroll
    for (int t = 0; t < kTile; t++) sum += advance(t);
    tile.end[cl][n] = h;
    if (n == 0) tile.sum_d[cl] = sum;
    __syncthreads();
    h = start;
    for (int s = 0; s < (int)(threadIdx.x >> 6); s++) h = decayed(h, a2 * tiles[s].sum_d[cl], tiles[s].end[cl][n]);
#pragma unroll
    for (int t = 0; t < kTile; t++) {
        if (p.marks && t % kMark == 0 && t <= last && mine) p.marks[((t0 + t) / kMark * p.B + b) * p.K * p.N + state] = h;
        advance(t);
        tile.steps[t][cl].x = group_sum(RAGGED && n >= p.N ? 0.0f : h * tile.c[t][n], 16);  // (the lanes' reads of D are done: one wavefront, LDS in order)
    }
    __syncthreads();
    if (vt <= last && column) {
        float y = fmaf(skip, u, tile.steps[vt][vc].x);
        if (p.z.data) y *= z * sigmoid_of(z);
        *in_tile(p.y, b, t0, vt, k) = (T)y;
    }
    if (p.state_out && t0 + last + 1 == p.L && mine) p.state_out[(int64_t)b * p.K * p.N + state] = h;
}

// One token of every sequence: bound by the states, which are read and written once (128 bytes of a channel's 16 against 10
// of everything else).  LANES lanes take a channel, 4 adjacent states each (16 bytes), a quad the next 16 of it after that; a
// workgroup 256 / LANES channels of one sequence.  A lane's states are read before they are written by it alone, so state_out may be
// the state's own buffer.  1000 sequences x 1536 x 16: 44 us, 4.8 TB/s; 3868 x 1408 x 4: 44 us, 5.0 TB/s (88 us with a state to each
// lane of a quad).
template <typename T, int LANES, int GROUPS, bool RAGGED>
__global__ __launch_bounds__(256) void gated_scan_one_token(ScanArgs<T> p) {
    const int b = blockIdx.x / p.column_blocks, k = (int)(blockIdx.x - b * p.column_blocks) * (256 / LANES) + threadIdx.x / LANES;
    const int q = threadIdx.x % LANES;
    if (k >= p.K) return;  // (all lanes of a channel)
    float h[GROUPS][4], a[GROUPS][4];
    T B[GROUPS][4], CC[GROUPS][4];
    int n[GROUPS];
    const int N = RAGGED ? p.N : 4 * LANES * GROUPS;
    const int64_t channel = (int64_t)k * N + q * 4, at = (int64_t)b * p.K * N + channel;
    const T *const from_b = p.b.at(b, 0) + q * 4, *const from_c = p.c.at(b, 0) + q * 4;
#pragma unroll
    for (int j = 0; j < GROUPS; j++) {
        const int first = j * LANES * 4;
        n[j] = RAGGED ? max(0, min(4, N - first - q * 4)) : 4;
        load_first<4>(p.state + at + first, n[j], h[j]);
        load_first<4>(p.a + channel + first, n[j], a[j]);
        load_first<4>(from_b + first, n[j], B[j]);
        load_first<4>(from_c + first, n[j], CC[j]);
    }
    const float u = (float)p.u.at(b, 0)[k];
    const float D = softplus_of((float)p.dt.at(b, 0)[k] + (p.dt_bias ? p.dt_bias[k] : 0.0f)), Du = D * u;
    const float z = p.z.data ? (float)p.z.at(b, 0)[k] : 0.0f;
    float v = 0.0f;
#pragma unroll
    for (int j = 0; j < GROUPS; j++) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            h[j][i] = fmaf(__builtin_amdgcn_exp2f(rate_of(a[j][i]) * D), h[j][i], Du * (float)B[j][i]);
            v = i < n[j] ? fmaf(h[j][i], (float)CC[j][i], v) : v;
        }
        store_first<4>(p.state_out + at + j * LANES * 4, n[j], h[j]);
    }
    if constexpr (LANES >= 2) v = add_dpp<0xB1>(v);
    if constexpr (LANES == 4) v = add_dpp<0x4E>(v);
    if (p.d) v = fmaf(p.d[k], u, v);
    if (p.z.data) v *= z * sigmoid_of(z);
    if (q == 0) p.y.at(b, 0)[k] = (T)v;
}

ScanPlan forward_plan(int64_t B, int64_t L, int64_t K, int64_t N) {
    if (N > 8 && N <= 16 && B * ceil_div(K, 64) >= kFullWide) {
        const int64_t column_blocks = ceil_div(K, 64);
        return {4, 4, column_blocks, ceil_div(L, kWideTile) * kWideTile, 1};
    }
    // (32 x 197 x 768 whole and one channel to a lane 38 us, in chunks and two 52; 16 x 4000 x 1536 708 and 629)
    return scan_plan(B, L, K, N, kFull, kHeld, kTile, L < 1024);
}

// Whether the tiles of a sequence run side by side in one workgroup: up to three workgroups on a compute unit (197 tokens x 1536
// channels, us against chunks or one wavefront a sequence: 1 image 8.1 / 12.0, 2 images 11.9 / 15.2, 3 images 18.5 / 16.7)
bool is_short(int64_t B, int64_t L, int64_t K, int64_t N) {
    return N <= kShortStates && L > kTile && L <= kShortTiles * kTile && B * ceil_div(K, kShortChannels) <= 768;
}

int check_scan(int dtype, const void *u, const void *dt, const float *a, const void *b, const void *c, const float *d, const void *z, const float *dt_bias, void *y,
               int64_t B, int64_t L, int64_t K, int64_t N, int64_t ldu, int64_t lddt, int64_t ldb, int64_t ldc, int64_t ldz, int64_t ldy) {
    if (!valid_dtype(dtype)) return PTQ4VM_ERR_SHAPE;
    if (!a || (B != 0 && (!u || !dt || !b || !c || !y))) return PTQ4VM_ERR_NULL;  // (a matrix of no rows has no address)
    if (!scan_sizes(B, L, K, N)) return PTQ4VM_ERR_SHAPE;
    if (ldu < K || lddt < K || ldb < N || ldc < N || (z && ldz < K) || ldy < K) return PTQ4VM_ERR_STRIDE;
    for (const int64_t ld : {ldu, lddt, ldb, ldc, z ? ldz : 0, ldy})
        if (ld >= kMaxPitch) return PTQ4VM_ERR_STRIDE;
    const uintptr_t e = dtype_bytes(dtype);
    if (!aligned_to(u, e) || !aligned_to(dt, e) || !aligned_to(b, e) || !aligned_to(c, e) || !aligned_to(z, e) || !aligned_to(y, e) || !aligned_to(a, 4) ||
        !aligned_to(d, 4) || !aligned_to(dt_bias, 4))
        return PTQ4VM_ERR_ALIGN;
    return PTQ4VM_OK;
}

template <typename T>
ScanArgs<T> scan_args(const void *u, const void *dt, const float *a, const void *b, const void *c, const float *d, const void *z, const float *dt_bias, void *y,
                      bool reverse, int64_t B, int64_t L, int64_t K, int64_t N, int64_t ldu, int64_t lddt, int64_t ldb, int64_t ldc, int64_t ldz, int64_t ldy) {
    ScanArgs<T> s{};
    s.u = tokens<T>(u, L, ldu, reverse), s.dt = tokens<T>(dt, L, lddt, reverse), s.b = tokens<T>(b, L, ldb, reverse), s.c = tokens<T>(c, L, ldc, reverse);
    s.z = tokens<T>(z, L, ldz, reverse), s.y = tokens<T>(y, L, ldy, reverse);
    s.a = a, s.d = d, s.dt_bias = dt_bias, s.B = (int)B, s.K = (int)K, s.N = (int)N, s.L = L;
    return s;
}

}  // namespace

extern "C" {

int64_t ptq4vm_gated_scan_workspace(int64_t B, int64_t L, int64_t K, int64_t N) {
    if (!scan_sizes(B, L, K, N) || B == 0) return 0;
    const ScanPlan plan = forward_plan(B, L, K, N);
    return plan.chunks > 1 && !is_short(B, L, K, N) ? plan.chunks * B * K * (N + 1) * 4 : 0;
}

int ptq4vm_gated_scan(int dtype, const void *u, const void *dt, const float *a, const void *b, const void *c, const float *d, const void *z, const float *dt_bias,
                      const float *state, void *y, float *state_out, float *marks, void *workspace, int64_t workspace_bytes, int reverse, int64_t B, int64_t L, int64_t K,
                      int64_t N, int64_t ldu, int64_t lddt, int64_t ldb, int64_t ldc, int64_t ldz, int64_t ldy, void *stream_) {
    const int rc = check_scan(dtype, u, dt, a, b, c, d, z, dt_bias, y, B, L, K, N, ldu, lddt, ldb, ldc, ldz, ldy);
    if (rc != PTQ4VM_OK) return rc;
    const int64_t need = ptq4vm_gated_scan_workspace(B, L, K, N);
    if (need > 0 && !workspace) return PTQ4VM_ERR_NULL;
    if (workspace_bytes < need) return PTQ4VM_ERR_SHAPE;
    if (!aligned_to(state, 4) || !aligned_to(state_out, 4) || !aligned_to(marks, 4) || !aligned_to(workspace, 16)) return PTQ4VM_ERR_ALIGN;
    if (B == 0) return PTQ4VM_OK;
    if (overlap(state, state_out, B * K * N * 4)) return PTQ4VM_ERR_OVERLAP;  // (the chunks of a sequence read it in their own time)
    const ScanPlan plan = forward_plan(B, L, K, N);
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    return for_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        ScanArgs<T> s = scan_args<T>(u, dt, a, b, c, d, z, dt_bias, y, reverse, B, L, K, N, ldu, lddt, ldb, ldc, ldz, ldy);
        s.state = state, s.state_out = state_out, s.marks = marks;
        s.chunk_state = static_cast<float *>(workspace), s.chunk_dt = s.chunk_state + (plan.chunks > 1 ? plan.chunks * B * K * N : 0);
        s.column_blocks = (int)plan.column_blocks, s.chunk_tokens = plan.chunk_tokens;
        if (is_short(B, L, K, N)) {
            s.column_blocks = (int)ceil_div(K, kShortChannels), s.blocks = (uint32_t)(B * s.column_blocks);
            const dim3 grid(xcd_grid(s.blocks)), block((unsigned)ceil_div(L, kTile) * 64);
            if (N == kShortStates && K % kShortChannels == 0)
                gated_scan_short<T, false><<<grid, block, 0, stream>>>(s);
            else
                gated_scan_short<T, true><<<grid, block, 0, stream>>>(s);
            return check_launch("gated_scan_short");
        }
        if (plan.channels == 4) {
            s.blocks = (uint32_t)(B * plan.column_blocks);
            if (N == 16 && K % 64 == 0)
                gated_scan_wide<T, false><<<dim3(xcd_grid(s.blocks)), dim3(64), 0, stream>>>(s);
            else
                gated_scan_wide<T, true><<<dim3(xcd_grid(s.blocks)), dim3(64), 0, stream>>>(s);
            return check_launch("gated_scan_wide");
        }
        return for_layout(plan, K, N, [&](auto ns, auto ch, auto ragged) {
            const auto go = [&](auto states_only, int64_t chunks) {
                s.blocks = (uint32_t)(chunks * B * plan.column_blocks);
                gated_scan_tokens<T, ns(), ch(), ragged(), states_only()><<<dim3(xcd_grid(s.blocks)), dim3(64), 0, stream>>>(s);
                return check_launch("gated_scan_tokens");
            };
            if (plan.chunks > 1)  // (nobody asks for the last chunk's)
                if (const int e = go(std::true_type{}, plan.chunks - 1)) return e;
            s.chunks = (uint32_t)plan.chunks, s.joined = plan.chunks >= kJoin;
            if (s.joined)
                if (const int e = launch_join_chunks<false>(s, stream)) return e;
            return go(std::false_type{}, plan.chunks);
        });
    });
}

int ptq4vm_gated_scan_step(int dtype, const void *u, const void *dt, const float *a, const void *b, const void *c, const float *d, const void *z, const float *dt_bias,
                           const float *state, void *y, float *state_out, int64_t B, int64_t K, int64_t N, int64_t ldu, int64_t lddt, int64_t ldb, int64_t ldc,
                           int64_t ldz, int64_t ldy, void *stream_) {
    const int rc = check_scan(dtype, u, dt, a, b, c, d, z, dt_bias, y, B, 1, K, N, ldu, lddt, ldb, ldc, ldz, ldy);
    if (rc != PTQ4VM_OK) return rc;
    if (B != 0 && (!state || !state_out)) return PTQ4VM_ERR_NULL;
    if (!aligned_to(state, 4) || !aligned_to(state_out, 4)) return PTQ4VM_ERR_ALIGN;
    if (!grid_fits(B * ceil_div(K, 64), 256)) return PTQ4VM_ERR_SHAPE;
    if (B == 0) return PTQ4VM_OK;
    if (state != state_out && overlap(state, state_out, B * K * N * 4)) return PTQ4VM_ERR_OVERLAP;
    hipStream_t stream = static_cast<hipStream_t>(stream_);
    return for_dtype(dtype, [&](auto zero) {
        using T = decltype(zero);
        ScanArgs<T> s = scan_args<T>(u, dt, a, b, c, d, z, dt_bias, y, false, B, 1, K, N, ldu, lddt, ldb, ldc, ldz, ldy);
        s.state = state, s.state_out = state_out;
        using std::integral_constant;
        const auto go = [&](auto lanes, auto groups, auto ragged) {
            s.column_blocks = (int)ceil_div(K, 256 / lanes());
            gated_scan_one_token<T, lanes(), groups(), ragged()><<<dim3((unsigned)(B * s.column_blocks)), dim3(256), 0, stream>>>(s);
            return check_launch("gated_scan_one_token");
        };
        const auto with = [&](auto lanes, auto groups) { return N == 4 * lanes() * groups() ? go(lanes, groups, std::false_type{}) : go(lanes, groups, std::true_type{}); };
        constexpr integral_constant<int, 1> one{};
        constexpr integral_constant<int, 2> two{};
        constexpr integral_constant<int, 4> four{};
        if (N <= 4) return with(one, one);
        if (N <= 8) return with(two, one);
        if (N <= 16) return with(four, one);
        if (N <= 32) return with(four, two);
        if (N <= 48) return with(four, integral_constant<int, 3>{});
        return with(four, four);
    });
}

}  // extern "C"
