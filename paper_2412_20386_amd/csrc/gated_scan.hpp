// The gated linear recurrence over tokens: what its kernels share.  For one sequence, channel k and state n:
//   D = softplus(dt + dt_bias),  h_t = exp(D a[k,n]) h_{t-1} + D u b[t,n],  s = sum_n c[t,n] h_t + d[k] u,  y = s z / (1 + e^-z)
// (the state equations of Sec. 2.1 with the input matrix to first order, Eqs. (1)-(8); u, dt, z and y have K columns, b and c
// have N, shared by all channels).
//
// A quad of lanes holds the states of C channels, NS of each to a lane, so that a wavefront runs 16 C channels through the
// tokens with the states in registers, sums over n are two DPP additions, and what belongs to a token and channel (softplus,
// gate) is computed once, by the lane that loaded it, and passed through LDS.  Bound by the vector ALU: a token, channel and
// state cost one exponential and four other instructions, against 8 bytes for all states of a channel.
#pragma once
#include <type_traits>

#include "token_ops.hpp"

namespace ptq4vm {

constexpr int kMark = PTQ4VM_SCAN_TILE;  // tokens from one mark to the next

template <typename T>
struct ScanArgs {
    Tokens<T> u, dt, b, c, z, y;
    const float *a, *d, *dt_bias, *state;
    float *state_out, *marks;
    float *chunk_state, *chunk_dt;  // [chunks][B][K][N] and [chunks][B][K]: a chunk's own end state and its sum of D
    // backward
    Tokens<T> dy, du, ddt, dz;
    float *partial_bc, *partial_a;
    int B, K, N, column_blocks;
    int64_t L, chunk_tokens;  // (whole tiles)
    uint32_t chunks, blocks;
    bool joined;  // chunk_state holds what comes into the next chunk, not what each leaves by itself
};

// What the layout of a wavefront makes of its lane number, where TOKENS tokens are staged at once
template <int NS, int C, int TOKENS>
struct ScanLane {
    static constexpr int kChannels = 16 * C;                // of a wavefront
    static constexpr int kStates = 4 * NS;                  // that a quad has room for
    static constexpr int kAcross = 64 / TOKENS;             // lanes side by side that load a token
    static constexpr int kVec = kChannels / kAcross;        // channels that a lane loads of its token
    static constexpr int kStateVec = (kStates * TOKENS + 63) / 64;  // states that a lane loads of b and of c
};

constexpr float kLog2e = 1.44269504088896340736f;
// a log2(e), so that e^{D a} = 2^{D rate}.  Not below the lowest number: what is staged behind the last token and joined behind the last chunk changes
// nothing because its D is 0, and 0 times minus infinity would be NaN (so would minus infinity times a gradient of 0).  2^{D rate} is 0 either
// way, for every D from 1e-36 on.
__device__ __forceinline__ float rate_of(float a) {
    const float rate = a * kLog2e;
    return rate < -3.402823466e38f ? -3.402823466e38f : rate;  // (a NaN stays one)
}

// 2^x h + end, for the decay over a whole chunk: with a rate above 0 it leaves the range of fp32 where h is 0 or small and the product does not, so
// it is multiplied in as its square root, twice.  (Where x is above 254, h has to be subnormal for the product to be a number.)
__device__ __forceinline__ float decayed(float h, float x, float end) {
    const float root = __builtin_amdgcn_exp2f(fminf(0.5f * x, 127.0f));
    return fmaf(h * root, root, end);
}

// States of a quad's lane: the power of two that has room for N
inline int states_per_lane(int64_t N) { return N <= 4 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }

// How a problem is cut: one chunk of tokens per sequence from 1024 wavefronts on, else chunks for `held` wavefronts, but no more of them than
// one for every 32 tokens begun (so of 17 at least), of whole tiles; two channels to a lane (fewer instructions for each) where that still
// leaves `full` wavefronts; not at the price of chunks if `whole`.  Above 16 states there is one channel to a lane only.  Whole and in chunks, us,
// forward / backward: 16 x 4000 x 1024 x 32 (1024 wavefronts) 756 / 3604 and 791 / 2199, with 64 states 1153 / 4460 and 1248 / 5021; 24 x 2000 x
// 1024 x 32 518 / 1881 and 534 / 1623; 31 sequences of them 514 / 1917 and 651 / 2149; 64 x 197 x 512 x 32 56 / 200 and 84 / 248.
// From kJoin chunks on, a kernel of its own runs through them; up to there each wavefront does, all loads in flight.
constexpr int kMostChunks = 256, kJoin = 9;
struct ScanPlan {
    int channels, states;
    int64_t column_blocks, chunk_tokens, chunks;
};
inline ScanPlan scan_plan(int64_t B, int64_t L, int64_t K, int64_t N, int64_t full, int64_t held, int tile, bool whole) {
    const int64_t most = ceil_div(L, 32) < kMostChunks ? ceil_div(L, 32) : kMostChunks;
    const auto cut = [&](int64_t waves) { return waves >= 1024 ? (int64_t)1 : ceil_div(held, waves > 0 ? waves : 1) < most ? ceil_div(held, waves > 0 ? waves : 1) : most; };
    const int64_t pairs = B * ceil_div(K, 32), singles = B * ceil_div(K, 16);
    ScanPlan p{N <= 16 && (whole && cut(singles) == 1 ? pairs : pairs * cut(pairs)) >= full ? 2 : 1, states_per_lane(N), 0, 0, 0};
    p.column_blocks = ceil_div(K, 16 * p.channels);
    p.chunk_tokens = ceil_div(ceil_div(L, cut(B * p.column_blocks)), tile) * tile;
    p.chunks = ceil_div(L, p.chunk_tokens);
    return p;
}

// f(NS, C, RAGGED): ragged where a wavefront's channels or a quad's states are not all there
template <typename F>
int for_layout(const ScanPlan &p, int64_t K, int64_t N, F &&f) {
    using std::bool_constant;
    using std::integral_constant;
    const auto with = [&](auto ns, auto c) { return N == 4 * ns() && K % (16 * c()) == 0 ? f(ns, c, bool_constant<false>{}) : f(ns, c, bool_constant<true>{}); };
    constexpr integral_constant<int, 1> one{};
    constexpr integral_constant<int, 2> two{};
    constexpr integral_constant<int, 4> four{};
    const auto pairs = [&](auto ns) { return p.channels == 2 ? with(ns, two) : with(ns, one); };
    switch (p.states) {
        case 1: return pairs(one);
        case 2: return pairs(two);
        case 4: return pairs(four);
        case 8: return with(integral_constant<int, 8>{}, one);
        default: return with(integral_constant<int, 16>{}, one);
    }
}

// Sizes that every entry point takes
inline bool scan_sizes(int64_t B, int64_t L, int64_t K, int64_t N) {
    return B >= 0 && L > 0 && K > 0 && N > 0 && N <= PTQ4VM_MAX_SCAN_N && L <= kMaxTokenRows && K <= kMaxTokenRows / 256 && (B == 0 || B <= kMaxTokenRows / L) &&
           B * ceil_div(K, 16) <= kMaxTokenRows / 64;
}

// Addresses of a tile are its first token's, the same for all lanes, and a lane's own 32-bit offset from there: 64-bit ones for
// every lane and matrix would be kept in registers.  (Pitches are below kMaxPitch for it.)
constexpr int64_t kMaxPitch = (int64_t)1 << 26;
template <typename T>
__device__ __forceinline__ T *in_tile(const Tokens<T> &v, int b, int64_t t0, int token, int column) {
    return v.at(b, t0) + (token * (int)v.token + column);
}
// b or c of one tile: a lane loads kStateVec states of one token, and keeps them in LDS ([TOKENS][kStates] floats), zero behind
// N and behind the last token.  (Where the states are fewer than the lanes, the others repeat them.)
template <typename S, bool RAGGED, typename T>
__device__ __forceinline__ void load_states(const Tokens<T> &v, int b, int64_t t0, int last, int N, T (&raw)[S::kStateVec]) {
    constexpr int V = S::kStateVec, kLanes = S::kStates / V;
    const int lane = threadIdx.x & 63, token = lane / kLanes % (64 / S::kAcross), n0 = lane % kLanes * V;
    const T *const from = in_tile(v, b, t0, min(token, last), n0);
    if constexpr (RAGGED)
        load_first<V>(from, max(0, min(V, N - n0)), raw);
    else
        load_whole<V>(from, raw);
    if (token > last)
#pragma unroll
        for (int i = 0; i < V; i++) raw[i] = (T)0.0f;
}
template <typename S, typename T>
__device__ __forceinline__ void keep_states(const T (&raw)[S::kStateVec], float (*to)[S::kStates]) {
    constexpr int V = S::kStateVec, kLanes = S::kStates / V;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < V; i++) to[lane / kLanes % (64 / S::kAcross)][lane % kLanes * V + i] = (float)raw[i];
}
// V channels from column k on, n of them inside K, of a tile's token; behind the tile's last token the last one's
template <int V, bool RAGGED, typename T>
__device__ __forceinline__ void load_token(const Tokens<T> &v, int b, int64_t t0, int token, int last, int k, int n, T (&raw)[V]) {
    const T *const from = in_tile(v, b, t0, min(token, last), k);
    if constexpr (RAGGED)
        load_first<V>(from, n, raw);
    else
        load_whole<V>(from, raw);
}
template <int V, bool RAGGED, typename T>
__device__ __forceinline__ void store_token(const Tokens<T> &v, int b, int64_t t0, int token, int k, int n, const float (&out)[V]) {
    store_first<V>(in_tile(v, b, t0, token, k), RAGGED ? n : V, out);
}

// NS states of one channel in a [.., K, N] array; `there`: the channel is one of K
template <int NS, bool RAGGED>
__device__ __forceinline__ void load_channel(const float *p, int64_t channel, int n0, int N, bool there, float (&v)[NS]) {
    if constexpr (RAGGED)
        load_first<NS>(p + (there ? channel : 0) * N + n0, there ? max(0, min(NS, N - n0)) : 0, v);
    else
        load_whole<NS>(p + channel * (4 * NS) + n0, v);
}
template <int NS, bool RAGGED>
__device__ __forceinline__ void store_channel(float *p, int64_t channel, int n0, int N, bool there, const float (&v)[NS]) {
    if constexpr (RAGGED) {
        if (there) store_first<NS>(p + channel * N + n0, max(0, min(NS, N - n0)), v);
    } else {
        store_first<NS>(p + channel * (4 * NS) + n0, NS, v);
    }
}

namespace {

// Runs through the chunks of a sequence for every state.  A chunk's slot i holds what it leaves by itself, end(i), and its sum of D;
// in(i + 1) = exp(a sum D(i)) in(i) + end(i) replaces end(i) (the first chunk's in is the state, or 0).  BACKWARD: the same from
// the last chunk to the first.  32 lanes take adjacent states, up to 16 of those groups a run of chunks each: a run's values are
// loaded at once, the runs are joined through LDS, and then the run writes what comes into its chunks.
constexpr int kJoinStates = 32, kJoinRuns = 16, kJoinRun = kMostChunks / kJoinRuns;
__host__ __device__ inline int join_length(int steps) { return steps <= 4 * kJoinRuns ? 4 : steps <= 8 * kJoinRuns ? 8 : kJoinRun; }  // (few runs: they are joined one after the other)
template <bool BACKWARD>
__global__ __launch_bounds__(kJoinStates *kJoinRuns) void join_chunks(float *__restrict__ chunk_state, const float *__restrict__ chunk_dt, const float *__restrict__ a,
                                                                     const float *__restrict__ state, int64_t channels, int K, int N, int chunks) {
    __shared__ float ends[kJoinRuns][kJoinStates], sums[kJoinRuns][kJoinStates];
    const int s = threadIdx.x % kJoinStates, run = threadIdx.x / kJoinStates;
    const int64_t at = (int64_t)blockIdx.x * kJoinStates + s;
    const bool there = at < channels * N;
    const int64_t channel = there ? at / N : 0;
    const int steps = chunks - 1;                                    // chunks that leave something to another one
    const int length = join_length(steps), first = run * length;
    const float a2 = there ? rate_of(a[channel % K * N + (at - channel * N)]) : 0.0f;
    float end[kJoinRun], D[kJoinRun], h = 0.0f, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinRun; i++) {
        const bool mine = there && i < length && first + i < steps;
        const int64_t slot = BACKWARD ? chunks - 1 - (first + i) : first + i;
        end[i] = mine ? chunk_state[slot * channels * N + at] : 0.0f;
        D[i] = mine ? chunk_dt[slot * channels + channel] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kJoinRun; i++) {
        h = decayed(h, a2 * D[i], end[i]);
        sum += D[i];
    }
    ends[run][s] = h, sums[run][s] = sum;
    __syncthreads();
    h = !BACKWARD && state && there ? state[at] : 0.0f;
    for (int r = 0; r < run; r++) h = decayed(h, a2 * sums[r][s], ends[r][s]);
#pragma unroll
    for (int i = 0; i < kJoinRun; i++) {
        h = decayed(h, a2 * D[i], end[i]);
        if (there && i < length && first + i < steps) chunk_state[(BACKWARD ? chunks - 1 - (first + i) : first + i) * channels * N + at] = h;
    }
}
template <bool BACKWARD, typename T>
int launch_join_chunks(const ScanArgs<T> &s, hipStream_t stream) {
    const int64_t channels = (int64_t)s.B * s.K;
    const int steps = (int)s.chunks - 1, runs = (int)ceil_div(ceil_div(steps, join_length(steps)), 4) * 4;  // (whole wavefronts)
    join_chunks<BACKWARD><<<dim3((unsigned)ceil_div(channels * s.N, kJoinStates)), dim3(kJoinStates * runs), 0, stream>>>(
        s.chunk_state, s.chunk_dt, s.a, s.state, channels, s.K, s.N, (int)s.chunks);
    return check_launch("join_chunks");
}

}  // namespace

}  // namespace ptq4vm
