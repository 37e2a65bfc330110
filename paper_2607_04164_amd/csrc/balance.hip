// How evenly the router's picks fall on the experts (or on their groups), and what to change in the logits:
//   p_t = softmax(z_t), lse_t = log sum exp z_t;  over the V tokens that count:
//   c_e = picks of expert e,  P_e = mean of p_te,  F_r = (sum of c_e over group r) / (k V)
//   balance = G sum_e F_g(e) P_e,   z loss = mean of lse_t^2
//   dz_te = b G / V p_te (F_g(e) - sum_j F_g(j) p_tj) + a 2 / V lse_t p_te      (the counts are constants)
//
// S lanes of a wave hold a token's row (lane s: experts s, s + S, .., or four neighbours at a time where rows are whole
// 16-byte chunks), so a wave takes 64 / S neighbouring rows at a time and a row's maximum and sums are register
// permutations. A lane keeps the sums of p of its experts over its tokens, in fp32 for kRounds of them; longer sums are
// kept in 64 bits in LDS. A workgroup's sums meet in LDS in wave order, in fp32. The last of every fold_of(E) workgroups
// to finish adds their sums, the last of those the rest, in 64 bits and by workgroup (arrival counters say who is last,
// the sums' order does not depend on it; no float atomics); a sum is rounded to fp32 where it is put away for the next
// level. So a sum of p is off by at most kRounds + 24 roundings of 2^-24, however many tokens there are; the z loss's
// squares are summed in 64 bits. That is one launch: a second one for these sums takes the host longer than them (8192
// tokens of 60 experts 12.2 -> 8.9 us a call; in a graph 9.2 and 9.0). Up to kOneGroup rounds of tokens one workgroup
// does it all.
//
// Bound by memory where there are many tokens (131072 of 256 experts: 36 us, 3.9 TB/s of 4.9; the read of the logits
// alone 29), by the host's call for few (64 tokens: kernel 4.3 us, call 8 to 9), and between them by two or three round trips
// past the caches for the sums.
#include "bmoe_common.h"

namespace bmoe {
namespace {

constexpr int kThreads = 1024;  // of the forward's workgroups
constexpr int kWaves = kThreads / 64;
constexpr int kMaxGroups = 256;  // workgroups of the forward, at most
constexpr int kOneGroup = 8;     // rounds of tokens that one workgroup takes by itself
constexpr int kRounds = 32;      // tokens of a lane that are added in fp32 (a running sum of thousands loses what its steps
                                 // round off, 3e-5 of it after 2048)
constexpr int kGradThreads = 256;

// sum / maximum over the S lanes of a token, the same bits in each of them
template <int CTRL>
__device__ __forceinline__ float permuted(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int S, typename OP>
__device__ __forceinline__ float over_lanes(float v, OP op) {
    static_assert(S == 4 || S == 16, "lanes of a token");
    v = op(v, permuted<0xb1>(v));  // xor 1
    v = op(v, permuted<0x4e>(v));  // xor 2
    if constexpr (S == 16) {
        v = op(v, permuted<0x141>(v));  // half-row mirror
        v = op(v, permuted<0x140>(v));  // row mirror
    }
    return v;
}

// e^x for x <= 0: exp2 of the rounded product, corrected by what the rounding left out
__device__ __forceinline__ float exp_neg(float x) {
    x = x < -104.f ? -104.f : x;  // (0 in fp32; a comparison, so that NaN stays)
    constexpr float L = 1.44269504f, L2 = 1.92596303e-8f;  // log2(e), and the rest of it
    const float t = x * L, r = fmaf(x, L2, fmaf(x, L, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, r * 0.693147182f, e);
}

// A row's logits to its probabilities; the row's log sum exp. Rows of nothing but -infinity: zeros.
template <int S, int V>
__device__ __forceinline__ float softmax_row(float (&z)[V]) {
    float m = z[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, z[v]);
    m = over_lanes<S>(m, [](float a, float b) { return fmaxf(a, b); });
    const float top = m == -__builtin_inff() ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        z[v] = exp_neg(z[v] - top);
        sum += z[v];
    }
    sum = over_lanes<S>(sum, [](float a, float b) { return a + b; });
    if (sum == 0.f) return 0.f;
    const float inv = 1.f / sum;
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] *= inv;
    return top + logf(sum);
}

// the expert of lane s's value v; B: neighbours at a time (1, or 4 with E a multiple of 4 and rows 16-byte aligned)
template <int S, int B>
__device__ __forceinline__ int expert_of(int s, int v) { return B * (s + S * (v / B)) + v % B; }

// the logits of token t that lane s holds; past E and T, -infinity
template <int S, int V, int B>
__device__ __forceinline__ void load_logits(float (&z)[V], const float* logits, int64_t t, int64_t T, int s, int E) {
    const float none = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < V; v += B) {
        const int e = expert_of<S, B>(s, v);
        if constexpr (B == 4) {
            const float4 q = t < T && e < E ? *(const float4*)(logits + t * E + e) : make_float4(none, none, none, none);
            z[v] = q.x, z[v + 1] = q.y, z[v + 2] = q.z, z[v + 3] = q.w;
        } else {
            z[v] = t < T && e < E ? logits[t * E + e] : none;
        }
    }
}

// A token's loads, issued together and ahead of their use: its logits, whether it counts, and its picks (the lane's
// i-th is slot s + S i).
template <int S, int V, int B, int PK>
struct Token {
    float z[V];
    int pick[PK > 0 ? PK : 1];
    int valid;
    __device__ __forceinline__ void load(const float* logits, const int32_t* picks, const uint8_t* mask, int64_t t,
                                         int64_t T, int s, int E, int k) {
        load_logits<S, V, B>(z, logits, t, T, s, E);
        valid = t < T ? (mask ? mask[t] : 1) : 0;
#pragma unroll
        for (int i = 0; i < PK; ++i) pick[i] = t < T && s + S * i < k ? picks[t * k + s + S * i] : -1;
    }
    // the logits of a token that does not count: -infinity, whatever they hold
    __device__ __forceinline__ void mask() {
#pragma unroll
        for (int v = 0; v < V; ++v) z[v] = valid ? z[v] : -__builtin_inff();
    }
};

// ---- the losses from the sums over all tokens

struct Sums {
    double p[BMOE_MAX_EXPERTS];  // of p_te
    int c[BMOE_MAX_EXPERTS + 1]; // picks; the last: tokens that count
    double z;                    // of lse^2
    // work of finish()
    int group[BMOE_MAX_EXPERTS];
    double part[kWaves];
};

// the group of expert `tid` (loaded before a kernel's other work), or -1
__device__ __forceinline__ int group_of(const int32_t* e2g, int E, int G, int tid) {
    if (tid >= E) return -1;
    const int g = e2g ? e2g[tid] : tid;
    return g < G ? g : -1;
}

// Ends a call: every thread of one workgroup of kThreads, s complete (a barrier behind it). g: group_of this thread.
__device__ __forceinline__ void finish(const BalanceArgs& a, Sums& s, int g) {
    const int tid = threadIdx.x, E = a.E;
    for (int r = tid; r < BMOE_MAX_EXPERTS; r += kThreads) s.group[r] = 0;
    __syncthreads();
    const int n = s.c[E];
    const double per = 1.0 / (n > 0 ? (double)n : 1.0);
    if (tid < E) {
        if (g >= 0) atomicAdd(&s.group[g], s.c[tid]);
        a.counts[tid] = s.c[tid];
        a.prob[tid] = (float)(s.p[tid] * per);
    }
    __syncthreads();
    double sum = g >= 0 ? (double)s.group[g] * s.p[tid] : 0.0;
#pragma unroll
    for (int off = 32; off; off >>= 1) sum += __shfl_xor(sum, off);
    if ((tid & 63) == 0) s.part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = 0.0;
        for (int w = 0; w < BMOE_MAX_EXPERTS / 64; ++w) sum += s.part[w];
        a.losses[0] = (float)((double)a.G * sum * per * per / (double)a.k);
        a.losses[1] = (float)(s.z * per);
        a.counts[E] = n;
    }
}

// ---- the sums of several workgroups
//
// Rows of sums in the workspace: z [rows] double, p [rows, E] float, c [rows, E + 1] int32. They are written and read
// past the XCDs' own L2 caches (relaxed atomics of device scope: sc1 stores and loads); a row is complete before its
// workgroup counts itself in.
//
// Rows a workgroup adds at a time. More make fewer levels (3 us each) but longer ones: up to 64 experts 4096 tokens in 64
// workgroups 7.8 us, in two levels of 32 9.9; 256 workgroups of 256 experts by 32 36 us, by 64 40.
__host__ __device__ constexpr int fold_of(int E) { return E <= 64 ? 64 : 32; }
constexpr int kTickets = 16;  // arrival counters: of all folds, and of each; zero between calls
static_assert(kMaxGroups / 32 < kTickets, "a counter for each fold");
struct Parts {
    double* z;
    float* p;
    int* c;
};
__host__ __device__ inline size_t parts_bytes(int rows, int E) {
    return ((size_t)rows * (8 + 4 * (size_t)E + 4 * (size_t)(E + 1)) + 7) / 8 * 8;
}
__host__ __device__ inline Parts parts_of(void* at, int rows, int E) {
    Parts q;
    q.z = (double*)at;
    q.p = (float*)(q.z + rows);
    q.c = (int*)(q.p + (size_t)rows * E);
    return q;
}
template <typename T>
__device__ __forceinline__ T load_far(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename T>
__device__ __forceinline__ void store_far(T* p, T v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// s to row `row`, by a workgroup whose threads see it complete
__device__ __forceinline__ void put_row(const Parts& q, int row, int E, const Sums& s) {
    const int tid = threadIdx.x;
    if (tid < E) store_far(q.p + (size_t)row * E + tid, (float)s.p[tid]);
    if (tid <= E) store_far(q.c + (size_t)row * (E + 1) + tid, s.c[tid]);
    if (tid == 0) store_far(q.z + row, s.z);
}

// Counts a workgroup in, after its row; whether it is the last of n (which leaves the counter zero).
__device__ __forceinline__ bool last_of(int* ticket, int n, int* flag) {
    wait_vmcnt<0>();  // this thread's part of the row is there
    __syncthreads();
    if (threadIdx.x == 0) {
        const bool last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == n - 1;
        if (last) store_far(ticket, 0);
        *flag = last ? 1 : 0;
    }
    __syncthreads();
    return *flag != 0;
}

// The sum of rows row0 .. row0 + n - 1 (n <= fold_of(EP)) in s, in their order. J = kThreads / ep threads an expert, ep a power
// of two, E or more.
struct Scratch {
    double p[kThreads];
    int c[kThreads];
};
template <int EP>
__device__ __forceinline__ void add_rows(const Parts& q, int row0, int n, int E, Sums& s, Scratch& w) {
    constexpr int J = kThreads / EP, PER = fold_of(EP) / J;
    static_assert(PER > 0, "a thread's rows");
    const int tid = threadIdx.x, e = tid % EP, j = tid / EP;
    float pv[PER];
    int cv[PER];
    // (those past the last row repeat it instead of branching)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const size_t row = row0 + min(j * PER + i, n - 1);
        pv[i] = load_far(q.p + row * E + min(e, E - 1));
        cv[i] = load_far(q.c + row * (E + 1) + min(e, E - 1));
    }
    // tokens that count, and the z loss: a thread a row
    int m = 0;
    double z = 0.0;
    if (tid < n) {
        m = load_far(q.c + (size_t)(row0 + tid) * (E + 1) + E);
        z = load_far(q.z + row0 + tid);
    }
    double p = 0.0;
    int c = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        p += j * PER + i < n ? (double)pv[i] : 0.0;
        c += j * PER + i < n ? cv[i] : 0;
    }
    w.p[tid] = p;
    w.c[tid] = c;
#pragma unroll
    for (int off = 32; off; off >>= 1) {
        m += __shfl_xor(m, off);
        z += __shfl_xor(z, off);
    }
    __syncthreads();
    if (tid < E) {  // (e == tid)
#pragma unroll
        for (int i = 1; i < J; ++i) {
            p += w.p[i * EP + tid];
            c += w.c[i * EP + tid];
        }
        s.p[tid] = p;
        s.c[tid] = c;
    }
    if (tid == 0) {
        s.c[E] = m;
        s.z = z;
    }
    __syncthreads();
}

// the sums over a wave's tokens of what its lanes hold, in all of them
template <int S, int V>
__device__ __forceinline__ void wave_sums(float (&p)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int off = S; off < 64; off *= 2) p[v] += __shfl_xor(p[v], off);
}

template <int S, int V, int B>
__global__ __launch_bounds__(kThreads) void balance_kernel(BalanceArgs a) {
    constexpr int PER = 64 / S;  // tokens of a wave at a time
    __shared__ float s_p[kWaves][S * V];
    __shared__ double s_long[kWaves][S * V];  // sums of p of a wave's whole kRounds (is_long; a wave's own until the end)
    __shared__ double s_z[kWaves];
    __shared__ Sums sums;
    __shared__ Scratch scratch;
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int E = a.E, k = a.k, s = lane % S;
    const int64_t step = (int64_t)gridDim.x * kWaves * PER;
    int64_t t = ((int64_t)blockIdx.x * kWaves + wave) * PER + lane / S;
    Token<S, V, B, BMOE_MAX_TOPK / S> next;
    next.load(a.logits, a.topk_idx, a.valid, t, a.T, s, E, k);
    const int g = group_of(a.e2g, E, a.G, tid);
    for (int e = tid; e <= E; e += kThreads) sums.c[e] = 0;
    const bool is_long = a.T > kRounds * step;
    if (is_long)
        for (int i = tid; i < kWaves * S * V; i += kThreads) s_long[i / (S * V)][i % (S * V)] = 0.0;
    __syncthreads();
    float p[V];
    double z2 = 0.0;  // (squares may leave fp32 where their mean does not)
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = 0.f;
    // (the lanes of a wave stay together: the permutations read their neighbours)
    for (int round = 0; __any(t < a.T); t += step, ++round) {
        if (round == kRounds) {
            wave_sums<S, V>(p);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (lane < S) s_long[wave][expert_of<S, B>(s, v)] += (double)p[v];
                p[v] = 0.f;
            }
            round = 0;
        }
        Token<S, V, B, BMOE_MAX_TOPK / S> now = next;
        next.load(a.logits, a.topk_idx, a.valid, t + step, a.T, s, E, k);
        now.mask();
        const float lse = softmax_row<S, V>(now.z);
        if (now.valid) {
#pragma unroll
            for (int v = 0; v < V; ++v) p[v] += now.z[v];
            z2 = fma((double)lse, (double)lse, z2);
#pragma unroll
            for (int i = 0; i < BMOE_MAX_TOPK / S; ++i)
                if (now.pick[i] >= 0 && now.pick[i] < E) atomicAdd(&sums.c[now.pick[i]], 1);
            if (s == 0) atomicAdd(&sums.c[E], 1);
        }
    }
    // the wave's tokens, then the waves in order
    wave_sums<S, V>(p);
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (lane < S) s_p[wave][expert_of<S, B>(s, v)] = p[v];
#pragma unroll
    for (int off = S; off < 64; off *= 2) z2 += __shfl_xor(z2, off);
    if (lane == 0) s_z[wave] = z2;
    __syncthreads();
    if (tid < E) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += s_p[w][tid];
        double all = (double)sum;
        if (is_long)
            for (int w = 0; w < kWaves; ++w) all += s_long[w][tid];
        sums.p[tid] = all;
    }
    if (tid == 0) {
        double sum = 0.0;
        for (int w = 0; w < kWaves; ++w) sum += s_z[w];
        sums.z = sum;
    }
    __syncthreads();
    const int groups = gridDim.x;
    if (groups > 1) {
        constexpr int EP = S * V < 64 ? 64 : S * V, kFold = fold_of(EP);
        int* tickets = (int*)a.ws;
        const Parts q = parts_of(tickets + kTickets, groups, E);
        const int fold = blockIdx.x / kFold, folds = ceil_div(groups, kFold), row0 = fold * kFold;
        put_row(q, blockIdx.x, E, sums);
        if (!last_of(tickets + 1 + fold, min(kFold, groups - row0), &s_last)) return;
        add_rows<EP>(q, row0, min(kFold, groups - row0), E, sums, scratch);
        if (folds > 1) {
            const Parts r = parts_of((char*)(tickets + kTickets) + parts_bytes(groups, E), folds, E);
            put_row(r, fold, E, sums);
            if (!last_of(tickets, folds, &s_last)) return;
            add_rows<EP>(r, 0, folds, E, sums, scratch);
        }
    }
    finish(a, sums, g);
}

template <int S, int V, int B>
__global__ __launch_bounds__(kGradThreads) void balance_grad_kernel(BalanceGradArgs a) {
    constexpr int PER = 64 / S;
    __shared__ int s_group[BMOE_MAX_EXPERTS];
    __shared__ float s_f[S * V];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, s = lane % S, E = a.E;
    const int64_t step = (int64_t)gridDim.x * (kGradThreads / 64) * PER;
    int64_t t = ((int64_t)blockIdx.x * (kGradThreads / 64) + wave) * PER + lane / S;
    Token<S, V, B, 0> next;
    next.load(a.logits, nullptr, a.valid, t, a.T, s, E, 0);
    const int g = group_of(a.e2g, E, a.G, tid);
    const int count = tid < E ? a.counts[tid] : 0, n = a.counts[E];
    const double per = 1.0 / (n > 0 ? (double)n : 1.0);
    // the losses' slopes by p (balance; every expert's) and by lse^2
    const double b = (double)a.d_losses[0] * per * per * (double)a.G / (double)a.k;
    const float zc = (float)(2.0 * (double)a.d_losses[1] * per);
    for (int r = tid; r < BMOE_MAX_EXPERTS; r += kGradThreads) s_group[r] = 0;
    __syncthreads();
    if (g >= 0) atomicAdd(&s_group[g], count);
    __syncthreads();
    if (tid < S * V) s_f[tid] = g >= 0 ? (float)(b * (double)s_group[g]) : 0.f;
    __syncthreads();
    float f[V];
#pragma unroll
    for (int v = 0; v < V; ++v) f[v] = s_f[expert_of<S, B>(s, v)];
    for (; __any(t < a.T); t += step) {
        Token<S, V, B, 0> now = next;
        next.load(a.logits, nullptr, a.valid, t + step, a.T, s, E, 0);
        now.mask();
        float (&z)[V] = now.z;
        const float lse = softmax_row<S, V>(z);
        float dot = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) dot = fmaf(f[v], z[v], dot);
        dot = over_lanes<S>(dot, [](float x, float y) { return x + y; });
        const float c = fmaf(zc, lse, -dot);
        if (t < a.T) {
#pragma unroll
            for (int v = 0; v < V; ++v) z[v] = now.valid ? z[v] * (f[v] + c) : 0.f;
#pragma unroll
            for (int v = 0; v < V; v += B) {
                const int e = expert_of<S, B>(s, v);
                if (e >= E) continue;
                if constexpr (B == 4) *(float4*)(a.d_logits + t * E + e) = make_float4(z[v], z[v + 1], z[v + 2], z[v + 3]);
                else a.d_logits[t * E + e] = z[v];
            }
        }
    }
}

int forward_groups(int T, int E) {
    const int per = kWaves * (E <= 16 ? 16 : 4);  // tokens of a workgroup at a time
    if (T <= kOneGroup * per) return 1;
    // (up to 64 experts no more workgroups than one fold, up to four rounds each: 8192 tokens 9.0 us in 64, 11.2 in 128)
    const int most = E <= 64 && T <= 4 * 64 * per ? 64 : kMaxGroups;
    return (int)min((int64_t)most, ceil_div64(T, per));
}

bool whole_chunks(int E, const void* a, const void* b) {
    return E % 4 == 0 && (((uintptr_t)a | (uintptr_t)b) & 15u) == 0;
}

template <int S, int V, int B>
hipError_t forward(const BalanceArgs& a, hipStream_t s) {
    const int groups = forward_groups(a.T, a.E);
    hipLaunchKernelGGL((balance_kernel<S, V, B>), dim3(groups), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

template <int S, int V, int B>
hipError_t gradient(const BalanceGradArgs& a, hipStream_t s) {
    const int64_t per = (kGradThreads / 64) * (64 / S);
    const int blocks = (int)min((int64_t)2048, ceil_div64(a.T, per));
    hipLaunchKernelGGL((balance_grad_kernel<S, V, B>), dim3(blocks), dim3(kGradThreads), 0, s, a);
    return hipGetLastError();
}

template <int B>
hipError_t pick(const BalanceArgs& a, hipStream_t s) {
    if (a.E <= 16) return forward<4, 4, B>(a, s);
    if (a.E <= 64) return forward<16, 4, B>(a, s);
    if (a.E <= 128) return forward<16, 8, B>(a, s);
    return forward<16, 16, B>(a, s);
}

template <int B>
hipError_t pick(const BalanceGradArgs& a, hipStream_t s) {
    if (a.E <= 16) return gradient<4, 4, B>(a, s);
    if (a.E <= 64) return gradient<16, 4, B>(a, s);
    if (a.E <= 128) return gradient<16, 8, B>(a, s);
    return gradient<16, 16, B>(a, s);
}

}  // namespace

size_t balance_ws_bytes(int T, int E) {
    const int g = forward_groups(T, E);
    return g == 1 ? 0 : 4 * kTickets + parts_bytes(g, E) + parts_bytes(ceil_div(g, fold_of(E)), E);
}

hipError_t launch_balance(const BalanceArgs& a, hipStream_t s) {
    return whole_chunks(a.E, a.logits, nullptr) ? pick<4>(a, s) : pick<1>(a, s);
}

hipError_t launch_balance_grad(const BalanceGradArgs& a, hipStream_t s) {
    return whole_chunks(a.E, a.logits, a.d_logits) ? pick<4>(a, s) : pick<1>(a, s);
}

}  // namespace bmoe
