// libcsr5: what stands around the products of a layer of experts -- the router, the way back to the tokens, the
// root-mean-square norm and the quantisation to 8 bits.  All of it is bound by memory or by latency; the products
// are in grouped.hip.  The C ABI is declared in include/csr5.h.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "csr5.h"
#include "numbers.h"

namespace {

// Calls f with a value of the type that dtype names.
template <typename F> int with_type(int dtype, F f) {
    switch (dtype) {
        case CSR5_DTYPE_BF16: return f(bf16());
        case CSR5_DTYPE_F16: return f(f16());
        case CSR5_DTYPE_F32: return f(float());
        default: return CSR5_EINVAL;
    }
}
size_t type_bytes(int dtype) { return dtype == CSR5_DTYPE_F32 ? 4 : dtype == CSR5_DTYPE_BF16 || dtype == CSR5_DTYPE_F16 ? 2 : 0; }

// The sum of v over the workgroup, for everybody, in a fixed order.  `part` holds a word per wavefront and is not used again
// before the next barrier.
__device__ __forceinline__ float group_sum(float v, float* part) {
    v = wave_sum(v);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < waves; w++) v += part[w];
    return v;
}

// ---------------------------------------------------------------------------------------------------------------
// Root-mean-square norm.  One workgroup per row, which it holds in registers between the sum of squares and the
// output: x and the residual are read once.  8 neighbouring values per thread, so a block of 128 values that share a
// scale is 16 neighbouring lanes; as many threads as the row has eights, up to 1024, then NV eights per thread.
// Squares are added up in 32 bits; h is rounded for memory only, y once.  Bound by memory: 32768 x 4096 in bf16, x and the
// residual to h and y, 173 us, 6.2 TB/s; to h and 8 bits with scales 166 us, 5.7 TB/s (a large copy: 4.8).  16 rows: 3.8 us, mostly
// the launch.
// ---------------------------------------------------------------------------------------------------------------
constexpr int NORM_THREADS = 1024;

template <typename T> struct NormArgs {
    int rows, n;
    const T *x, *residual, *gain;
    int64_t ldx, ldr;
    float eps;
    T *h, *y;
    int64_t ldh, ldy;
    uint8_t* q;
    int64_t ldq;
    float* scale;
    int64_t scale_row, scale_block;
    float* rstd;
};

template <typename T, int NV, bool VEC> __global__ __launch_bounds__(NORM_THREADS) void k_rmsnorm(NormArgs<T> a) {
    __shared__ float part[NORM_THREADS / 64];
    const int64_t row = workgroup();
    if (row >= a.rows) return;
    float v[NV][8];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NV; c++) {
        const int col = (c * int(blockDim.x) + int(threadIdx.x)) * 8;
        load_values<8, VEC>(a.x + row * a.ldx + col, a.n - col, v[c]);
        if (a.residual) {
            float r[8];
            load_values<8, VEC>(a.residual + row * a.ldr + col, a.n - col, r);
#pragma unroll
            for (int i = 0; i < 8; i++) v[c][i] += r[i];
        }
    }
#pragma unroll
    for (int c = 0; c < NV; c++) {
        const int col = (c * int(blockDim.x) + int(threadIdx.x)) * 8;
#pragma unroll
        for (int i = 0; i < 8; i++) sum += v[c][i] * v[c][i];
        if (a.h) store_values<8, VEC>(a.h + row * a.ldh + col, a.n - col, v[c]);
    }
    const float rstd = 1.f / sqrtf(group_sum(sum, part) / float(a.n) + a.eps);
    if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int c = 0; c < NV; c++) {
        const int col = (c * int(blockDim.x) + int(threadIdx.x)) * 8;
        float g[8];
        if (a.gain) load_values<8, VEC>(a.gain + col, a.n - col, g);
#pragma unroll
        for (int i = 0; i < 8; i++) v[c][i] = a.gain ? v[c][i] * rstd * g[i] : v[c][i] * rstd;
        if (a.y) store_values<8, VEC>(a.y + row * a.ldy + col, a.n - col, v[c]);
        if (a.q) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) most = max(most, i < a.n - col ? magnitude(v[c][i]) : 0u);
            const Scale s = f8_scale(lanes_max<16>(most));
            if (col < a.n) {
                f8_store<VEC>(a.q + row * a.ldq + col, a.n - col, v[c], s);
                if ((threadIdx.x & 15) == 0) a.scale[row * a.scale_row + (col / CSR5_F8_BLOCK) * a.scale_block] = s.scale;
            }
        }
    }
}

// Its gradients.  A workgroup takes rows by turns and keeps its share of the gain's gradient in registers; the shares
// go to the workspace and are added up by k_columns in a fixed order.  Bound by memory up to n = 16384 in 16 bits and 8192 in 32:
// 32768 x 4096 in bf16 with the residual's gradient 194 us, 5.5 TB/s.  Longer rows do not fit the registers, and what is spilled
// holds them up: 4096 x 32768 in bf16 892 us, 1.2 TB/s; in float32 4096 x 16384 252, 4.3, and x 32768 1749, 1.2.
template <typename T> struct NormBackArgs {
    int rows, n;
    const T *h, *gain, *dy, *residual_grad;
    int64_t ldh, lddy, ldrg;
    const float* rstd;
    T* dh;
    int64_t lddh;
    float* share;           // [gridDim.x][n], NULL: not wanted
};

// The next row's h and dy are asked for before this row's sum.
template <typename T, int NV, bool VEC> __global__ __launch_bounds__(NORM_THREADS) void k_rmsnorm_back(NormBackArgs<T> a) {
    __shared__ float part[2][NORM_THREADS / 64];
    float gain[NV][8], share[NV][8];
    auto at = [](int c) { return (c * int(blockDim.x) + int(threadIdx.x)) * 8; };
#pragma unroll
    for (int c = 0; c < NV; c++) {
        if (a.gain) load_values<8, VEC>(a.gain + at(c), a.n - at(c), gain[c]);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            share[c][i] = 0.f;
            if (!a.gain) gain[c][i] = 1.f;
        }
    }
    vec<T, 8> h[NV], dy[NV];
    auto ask = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < NV; c++) {
            h[c] = eight_values<VEC>(a.h + row * a.ldh + at(c), a.n - at(c));
            dy[c] = eight_values<VEC>(a.dy + row * a.lddy + at(c), a.n - at(c));
        }
    };
    if (blockIdx.x < a.rows) ask(blockIdx.x);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const float r = a.rstd[row];
        float v[NV][8], u[NV][8], sum = 0.f;
#pragma unroll
        for (int c = 0; c < NV; c++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                v[c][i] = float(h[c][i]) * r, u[c][i] = float(dy[c][i]);
                share[c][i] += u[c][i] * v[c][i];
                u[c][i] *= gain[c][i];
                sum += u[c][i] * v[c][i];
            }
        float d[NV][8];
        if (a.residual_grad)
#pragma unroll
            for (int c = 0; c < NV; c++) load_values<8, VEC>(a.residual_grad + row * a.ldrg + at(c), a.n - at(c), d[c]);
        if (row + gridDim.x < a.rows) ask(row + gridDim.x);
        const float mean = group_sum(sum, part[turn]) / float(a.n);
#pragma unroll
        for (int c = 0; c < NV; c++) {
#pragma unroll
            for (int i = 0; i < 8; i++) d[c][i] = r * (u[c][i] - v[c][i] * mean) + (a.residual_grad ? d[c][i] : 0.f);
            store_values<8, VEC>(a.dh + row * a.lddh + at(c), a.n - at(c), d[c]);
        }
    }
    if (a.share)
#pragma unroll
        for (int c = 0; c < NV; c++) store_values<8, false>(a.share + int64_t(blockIdx.x) * a.n + at(c), a.n - at(c), share[c]);
}

// out[col] = sum over `rows` rows; 32 columns and 32 rows side by side.
__global__ __launch_bounds__(1024) void k_columns(int rows, int n, const float* in, float* out) {
    __shared__ float part[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5, col = int(blockIdx.x) * 32 + c;
    float sum = 0.f;
    if (col < n)
#pragma unroll 8
        for (int i = r; i < rows; i += 32) sum += in[int64_t(i) * n + col];
    part[r][c] = sum;
    __syncthreads();
    if (r == 0 && col < n) {
        for (int i = 1; i < 32; i++) sum += part[i][c];
        out[col] = sum;
    }
}

// Threads of a row's workgroup, and how many times 8 values a thread holds.
int norm_threads(int n) {
    const int eights = divide_up(n, 8);
    return eights >= NORM_THREADS ? NORM_THREADS : divide_up(eights, 64) * 64;
}
template <typename F> void norm_shape(int n, F f) {
    const int eights = divide_up(n, 8), threads = norm_threads(n);
    if (eights <= NORM_THREADS) f(threads, std::integral_constant<int, 1>());
    else if (eights <= 2 * NORM_THREADS) f(threads, std::integral_constant<int, 2>());
    else f(threads, std::integral_constant<int, 4>());
}

// Workgroups of k_rmsnorm_back.  Each writes a share of the gain's gradient, n floats, so there are no more than fill the card:
// 4096 x 8192 with 256 of them 48 us, with 1024 69; 8191 x 2560 with 512 31, with 256 43, with 1024 35; 32768 x 1024 with
// 1024 47, with 512 70.
int norm_groups(int rows, int n) {
    const int threads = norm_threads(n), fill = threads >= 512 ? 256 : threads >= 192 ? 512 : 1024;
    return min(rows, fill);
}

// ---------------------------------------------------------------------------------------------------------------
// Quantisation.  ROWS = 1: 16 lanes per block of 128 values; ROWS = 128: a workgroup per block of 128 x 128.  A block stays in
// registers between its maximum and its values, so x is read once.  Bound by memory: 32768 x 4096 in bf16 81 us with either,
// 5.0 TB/s.
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int ROWS, bool VEC>
__global__ __launch_bounds__(256) void k_quantise(int rows, int n, const T* x, int64_t ldx, uint8_t* q, int64_t ldq, float* scale, int64_t scale_row, int64_t scale_block) {
    constexpr int PASSES = ROWS == 1 ? 1 : 8;
    const int blocks = (n + CSR5_F8_BLOCK - 1) / CSR5_F8_BLOCK, lane = threadIdx.x & 15, line = threadIdx.x >> 4;
    int64_t row0;
    int b;
    if (ROWS == 1) {
        const int64_t at = workgroup() * 16 + line;
        row0 = at / blocks, b = int(at % blocks);
        if (row0 >= rows) return;
    } else {
        row0 = workgroup() / blocks * ROWS, b = int(workgroup() % blocks);
        if (row0 >= rows) return;
        row0 += line;
    }
    const int col = b * CSR5_F8_BLOCK + lane * 8;
    float v[PASSES][8];
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < PASSES; p++) {
        const int64_t row = row0 + p * 16;
        load_values<8, VEC>(x + row * ldx + col, row < rows ? n - col : 0, v[p]);
#pragma unroll
        for (int i = 0; i < 8; i++) most = max(most, magnitude(v[p][i]));
    }
    if (ROWS == 1) {
        most = lanes_max<16>(most);
    } else {
        __shared__ uint32_t part[4];
        most = lanes_max<64>(most);
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(part[0], part[1]), max(part[2], part[3]));
    }
    const Scale s = f8_scale(most);
#pragma unroll
    for (int p = 0; p < PASSES; p++) {
        const int64_t row = row0 + p * 16;
        if (row < rows && col < n) f8_store<VEC>(q + row * ldq + col, n - col, v[p], s);
    }
    if (lane == 0 && (ROWS == 1 || line == 0)) scale[row0 / ROWS * scale_row + b * scale_block] = s.scale;
}

// ---------------------------------------------------------------------------------------------------------------
// The router.  A token's logits lie over LANES lanes, V neighbouring ones in each: 16 lanes, four tokens to a wavefront, for
// up to 256 experts and k up to 16, otherwise all 64.  k rounds of: largest of the token, who has it first, take it out.
// Logits are compared as whole numbers in the floats' order, 0 for what is never chosen (-inf, NaN); 16-bit ones carry their
// expert in the low half, so that the largest is the lowest expert's of the largest and names it.  256 experts in 16 bits take
// about 45 instructions a round, for four tokens (a wavefront per token: 25 for one; 32768 tokens, 8 of 256 experts, took 23 us).
//
// Grouping is a counting sort, stable by pair: every workgroup counts the experts of its chunk of tokens; then each
// adds up, per expert, the counts of all chunks and of those before it, and hands out rows to its pairs in order.
// Tokens of one chunk: one workgroup does both.  32768 tokens, 8 of 256 in bf16 (20 MB, 4 us at a copy's rate) take 21 us: about
// 13 to choose, of which the rounds' instructions are about half and waiting the rest (four wavefronts to a SIMD, two turns each, of
// data-parallel moves that wait for one another), and 8 to group, where every workgroup reads the counts of all chunks (64 MB from
// the L2).
// ---------------------------------------------------------------------------------------------------------------
constexpr int ROUTE_CHUNKS = 256;       // at most, each a workgroup
constexpr int ROUTE_WAVES = 16;
constexpr int ROUTE_ONE = 64;           // tokens that a single workgroup routes
constexpr int ROUTE_FEW = 16;           // ... by a wavefront each: 8 of 128 take 6.2 us so, four to a wavefront 7.3; 24 would take turns, 9.2 against 7.4

struct RouteArgs {
    int tokens, experts, k, chunk, chunks;      // chunk: tokens of a workgroup
    const void* logits;
    int64_t ld;
    bool vec;                                   // rows may be read V values at a time
    int32_t* expert;
    float* weight;
    int32_t *offset, *source, *place;
    int32_t* count;                             // [chunks][experts]
    bool fours;                                 // ... whose rows may be read four at a time
};

template <typename T, int V, int LANES> __device__ __forceinline__ void route_load(const RouteArgs& a, int64_t t, float (&v)[V]) {
    const int e = int(threadIdx.x % LANES) * V, have = max(a.experts - e, 0);
    const T* const row = static_cast<const T*>(a.logits) + t * a.ld + (have ? e : 0);
    if (a.vec && have >= V) {
        constexpr int N = V * sizeof(T) > 16 ? 16 / sizeof(T) : V;
#pragma unroll
        for (int i = 0; i < V; i += N) {
            float part[N];
            load_values<N, true>(row + i, N, part);
#pragma unroll
            for (int j = 0; j < N; j++) v[i + j] = part[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = i < have ? float(row[i]) : -INFINITY;
    }
}

// `there`: this lane's token is one.  chosen: also has the experts, in LDS, where it is not NULL.
template <typename T, int V, int LANES> __device__ __forceinline__ void route_token(const RouteArgs& a, int64_t t, bool there, const float (&logit)[V], int32_t* count, int32_t* chosen) {
    constexpr bool PACKED = sizeof(T) == 2, ROW = LANES == 16;
    const int lane = threadIdx.x % LANES, row = threadIdx.x & 48;
    uint32_t key[V];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; i++) {
        const float f = logit[i] + 0.f;                 // -0 and 0 are equal
        const uint32_t bits = __float_as_uint(f), order = bits >> 31 ? ~bits : bits | 0x80000000u;
        nan |= f != f;
        key[i] = f > -INFINITY ? (PACKED ? (order & 0xffff0000u) | (0xffffu - uint32_t(lane * V + i)) : order) : 0u;
        if constexpr (std::is_same<T, f16>::value) {    // 16 bits of its own: those of the float's are not all in the upper half
            const uint32_t half = __builtin_bit_cast(uint16_t, f16(f)), h = half >> 15 ? ~half & 0xffffu : half | 0x8000u;
            key[i] = f > -INFINITY ? h << 16 | (0xffffu - uint32_t(lane * V + i)) : 0u;
        }
    }
    const uint64_t nans = __ballot(nan);
    nan = ROW ? (nans >> row) & 0xffff : nans != 0;
    uint32_t mine = 0, best = 0;    // of lane j: the key of the j-th largest, and its expert; the largest's key
    int which = -1;
    for (int j = 0; j < a.k; j++) {
        uint32_t most = key[0];
#pragma unroll
        for (int i = 1; i < V; i++) most = max(most, key[i]);
        const uint32_t all = ROW ? row_max(most) : wave_max(most);
        if (!__any(all != 0)) break;
        int e;
        if (PACKED) {
            e = int(0xffffu - (all & 0xffffu));
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = key[i] == all ? 0u : key[i];
        } else {
            const uint64_t have = __ballot(most == all);
            const int first = ROW ? __ffs(uint32_t(have >> row) & 0xffffu) - 1 : __ffsll((unsigned long long)have) - 1;
            int at = 0;
#pragma unroll
            for (int i = V - 1; i >= 0; i--) at = key[i] == all ? i : at;
#pragma unroll
            for (int i = 0; i < V; i++) key[i] = lane == first && i == at ? 0u : key[i];
            e = first * V + __shfl(at, (ROW ? row : 0) + first);
        }
        if (j == 0) best = all;
        if (lane == j && all != 0) mine = all, which = e;
    }
    auto value = [](uint32_t all) {
        if constexpr (std::is_same<T, f16>::value) {
            const uint32_t h = all >> 16;
            return float(__builtin_bit_cast(f16, uint16_t(h & 0x8000u ? h & 0x7fffu : ~h)));
        }
        const uint32_t order = PACKED ? all & 0xffff0000u : all;
        // a packed negative number's lower half comes back as ones: cut
        const uint32_t bits = order >> 31 ? order & 0x7fffffffu : ~order;
        return __uint_as_float(PACKED ? bits & 0xffff0000u : bits);
    };
    const float top = value(best);
    float w = which >= 0 ? expf(value(mine) - top) : 0.f;
    const float sum = ROW ? row_sum(w) : wave_sum(w);
    w = w / fmaxf(sum, 1.f);                    // the largest is exp(0): the sum is 1 at least where there is one
    if (nan || top == INFINITY) w = NAN;
    if (there && lane < a.k) {
        a.expert[t * a.k + lane] = which;
        a.weight[t * a.k + lane] = w;
        if (chosen) chosen[t * a.k + lane] = which;
        if (which >= 0) atomicAdd(&count[which], 1);        // in LDS; a count does not depend on the order
    }
}

// Lanes whose `e` is this lane's, among those with `in`.
__device__ __forceinline__ uint64_t same_as(int e, bool in, int bits) {
    uint64_t m = __ballot(in);
    for (int b = 0; b < bits; b++) {
        const uint64_t set = __ballot((e >> b) & 1);
        m &= (e >> b) & 1 ? set : ~set;
    }
    return m;
}

// LDS: [ROUTE_WAVES + 2][experts] words, and one per pair where a single workgroup does it all
template <typename T, int V, int LANES, bool CHOOSE, bool GROUP> __global__ __launch_bounds__(ROUTE_WAVES * 64) void k_route(RouteArgs a) {
    extern __shared__ int32_t lds[];
    constexpr int THREADS = ROUTE_WAVES * 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, E = a.experts;
    int32_t *const total = lds + ROUTE_WAVES * E, *const before = total + E;     // rows of an expert in all chunks, in earlier ones
    int32_t* const chosen = before + E;                                          // a single workgroup's pairs' experts
    const int32_t t0 = int32_t(blockIdx.x) * a.chunk, t1 = min(t0 + a.chunk, a.tokens);
    for (int e = tid; e < 2 * E; e += THREADS) total[e] = 0;
    __syncthreads();
    if (CHOOSE && t0 < t1) {
        constexpr int STEP = THREADS / LANES;           // tokens of the workgroup at a time
        float v[V], next[V] = {};
        const int32_t mine = t0 + tid / LANES;
        route_load<T, V, LANES>(a, min(mine, a.tokens - 1), v);
        for (int32_t t = mine; t - tid / LANES < t1; t += STEP) {     // the same number of turns for everybody
            route_load<T, V, LANES>(a, min(t + STEP, a.tokens - 1), next);
            route_token<T, V, LANES>(a, t, t < t1, v, total, GROUP ? chosen : nullptr);
#pragma unroll
            for (int i = 0; i < V; i++) v[i] = next[i];
        }
    }
    if (CHOOSE) {
        __syncthreads();
        if (!GROUP)
            for (int e = tid; e < E; e += THREADS) a.count[int64_t(blockIdx.x) * E + e] = total[e];
    }
    if (!GROUP) return;
    __shared__ int32_t sums[ROUTE_WAVES];
    if (!CHOOSE) {
        // several threads per expert (per four), each some of the chunks
        auto add_up = [&](auto width) {
            constexpr int N = decltype(width)::value;
            const int parts = THREADS / (E / N), e = tid % (E / N) * N, part = tid / (E / N);
            if (part >= parts) return;
            int32_t sum[N] = {}, earlier[N] = {};
#pragma unroll 8
            for (int c = part; c < a.chunks; c += parts) {
                const vec<int32_t, N> x = *reinterpret_cast<const vec<int32_t, N>*>(a.count + int64_t(c) * E + e);
#pragma unroll
                for (int i = 0; i < N; i++) {
                    const int32_t v = N == 1 ? x[0] : x[i];
                    sum[i] += v, earlier[i] += c < int(blockIdx.x) ? v : 0;
                }
            }
#pragma unroll
            for (int i = 0; i < N; i++) {
                atomicAdd(&total[e + i], sum[i]);              // whole numbers, in LDS
                atomicAdd(&before[e + i], earlier[i]);
            }
        };
        if (a.fours) add_up(std::integral_constant<int, 4>());
        else add_up(std::integral_constant<int, 1>());
    }
    // each wavefront's own share of the chunk's pairs, in order
    const int32_t p0 = t0 * a.k, pairs = max(t1 - t0, 0) * a.k;
    const int32_t share = (pairs + THREADS - 1) / THREADS * 64;
    const int32_t first = p0 + min(wave * share, pairs), last = p0 + min((wave + 1) * share, pairs);
    int32_t* const mine = lds + wave * E;
    for (int e = lane; e < E; e += 64) mine[e] = 0;
    wave_order();
    const int32_t* const expert = CHOOSE ? chosen : a.expert;
    for (int32_t p = first + lane; p < last; p += 64) {
        const int e = expert[p];
        if (e >= 0) atomicAdd(&mine[e], 1);
    }
    __syncthreads();
    // exclusive sum of total over the experts: one expert per thread (experts <= threads)
    const int32_t n = tid < E ? total[tid] : 0;
    int32_t upto = wave_prefix(n);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int32_t rows = 0;
    for (int w = 0; w < ROUTE_WAVES; w++) {
        if (w < wave) upto += sums[w];
        rows += sums[w];
    }
    if (tid < E) {
        if (blockIdx.x == 0) a.offset[tid + 1] = upto;
        int32_t at = upto - n + before[tid];
        for (int w = 0; w < ROUTE_WAVES; w++) {         // where each wavefront's pairs of this expert begin
            const int32_t x = lds[w * E + tid];
            lds[w * E + tid] = at;
            at += x;
        }
    }
    if (blockIdx.x == 0 && tid == 0) a.offset[0] = 0;
    __syncthreads();
    const int bits = 32 - __clz(max(E - 1, 1));
    for (int32_t p = first + lane; p - lane < last; p += 64) {
        const int e = p < last ? expert[p] : -1;
        const uint64_t same = same_as(e, e >= 0, bits);
        int32_t at = -1;
        if (e >= 0) {
            const int32_t base = mine[e];
            at = base + __popcll(same & ((1ull << lane) - 1));
            a.source[at] = int32_t(uint32_t(p) / uint32_t(a.k));
            wave_order();
            if (63 - __clzll(same) == lane) mine[e] = at + 1;       // the last of its expert, after every lane's read
        }
        wave_order();
        if (p < last) a.place[p] = at;
    }
    const int32_t end = min(a.tokens * a.k - rows, p0 + pairs);
    for (int32_t r = p0 + tid; r < end; r += THREADS) a.source[rows + r] = -1;
}

int route_chunk(int32_t tokens) { return tokens <= ROUTE_ONE ? max(tokens, 1) : max(divide_up(tokens, ROUTE_CHUNKS), ROUTE_WAVES); }
bool route_fits(int32_t tokens, int32_t experts, int32_t k) {
    return experts <= CSR5_ROUTE_MAX_EXPERTS && k >= 1 && k <= experts && k <= CSR5_ROUTE_MAX_K && int64_t(tokens) * k <= MOST_SIZE;
}

// A wavefront per token: the row in LDS, zeros with k entries.
template <typename T> __global__ __launch_bounds__(256) void k_route_back(int tokens, int experts, int k, const int32_t* expert, const float* weight, const float* dweight, T* dlogits, int64_t ld) {
    __shared__ float rows[4][CSR5_ROUTE_MAX_EXPERTS];
    const int lane = threadIdx.x & 63;
    float* const row = rows[threadIdx.x >> 6];
    const int64_t t = workgroup() * 4 + (threadIdx.x >> 6);
    if (t >= tokens) return;                            // no barrier below: a wavefront's LDS accesses are in order
    for (int e = lane; e < experts; e += 64) row[e] = 0.f;
    wave_order();
    float w = 0.f, d = 0.f;
    int e = -1;
    if (lane < k) e = expert[t * k + lane], w = weight[t * k + lane], d = dweight[t * k + lane];
    if (uint32_t(e) >= uint32_t(experts)) e = -1, w = 0.f, d = 0.f;
    const float mean = wave_sum(w * d);
    if (e >= 0) row[e] = w * (d - mean);
    wave_order();
    for (int i = lane; i < experts; i += 64) dlogits[t * ld + i] = T(row[i]);
}

// ---------------------------------------------------------------------------------------------------------------
// Back to the tokens: a thread has 8 columns of a token, adds up its k rows in 32 bits and rounds once.  Bound by memory: 4 rows
// of 4096 in bf16 for each of 8192 tokens 77 us, 5.2 TB/s.
// ---------------------------------------------------------------------------------------------------------------
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_combine(int tokens, int k, int rows, int n, const T* z, int64_t ldz, const int32_t* place, const float* weight, const T* residual, int64_t ldr, T* y, int64_t ldy) {
    const int64_t t = workgroup();
    const int col = (int(blockIdx.z) * 256 + int(threadIdx.x)) * 8;
    if (t >= tokens || col >= n) return;
    float sum[8] = {};
    if (residual) load_values<8, VEC>(residual + t * ldr + col, n - col, sum);
    for (int j = 0; j < k; j++) {
        const int32_t r = place[t * k + j];
        if (uint32_t(r) >= uint32_t(rows)) continue;
        const float w = weight ? weight[t * k + j] : 1.f;
        float v[8];
        load_values<8, VEC>(z + r * ldz + col, n - col, v);
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] += w * v[i];
    }
    store_values<8, VEC>(y + t * ldy + col, n - col, sum);
}

// A wavefront per pair: dz and the sum for dweight in one pass over the row of z.  Bound by memory: at combine's size 127 us, 4.8
// TB/s.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_combine_back(int64_t pairs, int k, int rows, int n, const T* dy, int64_t lddy, const T* z, int64_t ldz, const int32_t* place, const float* weight, T* dz, int64_t lddz, float* dweight) {
    const int lane = threadIdx.x & 63;
    const int64_t p = workgroup() * 4 + (threadIdx.x >> 6);
    if (p >= pairs) return;
    const int32_t r = place[p];
    float sum = 0.f;
    if (uint32_t(r) < uint32_t(rows)) {
        const float w = weight[p];
        for (int col = lane * 8; col < n; col += 512) {
            float d[8], v[8];
            load_values<8, VEC>(dy + p / k * lddy + col, n - col, d);
            load_values<8, VEC>(z + r * ldz + col, n - col, v);
#pragma unroll
            for (int i = 0; i < 8; i++) sum += d[i] * v[i], d[i] *= w;
            store_values<8, VEC>(dz + r * lddz + col, n - col, d);
        }
    }
    sum = wave_sum(sum);
    if (lane == 0) dweight[p] = sum;
}

}  // namespace

extern "C" {

size_t csr5_route_workspace_bytes(int32_t tokens, int32_t experts, int32_t k) {
    if (tokens < 0 || experts < 0 || !route_fits(tokens, experts, k)) return 0;
    const int chunks = divide_up(tokens, route_chunk(tokens));
    return chunks <= 1 ? 0 : size_t(chunks) * size_t(experts) * 4;
}

int csr5_route(int32_t tokens, int32_t experts, int32_t k, int dtype, const void* logits, int64_t ld, int32_t* expert, float* weight,
               int32_t* offset, int32_t* source, int32_t* place, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || tokens < 0 || experts < 0 || !offset) return CSR5_EINVAL;
    if (!route_fits(tokens, experts, k)) return CSR5_ERANGE;
    if (!rows_ok(logits, tokens, ld, experts, size) || (tokens > 0 && (!expert || !weight || !source || !place))) return CSR5_EINVAL;
    const size_t need = csr5_route_workspace_bytes(tokens, experts, k);
    if (need && (!workspace || workspace_bytes < need)) return CSR5_ENOMEM;
    if (reinterpret_cast<uintptr_t>(workspace) & 3) return CSR5_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    RouteArgs a{tokens, experts, k, route_chunk(tokens), 0, logits, ld, false, expert, weight, offset, source, place, static_cast<int32_t*>(workspace), experts % 4 == 0 && (reinterpret_cast<uintptr_t>(workspace) & 15) == 0};
    a.chunks = max(divide_up(tokens, a.chunk), 1);
    const size_t lds = (size_t(ROUTE_WAVES + 2) * size_t(experts) + (a.chunks == 1 ? size_t(tokens) * size_t(k) : 0)) * 4;
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        auto go = [&](auto width, auto lanes) {
            constexpr int V = decltype(width)::value, LANES = decltype(lanes)::value;
            a.vec = aligned(logits, ld, size, V * size < 16 ? V * size : 16);
            if (a.chunks == 1) {
                k_route<T, V, LANES, true, true><<<1, ROUTE_WAVES * 64, lds, s>>>(a);
            } else {
                k_route<T, V, LANES, true, false><<<a.chunks, ROUTE_WAVES * 64, lds, s>>>(a);
                k_route<T, V, LANES, false, true><<<a.chunks, ROUTE_WAVES * 64, lds, s>>>(a);
            }
        };
        using std::integral_constant;
        if (k <= 16 && experts <= 256 && tokens > ROUTE_FEW) {
            if (experts <= 64) go(integral_constant<int, 4>(), integral_constant<int, 16>());
            else if (experts <= 128) go(integral_constant<int, 8>(), integral_constant<int, 16>());
            else go(integral_constant<int, 16>(), integral_constant<int, 16>());
        } else {
            if (experts <= 64) go(integral_constant<int, 1>(), integral_constant<int, 64>());
            else if (experts <= 256) go(integral_constant<int, 4>(), integral_constant<int, 64>());
            else go(integral_constant<int, 16>(), integral_constant<int, 64>());
        }
        return launched();
    });
}

int csr5_route_backward(int32_t tokens, int32_t experts, int32_t k, int dtype, const int32_t* expert, const float* weight,
                        const float* dweight, void* dlogits, int64_t ld, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || tokens < 0 || experts < 0) return CSR5_EINVAL;
    if (!route_fits(tokens, experts, k)) return CSR5_ERANGE;
    if (!rows_ok(dlogits, tokens, ld, experts, size) || (tokens > 0 && (!expert || !weight || !dweight))) return CSR5_EINVAL;
    if (tokens == 0) return CSR5_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        k_route_back<T><<<workgroups(divide_up(tokens, 4)), 256, 0, s>>>(tokens, experts, k, expert, weight, dweight, static_cast<T*>(dlogits), ld);
        return launched();
    });
}

int csr5_combine(int32_t tokens, int32_t k, int32_t rows, int32_t n, int dtype, const void* z, int64_t ldz, const int32_t* place,
                 const float* weight, const void* residual, int64_t ldr, void* y, int64_t ldy, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || tokens < 0 || k < 0 || rows < 0 || n < 0) return CSR5_EINVAL;
    if (int64_t(tokens) * k > INT32_MAX || n > MOST_SIZE) return CSR5_ERANGE;
    if (!rows_ok(z, rows, ldz, n, size) || !rows_ok(y, tokens, ldy, n, size) || (residual && !rows_ok(residual, tokens, ldr, n, size))) return CSR5_EINVAL;
    if (tokens == 0 || n == 0) return CSR5_OK;
    if (k > 0 && !place) return CSR5_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        dim3 grid = workgroups(tokens);
        grid.z = divide_up(n, 2048);
        auto go = [&](auto v) {
            k_combine<T, decltype(v)::value><<<grid, 256, 0, s>>>(tokens, k, rows, n, static_cast<const T*>(z), ldz, place, weight, static_cast<const T*>(residual), ldr, static_cast<T*>(y), ldy);
        };
        if (aligned(z, ldz, size, 16) && aligned(y, ldy, size, 16) && (!residual || aligned(residual, ldr, size, 16))) go(std::true_type());
        else go(std::false_type());
        return launched();
    });
}

int csr5_combine_backward(int32_t tokens, int32_t k, int32_t rows, int32_t n, int dtype, const void* dy, int64_t lddy, const void* z,
                          int64_t ldz, const int32_t* place, const float* weight, void* dz, int64_t lddz, float* dweight, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || tokens < 0 || k < 0 || rows < 0 || n < 0) return CSR5_EINVAL;
    if (int64_t(tokens) * k > INT32_MAX || n > MOST_SIZE) return CSR5_ERANGE;
    if (!rows_ok(z, rows, ldz, n, size) || !rows_ok(dy, tokens, lddy, n, size) || !rows_ok(dz, rows, lddz, n, size)) return CSR5_EINVAL;
    const int64_t pairs = int64_t(tokens) * k;
    if (pairs == 0) return CSR5_OK;
    if (!place || !weight || !dweight) return CSR5_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        auto go = [&](auto v) {
            k_combine_back<T, decltype(v)::value><<<workgroups(divide_up(pairs, 4)), 256, 0, s>>>(pairs, k, rows, n, static_cast<const T*>(dy), lddy, static_cast<const T*>(z), ldz, place, weight, static_cast<T*>(dz), lddz, dweight);
        };
        if (aligned(z, ldz, size, 16) && aligned(dy, lddy, size, 16) && aligned(dz, lddz, size, 16)) go(std::true_type());
        else go(std::false_type());
        return launched();
    });
}

int csr5_quantise(int32_t rows, int32_t n, int32_t block_rows, int dtype, const void* x, int64_t ldx, uint8_t* q, int64_t ldq, float* scale,
                  int64_t scale_row, int64_t scale_block, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || rows < 0 || n < 0 || (block_rows != 1 && block_rows != CSR5_F8_BLOCK)) return CSR5_EINVAL;
    if (rows > MOST_SIZE || n > MOST_SIZE) return CSR5_ERANGE;
    if (!rows_ok(x, rows, ldx, n, size) || !rows_ok(q, rows, ldq, n, 1)) return CSR5_EINVAL;
    if (rows == 0 || n == 0) return CSR5_OK;
    if (!scale || (reinterpret_cast<uintptr_t>(scale) & 3)) return CSR5_EINVAL;
    const int64_t blocks = divide_up(n, CSR5_F8_BLOCK);
    const int64_t groups = block_rows == 1 ? (int64_t(rows) * blocks + 15) / 16 : divide_up(rows, CSR5_F8_BLOCK) * blocks;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        auto go = [&](auto r, auto v) {
            k_quantise<T, decltype(r)::value, decltype(v)::value><<<workgroups(groups), 256, 0, s>>>(rows, n, static_cast<const T*>(x), ldx, q, ldq, scale, scale_row, scale_block);
        };
        auto by = [&](auto v) {
            if (block_rows == 1) go(std::integral_constant<int, 1>(), v);
            else go(std::integral_constant<int, CSR5_F8_BLOCK>(), v);
        };
        if (aligned(x, ldx, size, 16) && aligned(q, ldq, 1, 8)) by(std::true_type());
        else by(std::false_type());
        return launched();
    });
}

int csr5_rmsnorm(int32_t rows, int32_t n, int dtype, const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* gain,
                 float eps, void* h, int64_t ldh, void* y, int64_t ldy, uint8_t* q, int64_t ldq, float* scale, int64_t scale_row,
                 int64_t scale_block, float* rstd, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || rows < 0 || n < 0) return CSR5_EINVAL;
    if (n > CSR5_NORM_MAX_N) return CSR5_ERANGE;
    if (!rows_ok(x, rows, ldx, n, size) || (residual && !rows_ok(residual, rows, ldr, n, size)) || (h && !rows_ok(h, rows, ldh, n, size)) ||
        (y && !rows_ok(y, rows, ldy, n, size)) || (q && (!rows_ok(q, rows, ldq, n, 1) || !scale)) || (reinterpret_cast<uintptr_t>(gain) % size))
        return CSR5_EINVAL;
    if (rows == 0 || n == 0) return CSR5_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const NormArgs<T> a{rows, n, static_cast<const T*>(x), static_cast<const T*>(residual), static_cast<const T*>(gain), ldx, ldr, eps,
                            static_cast<T*>(h), static_cast<T*>(y), ldh, ldy, q, ldq, scale, scale_row, scale_block, rstd};
        const size_t wide = 16;
        const bool v = aligned(x, ldx, size, wide) && (!residual || aligned(residual, ldr, size, wide)) && aligned(gain, 0, size, wide) &&
                       (!h || aligned(h, ldh, size, wide)) && (!y || aligned(y, ldy, size, wide)) && (!q || aligned(q, ldq, 1, 8));
        norm_shape(n, [&](int threads, auto nv) {
            constexpr int NV = decltype(nv)::value;
            if (v) k_rmsnorm<T, NV, true><<<workgroups(rows), threads, 0, s>>>(a);
            else k_rmsnorm<T, NV, false><<<workgroups(rows), threads, 0, s>>>(a);
        });
        return launched();
    });
}

size_t csr5_rmsnorm_workspace_bytes(int32_t rows, int32_t n) {
    if (rows < 0 || n < 0 || n > CSR5_NORM_MAX_N) return 0;
    return n == 0 ? 0 : size_t(norm_groups(rows, n)) * size_t(n) * 4;
}

int csr5_rmsnorm_backward(int32_t rows, int32_t n, int dtype, const void* h, int64_t ldh, const void* gain, const float* rstd, const void* dy,
                          int64_t lddy, const void* residual_grad, int64_t ldrg, void* dh, int64_t lddh, float* dgain, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
    const size_t size = type_bytes(dtype);
    if (!size || rows < 0 || n < 0) return CSR5_EINVAL;
    if (n > CSR5_NORM_MAX_N) return CSR5_ERANGE;
    if (!rows_ok(h, rows, ldh, n, size) || !rows_ok(dy, rows, lddy, n, size) || !rows_ok(dh, rows, lddh, n, size) ||
        (residual_grad && !rows_ok(residual_grad, rows, ldrg, n, size)) || (reinterpret_cast<uintptr_t>(gain) % size) || (rows > 0 && !rstd))
        return CSR5_EINVAL;
    if (dgain && rows > 0 && n > 0 && (!workspace || workspace_bytes < csr5_rmsnorm_workspace_bytes(rows, n))) return CSR5_ENOMEM;
    if (reinterpret_cast<uintptr_t>(workspace) & 3) return CSR5_EINVAL;
    if (n == 0 || (rows == 0 && !dgain)) return CSR5_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const int groups = norm_groups(rows, n);
    return with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        const NormBackArgs<T> a{rows, n, static_cast<const T*>(h), static_cast<const T*>(gain), static_cast<const T*>(dy), static_cast<const T*>(residual_grad),
                                ldh, lddy, ldrg, rstd, static_cast<T*>(dh), lddh, dgain ? static_cast<float*>(workspace) : nullptr};
        const size_t wide = 16;
        const bool v = aligned(h, ldh, size, wide) && aligned(dy, lddy, size, wide) && aligned(dh, lddh, size, wide) && aligned(gain, 0, size, wide) &&
                       (!residual_grad || aligned(residual_grad, ldrg, size, wide));
        if (rows > 0)
            norm_shape(n, [&](int threads, auto nv) {
                constexpr int NV = decltype(nv)::value;
                if (v) k_rmsnorm_back<T, NV, true><<<groups, threads, 0, s>>>(a);
                else k_rmsnorm_back<T, NV, false><<<groups, threads, 0, s>>>(a);
            });
        if (dgain) k_columns<<<divide_up(n, 32), 1024, 0, s>>>(rows > 0 ? groups : 0, n, static_cast<const float*>(workspace), dgain);
        return launched();
    });
}

}  // extern "C"
