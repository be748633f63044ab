// libcsr5: what stands around the attention -- the pages of a step of serving, and rotary positions.  Bound by latency and by
// memory; the attention itself is in attention.hip.  The C ABI is declared in include/csr5.h.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "csr5.h"
#include "heads.h"
#include "numbers.h"

namespace {

// ---------------------------------------------------------------------------------------------------------------
// Pages.  A request's place among the new tokens, the pages taken and the pages given back is the sum of those before it: every
// workgroup adds all of them up (256 or 1024 requests at a time) and then writes its own share of the tokens, the new entries
// of the tables and the ring, finding the request of each by bisection over the sums in LDS; tokens, new entries and the ring are three workgroups', as each waits
// for memory.  Bound by the launch and four accesses to memory in turn: 48 requests 4.6 us, 700 that bring 30154 tokens 9.0 (one workgroup for everything
// 12.4 and 18.9; an empty launch 3.4).  So there is one launch and
// nothing to wait for between workgroups.
// ---------------------------------------------------------------------------------------------------------------
constexpr int PAGES_THREADS = 256, PAGES_SHARE = 1024;      // tokens, or entries, of a workgroup

struct PagesArgs {
    int requests, width, ring, shift, tokens;
    const int32_t *fresh, *length;
    int32_t* table;
    int64_t ldt;
    int32_t* pool;
    const int32_t* state;
    int32_t *offset, *position, *slot, *length_out, *state_out;
};

// Sums of three values over the threads before this one, and over all.
struct Sums {
    int64_t before[3], all[3];
};
template <int WAVES> __device__ __forceinline__ Sums sums_of(const int64_t (&v)[3], int64_t (&part)[3][WAVES]) {
    int64_t upto[3] = {v[0], v[1], v[2]};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        int64_t other[3];
#pragma unroll
        for (int k = 0; k < 3; k++) other[k] = __shfl_up(upto[k], d);
#pragma unroll
        for (int k = 0; k < 3; k++)
            if (lane >= d) upto[k] += other[k];
    }
    if (lane == 63) part[0][wave] = upto[0], part[1][wave] = upto[1], part[2][wave] = upto[2];
    __syncthreads();
    Sums s;
#pragma unroll
    for (int k = 0; k < 3; k++) {
        s.before[k] = upto[k] - v[k], s.all[k] = 0;
#pragma unroll
        for (int i = 0; i < WAVES; i++) {
            if (i < wave) s.before[k] += part[k][i];
            s.all[k] += part[k][i];
        }
    }
    return s;
}

// The last of the requests whose sum is at most `at`: the one that `at` lies in, as those after it without a share have a larger one.
__device__ __forceinline__ int request_at(const int32_t* first, int count, int32_t at) {
    int low = 0, high = count;
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        if (first[mid] <= at) low = mid;
        else high = mid;
    }
    return low;
}

template <int EACH> __global__ __launch_bounds__(PAGES_THREADS) void k_pages(PagesArgs a) {
    constexpr int THREADS = PAGES_THREADS, MANY = THREADS * EACH;     // requests at a time
    __shared__ int64_t part[3][THREADS / 64];
    __shared__ int32_t first[MANY];                                 // of what this workgroup writes; as far as there is room for it
    __shared__ int32_t wants[MANY];                                 // pages asked for before
    __shared__ int32_t lengths[MANY], held_pages[MANY];       // held_pages: -1 where a request is not served
    const int task = blockIdx.x % 3, group = blockIdx.x / 3, groups = gridDim.x / 3;     // tokens, new pages, pages that come back
    const int t = threadIdx.x;
    const int32_t mask = (1 << a.shift) - 1;
    const int64_t ring = max(a.ring, 1);
    const int32_t state = a.state[0];
    const int64_t head = state >= 0 && state < ring ? state : ((state % ring) + ring) % ring, count = min(max(int64_t(a.state[1]), int64_t(0)), int64_t(a.ring));
    const auto around = [&](int64_t i) { return i < ring ? i : i - ring; };         // of what is below 2 ring
    const int64_t most = int64_t(a.width) << a.shift;
    int64_t tokens = 0, asked = 0, taken = 0, back = 0;             // of the requests before these
    // this workgroup's part of `begin` to `last` of all
    const auto share = [&](int64_t begin, int64_t last, auto f) {
        if (begin >= last) return;                      // both are below 2^31 then
        const int32_t from = int32_t(begin), to = int32_t(last), skip = (group + groups - from / PAGES_SHARE % groups) % groups;
        for (int32_t base = from / PAGES_SHARE + skip; base <= (to - 1) / PAGES_SHARE; base += groups) {
            const int32_t end = base < to / PAGES_SHARE ? (base + 1) * PAGES_SHARE : to;
            for (int32_t i = max(base * PAGES_SHARE, from) + t; i < end; i += THREADS) f(i);
        }
    };
    const int64_t rooms[3] = {a.tokens, count, a.ring - count};
    const int64_t room = rooms[task];
    for (int r0 = 0; r0 < a.requests; r0 += MANY) {
        const int here = min(MANY, a.requests - r0);
        int32_t fresh[EACH], have[EACH];
#pragma unroll
        for (int e = 0; e < EACH; e++) {
            const int r = r0 + t * EACH + e;
            fresh[e] = r < a.requests ? a.fresh[r] : 0, have[e] = r < a.requests ? a.length[r] : 0;
        }
        int64_t v[3] = {0, 0, 0}, held[EACH], need[EACH];
        bool fits[EACH];
#pragma unroll
        for (int e = 0; e < EACH; e++) {
            have[e] = int32_t(min(int64_t(max(have[e], 0)), most));
            const int64_t wanted = (int64_t(have[e]) + max(fresh[e], 0) + mask) >> a.shift;
            held[e] = (int64_t(have[e]) + mask) >> a.shift;
            fits[e] = wanted <= a.width && fresh[e] >= 0;
            need[e] = fits[e] ? wanted - held[e] : 0;
            v[0] += max(fresh[e], 0), v[1] += need[e], v[2] += fresh[e] < 0 ? held[e] : 0;
        }
        if (r0 > 0) __syncthreads();
        const Sums s = sums_of<THREADS / 64>(v, part);
        int64_t token = tokens + s.before[0], want = asked + s.before[1], behind = back + s.before[2];
#pragma unroll
        for (int e = 0; e < EACH; e++) {
            const int r = r0 + t * EACH + e, i = t * EACH + e;
            // what is served is what all that is asked for up to it leaves room for
            const bool ok = fits[e] && (need[e] == 0 || want + need[e] <= count);
            first[i] = int32_t(min(room, task == 0 ? token : task == 1 ? want : behind)), wants[i] = int32_t(min(want, count)), lengths[i] = have[e], held_pages[i] = ok ? int32_t(held[e]) : -1;
            token += max(fresh[e], 0), want += need[e], behind += fresh[e] < 0 ? held[e] : 0;
            if (blockIdx.x == 0 && r < a.requests) {
                if (r == 0) a.offset[0] = 0;
                a.offset[r + 1] = int32_t(min(token, int64_t(a.tokens)));
                a.length_out[r] = fresh[e] < 0 ? 0 : ok ? have[e] + fresh[e] : have[e];
            }
            if (ok && need[e] > 0) taken = want;
        }
        __syncthreads();
        if (task == 0)
            share(tokens, min(tokens + s.all[0], room), [&](int32_t i) {
                const int q = request_at(first, here, i);
                const int32_t at = lengths[q] + (i - first[q]), holds = held_pages[q], p = at >> a.shift;
                int32_t slot = -1;
                if (holds >= 0) {
                    const int32_t page = p < holds ? a.table[int64_t(r0 + q) * a.ldt + p] : a.pool[around(head + wants[q] + (p - holds))];
                    if (page >= 0 && page <= (INT32_MAX >> a.shift)) slot = (page << a.shift) | (at & mask);       // others are no pages
                }
                a.position[i] = at, a.slot[i] = slot;
            });
        else if (task == 1)             // requests that are not served count here too, and are passed over
            share(asked, min(asked + s.all[1], room), [&](int32_t i) {
                const int q = request_at(first, here, i);
                if (held_pages[q] >= 0) a.table[int64_t(r0 + q) * a.ldt + held_pages[q] + (i - first[q])] = a.pool[around(head + i)];
            });
        else                            // behind the last free one; more than the ring has places for are not pages of it
            share(back, min(back + s.all[2], room), [&](int32_t i) {
                const int q = request_at(first, here, i);
                a.pool[around(around(head + count) + i)] = a.table[int64_t(r0 + q) * a.ldt + (i - first[q])];
            });
        tokens += s.all[0], asked += s.all[1], back += s.all[2];
    }
    if (task == 0)
        for (int64_t i = min(tokens, int64_t(a.tokens)) + int64_t(group) * THREADS + t; i < a.tokens; i += int64_t(groups) * THREADS) a.position[i] = 0, a.slot[i] = -1;
    if (blockIdx.x != 0) return;
    // the pages taken are those asked for up to the last request that got some: the most of all threads'
#pragma unroll
    for (int d = 1; d < 64; d *= 2) taken = max(taken, int64_t(__shfl_xor(taken, d)));
    __syncthreads();
    if ((t & 63) == 0) part[0][t >> 6] = taken;
    __syncthreads();
    if (t == 0) {
        for (int w = 1; w < THREADS / 64; w++) taken = max(taken, part[0][w]);
        if (a.requests == 0) a.offset[0] = 0;
        a.state_out[0] = int32_t(around(head + taken));
        a.state_out[1] = int32_t(count - taken + min(back, int64_t(a.ring) - count));
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Rotary positions.  A workgroup takes a few tokens; their angles' cosines and sines are computed once, into LDS, and serve all
// heads.  The angle, position * frequency, is a product of whole numbers below 2^31 and floats: in 32 bits a position of 10^6 would
// be off by 0.03 radians, so the product and its reduction to half a turn are in 64 bits, the cosine and sine of that in 32.
// Bound by memory: 16384 tokens of 28 + 4 heads of 128, three axes, 59 us (4.6 TB/s; value by value 177); 8191 of 16 + 16 heads of 64, backwards, 13.5 us (5.0; a
// large copy: 5.0); 24 tokens into the cache 3.7 us, a launch.
// ---------------------------------------------------------------------------------------------------------------
template <typename T> struct RotaryArgs {
    int tokens, heads, kv_heads, d, pairs, axes;
    const int32_t* position;
    int64_t ldp;
    const float* frequency;
    const int32_t* axis;
    bool inverse;
    Heads<T> q, q_out, k, k_out, v;
    const int32_t* slot;
    int32_t pages, shift;
    Cache<T> k_cache, v_cache;
};

constexpr int ROTARY_THREADS = 256, ROTARY_MANY = 1024;     // from so many tokens on a workgroup has four

// Cosines and sines of TOKENS tokens, in LDS: [token][pairs], then the sines.
template <int TOKENS, typename T> __device__ __forceinline__ void turns(const RotaryArgs<T>& a, int64_t token0, float* turn) {
    for (int i = threadIdx.x; i < TOKENS * a.pairs; i += ROTARY_THREADS) {
        const int t = TOKENS == 1 ? 0 : i / a.pairs, p = i - t * a.pairs;
        const int64_t token = min(token0 + t, int64_t(a.tokens - 1));
        const int32_t axis = a.axis ? a.axis[p] : 0;
        float c = 1.f, s = 0.f;
        if (uint32_t(axis) < uint32_t(a.axes)) {
            constexpr double TURN = 6.283185307179586476925;
            const double angle = double(a.position[axis * a.ldp + token]) * double(a.frequency[p]);
            sincosf(float(fma(-rint(angle * (1 / TURN)), TURN, angle)), &s, &c);
        }
        turn[i] = c, turn[TOKENS * a.pairs + i] = a.inverse ? -s : s;
    }
    __syncthreads();
}

// Value by value, for rows of any addresses.
template <typename T, bool INTERLEAVED> __global__ __launch_bounds__(ROTARY_THREADS) void k_rotary(RotaryArgs<T> a) {
    extern __shared__ float turn[];
    const int64_t token = workgroup();
    if (token >= a.tokens) return;
    turns<1>(a, token, turn);
    const int32_t slot = a.slot ? a.slot[token] : -1;
    const int32_t page = slot >> a.shift, place = slot & ((1 << a.shift) - 1);
    const bool cached = slot >= 0 && page < a.pages;
    const int each = a.d - a.pairs;                                 // a head: its pairs, and the values that stay
    for (int i = threadIdx.x; i < (a.heads + a.kv_heads) * each; i += ROTARY_THREADS) {
        const int h = i / each, e = i - h * each;
        const bool key = h >= a.heads;
        const int hk = h - a.heads;
        const T* const from = key ? a.k.p + token * a.k.row + hk * a.k.head : a.q.p + token * a.q.row + h * a.q.head;
        T* const to = key ? (a.k_out.p ? a.k_out.p + token * a.k_out.row + hk * a.k_out.head : nullptr) : a.q_out.p + token * a.q_out.row + h * a.q_out.head;
        T* const in = key && cached ? a.k_cache.p + page * a.k_cache.page + place * a.k_cache.row + hk * a.k_cache.head : nullptr;
        if (e < a.pairs) {
            const int x = INTERLEAVED ? 2 * e : e, y = INTERLEAVED ? 2 * e + 1 : e + a.pairs;
            const float p = float(from[x]), q = float(from[y]), c = turn[e], s = turn[a.pairs + e];
            const T u = T(p * c - q * s), w = T(p * s + q * c);
            if (to) to[x] = u, to[y] = w;
            if (in) in[x] = u, in[y] = w;
        } else {
            const T u = from[e + a.pairs];
            if (to) to[e + a.pairs] = u;
            if (in) in[e + a.pairs] = u;
        }
    }
    if (cached)
        for (int i = threadIdx.x; i < a.kv_heads * a.d; i += ROTARY_THREADS) {
            const int h = i / a.d, e = i - h * a.d;
            a.v_cache.p[page * a.v_cache.page + place * a.v_cache.row + h * a.v_cache.head + e] = a.v.p[token * a.v.row + h * a.v.head + e];
        }
}

// 16 bytes at a time.  A unit is 16 bytes of a head, or two times 16 whose values are pairs; a head has `units` of them (values have none to turn, and
// take the same number of places).  A workgroup's threads go through the units of its tokens.
template <typename T, bool INTERLEAVED, int TOKENS> __global__ __launch_bounds__(ROTARY_THREADS) void k_rotary_wide(RotaryArgs<T> a, int units, uint32_t inverse_units, int all_heads) {
    constexpr int V = 16 / sizeof(T), N = INTERLEAVED ? V / 2 : V;       // pairs of a unit
    extern __shared__ __align__(16) float turn[];
    const int64_t token0 = workgroup() * TOKENS;
    if (token0 >= a.tokens) return;
    turns<TOKENS>(a, token0, turn);
    const int tokens = int(min(int64_t(TOKENS), a.tokens - token0));
    const int total = all_heads * units, split = a.pairs / N;       // units that are turned
    int32_t page[TOKENS], place[TOKENS];
    bool cached[TOKENS];
#pragma unroll
    for (int t = 0; t < TOKENS; t++) {
        const int32_t slot = a.slot && t < tokens ? a.slot[token0 + t] : -1;
        page[t] = slot >> a.shift, place[t] = slot & ((1 << a.shift) - 1), cached[t] = slot >= 0 && page[t] < a.pages;
    }
    for (int i = threadIdx.x; i < total; i += ROTARY_THREADS) {
        const int h = units == 1 ? i : int(__umulhi(uint32_t(i), inverse_units)), u = i - h * units;
        const int hk = h - a.heads;
        if (hk >= a.kv_heads) {                                     // values, as they are
            const int hv = hk - a.kv_heads;
#pragma unroll
            for (int t = 0; t < TOKENS; t++) {
                if (!cached[t]) continue;
                const T* const from = a.v.p + (token0 + t) * a.v.row + hv * a.v.head;
                T* const in = a.v_cache.p + page[t] * a.v_cache.page + place[t] * a.v_cache.row + hv * a.v_cache.head;
                for (int c = u * V; c < a.d; c += units * V) *reinterpret_cast<uint4*>(in + c) = *reinterpret_cast<const uint4*>(from + c);
            }
            continue;
        }
        const bool key = hk >= 0, pair = u < split;
        // where the unit is: one place, or two
        const int c0 = INTERLEAVED || pair ? u * V : (u + split) * V, c1 = pair && !INTERLEAVED ? c0 + a.pairs : c0;
        const Heads<T> source = key ? a.k : a.q, result = key ? a.k_out : a.q_out;
        const int64_t from = (key ? hk : h) * source.head, to = (key ? hk : h) * result.head, in = hk * a.k_cache.head;
        vec<T, V> x[TOKENS], y[TOKENS];
#pragma unroll
        for (int t = 0; t < TOKENS; t++)
            if (t < tokens) {
                const T* const p = source.p + (token0 + t) * source.row + from;
                x[t] = *reinterpret_cast<const vec<T, V>*>(p + c0);
                if (!INTERLEAVED) y[t] = *reinterpret_cast<const vec<T, V>*>(p + c1);
            }
        if (pair) {
#pragma unroll
            for (int t = 0; t < TOKENS; t++)
                if (t < tokens) {
                    float c[N], s[N];
                    load_values<N, true>(turn + t * a.pairs + u * N, N, c);
                    load_values<N, true>(turn + (TOKENS + t) * a.pairs + u * N, N, s);
#pragma unroll
                    for (int e = 0; e < N; e++) {
                        if (INTERLEAVED) {
                            const float p = float(x[t][2 * e]), q = float(x[t][2 * e + 1]);
                            x[t][2 * e] = T(p * c[e] - q * s[e]), x[t][2 * e + 1] = T(p * s[e] + q * c[e]);
                        } else {
                            const float p = float(x[t][e]), q = float(y[t][e]);
                            x[t][e] = T(p * c[e] - q * s[e]), y[t][e] = T(p * s[e] + q * c[e]);
                        }
                    }
                }
        }
#pragma unroll
        for (int t = 0; t < TOKENS; t++)
            if (t < tokens) {
                if (!key || a.k_out.p) {
                    T* const p = result.p + (token0 + t) * result.row + to;
                    *reinterpret_cast<vec<T, V>*>(p + c0) = x[t];
                    if (!INTERLEAVED && pair) *reinterpret_cast<vec<T, V>*>(p + c1) = y[t];
                }
                if (key && cached[t]) {
                    T* const p = a.k_cache.p + page[t] * a.k_cache.page + place[t] * a.k_cache.row + in;
                    *reinterpret_cast<vec<T, V>*>(p + c0) = x[t];
                    if (!INTERLEAVED && pair) *reinterpret_cast<vec<T, V>*>(p + c1) = y[t];
                }
            }
    }
}

// Arrays of whole numbers of 32 bits: `rows` of `words`, ld apart.
struct Words {
    const void* p;
    int64_t words, rows = 1, ld = 0;
};
// Whether a, of one row, has a word that b has too.
bool share_words(const Words& a, const Words& b) {
    if (a.words == 0 || b.words == 0 || b.rows == 0) return false;
    const uint64_t from = reinterpret_cast<uintptr_t>(a.p), to = from + uint64_t(a.words) * 4, first = reinterpret_cast<uintptr_t>(b.p), row_bytes = uint64_t(b.words) * 4;
    if (to <= first) return false;
    const uint64_t begin = from > first ? from - first : 0, end = to - first;
    if (b.rows == 1) return begin < row_bytes;
    const uint64_t pitch = uint64_t(b.ld < (int64_t(1) << 60) ? b.ld : int64_t(1) << 60) * 4, row = begin / pitch;
    if (row >= uint64_t(b.rows)) return false;
    return begin - row * pitch < row_bytes || (row + 1 < uint64_t(b.rows) && end > (row + 1) * pitch);         // in the row, or as far as the next
}

}  // namespace

extern "C" {

int csr5_pages(int32_t requests, int32_t width, int32_t ring, int32_t page, int32_t tokens, const int32_t* fresh, const int32_t* length, int32_t* table,
               int64_t ldt, int32_t* pool, const int32_t* state, int32_t* offset, int32_t* position, int32_t* slot, int32_t* length_out, int32_t* state_out,
               void* hip_stream) {
    if (requests < 0 || width < 0 || ring < 0 || tokens < 0 || !power_of_two(page) || !state || !offset || !state_out) return CSR5_EINVAL;
    if (requests > MOST_SIZE || tokens > MOST_SIZE || int64_t(width) * page > INT32_MAX) return CSR5_ERANGE;
    if ((requests > 0 && (!fresh || !length || !length_out)) || !rows_ok(table, requests, ldt, width, 4) || (ring > 0 && !pool) || (tokens > 0 && (!position || !slot))) return CSR5_EINVAL;
    for (const void* p : {static_cast<const void*>(fresh), static_cast<const void*>(length), static_cast<const void*>(pool), static_cast<const void*>(state), static_cast<const void*>(offset),
                          static_cast<const void*>(position), static_cast<const void*>(slot), static_cast<const void*>(length_out), static_cast<const void*>(state_out)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return CSR5_EINVAL;
    // workgroups read the inputs, in no order, while others write
    const Words rows{table, width, requests, ldt};
    const Words one[] = {{pool, ring}, {offset, int64_t(requests) + 1}, {position, tokens}, {slot, tokens}, {length_out, requests}, {state_out, 2}, {fresh, requests}, {length, requests}, {state, 2}};
    constexpr int ALL = sizeof one / sizeof one[0], WRITTEN = 6;
    for (int i = 0; i < ALL; i++) {
        if (share_words(one[i], rows)) return CSR5_EINVAL;
        for (int j = i + 1; j < ALL && i < WRITTEN; j++)
            if (share_words(one[i], one[j])) return CSR5_EINVAL;
    }
    const PagesArgs a{requests, width, ring, __builtin_ctz(page), tokens, fresh, length, table, ldt, pool, state, offset, position, slot, length_out, state_out};
    const int64_t shares = divide_up(int64_t(tokens), PAGES_SHARE);
    const int groups = int(shares < 1 ? 1 : shares > 256 ? 256 : shares) * 3;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (requests <= PAGES_THREADS) k_pages<1><<<groups, PAGES_THREADS, 0, s>>>(a);
    else k_pages<4><<<groups, PAGES_THREADS, 0, s>>>(a);
    return launched();
}

int csr5_rotary(int32_t tokens, int32_t heads, int32_t kv_heads, int32_t d, int32_t rot, int dtype, int32_t axes, const int32_t* position, int64_t ldp,
                const float* frequency, const int32_t* axis, int interleaved, int inverse, csr5_heads_t q, csr5_heads_t q_out, csr5_heads_t k, csr5_heads_t k_out,
                csr5_heads_t v, const int32_t* slot, int32_t pages, int32_t page, csr5_cache_t k_cache, csr5_cache_t v_cache, void* hip_stream) {
    const size_t size = dtype == CSR5_DTYPE_F32 ? 4 : dtype == CSR5_DTYPE_BF16 || dtype == CSR5_DTYPE_F16 ? 2 : 0;
    if (!size || tokens < 0 || heads < 0 || kv_heads < 0 || d < 0 || rot < 0 || rot > d || rot % 2 || axes < 0) return CSR5_EINVAL;
    if (d > CSR5_ROTARY_MAX_D || tokens > MOST_SIZE || int64_t(heads) + kv_heads > CSR5_ATTENTION_MAX_HEADS || axes > MOST_SIZE) return CSR5_ERANGE;
    if (!heads_ok(q, tokens, heads, d, size) || !output_ok(q_out, tokens, heads, d, size) || !heads_ok(k, tokens, kv_heads, d, size) || (k_out.p && !output_ok(k_out, tokens, kv_heads, d, size))) return CSR5_EINVAL;
    if (slot && (pages < 0 || !power_of_two(page) || !heads_ok(v, tokens, kv_heads, d, size) || !cache_output_ok(k_cache, pages, page, kv_heads, d, size) || !cache_output_ok(v_cache, pages, page, kv_heads, d, size))) return CSR5_EINVAL;
    if (tokens > 0 && rot > 0 && axes > 0 && (!position || !frequency || ldp < tokens)) return CSR5_EINVAL;
    for (const void* p : {static_cast<const void*>(position), static_cast<const void*>(frequency), static_cast<const void*>(axis), static_cast<const void*>(slot)})
        if (reinterpret_cast<uintptr_t>(p) & 3) return CSR5_EINVAL;
    if (tokens == 0 || d == 0 || (heads == 0 && kv_heads == 0)) return CSR5_OK;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    auto typed_call = [&](auto zero) {
        using T = decltype(zero);
        const RotaryArgs<T> a{tokens, heads, kv_heads, d, rot / 2, axes, position, ldp, frequency, axis, inverse != 0, typed<T>(q), typed<T>(q_out), typed<T>(k), typed<T>(k_out),
                              typed<T>(v), slot, slot ? pages : 0, slot ? __builtin_ctz(page) : 0, typed<T>(k_cache), typed<T>(v_cache)};
        constexpr int V = 16 / sizeof(T);
        const int pairs = rot / 2, units = (interleaved ? d : d - pairs) / V, all_heads = heads + (slot ? 2 : 1) * kv_heads;
        const bool w = d % V == 0 && (interleaved ? rot : pairs) % V == 0 && units > 0 && int64_t(all_heads) * units < (1 << 22) && wide(q, size) && wide(q_out, size) && wide(k, size) &&
                       wide(k_out, size) && (!slot || (wide(v, size) && wide(k_cache, size) && wide(v_cache, size)));
        auto go = [&](auto inter) {
            constexpr bool I = decltype(inter)::value;
            const uint32_t inverse_units = units > 1 ? uint32_t(((uint64_t(1) << 32) + units - 1) / units) : 0;     // exact for what is below 2^32 / units
            if (!w) k_rotary<T, I><<<workgroups(tokens), ROTARY_THREADS, rot * 4, s>>>(a);
            else if (tokens >= ROTARY_MANY) k_rotary_wide<T, I, 4><<<workgroups(divide_up(tokens, 4)), ROTARY_THREADS, rot * 16, s>>>(a, units, inverse_units, all_heads);
            else k_rotary_wide<T, I, 1><<<workgroups(tokens), ROTARY_THREADS, rot * 4, s>>>(a, units, inverse_units, all_heads);
        };
        if (interleaved) go(std::true_type());
        else go(std::false_type());
        return launched();
    };
    return dtype == CSR5_DTYPE_F32 ? typed_call(float()) : dtype == CSR5_DTYPE_F16 ? typed_call(f16()) : typed_call(bf16());
}

}  // extern "C"
