// Distillation from a teacher's top logits on maps: a class's positions are adjacent (distill.hip has the formulas).
//
// Bound by memory as the rows: the logits are read and the gradient is written once where a tile's logits fit LDS or
// registers (up to 1024 classes); of more classes they are read twice.
//
// 1.88 million positions of 64 binary32 classes: 298 us, 3.6 TB/s with the lists, where no channel's positions are whole lines, and 243
// where they are; 198025 of 1000 bfloat16 classes 304 us (2.7 TB/s), 198016 235 (3.5); 20480 of 5000 binary32 classes 277 us.
#include <algorithm>
#include <type_traits>

#include "dev_common.h"
#include "distill.h"
#include "dss_internal.h"

namespace dss {

namespace {

// ------------------------------------------------------------------ few classes
// A lane for each position, its logits in a column of LDS that no other lane touches: lists are gathered, and what they take
// off the listed classes is taken off, there, with no barrier.  The column has the logits, then their exponentials, less
// what the list takes off them.
// kPlaces places of a list, loaded together: what a pass over a list costs is its loads' latency.  Lists of no more stay
// in registers.
constexpr int kPlaces = 8;
struct Places {
    int id[kPlaces];
    float t[kPlaces];

    __device__ __forceinline__ void load(const Distill& D, int64_t m, int j0) {
#pragma unroll
        for (int j = 0; j < kPlaces; ++j) {
            id[j] = class_of(D, m, min(j0 + j, D.k - 1));
            t[j] = teacher_of(D, m, min(j0 + j, D.k - 1));
        }
#pragma unroll
        for (int j = 0; j < kPlaces; ++j) {
            if (j0 + j >= D.k) id[j] = -1;
            if (id[j] < 0) t[j] = -INFINITY;
        }
    }
};

// The sum of N values by halves. A lane has all of a position's terms, and one after the other the small ones would be
// rounded away beside a large one: losses of 200000 positions of 100 classes with 60 places were off by 2.0e-7 of them (root mean
// square) that way, by 1.1e-7 by halves, in 430 and 432 us; with 8 places of 64 classes by 1.1e-7 and 0.9e-7.
template <int N>
__device__ __forceinline__ float by_halves(float (&v)[N]) {
#pragma unroll
    for (int n = 1; n < N; n *= 2)
#pragma unroll
        for (int i = 0; i + n < N; i += 2 * n) v[i] += v[i + n];
    return v[0];
}

// f(number, class) for all classes: 32, 8 and one at a time, so that what a class waits for is under way for others too.
template <typename F>
__device__ __forceinline__ void over_classes(int C, F f) {
    int c = 0;
    for (; c + 32 <= C; c += 32) f(std::integral_constant<int, 32>{}, c);
    for (; c + 8 <= C; c += 8) f(std::integral_constant<int, 8>{}, c);
    for (; c < C; ++c) f(std::integral_constant<int, 1>{}, c);
}

template <typename T, bool PAST>
__global__ __launch_bounds__(64) void distill_columns_kernel(Distill D) {
    extern __shared__ float columns[];
    const int C = (int)D.C, lane = threadIdx.x, k = D.k;
    float* const col = columns + lane;
    const int64_t own = xcd_order(blockIdx.x, gridDim.x) * 64 + lane, m = min(own, D.M - 1);
    Places a;
    a.load(D, m, 0);
    const float weight = D.weights ? D.weights[m] : 1.f;
    float z_max = -INFINITY;
    const T* z = static_cast<const T*>(D.z) + m;
    over_classes(C, [&](auto n, int c) {
        float v[n];
#pragma unroll
        for (int u = 0; u < n; ++u, z += D.cs) v[u] = to_f32(PAST ? __builtin_nontemporal_load(z) : *z);
#pragma unroll
        for (int u = 0; u < n; ++u) {
            col[(c + u) * 64] = v[u];
            z_max = fmaxf(z_max, v[u]);
        }
    });
    // f of the list's places, batch by batch
    auto over_places = [&](auto f) {
        for (int j0 = 0; j0 < k; j0 += kPlaces) {
            if (k > kPlaces) a.load(D, m, j0);
#pragma unroll
            for (int j = 0; j < kPlaces; ++j) f(a.id[j], a.t[j]);
        }
    };
    // Adds up N terms of each place, those that f(terms, class, logit) gives: a batch by halves, 8 batches, and then these.
    auto sums_of = [&](auto& all, auto f) {
        constexpr int N = std::extent_v<std::remove_reference_t<decltype(all)>>;
        for (int j1 = 0; j1 < k; j1 += 8 * kPlaces) {
            float some[N] = {};
            for (int j0 = j1; j0 < min(j1 + 8 * kPlaces, k); j0 += kPlaces) {
                if (k > kPlaces) a.load(D, m, j0);
                float v[N][kPlaces];
#pragma unroll
                for (int j = 0; j < kPlaces; ++j) {
                    float terms[N] = {};
                    f(terms, a.id[j], a.t[j]);
#pragma unroll
                    for (int n = 0; n < N; ++n) v[n][j] = terms[n];
                }
#pragma unroll
                for (int n = 0; n < N; ++n) some[n] += by_halves(v[n]);
            }
#pragma unroll
            for (int n = 0; n < N; ++n) all[n] += some[n];
        }
    };
    float t_max = -INFINITY, state = 0.f;
    over_places([&](int id, float t) {
        t_max = fmaxf(t_max, t);
        state = fmaxf(state, Place{id, t, 0.f}.state(D));
    });
    const bool live = weight != 0.f && state != 0.f;
    const float nan = state == 3.f ? quiet_nan() : 0.f;
    float sum_r = nan, sums_p[1] = {nan};
    sums_of(sums_p, [&](float (&terms)[1], int id, float t) { terms[0] = weight_of(D, t, t_max); });
    // the loss but for its last term, sum p log(sum_p / sum_r), and sum p
    const float sum_p = sums_p[0], per_p = 1.f / sum_p;
    float of_p[2] = {nan, 0.f};
    sums_of(of_p, [&](float (&terms)[2], int id, float t) {
        if (id < 0 || id >= C) return;
        const float p = weight_of(D, t, t_max) * per_p;
        terms[0] = loss_of(D, p, t, t_max, col[id * 64], z_max, 0.f);
        terms[1] = p;
    });
    over_classes(C, [&](auto n, int c) {
        float v[n];
#pragma unroll
        for (int u = 0; u < n; ++u) v[u] = col[(c + u) * 64];
#pragma unroll
        for (int u = 0; u < n; ++u) {
            v[u] = exp2_of((v[u] - z_max) * D.to_log2);
            col[(c + u) * 64] = v[u];
        }
        sum_r += by_halves(v);
    });
    const float loss = of_p[0] - of_p[1] * (logf(sum_p) - logf(sum_r));
    const float g = D.scale * weight * D.T;
    if (own < D.M) D.losses[m] = live ? g * (D.T * loss) : 0.f;
    if (!D.grad) return;
    over_places([&](int id, float t) {
        if (id >= 0 && id < C) col[id * 64] -= weight_of(D, t, t_max) * per_p * sum_r;
    });
    if (own >= D.M) return;
    const float per = g / sum_r;
    T* grad = static_cast<T*>(D.grad) + m;
    over_classes(C, [&](auto n, int c) {
        float v[n];
#pragma unroll
        for (int u = 0; u < n; ++u) v[u] = col[(c + u) * 64];
#pragma unroll
        for (int u = 0; u < n; ++u, grad += D.gcs) {
            T r;
            store_elem(&r, live ? v[u] * per : 0.f);
            if constexpr (PAST) __builtin_nontemporal_store(r, grad);
            else *grad = r;
        }
    });
}

// ------------------------------------------------------------------ tiles
// A workgroup has the 16 V positions of 16 lanes with W words each; a lane has 16 adjacent classes of its V positions, so a
// wave has 64 classes.
template <typename T, int W>
struct Tile {
    static constexpr int V = Logits<T, W>::E, kTokens = 16 * V;
    Logits<T, W> c[16];

    // The lane's classes c0 .. c0+15, those below C, of the V positions from p on; -infinity elsewhere.
    __device__ __forceinline__ void load(const T* p, int64_t cs, int c0, int C) {
        p += c0 * cs;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            c[r].clear();
            if (c0 + r < C) c[r].load(p);
            p += cs;
        }
    }
    // The same of the first n positions from p on.
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T* p, int64_t cs, int64_t c0, int64_t C, int64_t n) {
#pragma unroll
        for (int r = 0; r < 16; ++r) c[r].template load<PAST>(p + (c0 + r) * cs, c0 + r < C ? n : 0);
    }
    __device__ __forceinline__ void raise_into(float (&top)[V]) const {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v) top[v] = fmaxf(top[v], c[r].value(v));
    }
};

// Each position's value over the lanes that have it; room has V * 16 places for each wave.
template <typename Op, int V>
__device__ __forceinline__ void over_tile(float (&v)[V], float* room) {
    const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        v[j] = Op::of(v[j], __shfl_xor(v[j], 16));
        v[j] = Op::of(v[j], __shfl_xor(v[j], 32));
    }
    __syncthreads();
    if (lane < 16)
#pragma unroll
        for (int j = 0; j < V; ++j) room[((threadIdx.x >> 6) * 16 + lane) * V + j] = v[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = room[(lane & 15) * V + j];
    for (int w = 1; w < waves; ++w)
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = Op::of(v[j], room[(w * 16 + (lane & 15)) * V + j]);
}

// The lists of a tile's N positions in LDS: classes, the teacher's logits (-infinity at empty places; later their parts of
// the gradient) and the student's; and of each position what its loss is made of.
template <typename T, int N>
struct Lists {
    static constexpr int kTMax = 0, kPerP = N, kRef = 2 * N, kParts = 3 * N, kMass = 4 * N, kState = 5 * N, kPlace0 = 6 * N;
    float* at;
    int k;

    // (an odd number of places, so that positions start in different banks)
    static __host__ __device__ int pitch(int k) { return k | 1; }
    // Before the student's logits, and with them.
    static __host__ __device__ size_t bytes_of_t(int k) { return (size_t)N * (6 + 2 * pitch(k)) * 4; }
    static __host__ __device__ size_t bytes(int k) { return (size_t)N * (6 + 3 * pitch(k)) * 4; }
    // Place j of position n.
    __device__ __forceinline__ int& id(int j, int n) const { return reinterpret_cast<int*>(at)[kPlace0 + n * pitch(k) + j]; }
    __device__ __forceinline__ float& t(int j, int n) const { return at[kPlace0 + (N + n) * pitch(k) + j]; }
    __device__ __forceinline__ float& z(int j, int n) const { return at[kPlace0 + (2 * N + n) * pitch(k) + j]; }

    // f(place, position) of all places, a thread for each.
    template <typename F>
    __device__ __forceinline__ void over_places(F f) const {
        for (int i = threadIdx.x; i < k * N; i += blockDim.x) f(i / N, i % N);
    }
    __device__ __forceinline__ void read(const Distill& D, int64_t m0, const T* logits) const {
#pragma unroll 4
        for (int i = threadIdx.x; i < k * N; i += blockDim.x) {
            const int64_t m = min(m0 + i % N, D.M - 1);
            const int c = class_of(D, m, i / N);
            const float a = teacher_of(D, m, i / N);
            id(i / N, i % N) = c;
            t(i / N, i % N) = c >= 0 ? a : -INFINITY;
            z(i / N, i % N) = c >= 0 && c < (int)D.C ? to_f32(logits[m + c * D.cs]) : 0.f;
        }
    }
    // Of each position, from its list alone, 16 lanes for one: with p of the list, z' the largest of its student's logits and
    // d_j = (t_j - t_max) / T - (z_j - z') / T, the sums of p_j d_j and of p_j.  Its loss is then
    // sum p_j d_j - sum p_j ((z' - z_max) / T + log(sum_p / sum_r)).
    __device__ __forceinline__ void sum_up(const Distill& D, int64_t m0) const {
        const int lane = threadIdx.x & 15;
        for (int n = threadIdx.x >> 4; n < N; n += blockDim.x >> 4) {
            float tops[2] = {-INFINITY, 0.f};              // t_max, the list's state
            const bool there = m0 + n < D.M;
            for (int j = lane; j < k && there; j += 16) {
                const float a = t(j, n);
                tops[0] = fmaxf(tops[0], a);
                tops[1] = fmaxf(tops[1], Place{id(j, n), a, 0.f}.state(D));
            }
            over_lanes<Max, 16>(tops, nullptr);
            const float t_max = tops[0];
            float sum[1] = {0.f}, ref[1] = {-3.4028235e38f};
            for (int j = lane; j < k && there; j += 16) {
                const float p = weight_of(D, t(j, n), t_max);
                sum[0] += p;
                if (p > 0.f) ref[0] = fmaxf(ref[0], z(j, n));
            }
            over_lanes<Sum, 16>(sum, nullptr);
            over_lanes<Max, 16>(ref, nullptr);
            const float per_p = tops[1] == 3.f ? quiet_nan() : 1.f / sum[0];
            float sums[2] = {0.f, 0.f};                    // of p d, of p
            for (int j = lane; j < k && there; j += 16) {
                const float a = t(j, n), p = weight_of(D, a, t_max) * per_p;
                sums[0] += p <= 0.f ? 0.f : p * (((a - t_max) - (z(j, n) - ref[0])) * (D.to_log2 * kLn2));
                sums[1] += p;
            }
            over_lanes<Sum, 16>(sums, nullptr);
            if (lane != 0) continue;
            at[kTMax + n] = t_max;
            at[kPerP + n] = per_p;
            at[kRef + n] = ref[0];
            at[kParts + n] = sums[0];
            at[kMass + n] = sums[1];
            // 0: nothing is to be learnt
            at[kState + n] = there && D.weights && D.weights[m0 + n] == 0.f ? 0.f : tops[1];
        }
    }
    // Of position n, from its list and its logits' largest and sum: whether there is anything to learn, and the gradient's factor.
    __device__ __forceinline__ float factor(const Distill& D, int64_t m, int n) const {
        return D.scale * (D.weights ? D.weights[min(m, D.M - 1)] : 1.f) * D.T;
    }
    __device__ __forceinline__ void put_loss(const Distill& D, int64_t m0, int n, float top, float sum) const {
        const float state = at[kState + n], sum_r = state == 3.f ? quiet_nan() : sum;
        const float away = (at[kRef + n] - top) * (D.to_log2 * kLn2) - logf(at[kPerP + n]) - logf(sum_r);
        D.losses[m0 + n] = state == 0.f ? 0.f : factor(D, m0 + n, n) * (D.T * (at[kParts + n] - at[kMass + n] * away));
    }
    // Whether the class of place j is in position n's list at another place too.
    __device__ __forceinline__ bool again(int j, int n) const {
        const int c = id(j, n);
        bool other = false;
#pragma unroll 8
        for (int i = 0; i < k; ++i) other |= id(i, n) == c && i != j;
        return other && c >= 0;
    }
    // The teacher's logits become what they take off the gradient of their class, p_of(logit, position), and of a class that is
    // there more than once (twice(place, position)) all of it at its first place, whose other places are emptied.
    template <typename F, typename G>
    __device__ __forceinline__ void share_out(F p_of, G twice) const {
        over_places([&](int j, int n) { t(j, n) = p_of(t(j, n), n); });
        __syncthreads();
        uint64_t later = 0;              // a bit for each of the thread's places, of which there are at most 64
        int turn = 0;
        over_places([&](int j, int n) {
            if (twice(j, n)) {
                const int c = id(j, n);
                float p = t(j, n);
                bool first = true;
                for (int i = 0; i < k && first; ++i) {
                    if (i == j || id(i, n) != c) continue;
                    if (i < j) first = false;
                    else p += t(i, n);
                }
                if (first) t(j, n) = p;  // (nobody else reads a first place)
                else later |= 1ull << turn;
            }
            ++turn;
        });
        __syncthreads();
        turn = 0;
        over_places([&](int j, int n) {
            if (later >> turn++ & 1) id(j, n) = -1;
        });
    }
};

// Which place of its position's list a class has (counted from 1; 0: none), a byte for each class of a tile and
// position.  Gradients are then written once: stored over, a listed class's line would come back from memory and go there again.
template <int N>
struct Marks {
    uint8_t* at;

    static __host__ __device__ int bytes(int classes) { return (classes + 15) / 16 * 16 * N; }
    // (16 classes are a lane's: the same one of its neighbours' lies in other banks)
    __device__ __forceinline__ uint8_t* of(int c, int n) const { return at + (c ^ ((c >> 4) & 3)) * N + n; }
    __device__ __forceinline__ void clear(int classes) const {
        for (int i = threadIdx.x; i < bytes(classes) / 4; i += blockDim.x) reinterpret_cast<uint32_t*>(at)[i] = 0;
    }
};

// What the places of a part's listed classes take off their gradients.
template <int N>
struct Shares {
    float* at;
    int k;

    static __host__ __device__ size_t bytes(int k) { return (size_t)N * (k | 1) * 4; }
    __device__ __forceinline__ float& t(int j, int n) const { return at[n * (k | 1) + j]; }
};

// Takes off V adjacent positions' gradients of a class what its places take.
template <typename List, int N, int V>
__device__ __forceinline__ void take_off(float (&v)[V], const List& lists, const Marks<N>& marks, int c, int n) {
    using Word = std::conditional_t<V == 2, uint16_t, uint32_t>;
    const uint32_t places = *reinterpret_cast<const Word*>(marks.of(c, n));
    if (places == 0) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int place = places >> (8 * j) & 255;
        if (place) v[j] -= lists.t(place - 1, n + j);
    }
}

// Up to 1024 classes: the tile's logits stay in registers.  Whole tiles only: the last one ends with the last
// position and writes those from `first` on, which the one before it does not have.  (What it reads of the others
// may be their gradients already, if these are written over the logits; positions do not mix.)
template <typename T, int W, bool PAST>
__global__ __launch_bounds__(1024) __attribute__((amdgpu_waves_per_eu(16 / W))) void distill_tile_kernel(Distill D) {
    constexpr int V = Tile<T, W>::V, N = Tile<T, W>::kTokens;
    using List = Lists<T, N>;
    extern __shared__ __align__(16) char lds[];
    const List lists = {reinterpret_cast<float*>(lds), D.k};
    const int64_t tile0 = xcd_order(blockIdx.x, gridDim.x) * N, m0 = min(tile0, D.M - N);
    const int first = (int)(tile0 - m0), l16 = threadIdx.x & 15, C = (int)D.C;
    float* const room = reinterpret_cast<float*>(lds + List::bytes_of_t(D.k));
    // (the marks take the place of the student's logits)
    const Marks<N> marks = {reinterpret_cast<uint8_t*>(room + (blockDim.x >> 6) * N)};
    const T* z = static_cast<const T*>(D.z);
    int c0 = (threadIdx.x >> 4) * 16;
    // (the lists first: there are no registers for them beside the tile, but another workgroup's work)
    lists.read(D, m0, z);
    __syncthreads();
    lists.sum_up(D, m0);
    __syncthreads();
    if (D.grad) {
        marks.clear(C);
        lists.share_out([&](float t, int n) {
            return lists.factor(D, m0 + n, n) * (weight_of(D, t, lists.at[List::kTMax + n]) * lists.at[List::kPerP + n]);
        }, [&](int j, int n) { return lists.again(j, n); });
        lists.over_places([&](int j, int n) {
            const int c = lists.id(j, n);
            if (c >= 0 && c < C && lists.at[List::kState + n] != 0.f) *marks.of(c, n) = (uint8_t)(j + 1);
        });
    }
    __builtin_amdgcn_sched_barrier(0);
    Tile<T, W> tile;
    tile.load(z + m0 + l16 * V, D.cs, c0, C);
    float top[V], sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) top[v] = -INFINITY, sum[v] = 0.f;
    tile.raise_into(top);
#pragma unroll
    for (int r = 0; r < 16; ++r) tile.c[r].forget();
    over_tile<Max>(top, room);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float e = exp2_of((tile.c[r].value(v) - top[v]) * D.to_log2);
            if constexpr (sizeof(T) == 4) tile.c[r].w[v] = __float_as_uint(e);       // (bfloat16 has no room for it)
            sum[v] += e;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) tile.c[r].forget();
    over_tile<Sum>(sum, room);
    float per[V];
    uint32_t live = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int n = l16 * V + v;
        const float state = lists.at[List::kState + n];
        const float per_sum = state == 3.f ? quiet_nan() : 1.f / sum[v];
        live |= (state != 0.f ? 1u : 0u) << v;
        per[v] = lists.factor(D, m0 + n, n) * per_sum;
        if (threadIdx.x < 16 && n >= first) lists.put_loss(D, m0, n, top[v], sum[v]);
    }
    if (!D.grad) return;
    T* grad = static_cast<T*>(D.grad);
    asm volatile("" : "+v"(c0));         // (nothing of the loads' addresses is kept)
    T* p = grad + m0 + l16 * V + c0 * D.gcs;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        if (c0 + r < C) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[j] = sizeof(T) == 4 ? tile.c[r].value(j) : exp2_of((tile.c[r].value(j) - top[j]) * D.to_log2);
                v[j] = live >> j & 1 ? v[j] * per[j] : 0.f;
            }
            take_off(v, lists, marks, c0 + r, l16 * V);
            if (l16 * V >= first) {
                store_gradients<PAST>(p, v, V);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (l16 * V + j >= first) store_elem(p + j, v[j]);
            }
        }
        p += D.gcs;
        asm volatile("" : "+v"(p));      // (one address at a time: there are no registers for 16)
    }
}

// More classes, or too few positions for the units: `parts` workgroups share a tile's classes.  First each takes its
// part's largest logits and sums.
constexpr int kPartThreads = 256, kPartSpan = kPartThreads / 16 * 16;

// The workgroup's tile and part: neighbouring tiles of a part, which may share lines, on one XCD (20481 positions of 5000 binary32
// classes 330 us for 378; where they do not share any 277 for 267).
__device__ __forceinline__ int2 tile_and_part() {
    const int id = (int)xcd_order(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
    return {id % (int)gridDim.x, id / (int)gridDim.x};
}

template <typename T, bool PAST>
__global__ __launch_bounds__(kPartThreads) void distill_map_parts_kernel(Distill D, int64_t per_part, Part* parts) {
    constexpr int V = Tile<T, 4>::V;
    __shared__ float room[kPartThreads / 64 * 16 * V];
    const int2 own = tile_and_part();
    const int64_t m = (int64_t)own.x * Tile<T, 4>::kTokens + (threadIdx.x & 15) * V;
    const int64_t c1 = min((own.y + 1) * per_part, D.C);
    const T* z = static_cast<const T*>(D.z);
    float top[V], sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) top[v] = -INFINITY, sum[v] = 0.f;
    for (int64_t c0 = own.y * per_part; c0 < c1; c0 += kPartSpan) {
        Tile<T, 4> tile;
        tile.template load<PAST>(z + m, D.cs, c0 + (threadIdx.x >> 4) * 16, c1, D.M - m);
        float next[V];
#pragma unroll
        for (int v = 0; v < V; ++v) next[v] = top[v];
        tile.raise_into(next);
#pragma unroll
        for (int r = 0; r < 16; ++r) tile.c[r].forget();
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float to = next[v] == -INFINITY ? 0.f : next[v];
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) s += exp2_of((tile.c[r].value(v) - to) * D.to_log2);
            sum[v] = sum[v] * exp2_of((top[v] - to) * D.to_log2) + s;
            top[v] = next[v];
        }
    }
    float all[V];
#pragma unroll
    for (int v = 0; v < V; ++v) all[v] = top[v];
    over_tile<Max>(all, room);
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = joined(D, {all[v], 0.f}, {top[v], sum[v]}).sum;
    over_tile<Sum>(sum, room);
    if (threadIdx.x < 16)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (m + v < D.M) parts[(m + v) * gridDim.y + own.y] = {all[v], sum[v]};
}

// What the gradients of a slab's positions are made of, one array after the other.
constexpr int64_t kSlabPositions = 32768;
struct Stats {
    float* at;
    __device__ __forceinline__ float& z_max(int64_t m) const { return at[m]; }
    __device__ __forceinline__ float& per_sum(int64_t m) const { return at[kSlabPositions + m]; }
    __device__ __forceinline__ float& t_max(int64_t m) const { return at[2 * kSlabPositions + m]; }
    __device__ __forceinline__ float& per_p(int64_t m) const { return at[3 * kSlabPositions + m]; }
    __device__ __forceinline__ float& factor(int64_t m) const { return at[4 * kSlabPositions + m]; }
    // 0: nothing is to be learnt, 1: every class is in the list once, 2: one is there more than once.
    __device__ __forceinline__ float& kind(int64_t m) const { return at[5 * kSlabPositions + m]; }
};
constexpr int kStats = 6;

// Then the parts are joined and the lists summed up, 16 lanes for a position: the losses, and the positions' stats.
constexpr int kJoined = kPartThreads / 16;

template <typename T>
__global__ __launch_bounds__(kPartThreads) void distill_map_join_kernel(Distill D, const Part* parts, int n_parts, Stats stats) {
    using List = Lists<T, kJoined>;
    extern __shared__ __align__(16) char lds[];
    const List lists = {reinterpret_cast<float*>(lds), D.k};
    const int64_t m0 = (int64_t)blockIdx.x * kJoined, m = m0 + (threadIdx.x >> 4);
    const int lane = threadIdx.x & 15, n = threadIdx.x >> 4;
    lists.read(D, m0, static_cast<const T*>(D.z));
    __syncthreads();
    lists.sum_up(D, m0);
    Part own = {-INFINITY, 0.f};
#pragma unroll 8
    for (int p = lane; p < n_parts; p += 16) own = joined(D, own, parts[min(m, D.M - 1) * n_parts + p]);
    float top[1] = {own.top};
    over_lanes<Max, 16>(top, nullptr);
    float sum[1] = {joined(D, {top[0], 0.f}, own).sum}, twice[1] = {0.f};
    over_lanes<Sum, 16>(sum, nullptr);
    for (int j = lane; j < D.k; j += 16)
        if (lists.again(j, n)) twice[0] = 1.f;
    over_lanes<Max, 16>(twice, nullptr);
    __syncthreads();
    if (lane != 0 || m >= D.M) return;
    // (a position of -infinities has the sum 0 here, and no softmax)
    const float sum_r = top[0] == -INFINITY ? quiet_nan() : sum[0], state = lists.at[List::kState + n];
    stats.z_max(m) = top[0];
    stats.per_sum(m) = state == 3.f ? quiet_nan() : 1.f / sum_r;
    stats.t_max(m) = lists.at[List::kTMax + n];
    stats.per_p(m) = lists.at[List::kPerP + n];
    stats.factor(m) = lists.factor(D, m, n);
    stats.kind(m) = state == 0.f ? 0.f : 1.f + twice[0];
    lists.put_loss(D, m0, n, top[0], sum_r);
}

// Then the gradient, a part of a tile's classes for a workgroup, a span of them at a time.
template <typename T, bool PAST>
__global__ __launch_bounds__(kPartThreads) void distill_map_gradient_kernel(Distill D, int64_t per_part, Stats stats) {
    constexpr int W = (int)sizeof(T), V = Tile<T, W>::V, N = Tile<T, W>::kTokens;
    extern __shared__ __align__(16) char lds[];
    const Shares<N> shares = {reinterpret_cast<float*>(lds), D.k};
    const Marks<N> marks = {reinterpret_cast<uint8_t*>(lds + Shares<N>::bytes(D.k))};
    const int2 place = tile_and_part();
    const int64_t m0 = (int64_t)place.x * N, m = m0 + (threadIdx.x & 15) * V;
    const int64_t c_from = place.y * per_part, c1 = min(c_from + per_part, D.C);
    const T* z = static_cast<const T*>(D.z);
    T* grad = static_cast<T*>(D.grad);
    marks.clear(kPartSpan);
    // The part's listed classes, and what their places take off: of the thread's places a bit for each that there is.
    constexpr int U = 8;                 // classes under way
    uint64_t mine = 0;
    for (int turn = 0; turn * kPartThreads < D.k * N; turn += U) {
        int c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = (turn + u) * kPartThreads + threadIdx.x;
            c[u] = class_of(D, min(m0 + i % N, D.M - 1), min(i / N, D.k - 1));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = (turn + u) * kPartThreads + threadIdx.x, j = i / N, n = i % N;
            if (i >= D.k * N || m0 + n >= D.M || c[u] < c_from || c[u] >= c1) continue;
            const int64_t p = m0 + n;
            const float kind = stats.kind(p);
            auto share = [&](int place) { return weight_of(D, teacher_of(D, p, place), stats.t_max(p)) * stats.per_p(p); };
            float of_class = share(j);
            bool first = kind != 0.f;
            if (kind == 2.f)             // (a class that is there more than once: all of it at its first place)
                for (int o = 0; o < D.k && first; ++o) {
                    if (o == j || class_of(D, p, o) != c[u]) continue;
                    if (o < j) first = false;
                    else of_class += share(o);
                }
            if (!first) continue;
            shares.t(j, n) = stats.factor(p) * of_class;
            mine |= 1ull << (turn + u);
        }
    }
    // the marks of the span's listed classes, or none again
    auto mark = [&](int64_t c0, bool set) {
        for (uint64_t left = mine; left; left &= left - 1) {
            const int i = (int)(__ffsll((long long)left) - 1) * kPartThreads + threadIdx.x;
            const int64_t c = class_of(D, m0 + i % N, i / N) - c0;
            if (c >= 0 && c < kPartSpan) *marks.of((int)c, i % N) = (uint8_t)(set ? i / N + 1 : 0);
        }
    };
    __syncthreads();                     // the marks are clear
    float per[V], top[V];
    uint32_t live = 0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int64_t p = min(m + v, D.M - 1);
        live |= (stats.kind(p) != 0.f ? 1u : 0u) << v;
        per[v] = stats.factor(p) * stats.per_sum(p), top[v] = stats.z_max(p);
    }
    const int own = (threadIdx.x >> 4) * 16;
    for (int64_t span = c_from; span < c1; span += kPartSpan) {
        const int64_t c0 = span + own;
        Tile<T, W> tile;
        tile.load(z + m, D.cs, c0, c1, D.M - m);
        mark(span, true);
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (c0 + r >= c1 || m >= D.M) continue;
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = exp2_of((tile.c[r].value(j) - top[j]) * D.to_log2) * per[j];
            take_off(v, shares, marks, own + r, (threadIdx.x & 15) * V);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = live >> j & 1 ? v[j] : 0.f;
            store_gradients<PAST>(grad + m + (c0 + r) * D.gcs, v, D.M - m);
        }
        if (span + kPartSpan >= c1) break;
        __syncthreads();
        mark(span, false);
        __syncthreads();                 // (a class of the next span may have the same mark)
    }
}

// Whether the gradient goes around the caches: large, and of whole lines, which 16 lanes' stores fill.  198016 positions of 1000
// bfloat16 classes 235 us, through the caches 263; where lines are shared with other tiles' stores (198025) 404 and 308.
bool gradient_past(const Distill& D, dss_dtype dt) { return D.grad && outputs_past(D.M, D.C, D.gcs, D.grad, dt); }

template <typename T>
hipError_t run_columns(const Distill& D, dss_dtype dt, hipStream_t s) {
    const bool past = (!D.grad || gradient_past(D, dt)) && outputs_past(D.M, D.C, D.cs, D.z, dt);
    const auto kern = past ? distill_columns_kernel<T, true> : distill_columns_kernel<T, false>;
    // (a launch has fewer than 2^32 threads)
    for (int64_t m = 0; m < D.M; m += (int64_t)1 << 30) {
        const Distill S = positions(D, dt, m, std::min(D.M - m, (int64_t)1 << 30));
        kern<<<dim3((unsigned)ceil_div64(S.M, 64)), 64, (size_t)D.C * 256, s>>>(S);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int W>
hipError_t run_tiles(const Distill& D, dss_dtype dt, hipStream_t s) {
    constexpr int N = Tile<T, W>::kTokens;
    const int waves = (int)ceil_div64(D.C, 64);
    const size_t lds = std::max(Lists<T, N>::bytes_of_t(D.k) + (size_t)waves * N * 4 + Marks<N>::bytes((int)D.C), Lists<T, N>::bytes(D.k));
    const auto kern = gradient_past(D, dt) ? distill_tile_kernel<T, W, true> : distill_tile_kernel<T, W, false>;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    for (int64_t m = 0; m < D.M;) {
        // (what is left after this launch has a whole tile's positions)
        const int64_t n = D.M - m <= kSlabTokens ? D.M - m : kSlabTokens - N;
        const Distill S = positions(D, dt, m, n);
        kern<<<dim3((unsigned)ceil_div64(n, N)), waves * 64, lds, s>>>(S);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        m += n;
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_map_parts(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s) {
    // (the parts' tiles and the gradients', which are half as wide of bfloat16)
    constexpr int N = Tile<T, 4>::kTokens, G = Tile<T, (int)sizeof(T)>::kTokens;
    const size_t lists = Lists<T, kJoined>::bytes(D.k), gradient = Shares<G>::bytes(D.k) + Marks<G>::bytes(kPartSpan);
    const auto last = gradient_past(D, dt) ? distill_map_gradient_kernel<T, true> : distill_map_gradient_kernel<T, false>;
    const hipError_t allowed = allow_dynamic_lds((const void*)last, gradient);
    if (allowed != hipSuccess) return allowed;
    const Stats stats = {reinterpret_cast<float*>(parts)};
    parts += kStats * kSlabPositions * 4 / (int)sizeof(Part);
    constexpr int64_t room = kMostParts - kStats * kSlabPositions * 4 / (int)sizeof(Part);
    const auto first = D.M * D.C * (int64_t)sizeof(T) > (D.grad ? kNeverCached : kLarge) ? distill_map_parts_kernel<T, true>
                                                                                         : distill_map_parts_kernel<T, false>;
    for (int64_t m = 0; m < D.M; m += kSlabPositions) {
        const Distill S = positions(D, dt, m, std::min(D.M - m, kSlabPositions));
        // enough workgroups for the units, of at least a span of classes each
        const int64_t tiles = ceil_div64(S.M, N);
        const int64_t most = std::max<int64_t>(1, std::min({ceil_div64(1024, tiles), ceil_div64(D.C, kPartSpan), room / S.M}));
        const int64_t per_part = ceil_div64(ceil_div64(D.C, most), kPartSpan) * kPartSpan, n = ceil_div64(D.C, per_part);
        const dim3 grid((unsigned)tiles, (unsigned)n);
        first<<<grid, kPartThreads, 0, s>>>(S, per_part, parts);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        distill_map_join_kernel<T><<<dim3((unsigned)ceil_div64(S.M, kJoined)), kPartThreads, lists, s>>>(S, parts, (int)n, stats);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (D.grad)
            last<<<dim3((unsigned)ceil_div64(S.M, G), (unsigned)n), kPartThreads, gradient, s>>>(S, per_part, stats);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_map(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s) {
    // In microseconds for columns and for tiles, 8 places: 200000 positions of 100 binary32 classes 53 / 59, of 128 bfloat16 58 / 72, of
    // 200 binary32 101 / 80, of 250 bfloat16 153 / 80; 3000 positions of 200 11 / 12.  For tiles and for parts: 100000 positions of 800
    // binary32 classes 176 / 200.
    if (D.C <= kColumns) return run_columns<T>(D, dt, s);
    // (lists of up to 128 places: 64 positions' take 98 KB)
    if (D.k > 128) return launch_distill_any(D, dt, s);
    return D.C <= 1024 && D.M >= Tile<T, 2>::kTokens ? run_tiles<T, 2>(D, dt, s) : run_map_parts<T>(D, dt, parts, s);
}

}  // namespace

hipError_t launch_distill_map(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s) {
    return dt == DSS_BF16 ? run_map<uint16_t>(D, dt, parts, s) : run_map<float>(D, dt, parts, s);
}

}  // namespace dss
