// Log probabilities of scores, and their gradient.
//
// With scores x[i, v] of token i and word v, and a scale:
//   m = max_v x,   d_v = scale (x_v - m),   s = sum_v e^d_v,   t = sum_v e^d_v d_v,
//   lse = scale m + log s,   log p_v = d_v - log s,   entropy = log s - t / s.
// Every score is read once: lanes keep a maximum of their own and sums by it,
// and only where these are joined are they brought to one maximum.  Exponentials
// are taken to the base 2, with log2(e) in the scale.
#include "tre_internal.h"
#include "values.h"

#include <cfloat>

namespace tre {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

// Scores as rows (one tile) or as the tiles of a relation keyed by the word's
// tile: x[i, v] at (v / cols) tile_stride + i row_stride + v % cols.  A row is
// cut into runs of E elements that a lane takes with one access; a tile's last
// run may be short.
struct Scores {
    int64_t n, vocab, row_stride, tile_stride;
    uint32_t cols, runs, total;   // runs of a tile's row, of a row
    uint32_t mul, shift;          // q / runs = (q mul >> 32) >> shift for q < 2^31 (runs > 1)
};

Scores scores_of(const ScoreLayout& l, int elems) {
    Scores g{};
    g.n = l.n;
    g.vocab = l.vocab;
    g.row_stride = l.row_stride;
    g.tile_stride = l.tile_stride;
    g.cols = uint32_t(l.cols);
    g.runs = uint32_t((l.cols + elems - 1) / elems);
    g.total = uint32_t(l.vocab / l.cols) * g.runs;
    int s = 0;
    while ((int64_t(1) << s) < int64_t(g.runs)) s++;
    g.mul = uint32_t((uint64_t(1) << (31 + s)) / g.runs + 1);
    g.shift = uint32_t(s > 0 ? s - 1 : 0);
    return g;
}

struct Place {
    uint32_t tile, at;  // run `at` of the tile's row
};
__device__ inline Place place_of(const Scores& g, uint32_t q) {
    if (g.total == g.runs) return {0, q};
    if (g.runs == 1) return {q, 0};
    const uint32_t tile = __umulhi(q, g.mul) >> g.shift;
    return {tile, q - tile * g.runs};
}

// The E elements of a run, what lies behind a tile's row -inf.
template <int E, bool RAGGED, typename T>
__device__ inline void load_scores(const Scores& g, const T* row, Place p, float (&v)[E]) {
    const T* at = row + p.tile * g.tile_stride + int64_t(p.at) * E;
    if (!RAGGED || (p.at + 1) * E <= g.cols) {
        load_all(at, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < E; i++) v[i] = p.at * E + i < g.cols ? load1(at + i) : -kInf;
}

// ------------------------------------------------------------ top words
//
// The best words of a wavefront lie in its lanes, the best first, as keys of 64
// bits: the score in an order of whole numbers, then the word, lower words
// first.  0: none.  A NaN is taken as -inf.

__device__ inline uint32_t order_of(float x) {
    x = x != x ? -kInf : x + 0.f;  // (-0 is 0)
    const uint32_t b = __float_as_uint(x);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ inline float of_order(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
constexpr uint32_t kOrderLowest = 0x007fffffu;  // order_of(-inf)

__device__ inline uint64_t key_of(float x, uint32_t word) { return uint64_t(order_of(x)) << 32 | uint32_t(~word); }

template <int MASK>
__device__ inline uint32_t swap_lanes(uint32_t x) {
    if constexpr (MASK == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true);
    else if constexpr (MASK == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true);
    else if constexpr (MASK == 8) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true);
    else if constexpr (MASK < 32) return __builtin_amdgcn_ds_swizzle(x, MASK << 10 | 0x1f);
    else return __shfl_xor(x, MASK);
}
template <int MASK>
__device__ inline uint64_t swap_keys(uint64_t k) {
    return uint64_t(swap_lanes<MASK>(uint32_t(k >> 32))) << 32 | swap_lanes<MASK>(uint32_t(k));
}
template <int MASK>
__device__ inline void order_pair(uint64_t& k, bool low) {  // `low`: the lower lane of a pair gets the smaller key
    const uint64_t o = swap_keys<MASK>(k);
    const bool first = !(threadIdx.x & MASK);
    k = (first == low) == (k < o) ? k : o;
}
template <int STRIDE>
__device__ inline void merge_lanes(uint64_t& k, bool low) {
    order_pair<STRIDE>(k, low);
    if constexpr (STRIDE > 1) merge_lanes<STRIDE / 2>(k, low);
}
template <int SIZE>
__device__ inline void sort_lanes(uint64_t& k) {  // smallest first
    if constexpr (SIZE > 2) sort_lanes<SIZE / 2>(k);
    merge_lanes<SIZE / 2>(k, SIZE == 64 || !(threadIdx.x & SIZE));
}

struct Top {
    uint64_t key;  // of a lane, largest first
    uint64_t last; // the top-th
    int k;
    __device__ void init(int top) {
        key = last = 0;
        k = top;
    }
    __device__ uint64_t lane_key(int lane) const {
        return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(key >> 32), lane))) << 32 |
               uint32_t(__builtin_amdgcn_readlane(int(key), lane));
    }
    __device__ void settle() { last = lane_key(k - 1); }
    // 64 keys, smallest first
    __device__ void merge(uint64_t sorted) {
        key = key > sorted ? key : sorted;
        merge_lanes<32>(key, false);
        settle();
    }
    __device__ void insert(uint64_t c) {  // (the same in all lanes)
        if (c <= last) return;
        const int lane = threadIdx.x & 63;
        const int at = __popcll(__ballot(key > c));
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, uint32_t(key >> 32), 0x138, 0xf, 0xf, true);  // the lane before
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, uint32_t(key), 0x138, 0xf, 0xf, true);
        key = lane < at ? key : lane == at ? c : uint64_t(hi) << 32 | lo;
        settle();
    }
    // Keys of the lanes of `from`.  More than a few are sorted and merged: that
    // takes as long as some 12 insertions.
    __device__ void take(uint64_t mine, uint64_t from) {
        if (__popcll(from) > 12) {
            uint64_t k = from >> (threadIdx.x & 63) & 1 ? mine : 0;
            sort_lanes<64>(k);
            merge(k);
            return;
        }
        for (; from; from &= from - 1) {
            const int lane = __ffsll((unsigned long long)from) - 1;
            insert(uint64_t(uint32_t(__builtin_amdgcn_readlane(int(mine >> 32), lane))) << 32 |
                   uint32_t(__builtin_amdgcn_readlane(int(mine), lane)));
        }
    }
};

// -------------------------------------------------------------- forward

struct Sums {
    float m, s, t;  // t in units of log 2
};
__device__ inline Sums join(Sums a, Sums b, float scale2) {
    const float m = fmaxf(a.m, b.m);
    // (a difference without bound would meet sums of zero as inf * 0)
    const float da = fmaxf((a.m - m) * scale2, -2000.f), db = fmaxf((b.m - m) * scale2, -2000.f);
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    return {m, fa * a.s + fb * b.s, fa * (a.t + a.s * da) + fb * (b.t + b.s * db)};
}

struct ProbArgs {
    Scores g;
    const void* x;
    const void* ids;
    float *log_prob, *lse, *stats, *entropy;
    int32_t* top_ids;
    float* top_log_probs;
    int64_t* status;
    Sums* part;          // [row][split]
    uint64_t* part_keys; // [row][split][top]
    uint32_t splits, per; // workgroups of a row, runs of each
    float scale, scale2;
    int32_t id_bytes, top;
};

template <typename T>
__device__ inline void put_row(const ProbArgs& a, int64_t row, Sums u, const Top& top) {
    const int lane = threadIdx.x & 63;
    const bool empty = u.s == 0.f;
    const float m = empty ? -kInf : u.m, logs = logf(u.s);
    if (a.top_ids && lane < a.top) {
        const float v = of_order(uint32_t(top.key >> 32));
        a.top_ids[row * a.top + lane] = int32_t(~uint32_t(top.key));
        a.top_log_probs[row * a.top + lane] = empty ? -kInf : (v - m) * a.scale - logs;
    }
    if (lane) return;
    a.stats[2 * row] = m;
    a.stats[2 * row + 1] = logs;
    a.lse[row] = a.scale * m + logs;
    if (a.entropy) {
        const float h = logs - kLn2 * u.t / u.s;
        a.entropy[row] = empty || h < 0.f ? 0.f : h;  // (a sum that rounding took below zero)
    }
    if (a.log_prob) {
        const int64_t id = token(a.ids, a.id_bytes, row);
        float lp = 0.f;
        if (id >= 0 && id < a.g.vocab) {
            const int64_t tile = id / a.g.cols;
            const float v = load1(static_cast<const T*>(a.x) + tile * a.g.tile_stride + row * a.g.row_stride + (id - tile * a.g.cols));
            lp = empty ? -kInf : (v - m) * a.scale - logs;
        } else if (id >= 0 && a.status) {
            *a.status = TRE_E_KEYRANGE;
        }
        a.log_prob[row] = lp;
    }
}

// Runs of a lane in flight together.
constexpr int kRuns = 4;

// W wavefronts to a row, or to a part of it.
template <typename T, bool RAGGED, bool TOP, bool ENT, int W>
__global__ __launch_bounds__(kThreads) void k_probs(ProbArgs a) {
    constexpr int E = 16 / sizeof(T);
    constexpr uint32_t kStep = 64 * kRuns;
    __shared__ Sums sums[kWaves];
    __shared__ uint64_t keys[TOP && W > 1 ? W : 1][64];
    __shared__ uint32_t bar;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t task = W > 1 ? block_index() : block_index() * kWaves + wave;
    const int64_t row = a.splits > 1 ? task / a.splits : task;
    if (row >= a.g.n) return;
    const uint32_t split = uint32_t(task - row * a.splits);
    const uint32_t q0 = split * a.per, q1 = min(q0 + a.per, a.g.total);
    const T* x = static_cast<const T*>(a.x) + row * a.g.row_stride;
    Sums u{-FLT_MAX, 0.f, 0.f};
    Top top;
    if constexpr (TOP) {
        top.init(a.top);
        if constexpr (W > 1) {
            if (threadIdx.x == 0) bar = 0;
            __syncthreads();
        }
    }
    for (uint32_t b = q0 + (W > 1 ? wave : 0) * kStep; b < q1; b += W * kStep) {
        float v[kRuns][E];
        Place p[kRuns];
#pragma unroll
        for (int j = 0; j < kRuns; j++) {
            const uint32_t q = b + j * 64 + lane;
            p[j] = place_of(a.g, q);
            if (q < q1) {
                load_scores<E, RAGGED>(a.g, x, p[j], v[j]);
            } else {
#pragma unroll
                for (int i = 0; i < E; i++) v[j][i] = -kInf;
            }
        }
        float most = -FLT_MAX;
#pragma unroll
        for (int j = 0; j < kRuns; j++)
#pragma unroll
            for (int i = 0; i < E; i++) most = fmaxf(most, v[j][i]);
        if constexpr (TOP) {
            // what the other wavefronts have bars lower scores here too, but not equal ones, whose words may come first
            uint32_t others = 0;
            if constexpr (W > 1) others = *static_cast<volatile uint32_t*>(&bar);
            others = __builtin_amdgcn_readfirstlane(others);
            const bool full = top.last != 0, barred = others > kOrderLowest;
            float limit = full ? of_order(uint32_t(top.last >> 32)) : -kInf;
            if (barred) limit = fmaxf(limit, of_order(others == 0x80000000u ? others - 2 : others - 1));  // (0 and -0 are equal)
            const bool any = !full && !barred;
            if (any || __ballot(most > limit)) {
#pragma unroll
                for (int j = 0; j < kRuns; j++) {
                    const uint32_t q = b + j * 64 + lane;
#pragma unroll
                    for (int i = 0; i < E; i++) {
                        bool in = v[j][i] > limit;
                        if (any) in = q < q1 && p[j].at * E + i < a.g.cols;
                        const uint64_t from = __ballot(in);
                        if (from) top.take(key_of(v[j][i], p[j].tile * a.g.cols + p[j].at * E + i), from);
                    }
                }
                if constexpr (W > 1) {
                    if (lane == 0 && uint32_t(top.last >> 32) > others) atomicMax(&bar, uint32_t(top.last >> 32));
                }
            }
        }
        const float m = fmaxf(u.m, most), d = fmaxf((u.m - m) * a.scale2, -2000.f), f = __builtin_amdgcn_exp2f(d);
        if constexpr (ENT) u.t = f * (u.t + u.s * d);
        u.s *= f;
        u.m = m;
#pragma unroll
        for (int j = 0; j < kRuns; j++)
#pragma unroll
            for (int i = 0; i < E; i++) {
                const float z = (v[j][i] - m) * a.scale2, e = __builtin_amdgcn_exp2f(z);
                u.s += e;
                if constexpr (ENT) u.t += e * fmaxf(z, -2000.f);  // (no 0 * inf)
            }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const Sums v{__shfl_xor(u.m, o), __shfl_xor(u.s, o), ENT ? __shfl_xor(u.t, o) : 0.f};
        u = join(u, v, a.scale2);
    }
    if constexpr (W > 1) {
        if (lane == 0) sums[wave] = u;
        if constexpr (TOP) keys[wave][lane] = lane < a.top ? top.key : 0;
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < W; w++) {
            u = join(u, sums[w], a.scale2);
            if constexpr (TOP) top.merge(keys[w][63 - lane]);
        }
    }
    if (a.splits > 1) {
        if (lane == 0) a.part[task] = u;
        if (TOP && lane < a.top) a.part_keys[task * a.top + lane] = top.key;
    } else {
        put_row<T>(a, row, u, top);
    }
}

// The parts of a row joined: a wavefront to a row.
template <typename T>
__global__ __launch_bounds__(64) void k_probs_join(ProbArgs a) {
    const int lane = threadIdx.x;
    const int64_t row = block_index();
    if (row >= a.g.n) return;
    Sums u = lane < int(a.splits) ? a.part[row * a.splits + lane] : Sums{-FLT_MAX, 0.f, 0.f};
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) u = join(u, {__shfl_xor(u.m, o), __shfl_xor(u.s, o), __shfl_xor(u.t, o)}, a.scale2);
    Top top;
    top.init(a.top_ids ? a.top : 1);
    if (a.top_ids) {
        for (uint32_t i = 0; i < a.splits; i++) {
            const int from = 63 - lane;
            top.merge(from < a.top ? a.part_keys[(row * a.splits + i) * a.top + from] : 0);
        }
    }
    put_row<T>(a, row, u, top);
}

// A row of few scores is one wavefront's, and few rows are cut so that there are
// workgroups for the chip.
constexpr int64_t kWaveRuns = 4 * 64 * kRuns;   // up to so many runs
constexpr int64_t kFill = 512;                  // workgroups
constexpr uint32_t kMaxSplits = 32;

struct Cut {
    bool wave;
    uint32_t splits, per;
};
Cut cut_of(const Scores& g) {
    Cut c{int64_t(g.total) <= kWaveRuns, 1, g.total};
    if (c.wave) return c;
    const uint32_t step = kWaves * 64 * kRuns, steps = (g.total + step - 1) / step;
    uint32_t s = uint32_t(std::min<int64_t>(std::min<int64_t>(steps, kMaxSplits), std::max<int64_t>(1, kFill / std::max<int64_t>(g.n, 1))));
    c.per = (steps + s - 1) / s * step;
    c.splits = (g.total + c.per - 1) / c.per;
    return c;
}

template <typename T, bool RAGGED, bool TOP, bool ENT>
hipError_t probs3(ProbArgs a, Cut c, hipStream_t s) {
    if (c.wave) k_probs<T, RAGGED, TOP, ENT, 1><<<grid_of((a.g.n + kWaves - 1) / kWaves), kThreads, 0, s>>>(a);
    else k_probs<T, RAGGED, TOP, ENT, kWaves><<<grid_of(a.g.n * c.splits), kThreads, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.splits == 1) return e;
    k_probs_join<T><<<grid_of(a.g.n), 64, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, bool RAGGED>
hipError_t probs2(const ProbArgs& a, Cut c, hipStream_t s) {
    if (a.top_ids) return a.entropy ? probs3<T, RAGGED, true, true>(a, c, s) : probs3<T, RAGGED, true, false>(a, c, s);
    return a.entropy ? probs3<T, RAGGED, false, true>(a, c, s) : probs3<T, RAGGED, false, false>(a, c, s);
}
template <typename T>
hipError_t probs1(ProbArgs a, Cut c, hipStream_t s) {
    return a.g.cols % (16 / sizeof(T)) ? probs2<T, true>(a, c, s) : probs2<T, false>(a, c, s);
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// ------------------------------------------------------------- gradient
//
// With g, gl and gh the gradients by log_prob, lse and entropy H:
//   dx_v = scale (g [v = id] + p_v (gl - g - gh (log p_v + H))).

struct ProbGradArgs {
    Scores g;
    const void *x, *ids;
    const float *stats, *entropy, *by_log_prob, *by_lse, *by_entropy;
    void* out;
    int64_t* status;
    int64_t out_row_stride, out_tile_stride;
    uint32_t parts;      // wavefronts of a row
    float scale, scale2;
    int32_t id_bytes;
};

template <typename TI, typename TO, bool RAGGED, bool ENT>
__global__ __launch_bounds__(kThreads) void k_probs_grad(ProbGradArgs a) {
    constexpr int E = lane_elems<TI, TO>();
    const int lane = threadIdx.x & 63;
    const int64_t w = block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = w / a.parts;
    if (row >= a.g.n) return;
    const uint32_t part = uint32_t(w - row * a.parts);
    const float m = a.stats[2 * row], logs2 = a.stats[2 * row + 1] * kLog2e;
    int64_t id = a.ids ? token(a.ids, a.id_bytes, row) : -1;
    if (id >= a.g.vocab) {
        if (a.status && part == 0 && lane == 0) *a.status = TRE_E_KEYRANGE;
        id = -1;
    }
    float one = id >= 0 && a.by_log_prob ? a.by_log_prob[row] : 0.f;
    float c0 = (a.by_lse ? a.by_lse[row] : 0.f) - one, c1 = 0.f;
    if constexpr (ENT) {
        c1 = -a.by_entropy[row];
        c0 += c1 * a.entropy[row];
        c1 *= kLn2;
    }
    c0 *= a.scale;
    c1 *= a.scale;
    one *= a.scale;
    if (m == -kInf) one = c0 = c1 = 0.f;  // a row of no words
    const bool zero = c0 == 0.f && c1 == 0.f && one == 0.f;
    const int64_t id_tile = id >= 0 ? id / a.g.cols : -1, id_at = id >= 0 ? id - id_tile * a.g.cols : -1;
    const TI* x = static_cast<const TI*>(a.x) + row * a.g.row_stride;
    TO* out = static_cast<TO*>(a.out) + row * a.out_row_stride;
    float v[kRuns][E];
    Place p[kRuns];
#pragma unroll
    for (int j = 0; j < kRuns; j++) {
        const uint32_t q = (part * kRuns + j) * 64 + lane;
        p[j] = place_of(a.g, q);
        if (!zero && q < a.g.total) load_scores<E, RAGGED>(a.g, x, p[j], v[j]);
    }
#pragma unroll
    for (int j = 0; j < kRuns; j++) {
        const uint32_t q = (part * kRuns + j) * 64 + lane;
        if (q >= a.g.total) break;
        float y[E];
#pragma unroll
        for (int i = 0; i < E; i++) {
            y[i] = 0.f;
            if (!zero) {
                const float z = (v[j][i] - m) * a.scale2 - logs2, e = __builtin_amdgcn_exp2f(z);
                y[i] = e * (ENT ? c0 + c1 * fmaxf(z, -2000.f) : c0);
                if (p[j].tile == id_tile && p[j].at * E + i == id_at) y[i] += one;
            }
        }
        TO* at = out + p[j].tile * a.out_tile_stride + int64_t(p[j].at) * E;
        if (!RAGGED || (p[j].at + 1) * E <= a.g.cols) {
            store_all<true>(at, y);
        } else {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (p[j].at * E + i < a.g.cols) store1(at + i, y[i]);
        }
    }
}

template <typename TI, typename TO>
hipError_t probs_grad(ProbGradArgs a, const ScoreLayout& l, hipStream_t s) {
    constexpr int E = lane_elems<TI, TO>();
    a.g = scores_of(l, E);
    a.parts = (a.g.total + 64 * kRuns - 1) / (64 * kRuns);
    const dim3 grid = grid_of((l.n * a.parts + kWaves - 1) / kWaves);
    if (l.cols % E) {
        if (a.by_entropy) k_probs_grad<TI, TO, true, true><<<grid, kThreads, 0, s>>>(a);
        else k_probs_grad<TI, TO, true, false><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (a.by_entropy) k_probs_grad<TI, TO, false, true><<<grid, kThreads, 0, s>>>(a);
        else k_probs_grad<TI, TO, false, false><<<grid, kThreads, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t log_probs_ws_bytes(const ScoreLayout& l, int elem_bytes, int top) {
    const Cut c = cut_of(scores_of(l, 16 / elem_bytes));
    if (c.splits == 1) return 0;
    const size_t tasks = size_t(l.n) * c.splits;
    return align256(tasks * sizeof(Sums)) + align256(tasks * size_t(top) * 8);
}

hipError_t launch_log_probs(const ScoreLayout& l, const void* x, int dtype, const void* ids, int id_bytes, float scale, int top,
                            float* log_prob, float* lse, float* stats, float* entropy, int32_t* top_ids, float* top_log_probs,
                            int64_t* status, char* ws, hipStream_t s) {
    const bool half = dtype == TRE_BF16;
    ProbArgs a{};
    a.g = scores_of(l, half ? 8 : 4);
    const Cut c = cut_of(a.g);
    a.x = x;
    a.ids = ids;
    a.log_prob = ids ? log_prob : nullptr;
    a.lse = lse;
    a.stats = stats;
    a.entropy = entropy;
    a.top_ids = top > 0 ? top_ids : nullptr;
    a.top_log_probs = top_log_probs;
    a.status = status;
    a.splits = c.splits;
    a.per = c.per;
    if (c.splits > 1) {
        a.part = reinterpret_cast<Sums*>(ws);
        a.part_keys = reinterpret_cast<uint64_t*>(ws + align256(size_t(l.n) * c.splits * sizeof(Sums)));
    }
    a.scale = scale;
    a.scale2 = scale * kLog2e;
    a.id_bytes = id_bytes;
    a.top = top;
    return half ? probs1<uint16_t>(a, c, s) : probs1<float>(a, c, s);
}

hipError_t launch_log_probs_grad(const ScoreLayout& l, const void* x, int dtype, const float* stats, const void* ids, int id_bytes,
                                 float scale, const float* by_log_prob, const float* by_lse, const float* by_entropy,
                                 const float* entropy, void* out, int out_dtype, int64_t out_row_stride, int64_t out_tile_stride,
                                 int64_t* status, hipStream_t s) {
    ProbGradArgs a{};
    a.x = x;
    a.ids = ids;
    a.stats = stats;
    a.entropy = entropy;
    a.by_log_prob = by_log_prob;
    a.by_lse = by_lse;
    a.by_entropy = by_entropy;
    a.out = out;
    a.status = status;
    a.out_row_stride = out_row_stride;
    a.out_tile_stride = out_tile_stride;
    a.scale = scale;
    a.scale2 = scale * kLog2e;
    a.id_bytes = id_bytes;
    const bool half = out_dtype == TRE_BF16;
    if (dtype == TRE_BF16) return half ? probs_grad<uint16_t, uint16_t>(a, l, s) : probs_grad<uint16_t, float>(a, l, s);
    return half ? probs_grad<float, uint16_t>(a, l, s) : probs_grad<float, float>(a, l, s);
}

}  // namespace tre
