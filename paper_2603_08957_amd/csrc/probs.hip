// Log probabilities of scores, and their gradient.
//
// With scores x[i, v] of token i and word v, and a scale:
//   m = max_v x,   d_v = scale (x_v - m),   s = sum_v e^d_v,   t = sum_v e^d_v d_v,
//   lse = scale m + log s,   log p_v = d_v - log s,   entropy = log s - t / s.
// Every score is read once: lanes keep a maximum of their own and sums by it,
// and only where these are joined are they brought to one maximum.  Exponentials
// are taken to the base 2, with log2(e) in the scale.  x - m comes before the
// product with the scale, so that large scores lose nothing, and the maximum and
// log s are kept apart for the gradient for the same reason: a probability out of
// lse alone is off by 2^-24 |lse|.
//
// Memory bounds large calls: 8192 x 32768 bf16 scores with entropy take 98 us
// (5.5 TB/s; 10 vector operations a score, 77 us of the vector units' time), their
// gradient in bf16 196 us (5.2 TB/s read and written; 17 operations).  2048 x 32768
// take 24 us, with 8 top words 38 (17 operations, 31 us of the units' time).  A
// lane's four loads of 16 bytes are in flight together: with each waited for the
// first took 113 us.
#include "tre_internal.h"
#include "values.h"

#include <cfloat>

namespace tre {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();
// Runs of a lane in flight together.
constexpr int kRuns = 4;
constexpr int kMostWaves = 16;  // of a row

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

// How runs lie on a tile's row: it is made of whole ones, its last one is taken
// from the row's end (and overlaps the one before), or the row is shorter than one.
enum Fit { kWhole, kOverlap, kShort };
Fit fit_of(const Scores& g, int elems) {
    return g.cols % elems == 0 ? kWhole : int(g.cols) >= elems ? kOverlap : kShort;
}

typedef uint32_t u32x4_1 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_1 __attribute__((ext_vector_type(2), aligned(2)));

// E elements of one access, as they come: what is done with them waits, the loads do not.
template <typename T, int E>
struct Raw {
    uint32_t w[E * sizeof(T) / 4];
    __device__ void load(const T* at) {
        if constexpr (sizeof(w) == 16) {
            const u32x4_1 x = *reinterpret_cast<const u32x4_1*>(at);
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = x[i];
        } else {
            const u32x2_1 x = *reinterpret_cast<const u32x2_1*>(at);
            w[0] = x[0];
            w[1] = x[1];
        }
    }
    __device__ void load_some(const T* at, int n) {  // of at least one
#pragma unroll
        for (int i = 0; i < int(sizeof(w) / 4); i++) w[i] = 0;
#pragma unroll
        for (int i = 0; i < E; i++) {
            if (i >= n) break;
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(at[i]);
            else w[i / 2] |= uint32_t(at[i]) << (16 * (i & 1));
        }
    }
    __device__ float value(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};

// A run of a row and where it lies.
template <typename T, int E, int FIT>
struct Run {
    Raw<T, E> raw;
    uint32_t tile, start, own;  // columns from `start` on, its own from `own` on
    __device__ void find(const Scores& g, uint32_t q) {
        tile = 0;
        if (g.total != g.runs) tile = g.runs == 1 ? q : __umulhi(q, g.mul) >> g.shift;
        own = start = (q - tile * g.runs) * E;
        if constexpr (FIT == kOverlap) start = min(own, g.cols - E);
    }
    __device__ void load(const Scores& g, const T* row, uint32_t q) {
        const T* at;
        if (g.total == g.runs) {  // (one tile: 8 operations fewer)
            tile = 0;
            own = start = q * E;
            if constexpr (FIT == kOverlap) start = min(own, g.cols - E);
            at = row + start;
        } else {
            find(g, q);
            at = row + tile * g.tile_stride + start;
        }
        if constexpr (FIT == kShort) raw.load_some(at, int(g.cols));
        else raw.load(at);
    }
    // Its scores, -inf for columns that are not its own.
    __device__ void values(const Scores& g, float (&v)[E]) const {
#pragma unroll
        for (int i = 0; i < E; i++) {
            v[i] = raw.value(i);
            if constexpr (FIT == kOverlap) v[i] = start + i >= own ? v[i] : -kInf;
            if constexpr (FIT == kShort) v[i] = i < int(g.cols) ? v[i] : -kInf;
        }
    }
    __device__ bool whole() const { return FIT == kWhole || (FIT == kOverlap && start == own); }
    __device__ bool has(const Scores& g, int i) const { return FIT == kShort ? i < int(g.cols) : start + i >= own; }
};

// ------------------------------------------------------------ top words
//
// The best words of a wavefront lie in its lanes, the best first, as keys of 64
// bits: the score in an order of whole numbers, then the word, lower words
// first.  0: none.  Words that cannot come (-inf; a NaN is taken as that) have no
// place in it: where a row has too few others they are found at the end.

__device__ inline uint32_t order_of(float x) {
    x = x != x ? -kInf : x + 0.f;  // (-0 is 0)
    const uint32_t b = __float_as_uint(x);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ inline float of_order(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
constexpr uint32_t kOrderLowest = 0x007fffffu;  // order_of(-inf)
// The highest order, less its lower 16 bits, that at least k lanes reach; that of -inf if fewer have another.
__device__ inline uint32_t reached(uint32_t order, int k) {
    uint32_t t = 0;
#pragma unroll
    for (int b = 31; b >= 16; b--) {
        const uint32_t c = t | 1u << b;
        if (__popcll(__ballot(order >= c)) >= k) t = c;
    }
    return max(t, kOrderLowest);
}

__device__ inline uint64_t key_of(float x, uint32_t word) { return uint64_t(order_of(x)) << 32 | uint32_t(~word); }

// The value of the lane whose number differs by MASK: no LDS.
template <int MASK>
__device__ inline uint32_t swap_lanes(uint32_t x) {
    if constexpr (MASK == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, true);
    else if constexpr (MASK == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, true);
    else if constexpr (MASK == 4)  // eight lanes turned round, then each four
        return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
    else if constexpr (MASK == 8) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, true);
    else if constexpr (MASK == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
}
template <int MASK>
__device__ inline float swap_lanes(float x) {
    return __uint_as_float(swap_lanes<MASK>(__float_as_uint(x)));
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

// What a wavefront keeps of its scores: at first no more than the keys as they come
// (`pending`, LDS); 64 of them are sorted and merged into a list of the best that the
// lanes hold.  (Insertion one by one takes 300 cycles each, a wavefront's sort and
// merge 2700.)
constexpr int kPending = 128;
struct Top {
    uint64_t key;   // of a lane, largest first; none before the first merge
    uint64_t last;  // the top-th
    int n, k;       // pending, below 64; top
    __device__ void init(int top) {
        key = last = 0;
        n = 0;
        k = top;
    }
    // Whether any of these keys has a place in the list.
    __device__ bool beaten(uint64_t c) const { return __ballot(c > last) != 0; }
    // 64 keys, smallest first
    __device__ void merge(uint64_t sorted) {
        key = key > sorted ? key : sorted;
        merge_lanes<32>(key, false);
        last = uint64_t(uint32_t(__builtin_amdgcn_readlane(int(key >> 32), k - 1))) << 32 |
               uint32_t(__builtin_amdgcn_readlane(int(key), k - 1));
    }
    __device__ void merge_pending(uint64_t (&pending)[kPending]) {  // the first 64 of them
        const int lane = threadIdx.x & 63;
        uint64_t c = lane < n ? pending[lane] : 0;
        const uint64_t rest = lane + 64 < n ? pending[lane + 64] : 0;
        sort_lanes<64>(c);
        merge(c);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane + 64 < n) pending[lane] = rest;
        n = max(n - 64, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // Keys of the lanes of `from`.
    __device__ void take(uint64_t (&pending)[kPending], uint64_t mine, uint64_t from) {
        const int lane = threadIdx.x & 63;
        if (from >> lane & 1) pending[n + __popcll(from & ((uint64_t(1) << lane) - 1))] = mine;
        n += __popcll(from);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (other lanes read it)
        if (n >= 64) merge_pending(pending);
    }
    // The wavefront's best, a key a lane: as they came, or the list.
    __device__ uint64_t best(uint64_t (&pending)[kPending]) {
        const int lane = threadIdx.x & 63;
        if (last == 0) return lane < n ? pending[lane] : 0;
        if (n > 0) merge_pending(pending);
        return lane < k ? key : 0;
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

__device__ inline float first_lane(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
// The sums of lanes 0 to 2 END - 1 in one, in each of them up to its last bits.
template <int MASK, int END, bool ENT>
__device__ inline void join_lanes(Sums& u, float scale2) {
    u = join(u, {swap_lanes<MASK>(u.m), swap_lanes<MASK>(u.s), ENT ? swap_lanes<MASK>(u.t) : 0.f}, scale2);
    if constexpr (MASK < END) join_lanes<MASK * 2, END, ENT>(u, scale2);
}
__device__ inline Sums first_lane(Sums u) { return {first_lane(u.m), first_lane(u.s), first_lane(u.t)}; }

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
__device__ inline const T* score_at(const ProbArgs& a, int64_t row, int64_t word) {
    const int64_t tile = word / a.g.cols;
    return static_cast<const T*>(a.x) + tile * a.g.tile_stride + row * a.g.row_stride + (word - tile * a.g.cols);
}

// A token's given word.
__device__ inline int64_t given_word(const ProbArgs& a, int64_t row) {
    return a.log_prob ? token(a.ids, a.id_bytes, row) : -1;
}
// Its score as it comes (no word's: any), so that nothing waits for it.
template <typename T>
struct Given {
    T raw;
    bool is;
    __device__ float x() const {
        if constexpr (sizeof(T) == 4) return raw;
        else return __uint_as_float(uint32_t(raw) << 16);
    }
};
template <typename T>
__device__ inline Given<T> given_of(const ProbArgs& a, int64_t row, int64_t id) {
    const int64_t last = a.g.vocab - 1;
    return {*score_at<T>(a, row, min(max(id, int64_t(0)), last)), id >= 0 && id <= last};
}

// What a row's sums say.
struct Row {
    float m, logs;
    bool empty;
    __device__ explicit Row(Sums u) : m(u.s == 0.f ? -kInf : u.m), logs(logf(u.s)), empty(u.s == 0.f) {}
    __device__ float log_prob(float x, float scale) const { return empty ? -kInf : (x - m) * scale - logs; }
};

// (one thread)
template <typename T>
__device__ inline void put_sums(const ProbArgs& a, int64_t row, Sums u, Row r, Given<T> given, int64_t word) {
    a.stats[2 * row] = r.m;
    a.stats[2 * row + 1] = r.logs;
    a.lse[row] = a.scale * r.m + r.logs;
    if (a.entropy) {
        const float h = r.logs - kLn2 * u.t / u.s;
        a.entropy[row] = r.empty || h < 0.f ? 0.f : h;  // (a sum that rounding took below zero)
    }
    if (!a.log_prob) return;
    a.log_prob[row] = given.is ? r.log_prob(given.x(), a.scale) : 0.f;
    if (word >= a.g.vocab && a.status) *a.status = TRE_E_KEYRANGE;
}
// A word of rank `rank`, where that is one of the top ones.
__device__ inline void put_top(const ProbArgs& a, int64_t row, Row r, uint64_t key, int rank) {
    if (rank >= a.top) return;
    a.top_ids[row * a.top + rank] = int32_t(~uint32_t(key));
    a.top_log_probs[row * a.top + rank] = r.log_prob(of_order(uint32_t(key >> 32)), a.scale);
}
// The first words that cannot come, behind the `have` that can (a wavefront).
template <typename T>
__device__ inline void fill_top(const ProbArgs& a, int64_t row, Row r, int have) {
    const int lane = threadIdx.x & 63;
    for (int64_t b = 0; have < a.top && b < a.g.vocab; b += 64) {
        const int64_t w = b + lane;
        bool dead = false;
        if (w < a.g.vocab) dead = !(load1(score_at<T>(a, row, w)) > -kInf);
        const uint64_t all = __ballot(dead);
        if (dead) put_top(a, row, r, uint64_t(kOrderLowest) << 32 | uint32_t(~uint32_t(w)), have + __popcll(all & ((uint64_t(1) << lane) - 1)));
        have += __popcll(all);
    }
}

// Element `at` < N of a lane's runs, from FROM on.
template <int N, int E, int FROM = 0>
__device__ inline float pick(const float (&v)[kRuns][E], uint32_t at) {
    if constexpr (N == 1) return v[FROM / E][FROM % E];
    else {
        const float low = pick<N / 2, E, FROM>(v, at), high = pick<N / 2, E, FROM + N / 2>(v, at);
        return at & (N / 2) ? high : low;
    }
}

// W wavefronts to a row, or to a part of it; with one, a workgroup has kWaves rows.
//
// Top words.  A score may have a place if it is higher than the last of the
// wavefront's list, whose words come before, and not lower than what as many scores
// of the row as are wanted are known to reach (`known`): at first what top / W lanes
// of every wavefront reach, or top lanes of one, later the last of any list (`bar`).
// At the end what top / W keys of every wavefront reach leaves few; the rank of each
// of these is the number of those that are larger, a part of which every wavefront
// counts.  (Lists in order merged in pairs took 5 us of 12.5 for 20 of 32768.)
template <typename T, int FIT, bool TOP, bool ENT, int W>
__global__ __launch_bounds__(W > 1 ? W * 64 : kThreads) void k_probs(ProbArgs a) {
    constexpr int E = 16 / sizeof(T);
    constexpr uint32_t kStep = 64 * kRuns;
    __shared__ Sums sums[W];
    __shared__ uint64_t pending[TOP ? (W > 1 ? W : kWaves) : 1][TOP ? kPending : 1];
    __shared__ uint64_t pool[TOP && W > 1 ? W * 64 : 1];
    __shared__ int rank[TOP && W > 1 ? W * 64 : 1];
    __shared__ uint32_t bar, reach[W], reach_last[W];  // (a wavefront may be done while another still reads `reach`)
    __shared__ int count;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t task = W > 1 ? block_index() : block_index() * kWaves + wave;
    const int64_t row = a.splits > 1 ? task / a.splits : task;
    if (row >= a.g.n) return;
    const uint32_t split = uint32_t(task - row * a.splits);
    const uint32_t q0 = split * a.per, q1 = min(q0 + a.per, a.g.total);
    const T* x = static_cast<const T*>(a.x) + row * a.g.row_stride;
    // the given word, and its score when the row's first loads are on their way
    Given<T> given{};
    const int64_t word = (W == 1 || wave == 0) && a.splits == 1 ? given_word(a, row) : -1;
    Sums u{-FLT_MAX, 0.f, 0.f};
    Top top;
    uint32_t known = 0;
    if constexpr (TOP) {
        top.init(a.top);
        if constexpr (W > 1) {
            if (threadIdx.x == 0) {
                bar = 0;
                count = 0;
            }
            __syncthreads();
        }
    }
#pragma unroll 1
    for (uint32_t b0 = q0; b0 < q1; b0 += W * kStep) {
        const uint32_t b = b0 + (W > 1 ? wave : 0) * kStep;
        if (b >= q1 && !(TOP && W > 1 && b0 == q0)) break;  // (all come to the first barrier)
        Run<T, E, FIT> r[kRuns];
#pragma unroll
        for (int j = 0; j < kRuns; j++) r[j].load(a.g, x, min(b + j * 64 + lane, q1 - 1));
        if (b0 == q0 && (W == 1 || wave == 0) && a.log_prob && a.splits == 1) given = given_of<T>(a, row, word);
        float v[kRuns][E], most[kRuns];
#pragma unroll
        for (int j = 0; j < kRuns; j++) {
            r[j].values(a.g, v[j]);
            if (b + kStep > q1) {
#pragma unroll
                for (int i = 0; i < E; i++) v[j][i] = b + j * 64 + lane < q1 ? v[j][i] : -kInf;
            }
            most[j] = -FLT_MAX;
#pragma unroll
            for (int i = 0; i < E; i++) most[j] = fmaxf(most[j], v[j][i]);
        }
        float all = most[0];
#pragma unroll
        for (int j = 1; j < kRuns; j++) all = fmaxf(all, most[j]);
        if constexpr (TOP) {
            if (W > 1 && b0 == q0) {
                const uint32_t own = reached(order_of(all), (a.top + W - 1) / W);
                if (lane == 0) reach[wave] = own;
                __syncthreads();
                known = reach[0];
#pragma unroll
                for (int w = 1; w < W; w++) known = min(known, reach[w]);
            } else if (W > 1) {
                known = max(known, *static_cast<volatile uint32_t*>(&bar));
            }
            known = __builtin_amdgcn_readfirstlane(known);
            // (a wavefront of few words that can come bars nothing for the others)
            if (known <= kOrderLowest + 1 && top.last == 0) known = reached(order_of(all), a.top);
            const uint32_t least = max(max(uint32_t(top.last >> 32), kOrderLowest) + 1, known);
            float limit = of_order(least);
            if (__ballot(all >= limit)) {
                // a bit for each of a lane's scores that may have a place; then one of each lane at a time
                uint32_t mine = 0;
#pragma unroll
                for (int j = 0; j < kRuns; j++) {
                    if (!__ballot(most[j] >= limit)) continue;
#pragma unroll
                    for (int i = 0; i < E; i++) mine |= v[j][i] >= limit ? 1u << (j * E + i) : 0u;
                }
#pragma unroll 1
                while (__ballot(mine != 0)) {
                    const int at = mine ? __ffs(mine) - 1 : 0;
                    const float y = pick<kRuns * E, E>(v, uint32_t(at));
                    Run<T, E, FIT> run;
                    run.find(a.g, b + uint32_t(at) / E * 64 + lane);
                    const uint64_t from = __ballot(mine != 0 && y >= limit);
                    if (from) top.take(pending[wave], key_of(y, run.tile * a.g.cols + run.start + uint32_t(at) % E), from);
                    mine &= mine - 1;
                    limit = fmaxf(limit, of_order(max(uint32_t(top.last >> 32), kOrderLowest + 1)));
                }
                if constexpr (W > 1) {
                    if (lane == 0 && uint32_t(top.last >> 32) > known) atomicMax(&bar, uint32_t(top.last >> 32));
                }
            }
        }
        const float m = fmaxf(u.m, all), d = fmaxf((u.m - m) * a.scale2, -2000.f), f = __builtin_amdgcn_exp2f(d);
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
    join_lanes<1, 32, ENT>(u, a.scale2);
    uint64_t key = 0;
    if constexpr (TOP) key = top.best(pending[wave]);
    if constexpr (W == 1) {
        const Row r(first_lane(u));
        if constexpr (TOP) {
            int at = lane, n = a.top;
            if (top.last == 0) {
                n = top.n;
                at = 0;
                for (int j = 0; j < n; j++) at += pending[wave][j] > key;
            }
            if (key) put_top(a, row, r, key, at);
            if (n < a.top) fill_top<T>(a, row, r, n);  // (n: all that can come)
        }
        if (lane == 0) put_sums(a, row, u, r, given, word);
    } else {
        if (lane == 0) sums[wave] = u;
        if constexpr (TOP) {
            rank[threadIdx.x] = 0;
            const uint32_t own = reached(uint32_t(key >> 32), (a.top + W - 1) / W);
            if (lane == 0) reach_last[wave] = own;
            __syncthreads();
            uint32_t least = reach_last[0];
#pragma unroll
            for (int w = 1; w < W; w++) least = min(least, reach_last[w]);
            least = max(least, max(known, bar));
            const bool in = key && uint32_t(key >> 32) >= least;
            const uint64_t from = __ballot(in);
            int at = 0;
            if (lane == 0 && from) at = atomicAdd(&count, __popcll(from));
            at = __builtin_amdgcn_readfirstlane(at);
            if (in) pool[at + __popcll(from & ((uint64_t(1) << lane) - 1))] = key;
        }
        __syncthreads();
        if (wave == 0) {
            if constexpr (W == kMostWaves) {
                u = sums[lane & (W - 1)];
                join_lanes<1, W / 2, ENT>(u, a.scale2);
            } else {
#pragma unroll
                for (int w = 1; w < W; w++) u = join(u, sums[w], a.scale2);
            }
            if (TOP && lane == 0) sums[0] = u;  // (what the others take when all have counted)
        }
        if constexpr (TOP) {
            const int n = count, j0 = wave * n / W, j1 = (wave + 1) * n / W;
            for (int c = 0; c < n; c += 64) {
                const uint64_t mine = c + lane < n ? pool[c + lane] : 0;
                int larger = 0;
                for (int j = j0; j < j1; j++) larger += pool[j] > mine;
                if (larger) atomicAdd(&rank[c + lane], larger);
            }
            __syncthreads();
            u = sums[0];
        }
        const Row r(u);
        if constexpr (TOP) {
            const int n = count, i = threadIdx.x;
            if (a.splits > 1) {
                if (i < n && rank[i] < a.top) a.part_keys[task * a.top + rank[i]] = pool[i];
                if (i >= n && i < a.top) a.part_keys[task * a.top + i] = 0;
            } else {
                if (i < n) put_top(a, row, r, pool[i], rank[i]);
                if (n < a.top && wave == 0) fill_top<T>(a, row, r, n);  // (n: all that can come)
            }
        }
        if (threadIdx.x) return;  // (without top words the others' sums are their own)
        if (a.splits > 1) a.part[task] = u;
        else put_sums(a, row, u, r, given, word);
    }
}

// The parts of a row joined: a wavefront to a row, so many lists of top words in flight together.
constexpr int kLists = 8;

template <typename T>
__global__ __launch_bounds__(64) void k_probs_join(ProbArgs a) {
    const int lane = threadIdx.x;
    const int64_t row = block_index();
    if (row >= a.g.n) return;
    const int64_t word = given_word(a, row);
    Sums u = lane < int(a.splits) ? a.part[row * a.splits + lane] : Sums{-FLT_MAX, 0.f, 0.f};
    join_lanes<1, 32, true>(u, a.scale2);
    u = first_lane(u);
    Top top;
    top.init(a.top_ids ? a.top : 1);
    if (a.top_ids) {
        const int from = 63 - lane;
        const uint64_t* lists = a.part_keys + row * a.splits * a.top + from;
        for (uint32_t b = 0; b < a.splits; b += kLists) {
            uint64_t k[kLists];
#pragma unroll
            for (int i = 0; i < kLists; i++) k[i] = from < a.top && b + i < a.splits ? lists[(b + i) * a.top] : 0;
#pragma unroll
            for (int i = 0; i < kLists; i++)
                if (top.beaten(k[i])) top.merge(k[i]);
        }
    }
    const Row r(u);
    if (a.top_ids) {
        if (top.key) put_top(a, row, r, top.key, lane);
        if (top.last == 0) fill_top<T>(a, row, r, __popcll(__ballot(top.key != 0)));
    }
    Given<T> given{};
    if (a.log_prob) given = given_of<T>(a, row, word);
    if (lane == 0) put_sums(a, row, u, r, given, word);
}

// A row of few scores is one wavefront's, one of many four wavefronts'.  Many rows
// fill the device with a wavefront each, and four that wait for each other at a
// row's top words take longer: one and four take, a call in a graph, for 20000 bf16
// scores (2500 runs) with 8 top words, 20 and 14 us for 600 rows, 25 and 26 for 2048,
// 69 and 88 for 8192 (without top words 11, 8; 15, 16; 59, 58).  With 32768 (4096
// runs) 36 and 33 us for 2048 rows, 108 and 115 for 8192.
//
// Few rows have sixteen wavefronts each: with them and with four, 128 rows of 8192
// fp32 runs take 11 and 16 us with 8 top words, 5.3 and 6.4 without, 256 rows 13 and
// 18, 8.0 and 8.4.  From one row to a unit on four do better: 400 rows take 21 and 18,
// 11.0 and 10.2, 512 rows 22 and 20, 12.6 and 12.2 (of 4096 runs 18 and 13, 8.3 and
// 7.8), 513 rows 26 and 20, 13.9 and 12.3.
//
// One launch is less than the two of a row cut into parts, so these are cut only
// where that leaves long rows to few workgroups.  13 rows uncut and cut, with 8 top
// words and without: 12664 runs 12.2, 12.3 and 5.8, 6.1 us in fp32, 15.5, 13.1 and
// 8.2, 6.8 in bf16, whose runs have twice the scores; 16384 runs 13.5, 12.1 and 6.4,
// 6.2, in bf16 17.6, 13.2 and 9.3, 7.0; 65536 runs 35, 15 and 17, 6.5, in bf16 50, 17
// and 29, 8.4.  Up to 256 parts in all: 32 rows of 65536 runs take 17.5 us in 8 parts
// each, 24 in 16 and 20 in 4, 128 rows 31 in 2, 36 in 4 and 37 uncut (without top
// words 24 in 2 and 22 uncut), 200 rows 56 in 2 and 44 uncut.  Up to 32 a row: one of
// 131072 runs takes 15.3 us in 32, 15.0 in 16 and 17.8 in 8, without top words 5.7,
// 6.6 and 8.4.
constexpr int64_t kWaveRuns = 4 * 64 * kRuns;    // up to so many runs
constexpr int64_t kManyRows = 2048;              // from so many rows
constexpr int64_t kManyRuns = 14 * 64 * kRuns;   // up to so many runs
constexpr int64_t kFewRows = 512;
constexpr int64_t kLongRuns = 4 * kMostWaves * 64 * kRuns;
constexpr int64_t kFill = 256;                   // workgroups
constexpr uint32_t kMaxSplits = 32;

struct Cut {
    int waves;
    uint32_t splits, per;
};
Cut cut_of(const Scores& g) {
    const bool one = int64_t(g.total) <= (g.n < kManyRows ? kWaveRuns : kManyRuns);
    Cut c{one ? 1 : g.n > kFewRows ? kWaves : kMostWaves, 1, g.total};
    if (c.waves < kMostWaves || int64_t(g.total) <= kLongRuns || g.n > kFill / 2) return c;
    const uint32_t step = kMostWaves * 64 * kRuns, steps = (g.total + step - 1) / step;
    const uint32_t s = uint32_t(std::min<int64_t>(std::min<int64_t>(steps, kMaxSplits), kFill / std::max<int64_t>(g.n, 1)));
    c.per = (steps + s - 1) / s * step;
    c.splits = (g.total + c.per - 1) / c.per;
    return c;
}

template <typename T, int FIT, bool TOP, bool ENT>
hipError_t probs3(ProbArgs a, Cut c, hipStream_t s) {
    if (c.waves == 1) k_probs<T, FIT, TOP, ENT, 1><<<grid_of((a.g.n + kWaves - 1) / kWaves), kThreads, 0, s>>>(a);
    else if (c.waves == kWaves) k_probs<T, FIT, TOP, ENT, kWaves><<<grid_of(a.g.n), kThreads, 0, s>>>(a);
    else k_probs<T, FIT, TOP, ENT, kMostWaves><<<grid_of(a.g.n * c.splits), kMostWaves * 64, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.splits == 1) return e;
    k_probs_join<T><<<grid_of(a.g.n), 64, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int FIT>
hipError_t probs2(const ProbArgs& a, Cut c, hipStream_t s) {
    if (a.top_ids) return a.entropy ? probs3<T, FIT, true, true>(a, c, s) : probs3<T, FIT, true, false>(a, c, s);
    return a.entropy ? probs3<T, FIT, false, true>(a, c, s) : probs3<T, FIT, false, false>(a, c, s);
}
template <typename T>
hipError_t probs1(ProbArgs a, Cut c, hipStream_t s) {
    switch (fit_of(a.g, 16 / sizeof(T))) {
        case kWhole: return probs2<T, kWhole>(a, c, s);
        case kOverlap: return probs2<T, kOverlap>(a, c, s);
        default: return probs2<T, kShort>(a, c, s);
    }
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
    bool rows_first;     // wavefronts that follow each other take a part of one row after the other
    bool apart;          // the output is not the scores' memory: what two runs have in common may be written twice
    float scale, scale2;
    int32_t id_bytes;
};

template <typename TI, typename TO, int FIT, bool ENT>
__global__ __launch_bounds__(kThreads) void k_probs_grad(ProbGradArgs a) {
    constexpr int E = lane_elems<TI, TO>();
    const int lane = threadIdx.x & 63;
    const int64_t w = block_index() * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t by = a.rows_first ? a.g.n : int64_t(a.parts), q0 = w / by, q1 = w - q0 * by;
    const int64_t row = a.rows_first ? q1 : q0;
    const uint32_t part = uint32_t(a.rows_first ? q0 : q1);
    if (row >= a.g.n || part >= a.parts) return;
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
        if (c1 != 0.f) c0 += c1 * a.entropy[row];  // (which may be NaN)
        c1 *= kLn2;
    }
    c0 *= a.scale;
    c1 *= a.scale;
    one *= a.scale;
    if (m == -kInf) one = c0 = c1 = 0.f;  // a row of no words
    const bool zero = c0 == 0.f && c1 == 0.f && one == 0.f;
    const uint32_t id_tile = id >= 0 ? uint32_t(id) / a.g.cols : ~0u, id_at = uint32_t(id) - id_tile * a.g.cols;
    const TI* x = static_cast<const TI*>(a.x) + row * a.g.row_stride;
    TO* out = static_cast<TO*>(a.out) + row * a.out_row_stride;
    Run<TI, E, FIT> r[kRuns];
    if (!zero) {
#pragma unroll
        for (int j = 0; j < kRuns; j++) r[j].load(a.g, x, min((part * kRuns + j) * 64 + lane, a.g.total - 1));
    }
#pragma unroll
    for (int j = 0; j < kRuns; j++) {
        const uint32_t q = (part * kRuns + j) * 64 + lane;
        if (q >= a.g.total) break;
        float y[E];
        if (zero) {
            r[j].find(a.g, q);
#pragma unroll
            for (int i = 0; i < E; i++) y[i] = 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < E; i++) {
                const float v = r[j].raw.value(i);
                const float z = (v - m) * a.scale2 - logs2, e = __builtin_amdgcn_exp2f(z);
                y[i] = e * (ENT ? c0 + c1 * fmaxf(z, -2000.f) : c0);
            }
            if (r[j].tile == id_tile && id_at - r[j].start < uint32_t(E)) {
#pragma unroll
                for (int i = 0; i < E; i++) y[i] += r[j].start + i == id_at ? one : 0.f;
            }
        }
        TO* at = out + r[j].tile * a.out_tile_stride + r[j].start;
        if (r[j].whole() || (FIT == kOverlap && a.apart)) {
            store_all<FIT == kWhole>(at, y);
        } else {
#pragma unroll
            for (int i = 0; i < E; i++)
                if (r[j].has(a.g, i)) store1(at + i, y[i]);
        }
    }
}

template <typename TI, typename TO, int FIT>
void k_probs_grad_of(const ProbGradArgs& a, dim3 grid, hipStream_t s) {
    if (a.by_entropy) k_probs_grad<TI, TO, FIT, true><<<grid, kThreads, 0, s>>>(a);
    else k_probs_grad<TI, TO, FIT, false><<<grid, kThreads, 0, s>>>(a);
}
template <typename TI, typename TO>
hipError_t probs_grad(ProbGradArgs a, const ScoreLayout& l, hipStream_t s) {
    constexpr int E = lane_elems<TI, TO>();
    a.g = scores_of(l, E);
    a.parts = (a.g.total + 64 * kRuns - 1) / (64 * kRuns);
    // Where a tile's rows do not end with lines of 128 bytes, those of neighbours are written at about the same time, and a
    // line that two share once: 2458 x 23750 fp32 values in tiles of 250 take 93 us so, 114 row by row.  (Whole lines: 8192 x
    // 32768 fp32 values in tiles of 128 433 and 405.)
    a.rows_first = l.vocab > l.cols && l.cols * int64_t(sizeof(TO)) % 128 != 0;
    const dim3 grid = grid_of((l.n * a.parts + kWaves - 1) / kWaves);
    switch (fit_of(a.g, E)) {
        case kWhole: k_probs_grad_of<TI, TO, kWhole>(a, grid, s); break;
        case kOverlap: k_probs_grad_of<TI, TO, kOverlap>(a, grid, s); break;
        default: k_probs_grad_of<TI, TO, kShort>(a, grid, s); break;
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
    a.apart = out != x;
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
