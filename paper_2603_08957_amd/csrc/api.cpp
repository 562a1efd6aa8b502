// C-ABI entry points: argument checks, workspace layout, phase ordering,
// the join's one count read-back, capacity checks and timing.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

#include "tre_internal.h"

using namespace tre;

namespace {

constexpr uint64_t kMagic = 0x7472655f6a6f696eull;  // "tre_join"
constexpr int kTargetWorkgroups = 2048;              // 8 per CU on 256 CUs
constexpr int64_t kAsyncMaxKeys = 4096;              // output keys of the one-workgroup unit table

tre_status dev_fail(hipError_t e, const char* where) {
    set_error(std::string(where) + ": " + hipGetErrorString(e));
    return TRE_E_DEVICE;
}

tre_status key_error(int32_t flags) {
    if (flags & 4) return TRE_E_KEYRANGE;
    if (flags & 1) return TRE_E_UNSORTED;
    if (flags & 2) return TRE_E_DUPKEY;
    return TRE_OK;
}

int64_t blocks_per_unit(const Plan& p) {
    if (p.kclass == KC_GEMM) {
        const int64_t M = p.swap ? p.nN : p.nM, N = p.swap ? p.nM : p.nN;
        if (p.fast) return (M / 128) * (N / 128);
        const int64_t bm = 32 * p.tile_m, bn = 32 * p.tile_n;
        return p.nB * ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    }
    return (p.tile_elems[2] + 255) / 256;
}

// Number of U-index ranges for the 128x128 path (0 or 1 = off).  Worth
// it when the U tiles are reused by many keys (pairs per U tuple high) but do
// not fit in one XCD's 4 MB L2: cutting every key's pairs into ranges of U and
// dispatching range by range lets the workgroups resident on an XCD share
// about 2 MB of U tiles, which stay in its L2 while the V tiles stream past,
// at the price of one partial tile per (key, range).
int32_t choose_u_ranges(const Plan& p, const Layout& L, int64_t n_u, int64_t n_pairs, int64_t n_w) {
    if (!(p.kclass == KC_GEMM && p.fast) || p.opt.u_ranges < 0 || n_u < 2 || n_w < 1) return 0;
    int64_t R;
    if (p.opt.u_ranges > 0) {
        R = p.opt.u_ranges;
    } else {
        const int64_t u_bytes = n_u * p.tile_elems[0] * (p.dtype == TRE_BF16 ? 2 : 4);
        const int64_t reuse = n_pairs / n_u;
        if (u_bytes <= (int64_t(16) << 20) || reuse < 64 || n_w * blocks_per_unit(p) < kTargetWorkgroups) return 0;
        // ~2 MB of U per range: measured best on the 262,144-vertex chain
        // (4 MB ranges thrash the L2, 1 MB ranges pay for twice the partials)
        R = (u_bytes + (int64_t(2) << 20) - 1) >> 21;
    }
    R = std::min<int64_t>({R, n_u, kMaxURanges});
    while (R > 1 && R * n_w > L.part_cap) R /= 2;
    return R > 1 ? int32_t(R) : 0;
}

// Windows for the paced persistent kernel (0 = not used).  It applies where
// U ranges would (U tiles reused by many keys and too big for one L2) when a W
// tile is one 128x128 block, and is preferred there: it keeps U tiles in L2
// without partial tiles.  `slots` = workgroups resident at once.
int32_t choose_pacing(const Plan& p, int64_t n_u, int64_t n_pairs, int64_t n_w, int64_t slots) {
    if (!(p.kclass == KC_GEMM && p.fast) || blocks_per_unit(p) != 1 || p.opt.pace_windows < 0 ||
        p.opt.max_pairs_per_unit > 0 || n_u < 2 || n_w < 1 || slots <= 0)
        return 0;
    int64_t W;
    if (p.opt.pace_windows > 0) {
        W = p.opt.pace_windows;
    } else {
        if (p.opt.u_ranges != 0) return 0;  // an explicit U-range request wins
        const int64_t u_bytes = n_u * p.tile_elems[0] * (p.dtype == TRE_BF16 ? 2 : 4);
        const int64_t reuse = n_pairs / n_u;
        if (u_bytes <= (int64_t(16) << 20) || reuse < 64 || n_w < slots) return 0;
        // ~5.5 MB of U per window: measured best on the 262,144-vertex chain
        // (12 windows of its 64 MB; 16 or 10 windows are 0.5% slower, 8 and
        // 24 windows 1-3%: small windows wait more often, large ones miss L2)
        constexpr int64_t kWindowBytes = int64_t(11) << 19;
        W = (u_bytes + kWindowBytes - 1) / kWindowBytes;
    }
    W = std::max<int64_t>(1, std::min<int64_t>({W, n_u, 256}));
    const int64_t n_wg = std::min(n_w, slots);
    const int64_t rounds = (n_w + n_wg - 1) / n_wg;
    if (rounds * 8 * W > kPaceCounters) return 0;
    return int32_t(W);
}

// Workgroups one unit occupies: its output blocks (GEMM), or its threads /
// 256 for the vector class (several small units share a workgroup).
double unit_workgroups(const Plan& p) {
    if (p.kclass == KC_GEMM) return double(blocks_per_unit(p));
    const int64_t threads = p.vec_dot ? p.tile_elems[2] * 16 : (p.tile_elems[2] + p.vec_ept - 1) / p.vec_ept;
    if (threads > 128) return double((threads + 255) / 256);
    int64_t t = 1;
    while (t < threads) t <<= 1;
    return double(t) / 256.0;
}

// Unit length cap.  GEMM-class units are dispatched longest first, so once
// the keys' output blocks fill every resident slot (two workgroups per CU)
// one unit per key is the better schedule: measured on the block-sparse
// product (1,024 blocks of 6.4 pairs on average), cutting keys into units of
// 4-8 pairs cost 10% more in contraction and partial-tile sums.
int64_t choose_unit(const Plan& p, const Layout& L, int64_t n_pairs, int64_t n_w) {
    const double uw = unit_workgroups(p);
    int dev = 0, cus = 0;
    const int64_t fill = (hipGetDevice(&dev) == hipSuccess &&
                          hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && cus > 0)
                             ? 2 * int64_t(cus)
                             : int64_t(kTargetWorkgroups);
    int64_t pu;
    if (p.opt.max_pairs_per_unit > 0) {
        pu = p.opt.max_pairs_per_unit;
    } else if (p.kclass == KC_GEMM && !p.fast) {
        pu = tile_unit_pairs(p, n_pairs, n_w);
    } else if (p.kclass == KC_MX) {
        pu = mx_unit_pairs(p, n_pairs, n_w);
    } else if (double(n_w) * uw >= kTargetWorkgroups || (p.kclass == KC_GEMM && double(n_w) * uw >= fill)) {
        pu = std::max<int64_t>(n_pairs, 1);  // enough output blocks: one unit per key
    } else {
        pu = std::max<int64_t>(4, int64_t(std::ceil(double(n_pairs) * uw / kTargetWorkgroups)));
    }
    // partial tiles of split keys must fit: at most 2 * n_pairs / pu of them
    const int64_t need = (2 * n_pairs + L.part_cap - 2) / std::max<int64_t>(L.part_cap - 1, 1);
    return std::max<int64_t>(pu, std::max<int64_t>(need, 1));
}

// Most pairs a join of n_u and n_v tuples (unique keys) can make: the cross
// product, or one pair per tuple of the other side when one side's key is
// made of join labels only.  The GROUP BY grids are sized for min(this,
// workspace capacity).
int64_t pair_bound(const Plan& p, int64_t n_u, int64_t n_v) {
    int64_t b = (n_v > 0 && n_u > INT64_MAX / n_v) ? INT64_MAX : n_u * n_v;
    if (p.nk[0] == p.n_join) b = std::min(b, n_v);  // a V tuple meets at most one U tuple
    if (p.nk[1] == p.n_join) b = std::min(b, n_u);
    return b;
}

}  // namespace

namespace {

// What the join leaves for its read-back.
struct JoinState {
    int64_t max_pairs = 0;
    int64_t cap = 0;      // pairs the GROUP BY grids are sized for
    bool counts_known = false;  // pair and key counts known on the host (no read-back needed for them)
    bool small = false;
    int32_t path = 0;     // tre_timing.join_path
};

// tre_join up to its read-back: argument checks, workspace layout and every
// join launch.  `out` gets the sizes and the internal fields.
tre_status join_enqueue(tre_plan_t plan, const int32_t* u_keys, int64_t n_u, const int32_t* v_keys, int64_t n_v,
                        void* ws, size_t ws_bytes, hipStream_t s, tre_join_result* out, JoinState* st,
                        const int64_t* n_u_dev = nullptr) {
    if (!plan || !out || n_u < 0 || n_v < 0 || !ws) {
        set_error("tre_join: null plan/out/workspace or negative size");
        return TRE_E_ARG;
    }
    const Plan& p = plan->p;
    std::memset(out, 0, sizeof(*out));
    out->n_u = n_u;
    out->n_v = n_v;
    if ((p.nk[0] > 0 && n_u > 0 && !u_keys) || (p.nk[1] > 0 && n_v > 0 && !v_keys)) {
        set_error("tre_join: null key array");
        return TRE_E_ARG;
    }
    if (reinterpret_cast<uintptr_t>(ws) % 256) {
        set_error("tre_join: workspace must be 256-byte aligned");
        return TRE_E_ARG;
    }
    if ((p.nk[0] == 0 && n_u > 1) || (p.nk[1] == 0 && n_v > 1)) {
        set_error("tre_join: a relation without promoted labels holds at most one tuple");
        return TRE_E_DUPKEY;
    }
    if (n_u >= INT32_MAX || n_v >= INT32_MAX) {
        set_error("tre_join: more than 2^31 - 1 tuples");
        return TRE_E_SHAPE;
    }
    const int64_t max_pairs = tre_workspace_max_pairs(plan, n_u, n_v, ws_bytes);
    if (max_pairs < 0) {
        set_error("tre_join: workspace smaller than tre_workspace_bytes(plan, n_u, n_v, 0)");
        return TRE_E_WORKSPACE;
    }
    st->max_pairs = max_pairs;
    out->internal[0] = kMagic;
    out->internal[1] = reinterpret_cast<uint64_t>(plan);
    out->internal[2] = reinterpret_cast<uint64_t>(ws);
    out->internal[3] = uint64_t(ws_bytes);
    out->internal[4] = uint64_t(max_pairs);
    const Layout L = make_layout(p, n_u, n_v, max_pairs);
    char* w = reinterpret_cast<char*>(ws);
    hipError_t e;
    const bool validate = p.opt.validate_keys != 0;
    WsHeader* hdr = reinterpret_cast<WsHeader*>(w + L.hdr);
    if (n_u > 0 && n_v == 1 && keyed_by_u(p)) {
        // one pair and one group per U tuple: nothing to count
        if (n_u > max_pairs) {
            out->n_pairs = n_u;
            set_error("tre_join: workspace too small for the matched pairs (see n_pairs)");
            return TRE_E_WORKSPACE;
        }
        if ((e = launch_keyed_by_u(p, L, w, u_keys, s, n_u_dev, validate)) != hipSuccess) return dev_fail(e, "join");
        st->cap = n_u;
        st->counts_known = true;
        st->path = 4;
        out->n_pairs = n_u;
        out->n_w = n_u;
        return TRE_OK;
    }
    // the join counts the pairs into the header; the GROUP BY stage reads
    // that count on the device (its grids are sized for the workspace's
    // capacity), so one read-back at the end returns the key checks, the
    // pair count and the key count together
    const bool vd = n_u > 0 && n_v > 0 && v_dense(p, n_u), ud = n_u > 0 && n_v > 0 && u_dense(p, n_v);
    if ((vd || ud) && (vd ? n_v : n_u) > max_pairs) {
        // one pair per tuple of the driving relation, known without the device
        out->n_pairs = vd ? n_v : n_u;
        set_error("tre_join: workspace too small for the matched pairs (see n_pairs)");
        return TRE_E_WORKSPACE;
    }
    const int64_t cap = std::min(max_pairs, pair_bound(p, n_u, n_v));
    st->cap = (n_u > 0 && n_v > 0) ? std::max<int64_t>(cap, 0) : 0;
    st->small = n_u > 0 && n_v > 0 && small_join_ok(p, n_u, n_v, cap);
    if (st->small) {
        if ((e = launch_join_small(p, L, w, u_keys, v_keys, cap, s, validate)) != hipSuccess) return dev_fail(e, "join");
    } else if (vd || ud) {
        if ((e = launch_group(p, L, w, u_keys, v_keys, cap, s, validate)) != hipSuccess) return dev_fail(e, "group");
    } else if ((e = launch_fill_zero(hdr, sizeof(WsHeader), s)) != hipSuccess) {
        return dev_fail(e, "header");
    } else if (validate) {
        const ValJob jobs[2] = {{u_keys, n_u, p.nk[0], p.radix[0], &hdr->err_u, n_u_dev},
                                {v_keys, n_v, p.nk[1], p.radix[1], &hdr->err_v, nullptr}};
        if ((e = launch_validate(jobs, 2, s)) != hipSuccess) return dev_fail(e, "validate");
    }
    if (st->small || vd || ud) {
        // joined whole, with the key checks
    } else if (n_u > 0 && n_v > 0 && max_pairs > 0) {
        if ((e = launch_join(p, L, w, u_keys, v_keys, s, 0)) != hipSuccess) return dev_fail(e, "join");
        if ((e = launch_group(p, L, w, u_keys, v_keys, cap, s)) != hipSuccess) return dev_fail(e, "group");
    } else if (n_u > 0 && n_v > 0) {
        // no room for any pair: count only, to report the size needed
        if ((e = launch_join(p, L, w, u_keys, v_keys, s, 0)) != hipSuccess) return dev_fail(e, "join");
    }
    st->path = st->small                               ? 5
               : vd                                     ? 3
               : ud                                     ? 6
               : (p.v_outer && p.nk[0] == p.n_join)     ? 2
               : p.v_outer                              ? 1
                                                        : 0;
    return TRE_OK;
}

// The join's read-back: key checks and, unless known on the host, the pair
// and key counts.  With key checks off and counts known, nothing to wait for.
tre_status join_finish(const Plan& p, const JoinState& st, tre_join_result* out, hipStream_t s) {
    if (st.counts_known && !p.opt.validate_keys) return TRE_OK;
    const Layout L = make_layout(p, out->n_u, out->n_v, st.max_pairs);
    const char* w = reinterpret_cast<const char*>(out->internal[2]);
    WsHeader h{};
    hipError_t e;
    if ((e = hipMemcpyAsync(&h, w + L.hdr, sizeof(h), hipMemcpyDeviceToHost, s)) != hipSuccess)
        return dev_fail(e, "count read-back");
    if ((e = hipStreamSynchronize(s)) != hipSuccess) return dev_fail(e, "join sync");
    tre_status ks = key_error(h.err_u);
    if (ks == TRE_OK) ks = key_error(h.err_v);
    if (ks != TRE_OK) {
        set_error(std::string("tre_join: invalid keys in ") + (key_error(h.err_u) != TRE_OK ? "U" : "V"));
        return ks;
    }
    if (st.counts_known) return TRE_OK;
    const int64_t n_pairs = (out->n_u > 0 && out->n_v > 0) ? h.n_pairs : 0;
    out->n_pairs = n_pairs;
    if (n_pairs > st.max_pairs) {
        set_error("tre_join: workspace too small for the matched pairs (see n_pairs)");
        return TRE_E_WORKSPACE;
    }
    if (n_pairs >= INT32_MAX) {
        set_error("tre_join: more than 2^31 - 1 pairs");
        return TRE_E_SHAPE;
    }
    out->n_w = n_pairs > 0 ? h.n_w : 0;
    return TRE_OK;
}

void join_timing(tre_timing* timing, int32_t path) {
    if (!timing) return;
    const int32_t deferred = timing->deferred;
    std::memset(timing, 0, sizeof(*timing));
    timing->deferred = deferred;
    timing->join_path = path;
}

// tre_contract's launches, for the join's counts n_pairs and n_w, and the
// counts of an asynchronous call (counts not null).  With
// `dev` those are upper bounds and every kernel reads the join's counts from
// the workspace header (the caller has checked that the bounds need no U
// ranges and take a one-workgroup unit table or one unit per key).
tre_status contract_enqueue(tre_plan_t plan, const tre_join_result* jr, int64_t n_pairs, int64_t n_w,
                            const void* u_tiles, const void* v_tiles, int32_t* w_keys, void* w_out,
                            int32_t* pairs_out, hipStream_t s, tre_timing* timing, bool dev = false,
                            int64_t* counts = nullptr) {
    // W's element type is the plan's (fp32, or bf16 bits with w_bf16); the
    // kernels take the array as float* and store 16-bit elements through it
    // when the plan says bf16
    float* w_tiles = static_cast<float*>(w_out);
    const Plan& p = plan->p;
    if (n_pairs == 0) {
        if (!counts) return TRE_OK;
        const Layout L = make_layout(p, jr->n_u, jr->n_v, int64_t(jr->internal[4]));
        const hipError_t e = launch_write_outputs(p, L, reinterpret_cast<char*>(jr->internal[2]), nullptr, nullptr, 0, 0,
                                                  s, true, counts);
        return e == hipSuccess ? TRE_OK : dev_fail(e, "counts");
    }
    if (!u_tiles || !v_tiles || !w_tiles || (p.nk[2] > 0 && !w_keys)) {
        set_error("tre_contract: null tile or key buffer");
        return TRE_E_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(u_tiles) | reinterpret_cast<uintptr_t>(v_tiles) |
         reinterpret_cast<uintptr_t>(w_tiles)) & 15) {
        set_error("tre_contract: tile arrays must be 16-byte aligned");
        return TRE_E_ARG;
    }
    char* w = reinterpret_cast<char*>(jr->internal[2]);
    const Layout L = make_layout(p, jr->n_u, jr->n_v, int64_t(jr->internal[4]));
    // deferred timing: only the contraction kernel, by its own start / end
    // events (no marker packets); otherwise marks around every phase
    const bool deferred = timing && timing->deferred;
    PhaseTimer tm(timing != nullptr && !deferred);
    KernelEvents ke;
    if (deferred) {
        ke.start = event_acquire();
        ke.stop = event_acquire();
    }
    tm.mark(s);
    const int64_t slots = (p.kclass == KC_GEMM && p.fast) ? gemm_paced_slots(p) : 0;
    const int32_t pace = choose_pacing(p, jr->n_u, n_pairs, n_w, slots);
    const int32_t R = (pace || dev) ? 0 : choose_u_ranges(p, L, jr->n_u, n_pairs, n_w);
    // (a keyless one-tuple V with W keyed by U: one pair per key, nothing
    // to cut and no partial tiles to sum)
    const bool one_pair_keys = jr->n_v <= 1 && keyed_by_u(p);
    int64_t p_unit = (R > 1 || pace || one_pair_keys) ? n_pairs : choose_unit(p, L, n_pairs, n_w);
    // (no key holds more than n_pairs - n_w + 1 pairs, or more than the labels
    // that W does not keep have values: nothing to cut)
    if ((!dev && p_unit > n_pairs - n_w) || p_unit >= p.key_pairs_max) p_unit = n_pairs;
    // (a key to a unit, as the join left them)
    const bool whole_keys = p.kclass == KC_MX && !one_pair_keys && p_unit >= n_pairs && mx_whole_keys(p, n_pairs, n_w);
    hipError_t e;
    // (launch_units writes the tile offset tables itself)
    if (R > 1) {
        if ((e = launch_tables(p, reinterpret_cast<int32_t*>(w + L.tables), s)) != hipSuccess)
            return dev_fail(e, "tables");
        e = launch_range_units(p, L, w, n_w, jr->n_u, R, s);
    } else if (one_pair_keys || whole_keys) {
        // the join wrote the units, or the kernel takes its segments
        e = launch_tables(p, reinterpret_cast<int32_t*>(w + L.tables), s);
    } else {
        e = launch_units(p, L, w, n_pairs, n_w, p_unit, !pace, s, dev);
    }
    if (e != hipSuccess) return dev_fail(e, "units");
    tm.mark(s);
    // (4-bit tiles take the block of outputs and the grid from it: of whole keys
    // there are n_w units, no more)
    const int64_t unit_bound = R > 1                                      ? int64_t(R) * n_w
                               : p.kclass == KC_MX && p_unit >= n_pairs ? n_w
                                                                        : n_w + n_pairs / p_unit + 1;
    if (pace) {
        // one unit per key; every workgroup of the grid is resident at once
        const int64_t n_wg = std::min(n_w, slots);
        const int64_t rounds = (n_w + n_wg - 1) / n_wg;
        if ((e = launch_fill_zero(w + L.pace, sizeof(int32_t) * size_t(rounds * 8 * pace), s)) != hipSuccess)
            return dev_fail(e, "pace");
        if (ke.start && ke.stop) t_kernel_events = &ke;
        e = launch_gemm_paced(p, L, w, u_tiles, v_tiles, w_tiles, n_pairs, n_wg, pace, s);
    } else {
        if (ke.start && ke.stop) t_kernel_events = &ke;
        e = launch_contract(p, L, w, u_tiles, v_tiles, w_tiles, n_pairs, n_w, unit_bound, whole_keys, s);
    }
    t_kernel_events = nullptr;
    if (e != hipSuccess) return dev_fail(e, "contract");
    tm.mark(s);
    // units as long as the average key or longer: outliers are cut, and their
    // partial tiles summed on the way of the outputs
    const bool outliers =
        p.kclass != KC_VEC && !p.fast && R <= 1 && p_unit < n_pairs && p_unit * n_w >= n_pairs;
    const int64_t split_bound = R > 1 ? n_w : std::min<int64_t>(n_w, n_pairs / (p_unit + 1) + 1);
    if ((R > 1 || p_unit < n_pairs) && !outliers) {
        if ((e = launch_reduce(p, L, w, w_tiles, split_bound, s)) != hipSuccess) return dev_fail(e, "reduce");
    }
    if ((e = launch_write_outputs(p, L, w, w_keys, pairs_out, n_pairs, n_w, s, dev, counts,
                                  outliers ? w_tiles : nullptr, split_bound)) != hipSuccess)
        return dev_fail(e, "outputs");
    tm.mark(s);
    if (timing) {
        timing->contract_path = pace ? 3 : R > 1 ? 4 : p.kclass == KC_VEC ? 1 : p.kclass == KC_MX ? 5 : p.fast ? 2 : 0;
        timing->contract_block = p.kclass == KC_MX ? mx_block(p, n_pairs, unit_bound) : 0;
        if (deferred) {
            if (ke.launched) {
                timing->events[0] = reinterpret_cast<void*>(ke.start);
                timing->events[1] = reinterpret_cast<void*>(ke.stop);
                timing->pending = 1;
                ke.keep = true;
            }
        } else {
            timing->units_ms = tm.between(0, 1);
            timing->contract_ms = tm.between(1, 2);
            timing->reduce_ms = tm.between(2, 3);
            timing->total_ms += tm.between(0, 3);
        }
        WsHeader h{};
        if (!deferred && hipMemcpy(&h, w + L.hdr, sizeof(h), hipMemcpyDeviceToHost) == hipSuccess) {
            // (without a unit table nobody has written its counts)
            timing->n_units = whole_keys ? h.n_w : h.n_units;
            timing->n_split_segments = whole_keys ? 0 : h.n_split;
            timing->n_partials = whole_keys ? 0 : h.n_parts;
        }
    }
    return TRE_OK;
}

// Upper bounds on a join's pair and output key counts, from the sizes alone
// (exact when the host knows them), and whether the contraction can be
// enqueued on them with the counts read on the device: no pacing and no U
// ranges at the bounds, and a one-workgroup unit table or one unit per key
// (the paced persistent grid takes one unit per key and reads their count).
struct AsyncBounds {
    int64_t pairs = 0, keys = 0;
    bool ok = false;
};

AsyncBounds async_bounds(const Plan& p, int64_t n_u, int64_t n_v, int64_t max_pairs) {
    AsyncBounds b;
    if (n_u > 0 && n_v == 1 && keyed_by_u(p)) {
        b.pairs = b.keys = n_u;
    } else {
        b.pairs = (n_u > 0 && n_v > 0) ? std::max<int64_t>(0, std::min(max_pairs, pair_bound(p, n_u, n_v))) : 0;
        b.keys = std::min(b.pairs, key_space(p));
    }
    if (b.pairs <= 0) {
        b.ok = true;
        return b;
    }
    const Layout L = make_layout(p, n_u, n_v, max_pairs);
    const int64_t slots = (p.kclass == KC_GEMM && p.fast) ? gemm_paced_slots(p) : 0;
    if (choose_pacing(p, n_u, b.pairs, b.keys, slots) != 0) {
        b.ok = true;  // one unit per key; the persistent grid reads the unit count on the device
        return b;
    }
    if (choose_u_ranges(p, L, n_u, b.pairs, b.keys) != 0) return b;
    const int64_t p_unit = choose_unit(p, L, b.pairs, b.keys);
    b.ok = b.keys <= kAsyncMaxKeys || p_unit >= b.pairs;
    return b;
}

}  // namespace

extern "C" {

tre_status tre_join(tre_plan_t plan, const int32_t* u_keys, int64_t n_u, const int32_t* v_keys, int64_t n_v,
                    void* ws, size_t ws_bytes, void* stream, tre_join_result* out, tre_timing* timing) {
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    PhaseTimer tm(timing != nullptr && !timing->deferred);  // (deferred timing covers the contraction only)
    tm.mark(s);
    JoinState st;
    tre_status r = join_enqueue(plan, u_keys, n_u, v_keys, n_v, ws, ws_bytes, s, out, &st);
    if (r != TRE_OK) return r;
    // the end mark goes before the read-back, so reading the join time after
    // the wait needs no further wait
    tm.mark(s);
    if ((r = join_finish(plan->p, st, out, s)) != TRE_OK) return r;
    join_timing(timing, st.path);
    if (timing) {
        timing->join_ms = tm.between(0, 1);
        timing->total_ms = timing->join_ms;
    }
    return TRE_OK;
}

tre_status tre_contract(tre_plan_t plan, const tre_join_result* jr, const void* u_tiles, const void* v_tiles,
                        int32_t* w_keys, int64_t w_cap, void* w_out, int32_t* pairs_out, int64_t pair_cap,
                        void* stream, tre_timing* timing) {
    if (!plan || !jr) {
        set_error("tre_contract: null plan or join result");
        return TRE_E_ARG;
    }
    if (jr->internal[0] != kMagic || jr->internal[1] != reinterpret_cast<uint64_t>(plan)) {
        set_error("tre_contract: join result was not produced by tre_join with this plan");
        return TRE_E_STATE;
    }
    if (w_cap < jr->n_w || (pairs_out && pair_cap < jr->n_pairs)) {
        set_error("tre_contract: output capacity below n_w / n_pairs");
        return TRE_E_CAPACITY;
    }
    return contract_enqueue(plan, jr, jr->n_pairs, jr->n_w, u_tiles, v_tiles, w_keys, w_out, pairs_out,
                            reinterpret_cast<hipStream_t>(stream), timing);
}

tre_status tre_join_keys(tre_plan_t plan, const tre_join_result* jr, int32_t* w_keys, int64_t w_cap, void* stream) {
    if (!plan || !jr) {
        set_error("tre_join_keys: null plan or join result");
        return TRE_E_ARG;
    }
    if (jr->internal[0] != kMagic || jr->internal[1] != reinterpret_cast<uint64_t>(plan)) {
        set_error("tre_join_keys: join result was not produced by tre_join with this plan");
        return TRE_E_STATE;
    }
    const Plan& p = plan->p;
    if (w_cap < jr->n_w) {
        set_error("tre_join_keys: output capacity below n_w");
        return TRE_E_CAPACITY;
    }
    if (p.nk[2] == 0 || jr->n_w == 0) return TRE_OK;
    if (!w_keys) {
        set_error("tre_join_keys: null key buffer");
        return TRE_E_ARG;
    }
    char* w = reinterpret_cast<char*>(jr->internal[2]);
    const Layout L = make_layout(p, jr->n_u, jr->n_v, int64_t(jr->internal[4]));
    const hipError_t e = launch_write_outputs(p, L, w, w_keys, nullptr, jr->n_pairs, jr->n_w,
                                              reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "keys");
}

tre_status tre_timing_read(tre_timing* t) {
    if (!t) return TRE_E_ARG;
    if (!t->pending) return TRE_OK;
    // the contraction kernel's start and end
    t->contract_ms = event_elapsed(t->events[0], t->events[1]);
    t->total_ms += t->contract_ms;
    for (auto& e : t->events) {
        event_release(reinterpret_cast<hipEvent_t>(e));
        e = nullptr;
    }
    t->pending = 0;
    return TRE_OK;
}

tre_status tre_execute(tre_plan_t plan, const int32_t* u_keys, int64_t n_u, const void* u_tiles,
                       const int32_t* v_keys, int64_t n_v, const void* v_tiles, int32_t* w_keys, void* w_tiles,
                       int64_t w_cap, int64_t* n_w, int32_t* pairs_out, int64_t pair_cap, int64_t* n_pairs,
                       void* ws, size_t ws_bytes, void* stream, tre_timing* timing) {
    tre_join_result jr{};
    tre_status st = tre_join(plan, u_keys, n_u, v_keys, n_v, ws, ws_bytes, stream, &jr, timing);
    if (n_pairs) *n_pairs = jr.n_pairs;
    if (n_w) *n_w = jr.n_w;
    if (st != TRE_OK) return st;
    return tre_contract(plan, &jr, u_tiles, v_tiles, w_keys, w_cap, w_tiles, pairs_out, pair_cap, stream, timing);
}

tre_status tre_output_bounds(tre_plan_t plan, int64_t n_u, int64_t n_v, size_t ws_bytes, int64_t* pairs_bound,
                             int64_t* keys_bound, int32_t* async_ok) {
    if (!plan || n_u < 0 || n_v < 0 || !pairs_bound || !keys_bound || !async_ok) {
        set_error("tre_output_bounds: null argument or negative size");
        return TRE_E_ARG;
    }
    const int64_t max_pairs = tre_workspace_max_pairs(plan, n_u, n_v, ws_bytes);
    if (max_pairs < 0) {
        set_error("tre_output_bounds: workspace smaller than tre_workspace_bytes(plan, n_u, n_v, 0)");
        return TRE_E_WORKSPACE;
    }
    const AsyncBounds b = async_bounds(plan->p, n_u, n_v, max_pairs);
    *pairs_bound = b.pairs;
    *keys_bound = b.keys;
    *async_ok = b.ok ? 1 : 0;
    return TRE_OK;
}

tre_status tre_execute_async(tre_plan_t plan, const int32_t* u_keys, int64_t n_u, const int64_t* n_u_dev,
                             const void* u_tiles, const int32_t* v_keys, int64_t n_v, const void* v_tiles,
                             int32_t* w_keys, void* w_tiles, int64_t w_cap, int32_t* pairs_out, int64_t pair_cap,
                             int64_t* counts, void* ws, size_t ws_bytes, void* stream, tre_timing* timing) {
    if (!plan || !counts || n_u < 0 || n_v < 0) {
        set_error("tre_execute_async: null plan / counts or negative size");
        return TRE_E_ARG;
    }
    const Plan& p = plan->p;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (n_u_dev && !(n_v == 1 && keyed_by_u(p))) {
        set_error("tre_execute_async: a device-side U count needs a keyless one-tuple V with W keyed by U");
        return TRE_E_ARG;
    }
    const int64_t max_pairs = tre_workspace_max_pairs(plan, n_u, n_v, ws_bytes);
    if (max_pairs < 0) {
        set_error("tre_execute_async: workspace smaller than tre_workspace_bytes(plan, n_u, n_v, 0)");
        return TRE_E_WORKSPACE;
    }
    const AsyncBounds b = async_bounds(p, n_u, n_v, max_pairs);
    if (!b.ok) {
        if (n_u_dev) {
            set_error("tre_execute_async: a device-side U count needs an output within the device-count launches");
            return TRE_E_ARG;
        }
        // the counts are needed on the host: the synchronous call, then the
        // counts and the status to the device
        int64_t nw = 0, np = 0;
        const tre_status st = tre_execute(plan, u_keys, n_u, u_tiles, v_keys, n_v, v_tiles, w_keys, w_tiles, w_cap,
                                          &nw, pairs_out, pair_cap, &np, ws, ws_bytes, stream, timing);
        if (st == TRE_E_ARG || st == TRE_E_DEVICE || st == TRE_E_STATE) return st;
        const hipError_t e = launch_counts_set(np, nw, int64_t(st), counts, s);
        return e == hipSuccess ? st : dev_fail(e, "counts");
    }
    if (w_cap < b.keys || (pairs_out && pair_cap < b.pairs)) {
        set_error("tre_execute_async: output capacity below the bounds of tre_output_bounds");
        return TRE_E_CAPACITY;
    }
    tre_join_result jr{};
    JoinState js;
    PhaseTimer tm(timing != nullptr && !timing->deferred);
    tm.mark(s);
    tre_status st = join_enqueue(plan, u_keys, n_u, v_keys, n_v, ws, ws_bytes, s, &jr, &js, n_u_dev);
    if (st != TRE_OK) return st;
    tm.mark(s);
    join_timing(timing, js.path);
    if ((st = contract_enqueue(plan, &jr, b.pairs, b.keys, u_tiles, v_tiles, w_keys, w_tiles, pairs_out, s, timing,
                               true, counts)) != TRE_OK)
        return st;
    if (timing && !timing->deferred) {
        const float jm = tm.between(0, 1);
        timing->join_ms = jm;
        timing->total_ms += jm;
    }
    return TRE_OK;
}

tre_status tre_cast_f32_bf16(const float* x, uint16_t* y, int64_t n, void* stream) {
    if (n < 0 || (n > 0 && (!x || !y))) return TRE_E_ARG;
    hipError_t e = launch_cast_bf16(x, y, n, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "cast");
}

tre_status tre_scale_f32(const float* x, float* y, int64_t n, float scale, void* stream) {
    if (n < 0 || (n > 0 && (!x || !y))) return TRE_E_ARG;
    if (n > 0 && ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15)) {
        set_error("tre_scale_f32: arrays must be 16-byte aligned");
        return TRE_E_ARG;
    }
    hipError_t e = launch_scale(x, y, n, scale, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "scale");
}

namespace {

tre_status mx_args(tre_plan_t plan, int32_t operand, const void* tiles, int32_t dtype, int64_t n, const void* mx_tiles,
                   const char* where) {
    if (!plan || n < 0 || (operand != 0 && operand != 1) || (n > 0 && (!tiles || !mx_tiles))) {
        set_error(std::string(where) + ": null plan or array, negative size or no such operand");
        return TRE_E_ARG;
    }
    if (plan->p.dtype != TRE_MXFP4) {
        set_error(std::string(where) + ": the plan's tiles are not TRE_MXFP4");
        return TRE_E_DTYPE;
    }
    if (dtype != TRE_F32 && dtype != TRE_BF16) {
        set_error(std::string(where) + ": unquantised tiles must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    if ((reinterpret_cast<uintptr_t>(tiles) | reinterpret_cast<uintptr_t>(mx_tiles)) & 15) {
        set_error(std::string(where) + ": tile arrays must be 16-byte aligned");
        return TRE_E_ARG;
    }
    if (n >= INT32_MAX) {
        set_error(std::string(where) + ": more than 2^31 - 1 tiles");
        return TRE_E_SHAPE;
    }
    return TRE_OK;
}

}  // namespace

tre_status tre_mx_quantize(tre_plan_t plan, int32_t operand, const void* tiles, int32_t src_dtype, int64_t n,
                           void* mx_tiles, void* stream) {
    const tre_status st = mx_args(plan, operand, tiles, src_dtype, n, mx_tiles, "tre_mx_quantize");
    if (st != TRE_OK || n == 0) return st;
    const hipError_t e =
        launch_mx_quantize(plan->p, operand, tiles, src_dtype, n, mx_tiles, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "mx_quantize");
}

tre_status tre_mx_dequantize(tre_plan_t plan, int32_t operand, const void* mx_tiles, int64_t n, void* tiles,
                             int32_t dst_dtype, void* stream) {
    const tre_status st = mx_args(plan, operand, tiles, dst_dtype, n, mx_tiles, "tre_mx_dequantize");
    if (st != TRE_OK || n == 0) return st;
    const hipError_t e =
        launch_mx_dequantize(plan->p, operand, mx_tiles, n, tiles, dst_dtype, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "mx_dequantize");
}

namespace {

// Sizes of a table that the row entry points take: offsets in bytes and the
// launches' wavefronts stay within 63 bits.
bool rows_ok(int64_t n_ids, int64_t n_rows, int64_t elems) {
    return n_ids >= 0 && n_ids < INT32_MAX && n_rows >= 1 && n_rows < INT32_MAX && elems >= 1 && elems <= (int64_t(1) << 30);
}

}  // namespace

tre_status tre_lookup(const void* table, int32_t table_dtype, int64_t n_rows, int64_t row_elems, int64_t tile_rows,
                      const void* ids, int32_t id_bytes, int64_t n_ids, float scale, void* out, int32_t out_dtype,
                      int64_t* status, void* stream) {
    if (table_dtype != TRE_F32 && table_dtype != TRE_BF16 && table_dtype != TRE_MXFP4) {
        set_error("tre_lookup: table_dtype must be TRE_F32, TRE_BF16 or TRE_MXFP4");
        return TRE_E_DTYPE;
    }
    if (out_dtype != TRE_F32 && out_dtype != TRE_BF16) {
        set_error("tre_lookup: out_dtype must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    const bool mx = table_dtype == TRE_MXFP4;
    if (!rows_ok(n_ids, n_rows, row_elems) || (mx && (tile_rows < 1 || tile_rows > n_rows || n_rows % tile_rows))) {
        set_error("tre_lookup: size out of range, or tile_rows does not divide n_rows");
        return TRE_E_SHAPE;
    }
    if (mx && mx_tile_bytes(tile_rows, row_elems) > INT32_MAX) {
        set_error("tre_lookup: 4-bit tile larger than 2^31 - 1 bytes");
        return TRE_E_SHAPE;
    }
    if (n_ids == 0) return TRE_OK;
    if (!table || !ids || !out || (id_bytes != 4 && id_bytes != 8)) {
        set_error("tre_lookup: null array, or ids of neither 4 nor 8 bytes");
        return TRE_E_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(out)) & 15 ||
        reinterpret_cast<uintptr_t>(ids) % size_t(id_bytes) || reinterpret_cast<uintptr_t>(status) % 8) {
        set_error("tre_lookup: table and output must be 16-byte aligned, ids and status to their size");
        return TRE_E_ARG;
    }
    const hipError_t e = launch_lookup(table, table_dtype, n_rows, row_elems, mx ? tile_rows : 1, ids, id_bytes, n_ids, scale,
                                       out, out_dtype, status, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "lookup");
}

size_t tre_lookup_grad_workspace_bytes(int64_t n_ids, int64_t n_rows, int64_t row_elems) {
    return rows_ok(n_ids, n_rows, row_elems) ? lookup_grad_ws_bytes(n_ids, n_rows, row_elems) : 0;
}

tre_status tre_lookup_grad(const void* grad, int32_t grad_dtype, const void* ids, int32_t id_bytes, int64_t n_ids,
                           float scale, void* table_grad, int32_t out_dtype, int64_t n_rows, int64_t row_elems,
                           int32_t accumulate, int64_t* status, void* ws, size_t ws_bytes, void* stream) {
    if ((grad_dtype != TRE_F32 && grad_dtype != TRE_BF16) || (out_dtype != TRE_F32 && out_dtype != TRE_BF16)) {
        set_error("tre_lookup_grad: grad_dtype and out_dtype must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    if (!rows_ok(n_ids, n_rows, row_elems)) {
        set_error("tre_lookup_grad: size out of range");
        return TRE_E_SHAPE;
    }
    if (!table_grad || !ws || (n_ids > 0 && (!grad || !ids)) || (id_bytes != 4 && id_bytes != 8)) {
        set_error("tre_lookup_grad: null array, or ids of neither 4 nor 8 bytes");
        return TRE_E_ARG;
    }
    if ((reinterpret_cast<uintptr_t>(grad) | reinterpret_cast<uintptr_t>(table_grad)) & 15 ||
        reinterpret_cast<uintptr_t>(ids) % size_t(id_bytes) || reinterpret_cast<uintptr_t>(status) % 8 ||
        reinterpret_cast<uintptr_t>(ws) % 256) {
        set_error("tre_lookup_grad: grad and table_grad must be 16-byte, ws 256-byte aligned, ids and status to their size");
        return TRE_E_ARG;
    }
    if (ws_bytes < lookup_grad_ws_bytes(n_ids, n_rows, row_elems)) {
        set_error("tre_lookup_grad: workspace smaller than tre_lookup_grad_workspace_bytes");
        return TRE_E_WORKSPACE;
    }
    const hipError_t e = launch_lookup_grad(grad, grad_dtype, ids, id_bytes, n_ids, scale, table_grad, out_dtype, n_rows,
                                            row_elems, accumulate != 0, status, static_cast<char*>(ws),
                                            reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "lookup_grad");
}

namespace {

// Offsets into scores stay within 62 bits.
bool scores_ok(const ScoreLayout& l) {
    if (l.n < 0 || l.n >= INT32_MAX || l.vocab < 1 || l.vocab > (int64_t(1) << 30) || l.cols < 1 || l.cols > l.vocab ||
        l.vocab % l.cols)
        return false;
    const int64_t most = int64_t(1) << 60;
    return l.row_stride >= 0 && l.tile_stride >= 0 && l.row_stride <= most / std::max<int64_t>(l.n, 1) &&
           l.tile_stride <= most / (l.vocab / l.cols);
}
// Whether no two elements of the layout share a place.
bool scores_apart(const ScoreLayout& l) {
    int64_t size[2] = {l.n, l.vocab / l.cols}, stride[2] = {l.row_stride, l.tile_stride};
    if (stride[0] > stride[1]) {
        std::swap(size[0], size[1]);
        std::swap(stride[0], stride[1]);
    }
    int64_t reach = l.cols;
    for (int d = 0; d < 2; d++) {
        if (size[d] <= 1) continue;
        if (stride[d] < reach) return false;
        reach += stride[d] * (size[d] - 1);
    }
    return true;
}
// Whether [begin, end) meets an element (of so many bytes) of a layout at `at` that scores_apart holds for: its runs of
// `cols` elements come one after the other, so the last one that begins before `end` reaches farthest.
bool meets(uintptr_t begin, uintptr_t end, uintptr_t at, const ScoreLayout& l, int bytes) {
    if (begin >= end || end <= at) return false;
    int64_t size[2] = {l.n, l.vocab / l.cols}, stride[2] = {l.row_stride * bytes, l.tile_stride * bytes};
    if (size[1] > 1 && (size[0] <= 1 || stride[1] > stride[0])) {
        std::swap(size[0], size[1]);
        std::swap(stride[0], stride[1]);
    }
    int64_t left = int64_t(end - 1 - at), run = 0;
    for (int d = 0; d < 2; d++) {
        if (size[d] <= 1) continue;
        const int64_t k = std::min(left / stride[d], size[d] - 1);
        left -= k * stride[d];
        run += k * stride[d];
    }
    return at + uintptr_t(run) + uintptr_t(l.cols * bytes) > begin;
}
// Whether the gradient `o` at `out` surely meets the scores `l` at `x`: where the scores lie without gaps, or both in the
// same strides.  (Layouts of other kinds that lie between each other are the caller's to keep apart.)
bool meet(const ScoreLayout& l, uintptr_t x, int x_bytes, const ScoreLayout& o, uintptr_t out, int out_bytes) {
    int64_t size[2] = {l.n, l.vocab / l.cols}, stride[2] = {l.row_stride * x_bytes, l.tile_stride * x_bytes};
    const int64_t out_stride[2] = {o.row_stride * out_bytes, o.tile_stride * out_bytes};
    bool same = true;
    for (int d = 0; d < 2; d++) same = same && (size[d] <= 1 || stride[d] == out_stride[d]);
    if (stride[0] > stride[1]) {
        std::swap(size[0], size[1]);
        std::swap(stride[0], stride[1]);
    }
    int64_t reach = l.cols * x_bytes;
    bool whole = true;
    for (int d = 0; d < 2; d++) {
        if (size[d] <= 1) continue;
        whole = whole && stride[d] <= reach;
        reach += stride[d] * (size[d] - 1);
    }
    if (whole) return meets(x, x + uintptr_t(reach), out, o, out_bytes);
    if (!same) return false;
    // in the same strides a run of the one meets some run of the other if it meets one of those that a whole number of
    // strides apart lie nearest: the difference of the places, less strides of the larger and then of the smaller
    const int64_t apart = int64_t(x - out), len_x = l.cols * x_bytes, len_out = l.cols * out_bytes;
    const int big = size[1] > 1 ? 1 : 0, small = 1 - big;
    for (int64_t i = -3; i <= 3; i++) {
        const int64_t a = size[big] > 1 ? apart / stride[big] + i : 0;
        if (std::abs(a) >= size[big]) continue;
        const int64_t rest = apart - a * (size[big] > 1 ? stride[big] : 0);
        for (int64_t j = -3; j <= 3; j++) {
            const int64_t b = size[small] > 1 ? rest / stride[small] + j : 0;
            if (std::abs(b) >= size[small]) continue;
            const int64_t d = rest - b * (size[small] > 1 ? stride[small] : 0);
            if (d < len_out && d + len_x > 0) return true;
        }
    }
    return false;
}
tre_status scores_args(const char* where, const ScoreLayout& l, const void* x, int32_t dtype, const void* ids, int32_t id_bytes,
                       float scale, const int64_t* status) {
    const std::string w(where);
    if (dtype != TRE_F32 && dtype != TRE_BF16) {
        set_error(w + ": scores must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    if (!scores_ok(l)) {
        set_error(w + ": size or stride out of range, or cols does not divide vocab");
        return TRE_E_SHAPE;
    }
    const float scale2 = scale * 1.4426950408889634f;
    if (!(scale2 > 0.f) || !std::isfinite(scale2)) {
        set_error(w + ": scale must be positive and finite");
        return TRE_E_ARG;
    }
    if (l.n > 0 && !x) {
        set_error(w + ": null scores");
        return TRE_E_ARG;
    }
    if (ids && id_bytes != 4 && id_bytes != 8) {
        set_error(w + ": ids of neither 4 nor 8 bytes");
        return TRE_E_ARG;
    }
    if (reinterpret_cast<uintptr_t>(x) % (dtype == TRE_BF16 ? 2 : 4) || (ids && reinterpret_cast<uintptr_t>(ids) % size_t(id_bytes)) ||
        reinterpret_cast<uintptr_t>(status) % 8) {
        set_error(w + ": scores, ids and status must be aligned to their size");
        return TRE_E_ARG;
    }
    return TRE_OK;
}
bool floats_aligned(std::initializer_list<const void*> ps) {
    for (const void* p : ps)
        if (reinterpret_cast<uintptr_t>(p) % 4) return false;
    return true;
}

}  // namespace

size_t tre_log_probs_workspace_bytes(int64_t n, int64_t vocab, int64_t cols, int32_t dtype, int32_t top) {
    const ScoreLayout l{n, vocab, cols, 0, 0};
    if (!scores_ok(l) || (dtype != TRE_F32 && dtype != TRE_BF16) || top < 0 || top > 64) return 0;
    return n == 0 ? 0 : log_probs_ws_bytes(l, dtype == TRE_BF16 ? 2 : 4, top);
}

tre_status tre_log_probs(const void* x, int32_t dtype, int64_t n, int64_t vocab, int64_t cols, int64_t row_stride,
                         int64_t tile_stride, const void* ids, int32_t id_bytes, float scale, float* log_prob, float* lse,
                         float* stats, float* entropy, int32_t top, int32_t* top_ids, float* top_log_probs, int64_t* status,
                         void* ws, size_t ws_bytes, void* stream) {
    const ScoreLayout l{n, vocab, cols, row_stride, tile_stride};
    const tre_status st = scores_args("tre_log_probs", l, x, dtype, ids, id_bytes, scale, status);
    if (st != TRE_OK) return st;
    if (top < 0 || top > 64 || top > vocab) {
        set_error("tre_log_probs: top must be 0 to 64, at most vocab");
        return TRE_E_SHAPE;
    }
    if (n == 0) return TRE_OK;
    if (!lse || !stats || (ids && !log_prob) || (!ids && log_prob) || (top > 0 && (!top_ids || !top_log_probs))) {
        set_error("tre_log_probs: null array, or log_prob without ids");
        return TRE_E_ARG;
    }
    if (!floats_aligned({log_prob, lse, stats, entropy, top_ids, top_log_probs})) {
        set_error("tre_log_probs: results must be aligned to their size");
        return TRE_E_ARG;
    }
    const size_t need = log_probs_ws_bytes(l, dtype == TRE_BF16 ? 2 : 4, top);
    if (need > 0) {
        if (!ws || reinterpret_cast<uintptr_t>(ws) % 256) {
            set_error("tre_log_probs: workspace null or not 256-byte aligned");
            return TRE_E_ARG;
        }
        if (ws_bytes < need) {
            set_error("tre_log_probs: workspace smaller than tre_log_probs_workspace_bytes");
            return TRE_E_WORKSPACE;
        }
    }
    const hipError_t e = launch_log_probs(l, x, dtype, ids, id_bytes, scale, top, log_prob, lse, stats, entropy, top_ids,
                                          top_log_probs, status, static_cast<char*>(ws), reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "log_probs");
}

tre_status tre_log_probs_grad(const void* x, int32_t dtype, int64_t n, int64_t vocab, int64_t cols, int64_t row_stride,
                              int64_t tile_stride, const float* stats, const void* ids, int32_t id_bytes, float scale,
                              const float* by_log_prob, const float* by_lse, const float* by_entropy, const float* entropy,
                              void* grad, int32_t out_dtype, int64_t out_row_stride, int64_t out_tile_stride, int64_t* status,
                              void* stream) {
    const ScoreLayout l{n, vocab, cols, row_stride, tile_stride}, o{n, vocab, cols, out_row_stride, out_tile_stride};
    if (out_dtype != TRE_F32 && out_dtype != TRE_BF16) {
        set_error("tre_log_probs_grad: out_dtype must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    const tre_status st = scores_args("tre_log_probs_grad", l, x, dtype, ids, id_bytes, scale, status);
    if (st != TRE_OK) return st;
    if (!scores_ok(o) || !scores_apart(o)) {
        set_error("tre_log_probs_grad: strides of the gradient out of range, or rows that overlap");
        return TRE_E_SHAPE;
    }
    if (n == 0) return TRE_OK;
    if ((!by_log_prob && !by_lse && !by_entropy) || (by_log_prob && !ids) || (by_entropy && !entropy)) {
        set_error("tre_log_probs_grad: no gradient given, by_log_prob without ids or by_entropy without entropy");
        return TRE_E_ARG;
    }
    if (!stats || !grad) {
        set_error("tre_log_probs_grad: null array");
        return TRE_E_ARG;
    }
    if (reinterpret_cast<uintptr_t>(grad) % (out_dtype == TRE_BF16 ? 2 : 4) ||
        !floats_aligned({stats, by_log_prob, by_lse, by_entropy, entropy})) {
        set_error("tre_log_probs_grad: arrays must be aligned to their elements");
        return TRE_E_ARG;
    }
    if (grad == x && (out_dtype != dtype || out_row_stride != row_stride || out_tile_stride != tile_stride)) {
        set_error("tre_log_probs_grad: in place the gradient has the scores' type and strides");
        return TRE_E_ARG;
    }
    const uintptr_t to = reinterpret_cast<uintptr_t>(grad);
    const int out_bytes = out_dtype == TRE_BF16 ? 2 : 4;
    auto meets_row = [&](const void* p, int64_t bytes) {  // (values of every token)
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        return p && meets(at, at + uintptr_t(n * bytes), to, o, out_bytes);
    };
    if ((grad != x && meet(l, reinterpret_cast<uintptr_t>(x), dtype == TRE_BF16 ? 2 : 4, o, to, out_bytes)) || meets_row(stats, 8) ||
        meets_row(ids, id_bytes) || meets_row(by_log_prob, 4) || meets_row(by_lse, 4) || meets_row(by_entropy, 4) ||
        (by_entropy && meets_row(entropy, 4)) ||
        (status && meets(reinterpret_cast<uintptr_t>(status), reinterpret_cast<uintptr_t>(status) + 8, to, o, out_bytes))) {
        set_error("tre_log_probs_grad: the gradient overlaps an input");
        return TRE_E_ARG;
    }
    const hipError_t e = launch_log_probs_grad(l, x, dtype, stats, ids, id_bytes, scale, by_log_prob, by_lse, by_entropy, entropy,
                                               grad, out_dtype, out_row_stride, out_tile_stride, status,
                                               reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "log_probs_grad");
}

namespace {

bool sizes_ok(int32_t n, const int64_t* sizes) {
    if (n < 0 || (n > 0 && !sizes)) return false;
    int64_t total = 0;
    for (int32_t i = 0; i < n; i++) {
        if (sizes[i] < 0 || sizes[i] > (int64_t(1) << 37)) return false;
        total += (sizes[i] + 31) / 32 * 32;
        if (total > (int64_t(1) << 37)) return false;
    }
    return true;
}
int elem_size(int32_t type) { return type == TRE_BF16 ? 2 : 4; }

// Arrays of fp32 or bf16 of these sizes.
tre_status arrays_args(const std::string& where, int32_t n, const void* const* arrays, const int32_t* types, const int64_t* sizes) {
    if (n > 0 && (!arrays || !types)) {
        set_error(where + ": null argument");
        return TRE_E_ARG;
    }
    for (int32_t i = 0; i < n; i++) {
        if (types[i] != TRE_F32 && types[i] != TRE_BF16) {
            set_error(where + ": arrays must be TRE_F32 or TRE_BF16");
            return TRE_E_DTYPE;
        }
        if (sizes[i] > 0 && (!arrays[i] || reinterpret_cast<uintptr_t>(arrays[i]) % size_t(elem_size(types[i])))) {
            set_error(where + ": array null or not aligned to its elements");
            return TRE_E_ARG;
        }
    }
    return TRE_OK;
}
struct Span {
    uintptr_t begin, end;
};

}  // namespace

size_t tre_grad_norm_workspace_bytes(int32_t n_tensors, const int64_t* sizes) {
    return sizes_ok(n_tensors, sizes) ? grad_norm_ws_bytes(n_tensors, sizes) : 0;
}

tre_status tre_grad_norm(int32_t n_tensors, const void* const* tensors, const int32_t* types, const int64_t* sizes, float max_norm,
                         float* out, void* ws, size_t ws_bytes, void* stream) {
    if (!sizes_ok(n_tensors, sizes)) {
        set_error("tre_grad_norm: sizes out of range");
        return TRE_E_SHAPE;
    }
    const tre_status st = arrays_args("tre_grad_norm", n_tensors, tensors, types, sizes);
    if (st != TRE_OK) return st;
    if (max_norm != max_norm || !out || reinterpret_cast<uintptr_t>(out) % 4 || !ws || reinterpret_cast<uintptr_t>(ws) % 256) {
        set_error("tre_grad_norm: max_norm is NaN, or out or workspace null or misaligned");
        return TRE_E_ARG;
    }
    if (ws_bytes < grad_norm_ws_bytes(n_tensors, sizes)) {
        set_error("tre_grad_norm: workspace smaller than tre_grad_norm_workspace_bytes");
        return TRE_E_WORKSPACE;
    }
    const hipError_t e = launch_grad_norm(n_tensors, tensors, types, sizes, max_norm, out, static_cast<char*>(ws),
                                          reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "grad_norm");
}

size_t tre_adamw_state_bytes(int32_t n_tensors, const int64_t* sizes, int32_t bits) {
    if (!sizes_ok(n_tensors, sizes) || (bits != 8 && bits != 32)) return 0;
    const size_t total = size_t(adamw_room(n_tensors, sizes));
    return bits == 32 ? 8 * total : 2 * total + total / 16;
}

tre_status tre_adamw(int32_t n_tensors, void* const* params, const int32_t* param_types, const void* const* grads,
                     const int32_t* grad_types, const int64_t* sizes, void* state, const tre_adamw_options* opt, void* stream) {
    if (!sizes_ok(n_tensors, sizes)) {
        set_error("tre_adamw: sizes out of range");
        return TRE_E_SHAPE;
    }
    tre_status st = arrays_args("tre_adamw (parameters)", n_tensors, params, param_types, sizes);
    if (st == TRE_OK) st = arrays_args("tre_adamw (gradients)", n_tensors, grads, grad_types, sizes);
    if (st != TRE_OK) return st;
    if (!opt) {
        set_error("tre_adamw: null options");
        return TRE_E_ARG;
    }
    auto rate = [](double x) { return x >= 0. && std::isfinite(float(x)); };
    auto beta = [](double x) { return x >= 0. && x < 1.; };
    // (a reciprocal of less than 2^-126 is infinite: a weight without moments would become 0 * inf)
    if ((opt->bits != 8 && opt->bits != 32) || !beta(opt->beta1) || !beta(opt->beta2) || !rate(opt->eps) || !(float(opt->eps) >= 0x1p-126f) ||
        !rate(opt->weight_decay) || (!opt->lr_dev && !rate(opt->lr)) || (!opt->step_dev && opt->step < 1) ||
        (!opt->grad_scale_dev && !std::isfinite(float(opt->grad_scale)))) {
        set_error("tre_adamw: an option is out of range");
        return TRE_E_ARG;
    }
    if (reinterpret_cast<uintptr_t>(opt->lr_dev) % 4 || reinterpret_cast<uintptr_t>(opt->grad_scale_dev) % 4 ||
        reinterpret_cast<uintptr_t>(opt->step_dev) % 8 || reinterpret_cast<uintptr_t>(state) % 16) {
        set_error("tre_adamw: device values must be aligned to their size, the state to 16 bytes");
        return TRE_E_ARG;
    }
    if (adamw_room(n_tensors, sizes) == 0) return TRE_OK;
    if (!state) {
        set_error("tre_adamw: null state");
        return TRE_E_ARG;
    }
    // a parameter twice, or two that overlap, would be stepped twice at once
    std::unique_ptr<Span[]> spans(new (std::nothrow) Span[size_t(n_tensors)]);
    if (!spans) {
        set_error("tre_adamw: out of host memory");
        return TRE_E_ARG;
    }
    auto span = [&](const void* at, int32_t type, int64_t size) {
        const uintptr_t b = reinterpret_cast<uintptr_t>(at);
        return Span{b, b + uintptr_t(size) * uintptr_t(elem_size(type))};
    };
    int32_t live = 0;
    for (int32_t i = 0; i < n_tensors; i++)
        if (sizes[i] > 0) spans[live++] = span(params[i], param_types[i], sizes[i]);
    std::sort(spans.get(), spans.get() + live, [](const Span& a, const Span& b) { return a.begin < b.begin; });
    bool apart = true;
    for (int32_t i = 1; i < live; i++) apart = apart && spans[i].begin >= spans[i - 1].end;
    for (int32_t i = 0; i < n_tensors && apart; i++) {
        if (sizes[i] == 0) continue;
        const Span g = span(grads[i], grad_types[i], sizes[i]);
        const Span* after = std::lower_bound(spans.get(), spans.get() + live, g, [](const Span& a, const Span& b) { return a.begin < b.begin; });
        apart = (after == spans.get() + live || after->begin >= g.end) && (after == spans.get() || after[-1].end <= g.begin);
    }
    if (!apart) {
        set_error("tre_adamw: parameters overlap, or a gradient one");
        return TRE_E_ARG;
    }
    const hipError_t e = launch_adamw(n_tensors, params, param_types, grads, grad_types, sizes, state, *opt,
                                      reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "adamw");
}

tre_status tre_adamw_moments(const void* state, int64_t total, void* m, void* v, int32_t dtype, void* stream) {
    if (dtype != TRE_F32 && dtype != TRE_BF16) {
        set_error("tre_adamw_moments: dtype must be TRE_F32 or TRE_BF16");
        return TRE_E_DTYPE;
    }
    if (total < 0 || total % 32 || total > (int64_t(1) << 43)) {
        set_error("tre_adamw_moments: total must be a multiple of 32");
        return TRE_E_SHAPE;
    }
    if (total == 0) return TRE_OK;
    if (!state || !m || !v || (reinterpret_cast<uintptr_t>(state) | reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(v)) & 15) {
        set_error("tre_adamw_moments: array null or not 16-byte aligned");
        return TRE_E_ARG;
    }
    const hipError_t e = launch_adamw_moments(state, total, m, v, dtype, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "adamw_moments");
}

size_t tre_stack_workspace_bytes(int64_t n) { return n < 0 ? 0 : stack_ws_bytes(n); }

tre_status tre_stack_rows(const int32_t* keys, int64_t n, const void* tiles, int64_t row_elems, int32_t group,
                          int32_t elem_bytes, int32_t* out_keys, void* out_tiles, int64_t out_cap, int64_t* n_out,
                          void* ws, size_t ws_bytes, void* stream) {
    if (n < 0 || row_elems < 1 || group < 1 || (elem_bytes != 2 && elem_bytes != 4) || !n_out || !ws ||
        (n > 0 && (!keys || !tiles))) {
        set_error("tre_stack_rows: bad argument");
        return TRE_E_ARG;
    }
    if (ws_bytes < stack_ws_bytes(n)) return TRE_E_WORKSPACE;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    char* w = reinterpret_cast<char*>(ws);
    *n_out = 0;
    if (n == 0) return TRE_OK;
    hipError_t e = launch_stack(keys, n, tiles, row_elems, group, elem_bytes, nullptr, nullptr, 0, w, s, 0);
    if (e != hipSuccess) return dev_fail(e, "stack count");
    int64_t cnt = 0;
    const size_t cnt_off = (sizeof(int32_t) * size_t(n + 1) + 255) / 256 * 256;
    if ((e = hipMemcpyAsync(&cnt, w + cnt_off, sizeof(cnt), hipMemcpyDeviceToHost, s)) != hipSuccess)
        return dev_fail(e, "stack read-back");
    if ((e = hipStreamSynchronize(s)) != hipSuccess) return dev_fail(e, "stack sync");
    *n_out = cnt;
    if (cnt > out_cap || !out_keys || !out_tiles) {
        set_error("tre_stack_rows: output capacity below the number of stacked keys");
        return TRE_E_CAPACITY;
    }
    e = launch_stack(keys, n, tiles, row_elems, group, elem_bytes, out_keys, out_tiles, cnt, w, s, 1);
    return e == hipSuccess ? TRE_OK : dev_fail(e, "stack");
}

tre_status tre_tiles_from_entries(const int64_t* slot, const int64_t* offset, const void* value, int64_t n_entries,
                                  int32_t elem_bytes, void* tiles, int64_t n_tiles, int64_t tile_elems,
                                  void* stream) {
    if (n_entries < 0 || n_tiles < 0 || tile_elems < 1 || (elem_bytes != 2 && elem_bytes != 4) ||
        (n_entries > 0 && (!slot || !offset || !value)) || (n_tiles > 0 && !tiles)) {
        set_error("tre_tiles_from_entries: bad argument");
        return TRE_E_ARG;
    }
    hipError_t e = launch_tiles_from_entries(slot, offset, value, n_entries, elem_bytes, tiles, n_tiles, tile_elems,
                                             reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? TRE_OK : dev_fail(e, "tiles_from_entries");
}

}  // extern "C"
