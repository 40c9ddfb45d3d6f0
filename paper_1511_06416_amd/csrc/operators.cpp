// C ABI of the imputer's operators (declared in include/same.h): cross
// attention over ragged segments with its gradients, and dropout.  Argument
// checks, the work lists of a plan, its workspace and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <exception>
#include <limits>
#include <mutex>
#include <new>
#include <string>
#include <utility>
#include <vector>

#include "../../include/same.h"
#include "checks.hpp"
#include "cross.hpp"

namespace {

using same::align_up;
using same::aligned;
using same::check_apart;
using same::check_hip;
using same::CrossItem;
using same::CrossJoin;
using same::CrossSmallItem;
using same::extent;
using same::Extent;
using same::kAlign;
using same::overlap;
using same::record_error;

constexpr int64_t kMaxAxis = (int64_t)1 << 30;  // rows or keys of one segment
constexpr int64_t kMaxSegs = (int64_t)1 << 31;
constexpr int64_t kMaxBlocks = (int64_t)1 << 30;  // of a pass, before its last tiles are cut


// The work list of one pass on the host.
struct PassPlan {
    std::vector<CrossItem> items;
    std::vector<CrossJoin> joins;
    int32_t own_waves = 1, n_slots = 0;
};

struct DeviceLists {
    int device = -1;
    char *base = nullptr;
    CrossItem *items[3] = {nullptr, nullptr, nullptr};
    CrossJoin *joins[3] = {nullptr, nullptr, nullptr};
    CrossSmallItem *small = nullptr;
};

}  // namespace

struct same_cross_plan {
    int32_t heads_q = 0, heads_kv = 0, dim = 0, dtype = 0;
    int64_t n_q = 0, n_k = 0;  // tokens
    // Small segments: items of several; otherwise a work list for each PassKind.
    std::vector<CrossSmallItem> small;
    PassPlan pass[3];
    // workspace: parts and their statistics (forward); delta, then parts (gradient)
    size_t ws_ml = 0, ws_forward = 0, ws_part = 0, ws_backward = 0;
    std::vector<DeviceLists> dev;
    std::mutex mu;
};

namespace {

enum PassKind { kForward, kGradQuery, kGradKey };

constexpr int64_t kSmall = 32;  // query rows and keys that a wave takes

// Neighbouring segments into items of at most kSmall rows and keys; false if a
// segment has more.
bool build_small(std::vector<CrossSmallItem> &items, const std::vector<int64_t> &q_ptr,
                 const std::vector<int64_t> &k_ptr, int32_t group) {
    const int64_t n = (int64_t)q_ptr.size() - 1;
    for (int64_t s = 0; s < n; ++s)
        if ((q_ptr[s + 1] - q_ptr[s]) * group > kSmall || k_ptr[s + 1] - k_ptr[s] > kSmall) return false;
    CrossSmallItem it;
    auto start = [&](int64_t s) {
        std::memset((void *)&it, 0, sizeof(it));
        it.q0 = q_ptr[s];
        it.k0 = k_ptr[s];
    };
    auto flush = [&]() {
        if (it.n_rows || it.n_keys) items.push_back(it);
    };
    start(0);
    for (int64_t s = 0; s < n; ++s) {
        const int64_t rows = (q_ptr[s + 1] - q_ptr[s]) * group, keys = k_ptr[s + 1] - k_ptr[s];
        if (it.n_rows + rows > kSmall || it.n_keys + keys > kSmall) {
            flush();
            start(s);
        }
        for (int64_t r = 0; r < rows; ++r)
            it.range[it.n_rows + r] = (uint16_t)(it.n_keys | (it.n_keys + keys) << 8);
        it.n_rows += (int32_t)rows;
        it.n_keys += (int32_t)keys;
    }
    if (n) flush();
    return true;
}

// Waves of a block that own tiles of 32 and waves that share the other axis,
// and the time of an entry of that axis, that of 4 x 1 being one.
struct Geometry {
    int32_t own_waves, cut_waves;
    double entry;
};

// Waves of a pass's kernel that the estimate gives a SIMD.  One number for
// kernels that differ: by their registers, gradients up to 64 wide reach 2 to 4,
// the forward pass 3 in 1 x 4 at 64 wide and in 8 x 1 at 96, 5 in 4 x 1 at 32, and
// dK and dV at 128 wide 1 with dropout, which a plan does not know of.  The
// constants below were set with these numbers.
int waves_per_simd(PassKind kind, int32_t dim, const Geometry &g) {
    if (kind == kForward) return dim <= 64 ? 4 : 2;
    return dim > 64 && g.cut_waves > 1 ? 1 : 2;
}

// Tiles [0, whole) are left whole, the others cut into parts of `part` entries.
struct Cut {
    double cost = 0.0;
    int64_t whole = 0, part = kMaxAxis;
};

// In entries of a full chip (about 0.04 us): what a block costs before it
// begins, a join with its launch, and an element of a part written and read;
// set by the times of some 120 drawn sets of segments, whose mean is flat
// around them.  Parts are multiples of kPart.
constexpr double kBlock = 160.0, kJoin = 96.0, kElement = 1.0 / 32000;
constexpr int64_t kPart = 128;
constexpr double kUnits = 256.0;  // compute units

// How long the tiles (owners and other axis of every segment, longest axis
// first) take with a geometry of which the chip holds `room` blocks.  Whole
// rounds of blocks are left whole; the tiles of the last, partly filled round
// are cut into parts that fill it.  With many rounds the last one does not
// matter.  A block takes `alone` of its time where it has a compute unit to
// itself; a part holds `elements` of a row.
Cut plan_cut(const Geometry &g, const std::vector<std::pair<int64_t, int64_t>> &segs, int32_t heads_kv, double room,
             double alone, double elements) {
    const int64_t tile = 32 * g.own_waves, step = 32 * g.cut_waves;
    auto time_of = [&](int64_t cut) { return kBlock + g.entry * (double)((cut + step - 1) / step * step); };
    Cut c;
    int64_t tiles = 0;
    double total = 0.0;
    for (const auto &s : segs) {
        const int64_t t = (s.first + tile - 1) / tile;
        tiles += t;
        total += (double)t * time_of(s.second) * heads_kv;
    }
    c.whole = tiles;
    c.cost = total / room;
    if ((double)tiles * heads_kv > 16.0 * room) return c;
    c.whole = (int64_t)(std::floor((double)tiles * heads_kv / room) * room / heads_kv);
    struct Tail {
        int64_t tiles, owners, axis;
    };
    std::vector<Tail> tail;  // tiles of one length together
    int64_t at = 0, longest = 0;
    double before = 0.0;
    for (const auto &s : segs) {
        const int64_t t = (s.first + tile - 1) / tile, cut_tiles = std::max<int64_t>(0, std::min(t, at + t - c.whole));
        before += (double)(t - cut_tiles) * time_of(s.second) * heads_kv;
        at += t;
        if (!cut_tiles) continue;
        if (tail.empty() || tail.back().axis != s.second) tail.push_back({0, 0, s.second});
        tail.back().tiles += cut_tiles;
        tail.back().owners += s.first - (t - cut_tiles) * tile;
        longest = std::max(longest, s.second);
    }
    double best = 0.0;
    for (int64_t k = 1; k <= same::kMaxParts && !tail.empty(); ++k) {
        const int64_t p = k == 1 ? longest : ((longest + k - 1) / k + kPart - 1) / kPart * kPart;
        double blocks = 0.0, work = 0.0, split = 0.0;
        for (const Tail &t : tail) {
            const double parts = p ? (double)std::max<int64_t>(1, (t.axis + p - 1) / p) : 1.0;
            blocks += parts * (double)t.tiles * heads_kv;
            work += (parts * kBlock + g.entry * (double)t.axis) * (double)t.tiles * heads_kv;
            if (parts > 1) split += parts * (double)t.owners * heads_kv;
        }
        const double one = time_of(std::min(p, longest));
        const double full = std::ceil(blocks / kUnits) * kUnits / room;  // of the fullest compute unit
        const double cost = (full <= 1.0 ? one * (alone + (1.0 - alone) * full) : work / room + 0.5 * one) +
                            (split ? kJoin + split * elements * kElement : 0.0);
        if (k == 1 || cost < best) {
            best = cost;
            c.part = k == 1 ? kMaxAxis : p;
        }
        if (p <= kPart) break;
    }
    c.cost = before / room + best;
    return c;
}

// Splits the owners of every segment into tiles and, where the tiles alone
// leave compute units idle, the other axis into parts.
int build_pass(PassPlan &pp, const std::vector<int64_t> &q_ptr, const std::vector<int64_t> &k_ptr, int32_t group,
               int32_t heads_kv, int32_t dim, PassKind kind) {
    const int64_t n = (int64_t)q_ptr.size() - 1;
    const bool own_keys = kind == kGradKey;
    auto own_of = [&](int64_t s) { return own_keys ? k_ptr[s + 1] - k_ptr[s] : (q_ptr[s + 1] - q_ptr[s]) * group; };
    auto cut_of = [&](int64_t s) { return own_keys ? (q_ptr[s + 1] - q_ptr[s]) * group : k_ptr[s + 1] - k_ptr[s]; };
    std::vector<int64_t> order;  // longest first; the tiles of a segment stay together
    for (int64_t s = 0; s < n; ++s)
        if (own_of(s) > 0) order.push_back(s);
    if (order.empty()) return SAME_OK;
    std::stable_sort(order.begin(), order.end(), [&](int64_t a, int64_t b) { return cut_of(a) > cut_of(b); });
    std::vector<std::pair<int64_t, int64_t>> segs;
    for (int64_t s : order) segs.push_back({own_of(s), cut_of(s)});
    // The geometries a pass is compiled for.  Forward above 64 wide, 8 x 1: a
    // key read from LDS serves more waves (2 x 4,099 rows on 7,951 keys, 16
    // heads on 4 of 128, 547 against 584 us).  Gradients up to 64 wide, 2 x 1,
    // for segments that leave much of a tile of 128 empty.  1 x 4, few owners or
    // short tiles: one query over keys, or owners that 4 x 1 would have to split
    // and join.
    std::vector<Geometry> shapes = {{4, 1, 1.0}, {1, 4, 0.4}};
    if (kind == kForward && dim > 64) shapes.push_back({8, 1, 0.93});
    if (kind != kForward && dim <= 64) shapes.push_back({2, 1, 1.1});
    Cut cut;
    const Geometry *shape = nullptr;
    for (const Geometry &g : shapes) {
        // blocks the chip holds
        const int waves = waves_per_simd(kind, dim, g);
        const double room = 4 * kUnits * waves / (g.own_waves * g.cut_waves);
        // a gradient's entry takes longer than the forward's, its parts' elements less of it
        const Cut c = plan_cut(g, segs, heads_kv, room, waves > 2 ? 0.35 : waves == 1 ? 1.0 : kind == kForward ? 0.45 : 0.55,
                               (kind == kForward ? 1.0 : kind == kGradQuery ? 0.4 : 0.8) * dim);
        if (!shape || c.cost < cut.cost) {
            cut = c;
            shape = &g;
        }
    }
    pp.own_waves = shape->own_waves;
    const int64_t tile = 32 * pp.own_waves;
    // tiles, of which only a few are cut (see plan_cut)
    double tiles = 0.0;
    for (const auto &s : segs) tiles += (double)((s.first + tile - 1) / tile);
    if (tiles * heads_kv > (double)kMaxBlocks) return record_error(SAME_ESIZE, "the plan has more than 2^30 blocks");
    int64_t at = 0;
    for (int64_t s : order) {
        const int64_t own = own_of(s), len = cut_of(s);
        for (int64_t o = 0; o < own; o += tile, ++at) {
            const int64_t parts = at < cut.whole ? 1 : std::max<int64_t>(1, (len + cut.part - 1) / cut.part);
            const int64_t step = parts == 1 ? std::max<int64_t>(len, 1)
                                            : ((len + parts - 1) / parts + kPart - 1) / kPart * kPart;
            CrossItem it;
            it.q0 = q_ptr[s];
            it.k0 = k_ptr[s];
            it.own0 = (int32_t)o;
            it.n_own = (int32_t)std::min(tile, own - o);
            it.slot = -1;
            it.pad = 0;
            const int32_t first = pp.n_slots;
            int64_t b = 0;
            do {
                it.beg = (int32_t)b;
                it.end = (int32_t)std::min(len, b + step);
                if (step < len) it.slot = pp.n_slots++;
                pp.items.push_back(it);
                b += step;
            } while (b < len);
            if (step < len) pp.joins.push_back(CrossJoin{it.q0, it.k0, it.own0, it.n_own, first, pp.n_slots - first});
        }
    }
    return SAME_OK;
}

template <typename T>
size_t bytes_of(const std::vector<T> &v) {
    return align_up(v.size() * sizeof(T));
}

// The plan's lists on the current device, uploaded on first use (synchronous).
int lists_for_current_device(same_cross_plan *pl, DeviceLists *out) {
    int device = -1;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return record_error(SAME_EHIP, std::string("hipGetDevice: ") + hipGetErrorString(e));
    std::lock_guard<std::mutex> lock(pl->mu);
    if ((int)pl->dev.size() <= device) pl->dev.resize(device + 1);
    DeviceLists &d = pl->dev[device];
    if (d.device != device) {
        size_t off[7] = {0};
        for (int k = 0; k < 3; ++k) {
            off[2 * k + 1] = off[2 * k] + bytes_of(pl->pass[k].items);
            off[2 * k + 2] = off[2 * k + 1] + bytes_of(pl->pass[k].joins);
        }
        std::vector<char> host(off[6] + std::max<size_t>(bytes_of(pl->small), 1));
        auto put = [&](size_t o, const void *src, size_t bytes) {
            if (bytes) std::memcpy(host.data() + o, src, bytes);
        };
        for (int k = 0; k < 3; ++k) {
            put(off[2 * k], pl->pass[k].items.data(), pl->pass[k].items.size() * sizeof(CrossItem));
            put(off[2 * k + 1], pl->pass[k].joins.data(), pl->pass[k].joins.size() * sizeof(CrossJoin));
        }
        put(off[6], pl->small.data(), pl->small.size() * sizeof(CrossSmallItem));
        char *base = nullptr;
        e = hipMalloc((void **)&base, host.size());
        if (e == hipSuccess) e = hipMemcpy(base, host.data(), host.size(), hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            if (base) (void)hipFree(base);
            return record_error(e == hipErrorOutOfMemory ? SAME_ENOMEM : SAME_EHIP,
                                std::string("uploading the plan's lists: ") + hipGetErrorString(e));
        }
        d.base = base;
        for (int k = 0; k < 3; ++k) {
            d.items[k] = (CrossItem *)(base + off[2 * k]);
            d.joins[k] = (CrossJoin *)(base + off[2 * k + 1]);
        }
        d.small = (CrossSmallItem *)(base + off[6]);
        d.device = device;
    }
    *out = d;
    return SAME_OK;
}

// A strided input [tokens][heads][dim] of 16-bit elements.
int check_input(const char *name, const void *p, int64_t tokens, int64_t heads, int64_t dim, int64_t row, int64_t head,
                Extent *ext) {
    if (tokens == 0) return SAME_OK;
    if (!p) return record_error(SAME_EINVAL, std::string(name) + " is null");
    if (row < 0 || head < 0) return record_error(SAME_EINVAL, std::string(name) + ": strides must not be negative");
    if (!aligned(p, 16) || row % 8 != 0 || head % 8 != 0)
        return record_error(SAME_EALIGN,
                            std::string(name) + " must be 16-byte aligned, with strides that are multiples of 8");
    if (tokens > 1 && row >= (int64_t)1 << 25)
        return record_error(SAME_ESIZE, std::string(name) + ": a token's stride must stay below 2^25 elements");
    const double last = (double)(tokens - 1) * (double)row + (double)(heads - 1) * (double)head + (double)dim;
    if (last >= 4.6e18) return record_error(SAME_ESIZE, std::string(name) + ": strides pass 2^62 elements");
    *ext = extent(p, 2 * ((tokens - 1) * row + (heads - 1) * head + dim));
    return SAME_OK;
}

int check_output(const char *name, const void *p, int64_t elements, int64_t size, Extent *ext) {
    if (elements == 0) return SAME_OK;
    if (!p) return record_error(SAME_EINVAL, std::string(name) + " is null");
    if (!aligned(p, 16)) return record_error(SAME_EALIGN, std::string(name) + " must be 16-byte aligned");
    *ext = extent(p, elements * size);
    return SAME_OK;
}

// drop as a number of `steps`: what lies below it is dropped.
int drop_threshold(double drop, uint32_t steps, uint32_t *below) {
    *below = 0;
    if (!(drop >= 0.0 && drop < 1.0)) return record_error(SAME_EINVAL, "drop must lie in [0, 1)");
    if (drop == 0.0) return SAME_OK;
    *below = (uint32_t)std::nearbyint(drop * steps);
    if (*below == 0 || *below >= steps)
        return record_error(SAME_EINVAL, "drop must be 0 or round to 1 .. " + std::to_string(steps - 1) +
                                             " parts of " + std::to_string(steps));
    return SAME_OK;
}

// What both passes share: plan, inputs, scale, dropout, workspace.
struct Call {
    same::CrossParams p;
    DeviceLists d;
    std::vector<Extent> reads;
};

int prepare_call(same_cross_plan *pl, Call &c, const void *q, int64_t q_row, int64_t q_head, const void *k,
                 int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head, const uint8_t *key_mask,
                 double scale, double drop, uint64_t seed, uint32_t call_id, void *workspace, size_t need) {
    // what the kernels multiply scores by, among them the -inf of a hidden key
    const float per_bit = (float)scale * 1.4426950408889634f;
    if (!((float)scale >= std::numeric_limits<float>::min()) || !std::isfinite(per_bit))
        return record_error(SAME_EINVAL, "scale must be positive and finite, and so must scale * log2(e) in 32 bits");
    Extent e;
    int rc = check_input("q", q, pl->n_q, pl->heads_q, pl->dim, q_row, q_head, &e);
    if (rc) return rc;
    c.reads.push_back(e);
    e = Extent();
    rc = check_input("k", k, pl->n_k, pl->heads_kv, pl->dim, k_row, k_head, &e);
    if (rc) return rc;
    c.reads.push_back(e);
    e = Extent();
    rc = check_input("v", v, pl->n_k, pl->heads_kv, pl->dim, v_row, v_head, &e);
    if (rc) return rc;
    c.reads.push_back(e);
    if (key_mask) c.reads.push_back(extent(key_mask, pl->n_k));
    std::memset((void *)&c.p, 0, sizeof(c.p));
    rc = drop_threshold(drop, 256, &c.p.drop_below);
    if (rc) return rc;
    if (need && !workspace) return record_error(SAME_EINVAL, "workspace is null");
    if (!aligned(workspace, kAlign)) return record_error(SAME_EALIGN, "workspace must be 256-byte aligned");
    c.p.q = {q, q_row, q_head};
    c.p.k = {k, k_row, k_head};
    c.p.v = {v, v_row, v_head};
    c.p.key_mask = key_mask;
    c.p.heads_q = pl->heads_q;
    c.p.heads_kv = pl->heads_kv;
    c.p.group = pl->heads_q / pl->heads_kv;
    c.p.dim = pl->dim;
    c.p.scale = (float)scale;
    c.p.keep_gain = 256.0f / (256.0f - (float)c.p.drop_below);
    c.p.keep_part = (256.0f - (float)c.p.drop_below) / 256.0f;
    c.p.seed_lo = (uint32_t)seed;
    c.p.seed_hi = (uint32_t)(seed >> 32);
    c.p.call_id = call_id;
    return SAME_OK;
}

same::CrossPass pass_of(const same_cross_plan *pl, const DeviceLists &d, PassKind kind) {
    const PassPlan &pp = pl->pass[kind];
    same::CrossPass w;
    w.items = d.items[kind];
    w.joins = d.joins[kind];
    w.n_items = (int32_t)pp.items.size();
    w.n_joins = (int32_t)pp.joins.size();
    w.own_waves = pp.own_waves;
    return w;
}

int check_ptr(const char *name, int64_t n_segs, const int64_t *ptr, std::vector<int64_t> &out) {
    if (!ptr) return record_error(SAME_EINVAL, std::string(name) + " is null");
    out.assign(ptr, ptr + n_segs + 1);
    if (out[0] != 0) return record_error(SAME_EINVAL, std::string(name) + "[0] must be 0");
    for (int64_t s = 0; s < n_segs; ++s) {
        if (out[s + 1] < out[s]) return record_error(SAME_EINVAL, std::string(name) + " must not decrease");
        if (out[s + 1] - out[s] >= kMaxAxis)
            return record_error(SAME_ESIZE, std::string(name) + ": a segment has 2^30 entries or more");
    }
    return SAME_OK;
}

}  // namespace

extern "C" {

int same_cross_create(int64_t n_segs, const int64_t *q_ptr, const int64_t *k_ptr, int32_t heads_q, int32_t heads_kv,
                      int32_t head_dim, int32_t dtype, same_cross_plan **out) {
    if (!out) return record_error(SAME_EINVAL, "out is null");
    *out = nullptr;
    if (n_segs < 0) return record_error(SAME_EINVAL, "n_segs must not be negative");
    if (n_segs >= kMaxSegs) return record_error(SAME_ESIZE, "n_segs must stay below 2^31");
    if (heads_q < 1 || heads_kv < 1 || heads_q % heads_kv != 0)
        return record_error(SAME_EINVAL, "heads_q must be a positive multiple of heads_kv");
    if (heads_q > 65536) return record_error(SAME_ESIZE, "heads_q must be at most 65536");
    if (head_dim < 8 || head_dim > 128 || head_dim % 8 != 0)
        return record_error(SAME_EINVAL, "head_dim must be a multiple of 8 in [8, 128]");
    if (dtype != SAME_F16 && dtype != SAME_BF16) return record_error(SAME_EINVAL, "dtype must be SAME_F16 or SAME_BF16");
    same_cross_plan *pl = new (std::nothrow) same_cross_plan();
    if (!pl) return record_error(SAME_ENOMEM, "out of host memory");
    int rc;
    try {
        std::vector<int64_t> qp, kp;
        rc = check_ptr("q_ptr", n_segs, q_ptr, qp);
        if (!rc) rc = check_ptr("k_ptr", n_segs, k_ptr, kp);
        const int32_t group = heads_q / heads_kv;
        for (int64_t s = 0; !rc && s < n_segs; ++s)
            if ((qp[s + 1] - qp[s]) * group >= kMaxAxis)
                rc = record_error(SAME_ESIZE, "a segment has 2^30 query rows of one key head or more");
        if (!rc && !build_small(pl->small, qp, kp, group))
            for (int k = 0; !rc && k < 3; ++k) rc = build_pass(pl->pass[k], qp, kp, group, heads_kv, head_dim, (PassKind)k);
        if (!rc && (int64_t)pl->small.size() * heads_kv > kMaxBlocks)
            rc = record_error(SAME_ESIZE, "the plan has more than 2^30 blocks");
        if (!rc) {
            pl->heads_q = heads_q;
            pl->heads_kv = heads_kv;
            pl->dim = head_dim;
            pl->dtype = dtype;
            pl->n_q = qp[n_segs];
            pl->n_k = kp[n_segs];
            auto owners = [&](const PassPlan &pp) {
                return (size_t)pp.n_slots * (size_t)heads_kv * 32 * (size_t)pp.own_waves;
            };
            const size_t row = (size_t)head_dim * sizeof(float);
            const int64_t delta = pl->small.empty() ? pl->n_q : 0;  // small segments form theirs on the way
            pl->ws_ml = align_up(owners(pl->pass[kForward]) * row);
            pl->ws_forward = pl->ws_ml + align_up(owners(pl->pass[kForward]) * 2 * sizeof(float));
            pl->ws_part = align_up((size_t)delta * (size_t)heads_q * sizeof(float));
            pl->ws_backward = pl->ws_part + align_up(std::max(owners(pl->pass[kGradQuery]), 2 * owners(pl->pass[kGradKey])) * row);
        }
    } catch (const std::bad_alloc &) {
        rc = record_error(SAME_ENOMEM, "out of host memory");
    } catch (const std::exception &e) {  // nothing may leave a C entry
        rc = record_error(SAME_ESIZE, e.what());
    }
    if (rc) {
        delete pl;
        return rc;
    }
    *out = pl;
    return SAME_OK;
}

void same_cross_destroy(same_cross_plan *pl) {
    if (!pl) return;
    int cur = -1;
    for (DeviceLists &d : pl->dev)
        if (d.device >= 0) {
            if (cur < 0) (void)hipGetDevice(&cur);
            (void)hipSetDevice(d.device);
            (void)hipFree(d.base);
        }
    if (cur >= 0) (void)hipSetDevice(cur);
    delete pl;
}

int same_cross_workspace_size(const same_cross_plan *pl, int32_t backward, size_t *bytes) {
    if (!pl || !bytes) return record_error(SAME_EINVAL, "plan and bytes must be non-null");
    *bytes = backward ? pl->ws_backward : pl->ws_forward;
    return SAME_OK;
}

int same_cross_attention(same_cross_plan *pl, const void *q, int64_t q_row, int64_t q_head, const void *k,
                         int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                         const uint8_t *key_mask, double scale, double drop, uint64_t seed, uint32_t call_id,
                         void *out, float *lse, void *workspace, void *stream) {
    if (!pl) return record_error(SAME_EINVAL, "plan is null");
    try {
        Call c;
        int rc = prepare_call(pl, c, q, q_row, q_head, k, k_row, k_head, v, v_row, v_head, key_mask, scale, drop, seed,
                              call_id, workspace, pl->ws_forward);
        if (rc) return rc;
        const int64_t rows = pl->n_q * pl->heads_q;
        std::vector<Extent> writes(3);
        rc = check_output("out", out, rows * pl->dim, 2, &writes[0]);
        if (rc) return rc;
        if (lse) {
            if (!aligned(lse, 4)) return record_error(SAME_EALIGN, "lse must be 4-byte aligned");
            writes[1] = extent(lse, rows * 4);
        }
        writes[2] = extent(workspace, (int64_t)pl->ws_forward);
        rc = check_apart(writes, c.reads);
        if (rc) return rc;
        if (rows == 0) return SAME_OK;
        rc = lists_for_current_device(pl, &c.d);
        if (rc) return rc;
        c.p.out = out;
        c.p.lse = lse;
        c.p.part = (float *)workspace;
        c.p.part_ml = (float *)((char *)workspace + pl->ws_ml);
        c.p.small = c.d.small;
        c.p.n_items = (int32_t)pl->small.size();
        if (c.p.n_items)
            return check_hip(same::launch_cross_small(c.p, false, pl->dtype, (hipStream_t)stream),
                             "cross attention launch");
        return check_hip(same::launch_cross_forward(c.p, pass_of(pl, c.d, kForward), pl->dtype,
                                                    (hipStream_t)stream),
                         "cross attention launch");
    } catch (const std::bad_alloc &) {
        return record_error(SAME_ENOMEM, "out of host memory");
    } catch (const std::exception &e) {  // the plan's lock
        return record_error(SAME_EHIP, e.what());
    }
}

int same_cross_attention_backward(same_cross_plan *pl, const void *q, int64_t q_row, int64_t q_head, const void *k,
                                  int64_t k_row, int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                                  const uint8_t *key_mask, double scale, double drop, uint64_t seed, uint32_t call_id,
                                  const void *out, const float *lse, const void *dout, int64_t dout_row,
                                  int64_t dout_head, void *dq, void *dk, void *dv, void *workspace, void *stream) {
    if (!pl) return record_error(SAME_EINVAL, "plan is null");
    try {
        Call c;
        int rc = prepare_call(pl, c, q, q_row, q_head, k, k_row, k_head, v, v_row, v_head, key_mask, scale, drop, seed,
                              call_id, workspace, pl->ws_backward);
        if (rc) return rc;
        const int64_t rows = pl->n_q * pl->heads_q, keys = pl->n_k * pl->heads_kv;
        Extent e;
        rc = check_input("dout", dout, pl->n_q, pl->heads_q, pl->dim, dout_row, dout_head, &e);
        if (rc) return rc;
        c.reads.push_back(e);
        e = Extent();
        rc = check_output("out", out, rows * pl->dim, 2, &e);
        if (rc) return rc;
        c.reads.push_back(e);
        if (rows) {
            if (!lse) return record_error(SAME_EINVAL, "lse is null");
            if (!aligned(lse, 4)) return record_error(SAME_EALIGN, "lse must be 4-byte aligned");
            c.reads.push_back(extent(lse, rows * 4));
        }
        std::vector<Extent> writes(4);
        rc = check_output("dq", dq, rows * pl->dim, 2, &writes[0]);
        if (!rc) rc = check_output("dk", dk, keys * pl->dim, 2, &writes[1]);
        if (!rc) rc = check_output("dv", dv, keys * pl->dim, 2, &writes[2]);
        if (rc) return rc;
        writes[3] = extent(workspace, (int64_t)pl->ws_backward);
        rc = check_apart(writes, c.reads);
        if (rc) return rc;
        if (rows == 0 && keys == 0) return SAME_OK;
        rc = lists_for_current_device(pl, &c.d);
        if (rc) return rc;
        c.p.delta = (float *)workspace;
        c.p.part = (float *)((char *)workspace + pl->ws_part);
        c.p.dout = {dout, dout_row, dout_head};
        c.p.out_in = out;
        c.p.lse = (float *)lse;
        c.p.dq = dq;
        c.p.dk = dk;
        c.p.dv = dv;
        hipStream_t s = (hipStream_t)stream;
        c.p.small = c.d.small;
        c.p.n_items = (int32_t)pl->small.size();
        if (c.p.n_items)
            return check_hip(same::launch_cross_small(c.p, true, pl->dtype, s), "gradient launch");
        // dQ first: it leaves delta for the other pass
        rc = check_hip(same::launch_cross_dq(c.p, pass_of(pl, c.d, kGradQuery), pl->dtype, s),
                       "query gradient launch");
        if (rc) return rc;
        return check_hip(same::launch_cross_dkv(c.p, pass_of(pl, c.d, kGradKey), pl->dtype, s),
                         "key gradient launch");
    } catch (const std::bad_alloc &) {
        return record_error(SAME_ENOMEM, "out of host memory");
    } catch (const std::exception &e) {  // the plan's lock
        return record_error(SAME_EHIP, e.what());
    }
}

int same_dropout(int32_t dtype, const void *x, int64_t x_row, const void *residual, int64_t residual_row, int64_t rows,
                 int64_t cols, double drop, uint64_t seed, uint32_t call_id, void *y, int64_t y_row, void *stream) {
    if (dtype != SAME_F32 && dtype != SAME_F16 && dtype != SAME_BF16)
        return record_error(SAME_EINVAL, "dtype must be SAME_F32, SAME_F16 or SAME_BF16");
    if (rows < 0 || cols < 0) return record_error(SAME_EINVAL, "rows and cols must not be negative");
    same::DropoutParams p;
    int rc = drop_threshold(drop, 65536, &p.drop_below);
    if (rc) return rc;
    if (rows == 0 || cols == 0) return SAME_OK;
    if (!x || !y) return record_error(SAME_EINVAL, "x and y must be non-null");
    if (x_row < 0 || (residual && residual_row < 0))
        return record_error(SAME_EINVAL, "row strides must not be negative");
    if (rows > 1 && y_row < cols) return record_error(SAME_EINVAL, "y_row must be at least cols");
    const int64_t size = dtype == SAME_F32 ? 4 : 2;
    if (!aligned(x, size) || !aligned(y, size) || !aligned(residual, size))
        return record_error(SAME_EALIGN, "x, residual and y must be aligned to their elements");
    if ((double)rows * (double)cols >= 1e12) return record_error(SAME_ESIZE, "rows * cols must stay below 10^12");
    const double far = (double)(rows - 1) * (double)std::max(x_row, std::max(y_row, residual ? residual_row : 0));
    if (far >= 1e18) return record_error(SAME_ESIZE, "row strides pass 10^18 elements");
    if (rows == 1) x_row = y_row = residual_row = cols;
    // y may be x or residual itself, or lie apart; column blocks of one wider
    // buffer lie apart although their extents overlap
    auto apart = [&](const void *a, int64_t a_row) {
        if (a == y && a_row == y_row) return true;
        if (!overlap(extent(a, ((rows - 1) * a_row + cols) * size), extent(y, ((rows - 1) * y_row + cols) * size)))
            return true;
        if (a_row != y_row) return false;
        const int64_t step = y_row * size;
        const int64_t d = (((int64_t)((uintptr_t)a - (uintptr_t)y)) % step + step) % step;
        return d >= cols * size && d <= step - cols * size;
    };
    if (!apart(x, x_row)) return record_error(SAME_EINVAL, "y overlaps x without being x");
    if (residual && !apart(residual, residual_row))
        return record_error(SAME_EINVAL, "y overlaps residual without being residual");
    p.x = x;
    p.residual = residual;
    p.y = y;
    p.rows = rows;
    p.cols = cols;
    p.x_row = x_row;
    p.r_row = residual_row;
    p.y_row = y_row;
    p.keep_gain = 65536.0f / (65536.0f - (float)p.drop_below);
    p.seed_lo = (uint32_t)seed;
    p.seed_hi = (uint32_t)(seed >> 32);
    p.call_id = call_id;
    return check_hip(same::launch_dropout(p, dtype, (hipStream_t)stream), "dropout launch");
}

}  // extern "C"
