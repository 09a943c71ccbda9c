// Host planner: validates one step's batch, tiles it into (unit, KV chunk) work items, balances the
// items over persistent CTAs and uploads the packed plan with one asynchronous copy.
//
// The step being planned is the "next decoding step" after the interrupt manager has appended its
// queued interrupt tokens (paper Section 5.3): q_len 1 = decode, > 1 = interrupt span, 0 = a
// sequence paused by a trap (Section 3.2).  All work here is integer work on the host.
#include <cuda_runtime.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstring>
#include <exception>
#include <vector>

#include "asynclm.h"
#include "kernels.h"
#include "plan_internal.h"

namespace asynclm {

static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int resolve_num_sms(const asynclm_plan_options* opts, bool need_device, int* out) {
    if (opts && opts->num_sms > 0) { *out = opts->num_sms; return ASYNCLM_OK; }
    if (!need_device) { *out = 148; return ASYNCLM_OK; }
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return ASYNCLM_ERR_CUDA;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return ASYNCLM_ERR_CUDA;
    *out = n;
    return ASYNCLM_OK;
}

static int check_shape(const asynclm_shape* s) {
    if (!s) return ASYNCLM_ERR_INVALID_ARG;
    if (s->num_q_heads <= 0 || s->num_kv_heads <= 0 || s->num_pages < 0 || s->reserved != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    if (s->num_q_heads % s->num_kv_heads != 0) return ASYNCLM_ERR_UNSUPPORTED_SHAPE;
    const int g = s->num_q_heads / s->num_kv_heads;
    if (!(g == 1 || g == 2 || g == 4 || g == 8)) return ASYNCLM_ERR_UNSUPPORTED_SHAPE;
    if (!(s->head_dim == 64 || s->head_dim == 128)) return ASYNCLM_ERR_UNSUPPORTED_SHAPE;
    if (s->page_size != kPage) return ASYNCLM_ERR_UNSUPPORTED_SHAPE;
    return ASYNCLM_OK;
}

// Tokens of a span that one tensor-core work item covers: two row tiles of 128 (token, head) rows.
int tensor_tile_tokens(int group) { return 256 / group; }

// Rows (G * q_len) from which a (sequence, kv head) goes to the span body (tcgen05).  Below it the
// warp body reads the keys once per 8 (token, head) columns, which costs less than a span item's
// start-up; decode rows (G rows) always stay on the warp body, which runs at the memory rate for
// every supported G.  At head_dim 64 a re-read of the keys costs half as much.
static int default_tensor_min_rows(int head_dim) { return head_dim == 64 ? 64 : 32; }

// Sizes of the sections of the packed blob (identical offsets on host and device).
struct BlobLayout {
    size_t off_q_indptr, off_kv_len, off_page_indptr, off_page_indices, off_row_seq, off_row_slot, off_units,
        off_items, off_works, off_heads, off_cta_cuda, off_cta_tensor, off_split, off_merge, off_status,
        off_arrivals, off_joins, off_select_chunks, off_select_base, blob_bytes;
};

static BlobLayout layout_blob(int batch, int total_q, int64_t total_pages, int64_t n_units,
                              int64_t n_items, int ctas_cuda, int ctas_tensor, int64_t n_split,
                              int64_t n_merge_blocks, int64_t n_joins = 0, int64_t n_select_chunks = 0,
                              int64_t n_select_rows = 0) {
    BlobLayout L{};
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o = align_up(o + bytes, 256); return at; };
    L.off_status = take(256);
    L.off_q_indptr = take(sizeof(int32_t) * (size_t)(batch + 1));
    L.off_kv_len = take(sizeof(int32_t) * (size_t)std::max(batch, 1));
    L.off_page_indptr = take(sizeof(int32_t) * (size_t)(batch + 1));
    L.off_page_indices = take(sizeof(int32_t) * (size_t)std::max<int64_t>(total_pages, 1));
    L.off_row_seq = take(sizeof(int32_t) * (size_t)std::max(total_q, 1));
    L.off_row_slot = take(sizeof(int64_t) * (size_t)std::max(total_q, 1));
    L.off_units = take(sizeof(Unit) * (size_t)std::max<int64_t>(n_units, 1));
    L.off_items = take(sizeof(Item) * (size_t)std::max<int64_t>(n_items, 1));
    L.off_works = take(sizeof(Work) * (size_t)std::max<int64_t>(n_items, 1));
    L.off_heads = take(sizeof(int32_t) * kHeadWords * (size_t)std::max(ctas_cuda, ctas_tensor));
    L.off_cta_cuda = take(sizeof(int32_t) * (size_t)(ctas_cuda + 1));
    L.off_cta_tensor = take(sizeof(int32_t) * (size_t)(ctas_tensor + 1));
    L.off_split = take(sizeof(int32_t) * (size_t)std::max<int64_t>(n_split, 1));
    L.off_merge = take(sizeof(int32_t) * (size_t)std::max<int64_t>(n_merge_blocks, 1));
    L.off_arrivals = take(sizeof(int32_t) * (size_t)std::max<int64_t>(n_units, 1));
    L.off_joins = take(sizeof(Join) * (size_t)n_joins);
    L.off_select_chunks = take(sizeof(SelectChunk) * (size_t)n_select_chunks);
    L.off_select_base = take(sizeof(int64_t) * (size_t)n_select_rows);
    L.blob_bytes = o;
    return L;
}

static size_t partial_bytes(int64_t rows, int group, int head_dim) {
    return align_up((size_t)rows * (size_t)group * (size_t)head_dim * sizeof(float), 256) +
           align_up((size_t)rows * (size_t)group * sizeof(float), 256);
}

// Warp-body units: a sixth of the work is cut into short chunks for the end of the queue, about
// kTailChunksPerCta per CTA and never shorter than kMinChunkTiles tiles (see deal_dynamic), unless the shortest
// units, which stand at the end of the queue anyway, are short enough to even out the CTAs' finishing times: those
// that make up a sixth of the work are no longer than kShortUnitShare of a CTA's share.  Cutting costs item boundaries,
// partial rows and merges, and a CTA that is late streams faster once others have left the memory to it (which takes
// kSaturatingCtas to begin with).  (us of attention a layer, cut | not: 64 decoding sequences of 1-3 K keys 85.3 | 83.4, 256 of
// 0.3-2 K with 5 spans 192 | 186, 32 of 0.5-4 K with 8 spans 62.1 | 60.0, 40 of 64/8 heads with 8 123 | 114; the longest of the
// shortest sixth has 0.05 to 0.6 of a share there.  Near a share, cutting wins: 19 of 3 K keys 45.4 | 50.)
constexpr int kTailChunksPerCta = 2;
constexpr int kMinChunkTiles = 4;
constexpr int kMinSharedTiles = 2;      // of a span unit with a shared prefix
constexpr int kShortUnitShareNum = 2, kShortUnitShareDen = 3;
constexpr int kSaturatingCtas = 74;      // stream 6.2 TB/s of pages, 148 6.6, 37 4.4
// That alone leaves the last wave nearly empty where the units are of about one length and not a multiple of the CTAs, so
// an uncut queue is followed to its end (queue_ns) and cut after all if it ends later than the cut one by more than cutting
// costs.  (us of attention a layer, cut | not | chosen: sequences of one length, 38 of 4 K keys 104 | 117 | cut, 48 135 | 124 | not,
// 57 of 6 K 208 | 224 | cut, at head_dim 64 38 of 6 K 85.6 | 108 | cut, 74 156 | 145 | not.  Of 290 batches, half of them of one
// length or nearly, the chosen form takes 0.2 % longer than the faster one on average and 6 % at most, the rule above
// alone 2.1 % and 26 %.)
struct StreamCost {
    int64_t tile_ns, least_tile_ns;      // 128 keys on a CTA while kStreamCtas stream, and while few do
    int64_t cut_ns;                      // what a cut sixth costs at the end: more boundaries, partial rows, merges
};
// (Those of head_dim 64 were taken with a warp body that had one page of a stage for each warp; 640 and 570 are what it takes with two.
// 11 batches of one length and 11 others come out the same with either.)
constexpr int kStreamCtas = 148;
constexpr StreamCost stream_cost(int head_dim) {
    return head_dim == 64 ? StreamCost{700, 630, 2500} : StreamCost{1390, 834, 5000};
}
// The other units are cut into pieces of at most kBulkTiles tiles (50-90 us) or an eighth of a CTA's share: with
// contexts of 10^5 tokens, pieces of two fifths of the step, which used to be the only limit, left some CTAs on
// a last piece of half a millisecond.  (8 sequences of 32-131 K tokens, two 256-token spans: 1083 us of attention
// a layer without this limit, 910-970 with it, run to run; 32 and 128 tiles the same; 128 sequences of 64 / 8
// heads 489 at 32 tiles, 480 at 64 and 128.)
constexpr int kBulkTiles = 64;
// Span units of two row tiles are cut by keys instead of divided by rows where the pieces are at least this
// long, because the divided halves each stream the keys: 128 keys take a CTA 2.4 us for two row tiles and
// 1.55 us for one, when all CTAs stream.  (8 sequences of 32-131 K tokens, two 256-token spans: 1065-1096 us of
// attention a layer with divided units, 910-970 with as many cut ones as the fixed array has room for.)  Below,
// the partial rows and their merge cost more than they save (32 sequences of up to 4 K tokens, 8 spans: 62.5 us
// divided, 68.7 cut).
constexpr int kLongPieceTiles = 64;
// Tokens of one warp-body unit: its MMAs have 8 (token, head) columns.
static int warp_unit_tokens(int group) { return 8 / group; }

// Upper bounds on what the automatic policy produces, for C CTAs and W tiles of warp-body work in all.
//   Warp body, only units longer than 1.5 pieces are cut, into ceil(t / piece) <= 1.5 t / piece pieces (the
// worst is just over two).  A long piece is at least min(2/5 of a CTA's share, max(kBulkTiles, an eighth of
// it)) >= W / (8 C) tiles: at most 12 C pieces.  A short one is at least W / (12 C) less the rounding, and
// never below kMinChunkTiles, so below 1.25 times as many: 15 C pieces if one unit holds all the work; a unit
// goes to the short ones only until they hold a sixth of W, so all but the last add at most 1.5 * 15 C / 6.
// The worst mixture, a sixth of W in small units and the rest in the last one, stays below 17 C.
//   Span body: a unit is cut only if it is longer than what a fresh CTA takes, into pieces longer than half of
// that (or of one tile, which each need a CTA of their own), so a CTA holds fewer than three.
//   A unit that is not cut is one item, and a divided unit is two; only cut units hold partial rows.
static int64_t auto_item_bound(int64_t units, int ctas) { return 2 * units + (int64_t)20 * ctas; }
static int64_t auto_partial_row_bound(int ctas, int group) {
    return (int64_t)20 * ctas * warp_unit_tokens(group) + (int64_t)3 * ctas * tensor_tile_tokens(group);
}

}  // namespace asynclm

using namespace asynclm;

extern "C" int asynclm_plan_workspace_size(const asynclm_shape* shape,
                                           const asynclm_plan_options* opts, int32_t max_batch,
                                           int32_t max_total_q, int64_t max_total_pages,
                                           size_t* host_bytes, size_t* device_bytes) {
    int rc = check_shape(shape);
    if (rc != ASYNCLM_OK) return rc;
    if (max_batch < 0 || max_total_q < 0 || max_total_pages < 0 || !host_bytes || !device_bytes)
        return ASYNCLM_ERR_INVALID_ARG;
    int n_sms = 0;
    if (resolve_num_sms(opts, true, &n_sms) != ASYNCLM_OK) n_sms = 160;
    const int G = shape->num_q_heads / shape->num_kv_heads;
    const int ctas_cuda = n_sms * kCudaSlotsPerSm;
    const int ctas_tensor = n_sms;
    const int64_t max_units = (int64_t)max_total_q * shape->num_kv_heads;
    int64_t max_items, max_partial_rows;
    if (opts && opts->kv_chunk_tokens > 0) {
        // fixed chunk length: every unit may be cut into ceil(n/chunk) pieces
        const int64_t per_unit = (max_total_pages * kPage) / opts->kv_chunk_tokens + 1;
        max_items = max_units * per_unit;
        max_partial_rows = max_items;   // ntok tokens per unit are already counted in max_units
    } else {
        max_items = auto_item_bound(max_units, ctas_cuda);
        max_partial_rows = auto_partial_row_bound(ctas_cuda, G);      // only cut units hold partial rows
    }
    BlobLayout L = layout_blob(max_batch, max_total_q, max_total_pages, max_units, max_items,
                               ctas_cuda, ctas_tensor, max_units,
                               (int64_t)max_total_q * shape->num_q_heads / 4 + max_units);
    *host_bytes = align_up(sizeof(asynclm_plan_s), 256) + L.blob_bytes +
                  align_up(sizeof(int32_t) * (size_t)std::max<int64_t>(max_items, 1), 256);
    *device_bytes = L.blob_bytes + partial_bytes(max_partial_rows, G, shape->head_dim);
    return ASYNCLM_OK;
}

namespace {

struct UnitBuild {
    Unit u;
    int path;
    int64_t n_keys;   // keys visible to the unit's last token
    int32_t run = -1;      // shared prefix: the run of sequences that the unit's rows belong to
    bool flat = false;     // the unit holds the prefix that its run shares: all of its tokens see all of its keys
    // its rows are written as partial rows, whatever the number of chunks
    bool partial() const { return u.n_chunks > 1 || run >= 0; }
};

// Cuts the units of one path into items and deals them to `n_ctas` persistent CTAs.
// fixed_chunk > 0: equal chunks of that many tokens, then a contiguous equal-cost partition of the
// item sequence.  Otherwise: the concatenated tile sequence of all units is cut into n_ctas nearly
// equal contiguous ranges (a unit is split only where a range boundary falls inside it).
void cut_and_deal(const std::vector<int>& unit_ids, std::vector<UnitBuild>& units, int fixed_chunk,
                  int n_ctas, int item_overhead_tiles, std::vector<Item>& items,
                  std::vector<int32_t>& cta_indptr, std::vector<int32_t>& item_cta) {
    const size_t first_item = items.size();
    cta_indptr.assign((size_t)n_ctas + 1, (int32_t)first_item);
    if (unit_ids.empty() || n_ctas <= 0) return;
    auto tiles_of = [](int64_t tokens) { return (tokens + kKvTile - 1) / kKvTile; };
    if (fixed_chunk > 0) {
        for (int id : unit_ids) {
            UnitBuild& ub = units[id];
            int c = 0;
            for (int64_t k0 = 0; k0 < ub.n_keys; k0 += fixed_chunk, ++c) {
                Item it{id, (int32_t)k0, (int32_t)std::min<int64_t>(ub.n_keys, k0 + fixed_chunk), c};
                items.push_back(it);
            }
            ub.u.n_chunks = c;
        }
        int64_t total = 0;
        for (size_t i = first_item; i < items.size(); ++i)
            total += item_overhead_tiles + tiles_of(items[i].kv1 - items[i].kv0);
        // contiguous partition: an item goes to the CTA in whose share of the total its midpoint falls
        int64_t cum = 0;
        for (size_t i = first_item; i < items.size(); ++i) {
            const int64_t c = item_overhead_tiles + tiles_of(items[i].kv1 - items[i].kv0);
            const int64_t cta = std::min<int64_t>(n_ctas - 1, ((2 * cum + c) * n_ctas) / (2 * total));
            item_cta.push_back((int32_t)cta);
            cum += c;
        }
    } else {
        int64_t total_tiles = 0;
        for (int id : unit_ids) total_tiles += tiles_of(units[id].n_keys);
        const int64_t total_cost =
            total_tiles + (int64_t)item_overhead_tiles * ((int64_t)unit_ids.size() + n_ctas);
        const int64_t quota = std::max<int64_t>(1 + item_overhead_tiles,
                                                (total_cost + n_ctas - 1) / n_ctas);
        int cta = 0;
        int64_t budget = quota;
        for (int id : unit_ids) {
            UnitBuild& ub = units[id];
            int64_t tiles_left = tiles_of(ub.n_keys);
            int64_t k0 = 0;
            int c = 0;
            while (tiles_left > 0) {
                if (budget <= item_overhead_tiles && cta + 1 < n_ctas) {
                    ++cta;
                    budget = quota;
                }
                int64_t take = cta + 1 < n_ctas
                                   ? std::min<int64_t>(tiles_left, std::max<int64_t>(1, budget - item_overhead_tiles))
                                   : tiles_left;
                const int64_t k1 = std::min<int64_t>(ub.n_keys, k0 + take * kKvTile);
                items.push_back(Item{id, (int32_t)k0, (int32_t)k1, c});
                item_cta.push_back(cta);
                budget -= item_overhead_tiles + take;
                tiles_left -= take;
                k0 = k1;
                ++c;
            }
            ub.u.n_chunks = c;
        }
    }
    // items were emitted in CTA order; build the CSR
    std::vector<int32_t> count((size_t)n_ctas, 0);
    for (size_t i = first_item; i < items.size(); ++i) count[(size_t)item_cta[i]]++;
    int32_t at = (int32_t)first_item;
    for (int k = 0; k < n_ctas; ++k) {
        cta_indptr[(size_t)k] = at;
        at += count[(size_t)k];
    }
    cta_indptr[(size_t)n_ctas] = at;
}

// Costs of the attention kernels on B200 as the packing sees them, in nanoseconds, used only to size the span
// CTAs.  At head_dim 128 they are those of an earlier form of the span body with 128-key tiles, which the margins
// below were chosen with; the present body takes, per 128 keys with one | two row tiles, 0.9 | 1.55 us on a CTA
// alone and 1.4 | 2.4 on all 148, where memory and power bound it (with 900 | 1800 here, 48 sequences with 6 spans took
// 120 us instead of 112).  At head_dim 64 it takes 0.93 | 1.55 alone and 1.0 | 1.9 on all.
struct PathCost {
    static constexpr int gran = kKvTile;      // tokens per tile of every path (cuts fall on multiples of it); a constant, because planning divides by it a lot
    int64_t tile_ns;     // one tile in steady state
    int64_t item_ns;     // starting and finishing an item (pipeline fill and drain, merge, write)
    int64_t phase_ns;    // first item of the path on a CTA (descriptor chain, first loads)
};
// Span body: a KV tile of 128 keys against one row tile, an item, the body's start on a CTA.
constexpr PathCost kTensorCost{1170, 8000, 11800};
constexpr int64_t kTensorDualTileNs = 2435;   // a KV tile of an item with two row tiles (more than 128 rows)
// When every unit runs on the span body all SMs stream K/V tiles at once and the tile time is set by
// the memory system (64 KB per tile and SM); the producers run ahead across item boundaries.
constexpr PathCost kTensorOnlyCost{1543, 8000, 2400};
constexpr int64_t kTensorOnlyDualTileNs = 3126;
// Warp body: 64 KB per 128-key tile (32 KB at head_dim 64).  It is bound by memory, so its tile time depends on
// how many SMs stream at once: 1.39 us when all 148 do, 1.05 us (62 KB/us) when half of them run span tiles,
// which draw some bandwidth too, 0.79 us for 74 and 0.73 for one by themselves; at head_dim 64 0.64, 0.58 for 37 to
// 100 and 0.53 for one.  The model takes the second figure for both.  (At head_dim 64 900 here gives layers of 0.88 to 1.08 of the time
// with 1050, 750 of 0.90 to 1.11, without a rule to tell which batch gains.)
constexpr PathCost kWarpCost{1050, 400, 2000};
// No step ends before its bytes have crossed the memory bus: K/V pages stream at about 6 bytes per
// nanosecond on this access pattern (4 KB runs through a shuffled page table), after about 3 us in
// which the CTAs start.  Without this floor the model would spread the span units over so many CTAs
// that too few were left streaming to keep the memory busy (one SM streams 60-75 KB/us at most).
// Each (sequence, kv head) counts once: the row tiles of a long span re-read it, mostly from L2.
constexpr int64_t kDramBytesPerUs = 6000000;
// A span CTA that finishes early joins the queue; one that finishes late delays the whole step, so the span CTAs
// are filled to the load limit divided by this margin (in 1/64).  The costs above are head_dim 128's of a
// slower body, which leaves a margin by itself.  Attention of a layer in us at 66 | 68 | 72 | 88, head_dim 128: 32
// sequences with 8 spans 60.0 | 61.5 | 61.4 | 61.6, 64 with 12 73.3 | 73.1 | 72.8 | 79.2, 40 of 16/8 heads with 10 65.1 | 64.7 |
// 64.5 | 69.2, 40 of 64/8 heads with 8 114 | 121 | 120 | 122, 128 of 64/8 heads with 13 492 | 489 | 488 | 479 (469 | 465 | 463 |
// 463 at best: power); at head_dim 64, 64 | 72 | 76 | 88: 32 with 8 50.0 | 49.8 | 49.4 | 55.4, 64 with 16 83.3 | 81.1 | 80.7 |
// 80.2, 64 of 8/8 heads with 8 103 | 103 | 104 | 106, 100 of 8/2 heads with 20 48.1 | 50.4 | 50.7 | 55.1.
constexpr int64_t span_margin64(int head_dim) { return head_dim == 64 ? 72 : 66; }
// The same, for the decision to divide a unit by rows.  At head_dim 128 it lies above the span CTAs' margin, so that a unit
// between the two limits is divided although it would fit a CTA whole.  Both ways measured: with 66 here 28 of 1632 random
// batches come out otherwise, attention of a layer 0.80 to 1.18 of the time with 72, 1.002 on average.
constexpr int64_t kDivideMargin64 = 72;
// Share (in 1/64) of the queue that the CTAs without span work must be able to stream by themselves.
constexpr int64_t kStreamShare64 = 58;
constexpr int64_t kStartNs = 3000;

// The costs that a plan is made with: the above for the bf16 cache, and for the 8-bit one (ASYNCLM_PLAN_KV8) these.  Its
// warp body takes, per 128 keys, 0.78 us when all SMs stream (6.3 TB/s) and 0.66 on a CTA alone (a warp's work on two
// pages), half of what 16 bits take, while an item's boundary costs as much as there.  Its span body takes, per 128 keys
// with one | two row tiles, 1.7 | 2.7 us on a CTA alone and 2.3 | 2.7 on all (1.9 | 3.0 and 2.6 | 3.3 when these costs were
// chosen).  An item of it is taken as longer than it is, 8 us, which keeps spans in longer pieces.  (18 mixed batches at 6 | 8 | 10
// us: 12 within 2 %; 128 sequences with 6 spans 81 | 75.6 | 76, 32 with 24 of 33-96 tokens 169 | 166 | 165, 32 with 8 61 | 63 |
// 63 and 76 | 76 | 82, 48 with 3 97 | 97 | 86, 16 with 4 of 100-300 tokens 214 | 215 | 211.)
struct Model {
    PathCost tensor, tensor_only, warp;
    int64_t dual_ns, dual_only_ns;
    StreamCost stream;
    bool kv8;
};
constexpr Model model_of(int head_dim, bool kv8) {
    if (!kv8) return Model{kTensorCost, kTensorOnlyCost, kWarpCost, kTensorDualTileNs, kTensorOnlyDualTileNs, stream_cost(head_dim), false};
    const bool narrow = head_dim == 64;
    return Model{PathCost{2200, 8000, 10000}, PathCost{2580, 8000, 2400}, PathCost{narrow ? 540 : 720, 1200, 2000}, 3200, 3270,
                 narrow ? StreamCost{850, 750, 2500} : StreamCost{780, 660, 2500}, true};
}

// Sorts `v` by falling key, equal keys in the order they stand in.  What stands here comes in runs of equal keys (the
// kv heads of a sequence, a unit's pieces), so the runs are sorted and written out again.
template <typename T, typename Key>
void sort_falling(std::vector<T>& v, Key key) {
    struct Run { int64_t key; uint32_t at, count; };
    std::vector<Run> runs;
    runs.reserve(v.size() / 4 + 8);
    for (size_t i = 0; i < v.size(); ++i) {
        const int64_t k = key(v[i]);
        if (!runs.empty() && runs.back().key == k) ++runs.back().count;
        else runs.push_back(Run{k, (uint32_t)i, 1});
    }
    auto before = [](const Run& x, const Run& y) { return x.key != y.key ? x.key > y.key : x.at < y.at; };
    if (std::is_sorted(runs.begin(), runs.end(), before)) return;
    std::sort(runs.begin(), runs.end(), before);
    std::vector<T> sorted;
    sorted.reserve(v.size());
    for (const Run& r : runs) sorted.insert(sorted.end(), v.begin() + r.at, v.begin() + r.at + r.count);
    v.swap(sorted);
}

// How span units and long decode units are cut.  The default is the fastest; asynclm_plan asks for fewer cuts
// where the partial results would outgrow the fixed array of asynclm_attn_mixed_static.
struct CutPolicy {
    int units_by_keys = INT_MAX;      // long span units (kLongPieceTiles) that may be cut by keys, the longest first
    bool bound_pieces = true;         // kBulkTiles
};

// Modelled time until the last CTA is through with the warp body's queue: `joins` holds when the CTAs with span work join
// (the others are there from the start), each takes the next item as soon as it is through with one, and those that are
// still busy when nothing is left stream faster.  Time runs in steps of 1/1024 of the mean (longer ones where
// an item or a join is very long); *mean_ns, the mean finish, is what no other order of the same items ends before.
int64_t queue_ns(const std::vector<Item>& queue, const std::vector<int64_t>& joins, int n_ctas, const Model& model, int64_t* mean_ns) {
    const StreamCost cost = model.stream;
    auto tile_ns = [&](int64_t ctas) { return std::max(cost.least_tile_ns, cost.tile_ns * ctas / kStreamCtas); };
    const int64_t tile = tile_ns(n_ctas);
    struct Run { int64_t ns, count; };      // items of equal cost
    std::vector<Run> runs;
    int64_t sum = 0, tiles_before = -1, longest = 0;
    for (const Item& it : queue) {
        const int64_t tiles = ((int64_t)it.kv1 - it.kv0 + kWarpCost.gran - 1) / kWarpCost.gran;
        if (tiles != tiles_before) runs.push_back(Run{model.warp.item_ns + tiles * tile, 0});
        tiles_before = tiles;
        ++runs.back().count;
        sum += runs.back().ns;
        longest = std::max(longest, runs.back().ns);
    }
    for (int64_t at : joins) sum += at, longest = std::max(longest, at);
    const int64_t step = std::max<int64_t>(16, std::max(sum / n_ctas / 1024, longest / 4096));
    std::vector<int32_t> free(2048);      // CTAs that are free from step i on
    auto add = [&](int64_t at, int64_t ctas) {
        if (at >= (int64_t)free.size()) free.resize((size_t)at + 1024);
        free[(size_t)at] += (int32_t)ctas;
    };
    add(0, n_ctas - (int64_t)joins.size());
    for (int64_t at : joins) add(at / step, 1);
    size_t now = 0;
    for (const Run& r : runs) {
        const int64_t need = std::max<int64_t>(1, (r.ns + step / 2) / step);
        for (int64_t left = r.count; left > 0;) {
            while (free[now] == 0) ++now;
            const int64_t n = std::min<int64_t>(left, free[now]);
            free[now] -= (int32_t)n;
            add((int64_t)now + need, n);
            left -= n;
        }
    }
    // (CTAs that join when nothing is left have no part in it)
    int64_t late = 0;
    for (int64_t at : joins)
        if (at / step > (int64_t)now) --free[(size_t)(at / step)], ++late, sum -= at;
    *mean_ns = sum / (n_ctas - late);
    int64_t end = (int64_t)now * step, busy = n_ctas - late - free[now];
    for (size_t at = now + 1; busy > 0; ++at) {
        if (free[at] == 0) continue;
        end += (int64_t)(at - now) * step * tile_ns(busy) / tile;
        now = at;
        busy -= free[at];
    }
    return end;
}

// Default policy for the fused kernel.
//   Span units (tensor-core body) are compute-heavy and predictable: they are packed whole onto as few
// persistent CTAs as the load limit allows (largest first, each into the fullest CTA that still has
// room; a unit larger than a CTA's share is cut into equal pieces), so that most of them write final
// bf16 rows instead of fp32 partial rows.
//   Warp-body units (decode rows, short spans) are bandwidth-bound, and how fast a CTA streams depends
// on what the other SMs are doing, which no static cost predicts.  They are cut into chunks of a few
// tiles, sorted by length (longest first), and handed out at run time: the CTAs without span work
// start on one chunk each, every other chunk waits in a queue from which a CTA that runs out of work
// (a span CTA included) takes the next one with one atomic add.  Partial results are indexed by chunk
// and merged in chunk order, so the output does not depend on which CTA ran what.
//   The load limit is the smallest one under which the span units fit and the room left on all CTAs
// covers the modelled time of the queue; it is found by bisection.
//   selected: the units are those of selected pages.
//   Returns false, with only the units (their division and n_chunks) filled in, if the cuts leave more than
// max_partial_rows partial rows.
bool deal_dynamic(std::vector<int>& ids_tensor, const std::vector<int>& ids_warp,
                  std::vector<UnitBuild>& units, int group, int head_dim, const Model& model, int64_t kv_bytes, int n_ctas, const CutPolicy& policy,
                  int64_t max_partial_rows, bool selected, int64_t* limit_ns, std::vector<Item>& items,
                  std::vector<int32_t>& cta_indptr_warp, std::vector<int32_t>& cta_indptr_tensor,
                  std::vector<int32_t>& item_cta, int32_t* queue_first, int32_t* queue_count) {
    struct Piece { Item it; int32_t cta; };
    const bool tensor_only = ids_warp.empty();
    const PathCost tc = tensor_only ? model.tensor_only : model.tensor;
    const PathCost kWarpCost = model.warp;
    const int64_t dual_tile_ns = tensor_only ? model.dual_only_ns : model.dual_ns;
    auto tiles_of = [](int64_t keys, int gran) { return (keys + gran - 1) / gran; };

    // ---- warp-body work as the model sees it (the chunks are cut below, once the number of CTAs
    // that start on the queue is known)
    int64_t warp_tiles = 0;
    for (int id : ids_warp) warp_tiles += tiles_of(units[id].n_keys, kWarpCost.gran);
    const int64_t warp_ns = warp_tiles * kWarpCost.tile_ns + (int64_t)ids_warp.size() * 2 * kWarpCost.item_ns;

    // ---- span units with two row tiles that would not fit a CTA whole are divided by rows into two
    // units of one row tile each (the second reader of the keys finds most of them in L2) rather than by
    // keys, which would cost fp32 partial rows and a merge, unless the pieces would be long (kLongPieceTiles).
    // The limit used for the decision is the lower bound of the one found below.
    {
        int64_t work = warp_ns;
        for (int id : ids_tensor)
            work += tc.item_ns + tiles_of(units[id].n_keys, tc.gran) * (units[id].u.ntok * group > 128 ? dual_tile_ns : tc.tile_ns);
        const int64_t limit0 = std::max(work / n_ctas, kStartNs + kv_bytes * 1000 / kDramBytesPerUs) * 64 / kDivideMargin64;
        const int half = 128 / group;      // tokens of one row tile
        // which of them are left to be cut by keys (below): the longest, because a divided half stays whole and would
        // be a CTA's longest item
        std::vector<char> by_keys;
        if (policy.units_by_keys > 0 && limit0 - tc.phase_ns - tc.item_ns >= kLongPieceTiles * dual_tile_ns) {
            std::vector<int> longest(ids_tensor);
            std::stable_sort(longest.begin(), longest.end(), [&](int x, int y) { return units[x].n_keys > units[y].n_keys; });
            by_keys.assign(units.size(), 0);
            int n = 0;
            for (int id : longest)
                if (units[(size_t)id].u.ntok * group > 128 && n < policy.units_by_keys) by_keys[(size_t)id] = 1, ++n;
        }
        const size_t n0 = ids_tensor.size();
        for (size_t i = 0; i < n0; ++i) {
            const int id = ids_tensor[i];
            UnitBuild& ub = units[(size_t)id];
            if (ub.u.ntok * group <= 128 || ub.flat) continue;      // (a shared prefix has partial rows anyway)
            if (tc.phase_ns + tc.item_ns + tiles_of(ub.n_keys, tc.gran) * dual_tile_ns <= limit0) continue;
            if (!by_keys.empty() && by_keys[(size_t)id]) continue;
            UnitBuild second = ub;
            second.u.q_row0 += half;
            second.u.ntok -= half;
            second.u.kv_limit0 += half;
            ub.u.ntok = half;
            ub.n_keys = (int64_t)ub.u.kv_limit0 + ub.u.ntok - 1;
            ids_tensor.push_back((int)units.size());
            units.push_back(second);
        }
    }

    // ---- span units under a load limit
    // (those with a shared prefix apart: they are cut wherever a CTA is full)
    std::vector<int> order, shared_order;
    std::vector<int64_t> tiles(units.size()), tns(units.size());
    for (int id : ids_tensor) {
        (units[(size_t)id].flat ? shared_order : order).push_back(id);
        tiles[(size_t)id] = tiles_of(units[id].n_keys, tc.gran);
        tns[(size_t)id] = units[id].u.ntok * group > 128 ? dual_tile_ns : tc.tile_ns;
    }
    sort_falling(order, [&](int id) { return tiles[(size_t)id] * tns[(size_t)id]; });
    // units of the same cost one after the other: (first in `order`, how many)
    struct Batch { int64_t tiles, ns; uint32_t at, count; };
    std::vector<Batch> batches;
    for (size_t i = 0; i < order.size(); ++i) {
        const int64_t t = tiles[(size_t)order[i]], ns = tns[(size_t)order[i]];
        if (!batches.empty() && batches.back().tiles == t && batches.back().ns == ns) ++batches.back().count;
        else batches.push_back(Batch{t, ns, (uint32_t)i, 1});
    }
    struct Cta { int64_t load; int32_t id; };
    std::vector<Cta> ctas((size_t)n_ctas);      // those in use, the fullest first, equal loads by id
    std::vector<Piece> pieces_out;
    int used = 0;
    // Packs the span units under `cap`; returns false if they do not fit or leave too little room for
    // the queue.  With emit == false only the verdict is computed (the bisection's probes).
    int64_t span_work = 0;      // all span items without the per-CTA start
    for (int id : ids_tensor) span_work += tc.item_ns + tiles[(size_t)id] * tns[(size_t)id];
    const int64_t floor_ns = kStartNs + kv_bytes * 1000 / kDramBytesPerUs;
    const int64_t bound = std::max<int64_t>(std::max<int64_t>(1, (warp_ns + span_work) / n_ctas), floor_ns);      // of the load limit
    auto fill = [&](int64_t limit, bool emit) {
        // CTAs that may hold span work: the others have to be able to stream most of the queue by
        // themselves (span CTAs draw little bandwidth, and one SM streams only so much)
        const int64_t stream_ctas = limit > kStartNs
            ? (warp_tiles * kWarpCost.tile_ns * kStreamShare64 / 64 + (limit - kStartNs) - 1) / (limit - kStartNs) : n_ctas;
        // (a lone CTA does both)
        const int64_t span_ctas = ids_warp.empty() || n_ctas == 1 ? n_ctas : n_ctas - stream_ctas;
        if (!ids_tensor.empty() && span_ctas < 1) return false;
        // what a span CTA may be given: the span work spread over those CTAs with some slack for the
        // packing, at most the load limit less the safety margin.  Spreading the spans thin costs little (a
        // span CTA that is done early joins the queue), filling span CTAs to the brim risks a late finish.
        const int64_t thin = ids_tensor.empty() ? 0 : span_work / span_ctas * 5 / 4 + tc.phase_ns + tc.item_ns + dual_tile_ns;
        // (Past twice the lower bound the spread is given up: items of more than half of `thin` take a CTA each,
        // and there may be more of them than CTAs.)
        const int64_t full = limit * 64 / span_margin64(head_dim);
        const int64_t cap = limit > 2 * bound ? full : std::min(full, std::max(thin, 2 * (tc.phase_ns + tc.item_ns)));
        pieces_out.clear();
        used = 0;
        // moves the CTA at position `at` of `ctas` to where its new load belongs
        auto add_load = [&](int at, int64_t more) {
            Cta c = ctas[(size_t)at];
            c.load += more;
            auto fuller = [](const Cta& x, const Cta& y) { return x.load != y.load ? x.load > y.load : x.id < y.id; };
            if (at == 0 || fuller(ctas[(size_t)at - 1], c)) {
                ctas[(size_t)at] = c;
                return;
            }
            const int to = (int)(std::upper_bound(ctas.begin(), ctas.begin() + at, c, fuller) - ctas.begin());
            std::move_backward(ctas.begin() + to, ctas.begin() + at, ctas.begin() + at + 1);
            ctas[(size_t)to] = c;
        };
        // Shared prefixes first: their rows are partial ones and joined whatever the cuts, so each unit goes on where the last one ended, and CTAs
        // are filled to the brim.  (us, pieces of one length for a unit | so: 30 sequences with 6 spans of 4-100 tokens 84 | 79, 30 with 3 of 300-600
        // 193 | 173, 10 over the 8-bit cache with 3 of 200-500 310 | 202, 96 with one token each at 8/2 heads of 64 21.0 | 19.5, 64 with one 46 | 46.)
        for (int id : shared_order) {
            const int64_t t = tiles[(size_t)id], ns = tns[(size_t)id];
            int32_t c = 0;
            for (int64_t k0 = 0; k0 < t; ++c) {
                auto room = [&]() { return (cap - ctas[(size_t)used - 1].load - tc.item_ns) / ns; };
                if (used == 0 || room() < std::min(t - k0, (int64_t)kMinSharedTiles)) {
                    if (used < n_ctas) {
                        ctas[(size_t)used] = Cta{tc.phase_ns, (int32_t)used};
                        ++used;
                    }
                    if (!emit && used > span_ctas) return false;
                }
                const bool last = used == n_ctas && room() < kMinSharedTiles;      // (no CTA is left)
                if (last && !emit) return false;
                int64_t take = last ? t - k0 : std::min(t - k0, std::max<int64_t>(1, room()));
                if (t - k0 - take < kMinSharedTiles) take = t - k0;
                if (emit)
                    pieces_out.push_back(Piece{Item{id, (int32_t)(k0 * tc.gran), (int32_t)std::min<int64_t>(units[id].n_keys, (k0 + take) * tc.gran), c},
                                               ctas[(size_t)used - 1].id});
                ctas[(size_t)used - 1].load += tc.item_ns + take * ns;
                k0 += take;
            }
        }
        std::sort(ctas.begin(), ctas.begin() + used, [](const Cta& x, const Cta& y) { return x.load != y.load ? x.load > y.load : x.id < y.id; });
        for (const Batch& batch : batches) {
            const int64_t t = batch.tiles, ns = batch.ns;
            const int64_t fresh_room = std::max<int64_t>(1, (cap - tc.phase_ns - tc.item_ns) / ns);
            const int64_t pieces = t <= fresh_room ? 1 : (t + fresh_room - 1) / fresh_room;
            // pieces of a unit one after the other, units one after the other; whole units go to one CTA several at once
            // as long as it stays the fullest that has room (nobody fuller has, and it only gets fuller)
            const int64_t todo = pieces * batch.count;
            for (int64_t k = 0; k < todo;) {
                const int64_t c = k % pieces;
                const int64_t take = pieces == 1 ? t : t / pieces + (c < t % pieces ? 1 : 0);
                const int64_t need = tc.item_ns + take * ns;
                int at = used;
                if (used > 0 && ctas[(size_t)used - 1].load + need <= cap)
                    at = (int)(std::partition_point(ctas.begin(), ctas.begin() + used, [&](const Cta& x) { return x.load + need > cap; }) - ctas.begin());
                if (at == used) {
                    if (used < n_ctas) {
                        ctas[(size_t)used] = Cta{tc.phase_ns, (int32_t)used};
                        ++used;
                        if (!emit && used > span_ctas) return false;
                    } else {
                        if (!emit) return false;
                        --at;      // the least loaded
                        while (at > 0 && ctas[(size_t)at - 1].load == ctas[(size_t)at].load) --at;
                    }
                }
                const int64_t n = pieces > 1 ? 1 : std::min(todo - k, 1 + std::max<int64_t>(0, cap - need - ctas[(size_t)at].load) / need);
                if (emit)
                    for (int64_t j = k; j < k + n; ++j) {
                        const int id = order[batch.at + (size_t)(j / pieces)];
                        const int64_t k0 = c * (t / pieces) + std::min(c, t % pieces);      // tiles before piece c
                        pieces_out.push_back(Piece{Item{id, (int32_t)(k0 * tc.gran), (int32_t)std::min<int64_t>(units[id].n_keys, (k0 + take) * tc.gran),
                                                        (int32_t)c}, ctas[(size_t)at].id});
                    }
                add_load(at, n * need);
                k += n;
            }
        }
        // room for the queue: what the span CTAs have left after restarting on the warp body, and the
        // whole limit on the others
        int64_t room = (n_ctas - used) * std::max<int64_t>(0, limit - kWarpCost.phase_ns);
        for (int k = 0; k < used; ++k)
            room += std::max<int64_t>(0, limit - ctas[(size_t)k].load - kWarpCost.phase_ns);
        return used <= span_ctas && room >= warp_ns;
    };
    int64_t lo = bound;
    int64_t hi = lo + lo / 4 + tc.item_ns + tc.phase_ns + kWarpCost.phase_ns;
    while (!fill(hi, false)) { lo = hi; hi += hi / 2; }
    for (int iter = 0; iter < 24 && hi - lo > std::max<int64_t>(50, hi / 128); ++iter) {      // to 0.8 %
        const int64_t mid = (lo + hi) / 2;
        if (fill(mid, false)) hi = mid; else lo = mid;
    }
    fill(hi, true);
    *limit_ns = hi;
    for (const Piece& pz : pieces_out) units[pz.it.unit].u.n_chunks = std::max(units[pz.it.unit].u.n_chunks, pz.it.chunk + 1);

    // ---- warp-body chunks.  An item boundary costs time and a split unit costs partial rows and a
    // merge, so most of the work stays in long pieces: where the shortest units are long themselves (kShortUnitShare), a
    // few units, a sixth of all tiles, are cut into short chunks that go to the END of the queue, where they even out
    // the CTAs' finishing times; every other unit stays whole unless it is longer than two fifths of the step (or than kBulkTiles tiles
    // and an eighth of a CTA's share), in which case it is cut into equal pieces.  The queue holds the long pieces longest first, then the short chunks.
    std::vector<int> warp_order(ids_warp);
    sort_falling(warp_order, [&](int id) { return units[id].n_keys; });
    std::vector<Item> chunks, tail;
    chunks.reserve(ids_warp.size() + (size_t)n_ctas * 4);
    auto longest_piece = [&](int64_t limit) {
        int64_t t = limit * 2 / 5 / kWarpCost.tile_ns;
        if (policy.bound_pieces) t = std::min(t, std::max<int64_t>(kBulkTiles, warp_tiles / (8 * (int64_t)n_ctas)));
        return std::max<int64_t>(t, kMinChunkTiles);
    };
    int64_t bulk_max = longest_piece(hi);
    const int64_t tail_target = warp_tiles / 6;
    const int64_t tail_chunk = std::max<int64_t>(kMinChunkTiles, tail_target / ((int64_t)n_ctas * kTailChunksPerCta));
    // cuts the units; which are cut short: first those of up to four chunks (their merge is one round trip to
    // L2), longest first; longer ones only if that does not give a sixth of the tiles
    std::vector<char> to_tail(units.size());
    auto cut = [&](bool cut_tail) {
        chunks.clear();
        tail.clear();
        std::fill(to_tail.begin(), to_tail.end(), 0);
        int64_t tail_tiles = 0;
        for (int pass = 0; pass < 2 && cut_tail && tail_tiles < tail_target; ++pass)
            for (int id : warp_order) {
                const int64_t t = tiles_of(units[id].n_keys, kWarpCost.gran);
                if (tail_tiles >= tail_target) break;
                if (to_tail[(size_t)id] || t <= tail_chunk + tail_chunk / 2 || (pass == 0 && t > 4 * tail_chunk)) continue;
                to_tail[(size_t)id] = 1;
                tail_tiles += t;
            }
        for (int id : warp_order) {
            const int64_t t = tiles_of(units[id].n_keys, kWarpCost.gran);
            const bool short_chunks = to_tail[(size_t)id] != 0;
            const int64_t piece_max = short_chunks ? tail_chunk : bulk_max;
            const int64_t pieces = t <= piece_max + piece_max / 2 ? 1 : (t + piece_max - 1) / piece_max;
            int64_t k0 = 0;
            for (int64_t c = 0; c < pieces; ++c) {
                const int64_t take = t / pieces + (c < t % pieces ? 1 : 0);
                const int64_t k1 = std::min<int64_t>(units[id].n_keys, k0 + take * kWarpCost.gran);
                (short_chunks ? tail : chunks).push_back(Item{id, (int32_t)k0, (int32_t)k1, (int32_t)c});
                k0 = k1;
            }
            units[id].u.n_chunks = (int32_t)pieces;
        }
    };
    // the queue in its order: long pieces, then short chunks, the longest first
    bool queued = false;
    auto queue_up = [&]() {
        auto length = [](const Item& x) { return (int64_t)x.kv1 - x.kv0; };
        sort_falling(chunks, length);
        sort_falling(tail, length);
        chunks.insert(chunks.end(), tail.begin(), tail.end());
        queued = true;
    };
    // The 8-bit cache: an item takes half the time and its boundary no less, so short chunks for the end of the queue cost
    // more than they even out.  Units are cut into pieces of one length, the least that makes at most 1, 2, 3 or 4 pieces
    // for a CTA, or not at all, whichever the model of the queue has end first, with what joining the pieces of a unit
    // takes behind it.  (us of attention, cut as the 16-bit cache's | so: one sequence of 60 K keys, 8 kv heads, 56.7 |
    // 30.9; 16 of 4 K 35.3 | 31.1; 5 of 32-110 K 166 | 144.8; 64 of 1-3 K 52.6 | 51.2.)  The search costs the host 50 to 80 us at such
    // sizes.  Not at head_dim 64 with a unit or more for every CTA, where it is worth 2 % on average over 20 batches, 0.91 to 1.2 of the time by turns: 40
    // sequences of 2-6 K keys, 8 kv heads, 58-60 | 53-55, 20 of 4-30 K 104-109 | 96-101, 64 of 1-3 K 42-43 | 41-43, 32 of 0.5-8 K 47, 56 | 57,
    // 54, 100 of 1-10 K, 2 kv heads, 44-51 | 45-56, short ones and 128 of 16 kv heads equal.
    // Selected pages of either cache, too: their units are of one length or nearly (16 sequences with 128 pages of 16 bits, 128 units on 148 CTAs, 30.7 | 26.2).
    const bool even = (model.kv8 || selected) && (head_dim != 64 || (int64_t)warp_order.size() < n_ctas);
    if (even) {
        std::vector<int64_t> joins;
        for (int k = 0; k < used; ++k) joins.push_back(ctas[(size_t)k].load);
        int64_t longest = 0;
        for (int id : warp_order) longest = std::max(longest, tiles_of(units[id].n_keys, kWarpCost.gran));
        // pieces of `most` tiles; of a unit: its tiles in equal parts
        auto pieces_of = [&](int64_t t, int64_t most) { return (t + most - 1) / most; };
        auto cut_even = [&](int64_t most) {
            chunks.clear();
            int64_t worst = 1;
            for (int id : warp_order) {
                const int64_t t = tiles_of(units[id].n_keys, kWarpCost.gran), pieces = pieces_of(t, most);
                int64_t k0 = 0;
                for (int64_t c = 0; c < pieces; ++c) {
                    const int64_t take = t / pieces + (c < t % pieces ? 1 : 0);
                    const int64_t k1 = std::min<int64_t>(units[id].n_keys, k0 + take * kWarpCost.gran);
                    chunks.push_back(Item{id, (int32_t)k0, (int32_t)k1, (int32_t)c});
                    k0 = k1;
                }
                units[id].u.n_chunks = (int32_t)pieces;
                worst = std::max(worst, pieces);
            }
            sort_falling(chunks, [](const Item& x) { return (int64_t)x.kv1 - x.kv0; });
            return worst;
        };
        int64_t best_most = longest, best_ns = -1, tried = -1;
        for (int per_cta = 0; per_cta <= 4 && longest > 0; ++per_cta) {
            int64_t most = longest;
            if (per_cta > 0) {
                int64_t lo = kMinChunkTiles - 1, hi = longest;      // (lo: too many pieces, or too short)
                while (hi - lo > 1) {
                    const int64_t mid = (lo + hi) / 2;
                    int64_t n = 0;
                    for (int id : warp_order) n += pieces_of(tiles_of(units[id].n_keys, kWarpCost.gran), mid);
                    if (n <= (int64_t)per_cta * n_ctas) hi = mid; else lo = mid;
                }
                most = hi;
            }
            if (most == tried) continue;
            tried = most;
            const int64_t worst = cut_even(most);
            int64_t mean = 0;
            const int64_t ns = queue_ns(chunks, joins, n_ctas, model, &mean) + (worst > 1 ? 1500 + 250 * worst : 0);
            if (best_ns < 0 || ns < best_ns) best_ns = ns, best_most = most;
            if (per_cta == 0 && (int64_t)chunks.size() > 12 * (int64_t)n_ctas) break;      // (many units: nothing to gain)
        }
        if (longest > 0) cut_even(best_most);
        tail.clear();
        queued = true;
    }
    bool cut_tail = n_ctas < kSaturatingCtas;
    int64_t shortest = 0;
    for (size_t i = warp_order.size(); i-- > 0 && shortest < tail_target && !cut_tail;) {
        const int64_t t = tiles_of(units[(size_t)warp_order[i]].n_keys, kWarpCost.gran);
        shortest += t;
        cut_tail = t * n_ctas * kShortUnitShareDen > warp_tiles * kShortUnitShareNum;
    }
    int64_t decode_tiles = 0;
    for (int id : ids_warp)
        if (units[(size_t)id].u.ntok == 1) decode_tiles += tiles_of(units[(size_t)id].n_keys, kWarpCost.gran);
    cut_tail = cut_tail || 2 * decode_tiles < warp_tiles;      // (spans on the warp body: not measured without)
    if (!even) cut(cut_tail);
    // Two fifths of the limit were chosen when the span CTAs had a margin of 88 and the limit came out that much higher. Where
    // pieces of that length leave no queue, they are taken: a CTA that comes from span tiles passes through the warp
    // body's start and end (3 us) to find a queue empty.  (us of attention a layer, with a queue | without: 4 sequences of 4/2
    // heads over 5-7 K keys, one with 75 tokens, 41 pieces on 40 CTAs 29.3 | 26.1; 23 of 4/2 heads with 2-44 tokens 30.3 | 23.2.)
    if (!even && used > 0 && chunks.size() + tail.size() > (size_t)(n_ctas - used) && warp_order.size() <= (size_t)(n_ctas - used)) {
        const int64_t shorter = bulk_max;
        bulk_max = longest_piece(hi * 88 / span_margin64(head_dim));
        cut(cut_tail);
        if (chunks.size() + tail.size() > (size_t)(n_ctas - used)) {
            bulk_max = shorter;
            cut(cut_tail);
        }
    }
    if (!even && !cut_tail && chunks.size() > (size_t)(n_ctas - used)) {      // (else every CTA has one to begin with and nothing is left)
        std::vector<int64_t> joins;
        for (int k = 0; k < used; ++k) joins.push_back(ctas[(size_t)k].load);
        int64_t mean = 0;
        queue_up();
        const int64_t whole = queue_ns(chunks, joins, n_ctas, model, &mean);
        // (Span CTAs join at times of their own, which evens the waves out better than modelled: where a gain of 6 to 11 % of the
        // mean was predicted, cutting was 1 to 7 % slower; where 20 %, 6 % faster.)
        const int64_t cut_ns = std::max(model.stream.cut_ns, used > 0 ? mean / 8 : 0);
        if (whole - mean > cut_ns) {
            const std::vector<Item> uncut(chunks);
            cut(true);
            queue_up();
            if (whole - queue_ns(chunks, joins, n_ctas, model, &mean) <= cut_ns) {
                chunks = uncut;
                for (int id : warp_order) units[(size_t)id].u.n_chunks = 1;
                for (const Item& it : chunks) units[(size_t)it.unit].u.n_chunks = std::max(units[(size_t)it.unit].u.n_chunks, it.chunk + 1);
            }
        }
    }
    int64_t partial_rows = 0;
    for (const UnitBuild& ub : units)
        if (ub.partial()) partial_rows += (int64_t)ub.u.n_chunks * ub.u.ntok;
    if (partial_rows > max_partial_rows) return false;
    if (!queued) queue_up();

    // ---- emit: warp-body items first (one start chunk for every CTA without span work, then the
    // queue), then the span items grouped by CTA
    cta_indptr_warp.assign((size_t)n_ctas + 1, 0);
    cta_indptr_tensor.assign((size_t)n_ctas + 1, 0);
    const int n_start = (int)std::min<size_t>(chunks.size(), (size_t)(n_ctas - used));
    items.reserve(chunks.size() + pieces_out.size());
    item_cta.reserve(chunks.size() + pieces_out.size());
    for (size_t i = 0; i < chunks.size(); ++i) {
        items.push_back(chunks[i]);
        item_cta.push_back(i < (size_t)n_start ? used + (int32_t)i : -1);
    }
    for (int k = 0; k <= n_ctas; ++k)
        cta_indptr_warp[(size_t)k] = std::min(std::max(k - used, 0), n_start);
    *queue_first = n_start;
    *queue_count = (int32_t)chunks.size() - n_start;
    const int32_t first = (int32_t)items.size();
    std::stable_sort(pieces_out.begin(), pieces_out.end(), [](const Piece& x, const Piece& y) { return x.cta < y.cta; });
    std::vector<int32_t> count((size_t)n_ctas, 0);
    for (const Piece& pz : pieces_out) {
        items.push_back(pz.it);
        item_cta.push_back(pz.cta);
        count[(size_t)pz.cta]++;
    }
    int32_t at = first;
    for (int k = 0; k < n_ctas; ++k) {
        cta_indptr_tensor[(size_t)k] = at;
        at += count[(size_t)k];
    }
    cta_indptr_tensor[(size_t)n_ctas] = at;
    return true;
}

// What a plan may have beyond the ordinary one.
struct PlanExtra {
    const asynclm_prefix_group* groups = nullptr;
    int32_t n_groups = 0;
    const asynclm_sparse* sparse = nullptr;
};

// Sequences next to each other in the batch that share their first `tokens` keys: the units of `first` hold these for all rows
// [row0, row0 + rows).
struct Run {
    int32_t first, tokens, row0, rows, seqs;
};

// Selected pages: a chunk of scores is a multiple of these pages (16 for each warp of a CTA), about so many for an SM.  (us of bounds, selection and attention,
// chunks of 64 | 128 | 192 | 256 | 320 pages: 4 sequences of 16-60 K tokens 39.7 | 37.8 | 37.6 | 38.7 | 39.8, 48 of 3-12 K with 1-4 new tokens 120 | 114 |
// 113 | 112 | 113, 150 of 0.3-9 K at 8/2 heads of 64 43.5 | 43.8 | 43.6 | 45.9 | 47.3; the rule takes 128, 192 and 128.)
constexpr int kSelectChunkUnit = 64, kSelectChunksPerSm = 8;

// Rows of a kv head (G * q_len) up to which a sequence always shares its prefix.  Longer spans' items are bound by the products, of which sharing
// saves none, and their partial rows are many, but their prefixes are cut by keys and evened out where they share it: for batches with such spans the planner
// compares the ways by their modelled time.  (us of attention, unshared | shared by sequences of up to 128 rows | 512 | 1024 | 4096, 32/8 heads of 128 but
// for the third: 30 sequences with 6 spans of 4-100 tokens 103 | 127 | 84 | 84 | 84; 8 spans of 100-200 177 | 179 | 119 | 104 | 109; 40 with 8 of 20-200 at
// head_dim 64 134 | 124 | 112 | 93 | 93; 30 with 3 of 300-600 193 | 267 | 266 | 265 | 193; 6 of 250-500 alone 151 | 151 | 152 | 152 | 184; 4 prompts of
// 500-1500 358-389 | 358 | 358 | 358 | 358, and 496 if all share.)
constexpr int64_t kMostSharedRows = 1024;
// Where short sequences alone share nothing (single tokens between long spans, which end their runs, or long spans alone), all share if the model has that take less
// by a sixteenth: it makes too much of the time of long spans, and more of it where they share nothing.  (us, unshared | all share, and the model's ratio, 32/8 heads of
// 128: 10 single tokens and 10 spans of 300 in turn behind 16 000 keys 802 | 779, 0.93, over the 8-bit cache 1197 | 1233, 0.91; 20 and 20 of 257 behind 8000 908 |
// 766, 0.91; 2 and 2 of 300 behind 30 000 498 | 339, 0.51; 6 of 300 behind 4096 151 | 189, 0.97; 3 and 3 of 600 behind 3008, 8 bits, 180 | 205, 0.98;
// 4 and 4 of 300 behind 2000, 8 bits, 132 | 122, 0.77, at head_dim 64 66 | 69, 0.95.)
constexpr int kSharedMargin = 16;
// Sharing costs partial rows and the join behind the attention; it has to save as many bytes of K and V as cross the bus in this time.
constexpr int64_t kLeastSavedNs = 2500;

// The runs of the groups (checked: ASYNCLM_OK, or what is wrong with them) of sequences with up to most_rows rows, and shared[b], 1 + sequence b's run or 0.
int find_runs(const PlanExtra& extra, const asynclm_batch& batch, int B, int page, int group, int64_t bytes_per_key, bool all, int64_t most_rows,
              std::vector<Run>& runs, std::vector<int32_t>& shared) {
    runs.clear();
    shared.assign((size_t)B, 0);
    int end = 0;
    int64_t saved = 0;
    for (int g = 0; g < extra.n_groups; ++g) {
        const asynclm_prefix_group& x = extra.groups[g];
        if (x.first_seq < end || x.n_seqs < 1 || x.n_seqs > B - x.first_seq || x.prefix_tokens < 0 || x.prefix_tokens % page != 0 || x.reserved != 0)
            return ASYNCLM_ERR_INVALID_ARG;
        end = x.first_seq + x.n_seqs;
        const size_t n_pages = (size_t)(x.prefix_tokens / page);
        const int32_t* pages = nullptr;      // of the first sequence that has new tokens
        bool open = false;                   // the last run may go on
        for (int b = x.first_seq; b < end; ++b) {
            const int ql = batch.q_indptr[b + 1] - batch.q_indptr[b];
            if (ql == 0) continue;
            if (batch.kv_len_before[b] < x.prefix_tokens) return ASYNCLM_ERR_INVALID_ARG;
            const int32_t* own = batch.page_indices + batch.page_indptr[b];
            if (pages == nullptr) pages = own;
            else if (n_pages > 0 && std::memcmp(pages, own, n_pages * sizeof(int32_t)) != 0) return ASYNCLM_ERR_PAGE_TABLE;
            if (n_pages == 0 || (int64_t)ql * group > most_rows) {
                open = false;
                continue;
            }
            if (!open) runs.push_back(Run{b, x.prefix_tokens, batch.q_indptr[b], 0, 0});
            open = true;
            runs.back().rows += ql;
            ++runs.back().seqs;
            shared[(size_t)b] = (int32_t)runs.size();
        }
    }
    for (Run& r : runs) {
        if (r.seqs < 2) r.tokens = 0;
        saved += (int64_t)(r.seqs - 1) * r.tokens * bytes_per_key;
    }
    if (saved == 0 || (!all && saved * 1000 / kDramBytesPerUs < kLeastSavedNs)) runs.clear();
    for (int32_t& at : shared) at = at > 0 && !runs.empty() && runs[(size_t)at - 1].tokens > 0 ? at : 0;
    return ASYNCLM_OK;
}

int make_plan(const asynclm_shape* shape, const asynclm_plan_options* opts, const asynclm_batch* batch, const PlanExtra& extra, void* host_ws,
              size_t host_bytes, void* dev_ws, size_t dev_bytes, void* stream, asynclm_plan_t** out_plan) {
    int rc = check_shape(shape);
    if (rc != ASYNCLM_OK) return rc;
    if (!batch || !host_ws || !out_plan || batch->batch < 0) return ASYNCLM_ERR_INVALID_ARG;
    if (((uintptr_t)host_ws & 15) != 0 || ((uintptr_t)dev_ws & 255) != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    const int B = batch->batch;
    if (B > 0 && (!batch->q_indptr || !batch->kv_len_before || !batch->page_indptr))
        return ASYNCLM_ERR_INVALID_ARG;
    if (opts && (opts->kv_chunk_tokens < 0 || opts->num_sms < 0 || opts->tensor_min_rows < 0))
        return ASYNCLM_ERR_INVALID_ARG;
    if (opts && opts->kv_chunk_tokens > 0 && opts->kv_chunk_tokens % 64 != 0)
        return ASYNCLM_ERR_INVALID_ARG;
    const bool host_only = dev_ws == nullptr;
    if (host_only && !(opts && opts->num_sms > 0)) return ASYNCLM_ERR_INVALID_ARG;

    int device = -1;
    if (!host_only) {
        if (cudaGetDevice(&device) != cudaSuccess) return ASYNCLM_ERR_CUDA;
        int major = 0;
        if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess)
            return ASYNCLM_ERR_CUDA;
        if (major != 10) return ASYNCLM_ERR_ARCH;
    }
    int n_sms = 0;
    rc = resolve_num_sms(opts, !host_only, &n_sms);
    if (rc != ASYNCLM_OK) return rc;

    const int Hkv = shape->num_kv_heads;
    const int G = shape->num_q_heads / Hkv;
    const int P = shape->page_size;

    // ---- validation -------------------------------------------------------------------------
    static const int32_t zero_indptr[1] = {0};
    const int32_t* q_indptr = B > 0 ? batch->q_indptr : zero_indptr;
    const int32_t* page_indptr = B > 0 ? batch->page_indptr : zero_indptr;
    if (q_indptr[0] != 0 || page_indptr[0] != 0) return ASYNCLM_ERR_INVALID_ARG;
    int64_t total_kv = 0;
    for (int b = 0; b < B; ++b) {
        const int64_t ql = (int64_t)q_indptr[b + 1] - q_indptr[b];
        const int64_t np = (int64_t)page_indptr[b + 1] - page_indptr[b];
        if (ql < 0 || np < 0 || batch->kv_len_before[b] < 0) return ASYNCLM_ERR_INVALID_ARG;
        const int64_t n = (int64_t)batch->kv_len_before[b] + ql;
        if (n > INT32_MAX - kKvTile) return ASYNCLM_ERR_INVALID_ARG;
        if (ql > 0) {
            if (np * P < n) return ASYNCLM_ERR_PAGE_TABLE;
            total_kv += n;
        }
    }
    const int T = q_indptr[B];
    const int64_t total_pages = page_indptr[B];
    if (total_pages > 0 && !batch->page_indices) return ASYNCLM_ERR_INVALID_ARG;
    for (int b = 0; b < B; ++b) {
        const int64_t ql = (int64_t)q_indptr[b + 1] - q_indptr[b];
        if (ql == 0) continue;   // paused sequences are not read or written: their ids are not checked
        const int64_t need = ((int64_t)batch->kv_len_before[b] + ql + P - 1) / P;
        // (as unsigned numbers, the negative ids are the largest; no exit inside the loop, so that it runs in vectors)
        const int32_t* ids = batch->page_indices + page_indptr[b];
        const uint32_t end = (uint32_t)std::min<int64_t>(shape->num_pages, (int64_t)INT32_MAX + 1);
        uint32_t bad = 0;
        for (int64_t j = 0; j < need; ++j) bad |= (uint32_t)((uint32_t)ids[j] >= end);
        if (bad) return ASYNCLM_ERR_PAGE_TABLE;
    }
    if (opts && (opts->flags & ASYNCLM_PLAN_REJECT_ALIASED_WRITES)) {
        std::vector<int32_t> written;
        for (int b = 0; b < B; ++b) {
            const int ql = q_indptr[b + 1] - q_indptr[b];
            if (ql == 0) continue;
            const int lo = batch->kv_len_before[b] / P;
            const int hi = (batch->kv_len_before[b] + ql - 1) / P;
            for (int j = lo; j <= hi; ++j) written.push_back(batch->page_indices[page_indptr[b] + j]);
        }
        std::sort(written.begin(), written.end());
        if (std::adjacent_find(written.begin(), written.end()) != written.end())
            return ASYNCLM_ERR_PAGE_TABLE;
    }

    // ---- what is shared, what is selected --------------------------------------------------------
    const bool kv8 = opts && (opts->flags & ASYNCLM_PLAN_KV8);
    const int64_t bytes_per_key = (int64_t)Hkv * (kv8 ? 2 * ((int64_t)shape->head_dim + 1) : 4 * (int64_t)shape->head_dim);
    std::vector<Run> runs;
    std::vector<int32_t> shared;      // 1 + the sequence's run, or 0
    const bool share_all = opts && (opts->flags & ASYNCLM_PLAN_SHARE_ALL);
    auto share = [&](int64_t most_rows) { return find_runs(extra, *batch, B, P, G, bytes_per_key, share_all, most_rows, runs, shared); };
    if (extra.n_groups > 0) {
        rc = share(share_all ? INT64_MAX : kMostSharedRows);
        if (rc != ASYNCLM_OK) return rc;
    }
    auto run_of = [&](int b) { return shared.empty() ? -1 : shared[(size_t)b] - 1; };
    const asynclm_sparse* sparse = extra.sparse;
    const int64_t n_select = sparse ? (int64_t)T * Hkv * sparse->budget_pages : 0;
    std::vector<SelectChunk> select_chunks;
    std::vector<int64_t> select_base;
    int64_t select_keys = 0;      // scores of one kv head
    int32_t chunk_pages = kSelectChunkUnit, most_pages = 0;
    if (sparse) {
        auto pages_of = [&](int r, int b) { return (batch->kv_len_before[b] + (r - q_indptr[b])) / P + 1; };
        // Rows that have more pages than the budget are scored, as many together as a chunk takes (they read the same bounds).
        struct Group { int seq, row0, rows, pages; };
        std::vector<Group> groups;
        int64_t scored = 0;
        select_base.reserve((size_t)T);
        for (int b = 0; b < B; ++b)
            for (int r = q_indptr[b]; r < q_indptr[b + 1]; ++r) {
                const int pages = pages_of(r, b);
                select_base.push_back(select_keys);
                if (pages <= sparse->budget_pages) continue;
                select_keys += pages;
                most_pages = std::max(most_pages, pages);
                if (r > q_indptr[b] && !groups.empty() && groups.back().row0 + groups.back().rows == r && groups.back().rows < kSelectQueries / G) {
                    ++groups.back().rows;
                    scored += pages - groups.back().pages;
                    groups.back().pages = pages;
                } else {
                    groups.push_back(Group{b, r, 1, pages});
                    scored += pages;
                }
            }
        const int64_t chunks = (int64_t)kSelectChunksPerSm * n_sms;
        chunk_pages = (int32_t)std::min<int64_t>(std::max<int64_t>((scored * Hkv + chunks * kSelectChunkUnit - 1) / (chunks * kSelectChunkUnit), 1) * kSelectChunkUnit, 1 << 24);
        for (const Group& g : groups)
            for (int64_t j = 0; j < g.pages; j += chunk_pages)
                select_chunks.push_back(SelectChunk{g.row0, g.rows, (int32_t)j, batch->kv_len_before[g.seq] + (g.row0 - q_indptr[g.seq]), page_indptr[g.seq], {0, 0, 0}});
        if ((int64_t)select_chunks.size() * Hkv > INT32_MAX || (int64_t)T * Hkv > INT32_MAX || total_pages + n_select > (int64_t)1 << 40)
            return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
    }

    // ---- units ------------------------------------------------------------------------------
    const bool tensor_wanted = !sparse && !(opts && (opts->flags & ASYNCLM_PLAN_NO_TENSOR_PATH));
    const int tensor_min_rows =
        (opts && opts->tensor_min_rows > 0) ? opts->tensor_min_rows : default_tensor_min_rows(shape->head_dim);
    const int TQ = tensor_tile_tokens(G);
    const int fixed_chunk = opts ? opts->kv_chunk_tokens : 0;
    const int ctas_cuda = n_sms * kCudaSlotsPerSm;
    const int ctas_tensor = n_sms;
    std::vector<UnitBuild> units;
    std::vector<int> ids_cuda, ids_tensor;
    std::vector<Item> items;
    std::vector<int32_t> item_cta, cta_indptr_cuda, cta_indptr_tensor;
    int n_items_cuda = 0;
    int32_t queue_first = 0, queue_count = 0;
    std::vector<int32_t> split_units, merge_blocks;   // merge block: 4 (token, head) rows of a split unit
    int64_t partial_rows = 0;
    int64_t limit_ns = 0;             // the load limit that the cuts were made for: the step's modelled time
    // (too_many: the cuts leave more than max_partial_rows partial rows, and nothing is dealt)
    bool too_many = false;
    auto deal = [&](const CutPolicy& policy, bool tensor_on, int64_t max_partial_rows) -> int {
        units.clear(); ids_cuda.clear(); ids_tensor.clear(); items.clear(); item_cta.clear();
        units.reserve(std::min<size_t>((size_t)std::min(B, T) * Hkv, 65536));
        ids_cuda.reserve(units.capacity());
        split_units.clear(); merge_blocks.clear();
        n_items_cuda = queue_first = queue_count = 0;
        partial_rows = 0;
        int64_t read_keys = total_kv;      // keys the step has to read, each (sequence, kv head) counted once
        for (size_t k = 0; k < runs.size(); ++k) {
            const Run& run = runs[k];
            if (run.tokens == 0) continue;
            read_keys -= (int64_t)(run.seqs - 1) * run.tokens;
            const bool tensor = tensor_on && (int64_t)G * run.rows >= tensor_min_rows;
            const int step = tensor ? TQ : warp_unit_tokens(G);
            for (int h = 0; h < Hkv; ++h) {
                for (int t0 = 0; t0 < run.rows; t0 += step) {
                    UnitBuild ub{};
                    ub.u.seq = run.first;
                    ub.u.kv_head = h;
                    ub.u.q_row0 = run.row0 + t0;
                    ub.u.ntok = std::min(step, run.rows - t0);
                    ub.u.kv_limit0 = run.tokens;      // of every token: no item reaches beyond
                    ub.u.partial_base = -1;
                    ub.u.page_base = page_indptr[run.first];
                    ub.path = tensor ? kPathTensor : kPathCuda;
                    ub.n_keys = run.tokens;
                    ub.run = (int32_t)k;
                    ub.flat = true;
                    (tensor ? ids_tensor : ids_cuda).push_back((int)units.size());
                    units.push_back(ub);
                }
            }
        }
        if (sparse) {
            // A unit for every row and kv head, whose page list the selection writes: full pages, and the last one up to the row's own key.
            read_keys = 0;
            for (int b = 0; b < B; ++b)
                for (int r = q_indptr[b]; r < q_indptr[b + 1]; ++r) {
                    const int pos = batch->kv_len_before[b] + (r - q_indptr[b]);
                    const int pages = std::min(pos / P + 1, (int)sparse->budget_pages);
                    for (int h = 0; h < Hkv; ++h) {
                        UnitBuild ub{};
                        ub.u.seq = b;
                        ub.u.kv_head = h;
                        ub.u.q_row0 = r;
                        ub.u.ntok = 1;
                        ub.u.kv_limit0 = (pages - 1) * P + pos % P + 1;
                        ub.u.partial_base = -1;
                        ub.path = kPathCuda;
                        ub.n_keys = ub.u.kv_limit0;
                        ids_cuda.push_back((int)units.size());
                        units.push_back(ub);
                    }
                    read_keys += units.back().n_keys;
                }
        }
        for (int b = 0; b < B && !sparse; ++b) {
            const int ql = q_indptr[b + 1] - q_indptr[b];
            if (ql == 0) continue;
            const int run = run_of(b), front = run >= 0 ? runs[(size_t)run].tokens : 0;      // keys that the run holds
            const int ctx = batch->kv_len_before[b] - front;
            const bool tensor = tensor_on && (int64_t)G * ql >= tensor_min_rows;
            const int step = tensor ? TQ : warp_unit_tokens(G);
            for (int h = 0; h < Hkv; ++h) {
                for (int t0 = 0; t0 < ql; t0 += step) {
                    UnitBuild ub{};
                    ub.u.seq = b;
                    ub.u.kv_head = h;
                    ub.u.q_row0 = q_indptr[b] + t0;
                    ub.u.ntok = std::min(step, ql - t0);
                    ub.u.kv_limit0 = ctx + t0 + 1;
                    ub.u.n_chunks = 0;
                    ub.u.partial_base = -1;
                    ub.u.page_base = page_indptr[b] + front / P;
                    ub.path = tensor ? kPathTensor : kPathCuda;
                    ub.n_keys = (int64_t)ub.u.kv_limit0 + ub.u.ntok - 1;
                    ub.run = run;
                    (tensor ? ids_tensor : ids_cuda).push_back((int)units.size());
                    units.push_back(ub);
                }
            }
        }

        // ---- items and CTA assignment --------------------------------------------------------------
        if ((fixed_chunk > 0 && !sparse) || ctas_cuda != ctas_tensor) {
            cut_and_deal(ids_cuda, units, fixed_chunk, ctas_cuda, kCudaItemOverheadTiles, items,
                         cta_indptr_cuda, item_cta);
            n_items_cuda = (int)items.size();
            cut_and_deal(ids_tensor, units, fixed_chunk, ctas_tensor, kTensorItemOverheadTiles, items,
                         cta_indptr_tensor, item_cta);
        } else {
            too_many = !deal_dynamic(ids_tensor, ids_cuda, units, G, shape->head_dim, model_of(shape->head_dim, kv8), read_keys * bytes_per_key, ctas_cuda, policy,
                                     max_partial_rows, sparse != nullptr, &limit_ns, items, cta_indptr_cuda, cta_indptr_tensor, item_cta, &queue_first, &queue_count);
            if (too_many) return ASYNCLM_OK;
            n_items_cuda = queue_first + queue_count;
        }

        // ---- partial rows ------------------------------------------------------------------------
        for (size_t i = 0; i < units.size(); ++i) {
            if (units[i].partial()) {
                units[i].u.partial_base = (int32_t)partial_rows;
                partial_rows += (int64_t)units[i].u.n_chunks * units[i].u.ntok;
                if (partial_rows > INT32_MAX / 2) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
                if (units[i].run >= 0) continue;      // joined with the other unit of its rows, below
                split_units.push_back((int32_t)i);
                if (i >= (size_t)(INT32_MAX >> 6)) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
                // split units of the warp body are merged inside the attention kernel; those of the span
                // body by the merge kernel
                if (units[i].path == kPathTensor)
                    for (int rb = 0; rb * 4 < units[i].u.ntok * G; ++rb) merge_blocks.push_back((int32_t)((i << 6) | (size_t)rb));
            }
        }
        return ASYNCLM_OK;
    };
    // The fastest cuts, as long as their partial results fit the fixed array of asynclm_attn_mixed_static; else as
    // many of the long span units cut by keys as it has room for, none of them, long pieces in the queue as
    // well, and at head_dim 64 no span units at all (warp units have far fewer partial rows).  If nothing fits,
    // the fastest again: that call then refuses the plan.  A try that does not fit ends when its cuts are
    // known, before the items are sorted and dealt.
    int64_t static_rows = (int64_t)(ASYNCLM_STATIC_SCRATCH_BYTES / ((size_t)G * (shape->head_dim + 1) * sizeof(float)));
    while (partial_bytes(static_rows, G, shape->head_dim) > ASYNCLM_STATIC_SCRATCH_BYTES) --static_rows;
    auto fits_static = [&]() { return !too_many && partial_rows <= static_rows; };
    const CutPolicy fastest;
    if (extra.n_groups > 0 && !share_all && fixed_chunk == 0) {
        int64_t longest = 0;      // rows of a sequence in a group
        for (int g = 0; g < extra.n_groups; ++g)
            for (int b = extra.groups[g].first_seq; b < extra.groups[g].first_seq + extra.groups[g].n_seqs; ++b)
                longest = std::max<int64_t>(longest, (int64_t)(q_indptr[b + 1] - q_indptr[b]) * G);
        // (also where short sequences alone share nothing, as between long spans, which end their runs)
        if (longest > kMostSharedRows && (share(INT64_MAX), !runs.empty())) {
            // partial rows are written and read, past what the model has in its load limit
            int64_t best = -1, best_ns = 0;
            bool unshared = false;
            for (const int64_t most : {kMostSharedRows, INT64_MAX, (int64_t)0}) {
                (void)share(most);
                if (runs.empty() && unshared) continue;
                unshared = unshared || runs.empty();
                rc = deal(fastest, tensor_wanted, INT64_MAX);
                if (rc != ASYNCLM_OK) continue;
                const int64_t ns = limit_ns + partial_rows * G * (shape->head_dim + 1) * 8 * 1000 / kDramBytesPerUs;
                const int64_t margin = unshared && !runs.empty() ? best_ns / kSharedMargin : 0;
                if (best < 0 || ns < best_ns - margin) best = most, best_ns = ns;
            }
            (void)share(best < 0 ? 0 : best);
        }
    }
    // (rows that share a prefix have partial rows whatever the cuts: such a plan is not cut down for that array)
    rc = deal(fastest, tensor_wanted, runs.empty() ? static_rows : INT64_MAX);
    if (rc == ASYNCLM_OK && !fits_static() && runs.empty()) {
        if (fixed_chunk == 0) {
            int64_t span_rows = 0, span_units = 0, warp_rows = 0;
            for (const UnitBuild& ub : units) {
                const int64_t rows = ub.partial() ? (int64_t)ub.u.n_chunks * ub.u.ntok : 0;
                if (ub.path != kPathTensor) warp_rows += rows;
                else if (rows > 0 && !ub.flat) span_rows += rows, ++span_units;
            }
            const int64_t room = (int64_t)(ASYNCLM_STATIC_SCRATCH_BYTES / ((size_t)G * (shape->head_dim + 1) * sizeof(float))) - warp_rows;
            CutPolicy fewer;
            fewer.units_by_keys = room <= 0 ? 0 : (int)(span_units * room / std::max<int64_t>(1, span_rows) * 15 / 16);
            if (fewer.units_by_keys > 0) rc = deal(fewer, tensor_wanted, static_rows);
            if (rc == ASYNCLM_OK && !fits_static()) rc = deal(CutPolicy{0, true}, tensor_wanted, static_rows);
            if (rc == ASYNCLM_OK && !fits_static()) rc = deal(CutPolicy{0, false}, tensor_wanted, static_rows);
        }
        if (rc == ASYNCLM_OK && !fits_static() && tensor_wanted && shape->head_dim == 64)
            rc = deal(CutPolicy{0, false}, false, static_rows);
        if (rc == ASYNCLM_OK && !fits_static()) rc = deal(fastest, tensor_wanted, INT64_MAX);
    }
    if (rc != ASYNCLM_OK) return rc;
    const int n_items = (int)items.size();

    const int n_split = (int)split_units.size();

    // ---- rows of a run: the unit with the sequence's own keys beside the one with the shared keys ----
    std::vector<Join> joins;
    if (!runs.empty()) {
        std::vector<std::vector<int32_t>> flat(runs.size() * (size_t)Hkv);      // a run's units with its prefix, by rows
        for (size_t i = 0; i < units.size(); ++i)
            if (units[i].flat) flat[(size_t)units[i].run * Hkv + units[i].u.kv_head].push_back((int32_t)i);
        for (const UnitBuild& own : units) {
            if (own.run < 0 || own.flat) continue;
            for (int32_t id : flat[(size_t)own.run * Hkv + own.u.kv_head]) {
                const Unit& pre = units[(size_t)id].u;
                const int r0 = std::max(own.u.q_row0, pre.q_row0), r1 = std::min(own.u.q_row0 + own.u.ntok, pre.q_row0 + pre.ntok);
                if (r0 >= r1) continue;
                if (joins.size() >= (size_t)(INT32_MAX / kJoinRows)) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
                for (int k = 0; k < (r1 - r0) * G; k += kJoinRows)
                    joins.push_back(Join{r0, k, (r1 - r0) * G, own.u.kv_head, own.u.partial_base + r0 - own.u.q_row0, own.u.ntok, own.u.n_chunks,
                                         pre.partial_base + r0 - pre.q_row0, pre.ntok, pre.n_chunks, {0, 0}});
            }
        }
    }

    // CTAs without an item, which stand at the end, have something to do only where there is a queue: else they are not
    // launched, and their headers (384 bytes each, of which a small plan mostly consists) are neither cleared nor uploaded.
    int grid_cuda = ctas_cuda, grid_tensor = ctas_tensor;
    if (queue_count == 0 && ctas_cuda == ctas_tensor) {
        auto idle = [&](int c) { return cta_indptr_cuda[(size_t)c] == cta_indptr_cuda[(size_t)c + 1] && cta_indptr_tensor[(size_t)c] == cta_indptr_tensor[(size_t)c + 1]; };
        while (grid_cuda > 1 && idle(grid_cuda - 1)) --grid_cuda;
        grid_tensor = grid_cuda;
    }

    // ---- pack ---------------------------------------------------------------------------------
    BlobLayout L = layout_blob(B, T, total_pages, (int64_t)units.size(), n_items, grid_cuda,
                               grid_tensor, (int64_t)n_split, (int64_t)merge_blocks.size(), (int64_t)joins.size(),
                               (int64_t)select_chunks.size(), (int64_t)select_base.size());
    const size_t plan_bytes = align_up(sizeof(asynclm_plan_s), 256);
    const size_t item_cta_bytes = align_up(sizeof(int32_t) * (size_t)std::max(n_items, 1), 256);
    const size_t shift_bytes = runs.empty() ? 0 : align_up(sizeof(int32_t) * units.size(), 256);
    const size_t host_need = plan_bytes + L.blob_bytes + item_cta_bytes + shift_bytes;
    // behind the blob: partial rows, then a selection's error bounds, page lists and scores
    const size_t off_error = L.blob_bytes + partial_bytes(partial_rows, G, shape->head_dim);
    const size_t off_select = off_error + (sparse ? align_up(sizeof(float) * (size_t)T * Hkv, 256) : 0);
    const size_t off_keys = off_select + align_up(sizeof(int32_t) * (size_t)n_select, 256);
    const size_t off_exact = off_keys + align_up(sizeof(uint32_t) * (size_t)select_keys * Hkv, 256);
    const size_t dev_need = off_exact + align_up(sizeof(uint64_t) * (size_t)select_keys * Hkv, 256);
    // the lists as indices of the page table: 2^31 of them are 8 GB
    const int64_t select_at = ((int64_t)off_select - (int64_t)L.off_page_indices) / (int64_t)sizeof(int32_t);
    if (sparse && select_at + n_select > INT32_MAX) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
    if (host_bytes < host_need) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;
    if (!host_only && dev_bytes < dev_need) return ASYNCLM_ERR_WORKSPACE_TOO_SMALL;

    char* hb = (char*)host_ws + plan_bytes;
    std::memset(hb + L.off_status, 0, 256);
    std::memset(hb + L.off_arrivals, 0, sizeof(int32_t) * std::max<size_t>(units.size(), 1));
    if (B > 0) {
        std::memcpy(hb + L.off_q_indptr, q_indptr, sizeof(int32_t) * (size_t)(B + 1));
        std::memcpy(hb + L.off_kv_len, batch->kv_len_before, sizeof(int32_t) * (size_t)B);
        std::memcpy(hb + L.off_page_indptr, page_indptr, sizeof(int32_t) * (size_t)(B + 1));
    } else {
        std::memset(hb + L.off_q_indptr, 0, sizeof(int32_t));
        std::memset(hb + L.off_page_indptr, 0, sizeof(int32_t));
    }
    if (total_pages > 0)
        std::memcpy(hb + L.off_page_indices, batch->page_indices, sizeof(int32_t) * (size_t)total_pages);
    int32_t* row_seq = (int32_t*)(hb + L.off_row_seq);
    int64_t* row_slot = (int64_t*)(hb + L.off_row_slot);
    for (int b = 0; b < B; ++b)
        for (int r = q_indptr[b]; r < q_indptr[b + 1]; ++r) {
            row_seq[r] = b;
            const int pos = batch->kv_len_before[b] + (r - q_indptr[b]);
            row_slot[r] = (int64_t)batch->page_indices[page_indptr[b] + pos / P] * P + pos % P;
        }
    Unit* h_units = (Unit*)(hb + L.off_units);
    for (size_t i = 0; i < units.size(); ++i) {
        if (sparse) units[i].u.page_base = (int32_t)(select_at + ((int64_t)units[i].u.q_row0 * Hkv + units[i].u.kv_head) * sparse->budget_pages);
        h_units[i] = units[i].u;
    }
    if (n_items > 0) std::memcpy(hb + L.off_items, items.data(), sizeof(Item) * (size_t)n_items);
    int32_t* h_heads = (int32_t*)(hb + L.off_heads);
    std::memset(h_heads, 0, sizeof(int32_t) * kHeadWords * (size_t)std::max(grid_cuda, grid_tensor));
    Work* h_works = (Work*)(hb + L.off_works);
    for (int i = 0; i < n_items; ++i) {
        const Item& it = items[(size_t)i];
        const Unit& u = units[(size_t)it.unit].u;
        Work w;
        w.kv0 = it.kv0;
        w.kv_end = std::min(it.kv1, u.kv_limit0 + u.ntok - 1);
        w.q_row0 = u.q_row0;
        w.ntok = u.ntok;
        w.kv_limit0 = u.kv_limit0;
        w.kv_head = u.kv_head;
        w.partial_row0 = u.partial_base < 0 ? -1 : u.partial_base + it.chunk * u.ntok;
        w.page0 = u.page_base + it.kv0 / kPage;
        w.unit = it.unit;
        w.n_chunks = units[(size_t)it.unit].run >= 0 ? 0 : u.n_chunks;      // 0: the attention kernel merges none of them
        w.partial_base = u.partial_base;
        w.q_seq0 = q_indptr[u.seq];
        h_works[i] = w;
    }
    for (int c = 0; c < std::max(grid_cuda, grid_tensor); ++c) {
        int32_t* h = h_heads + (size_t)c * kHeadWords;
        const int32_t range[4] = {c < grid_tensor ? cta_indptr_tensor[(size_t)c] : 0,
                                  c < grid_tensor ? cta_indptr_tensor[(size_t)c + 1] : 0,
                                  c < grid_cuda ? cta_indptr_cuda[(size_t)c] : 0,
                                  c < grid_cuda ? cta_indptr_cuda[(size_t)c + 1] : 0};
        std::memcpy(h, range, sizeof(range));
        for (int path = 0; path < 2; ++path) {
            const int first = range[2 * path], last = range[2 * path + 1];
            if (first >= last) continue;
            const Work& w = h_works[first];
            std::memcpy(h + (path == 0 ? kHeadWorkTensor : kHeadWorkCuda), &w, sizeof(Work));
            const int npg = (w.kv_end - w.kv0 + kPage - 1) / kPage;
            for (int k = 0; k < 32 && k < npg && !sparse; ++k)      // (selected pages are not known yet)
                h[(path == 0 ? kHeadPagesTensor : kHeadPagesCuda) + k] = batch->page_indices[w.page0 + k];
        }
    }
    std::memcpy(hb + L.off_cta_cuda, cta_indptr_cuda.data(), sizeof(int32_t) * (size_t)(grid_cuda + 1));
    std::memcpy(hb + L.off_cta_tensor, cta_indptr_tensor.data(),
                sizeof(int32_t) * (size_t)(grid_tensor + 1));
    if (n_split > 0) std::memcpy(hb + L.off_split, split_units.data(), sizeof(int32_t) * split_units.size());
    if (!merge_blocks.empty())
        std::memcpy(hb + L.off_merge, merge_blocks.data(), sizeof(int32_t) * merge_blocks.size());
    if (!joins.empty()) std::memcpy(hb + L.off_joins, joins.data(), sizeof(Join) * joins.size());
    if (!select_chunks.empty()) {
        std::memcpy(hb + L.off_select_chunks, select_chunks.data(), sizeof(SelectChunk) * select_chunks.size());
        std::memcpy(hb + L.off_select_base, select_base.data(), sizeof(int64_t) * select_base.size());
    }
    int32_t* h_item_cta = (int32_t*)(hb + L.blob_bytes);
    int32_t* h_shift = runs.empty() ? nullptr : (int32_t*)(hb + L.blob_bytes + item_cta_bytes);
    for (size_t i = 0; i < units.size() && h_shift; ++i)
        h_shift[i] = units[i].flat ? -1 : units[i].run >= 0 ? runs[(size_t)units[i].run].tokens : 0;
    if (n_items > 0) std::memcpy(h_item_cta, item_cta.data(), sizeof(int32_t) * (size_t)n_items);

    asynclm_plan_s* plan = (asynclm_plan_s*)host_ws;
    std::memset(plan, 0, sizeof(*plan));
    plan->magic = kPlanMagic;
    plan->shape = *shape;
    plan->device = device;
    plan->host_only = host_only ? 1 : 0;
    plan->h_units = h_units;
    plan->h_items = (const Item*)(hb + L.off_items);
    plan->h_item_cta = h_item_cta;
    plan->h_q_indptr = (const int32_t*)(hb + L.off_q_indptr);
    plan->h_unit_shift = h_shift;
    plan->h_units_path_split = n_items_cuda;
    plan->shared = runs.empty() ? 0 : 1;
    plan->sparse = sparse ? 1 : 0;
    for (int b = 0; b < B; ++b) plan->max_q_len = std::max(plan->max_q_len, q_indptr[b + 1] - q_indptr[b]);

    char* db = (char*)dev_ws;
    DevPlan& d = plan->dev;
    auto dp = [&](size_t off) { return host_only ? nullptr : (void*)(db + off); };
    d.status = (int32_t*)dp(L.off_status);
    d.counters = (int32_t*)dp(L.off_status + 64);
    d.queue_first = queue_first;
    d.queue_count = queue_count;
    d.q_indptr = (const int32_t*)dp(L.off_q_indptr);
    d.kv_len_before = (const int32_t*)dp(L.off_kv_len);
    d.page_indptr = (const int32_t*)dp(L.off_page_indptr);
    d.page_indices = (const int32_t*)dp(L.off_page_indices);
    d.row_seq = (const int32_t*)dp(L.off_row_seq);
    d.row_slot = (const int64_t*)dp(L.off_row_slot);
    d.units = (const Unit*)dp(L.off_units);
    d.items = (const Item*)dp(L.off_items);
    d.works = (const Work*)dp(L.off_works);
    d.cta_heads = (const int32_t*)dp(L.off_heads);
    d.cta_indptr_cuda = (const int32_t*)dp(L.off_cta_cuda);
    d.cta_indptr_tensor = (const int32_t*)dp(L.off_cta_tensor);
    d.split_units = (const int32_t*)dp(L.off_split);
    d.merge_blocks = (const int32_t*)dp(L.off_merge);
    d.unit_arrivals = (int32_t*)dp(L.off_arrivals);
    d.partial_o = (float*)dp(L.blob_bytes);
    d.partial_lse = (float*)dp(L.blob_bytes + align_up((size_t)partial_rows * (size_t)G *
                                                           (size_t)shape->head_dim * sizeof(float), 256));
    d.joins = (const Join*)dp(L.off_joins);
    d.num_join_blocks = (int32_t)joins.size();
    d.total_pages = total_pages;
    if (sparse) {
        d.select_chunks = (const SelectChunk*)dp(L.off_select_chunks);
        d.select_base = (const int64_t*)dp(L.off_select_base);
        d.select_pages = (int32_t*)dp(off_select);
        d.select_keys = (unsigned*)dp(off_keys);
        d.select_exact = (unsigned long long*)dp(off_exact);
        d.select_error = (unsigned*)dp(off_error);
        d.num_select_chunks = (int32_t)select_chunks.size();
        d.select_chunk_pages = chunk_pages;
        d.select_most_pages = most_pages;
        d.select_budget = sparse->budget_pages;
        d.select_first = sparse->first_pages;
        d.select_last = sparse->last_pages;
    }
    d.batch = B;
    d.total_q = T;
    d.num_units = (int32_t)units.size();
    d.num_items = n_items;
    d.num_items_cuda = n_items_cuda;
    d.num_items_tensor = n_items - n_items_cuda;
    d.num_split_units = n_split;
    d.num_merge_blocks = (int32_t)merge_blocks.size();
    d.num_ctas_cuda = grid_cuda;
    d.num_ctas_tensor = grid_tensor;
    d.num_q_heads = shape->num_q_heads;
    d.num_kv_heads = Hkv;
    d.head_dim = shape->head_dim;
    d.group = G;
    d.num_pages = shape->num_pages;
    // at least the smallest normal number: the kernels flush smaller ones to zero, and the span body scales masked
    // scores (-inf) as well
    d.sm_scale = shape->sm_scale > 0.f ? std::max(shape->sm_scale, FLT_MIN) : 1.0f / sqrtf((float)shape->head_dim);

    asynclm_plan_info& info = plan->info;
    info.total_q = T;
    info.num_units = d.num_units;
    info.num_items = n_items;
    info.num_split_units = d.num_split_units;
    info.partial_rows = (int32_t)partial_rows;
    int max_chunk = 0;
    for (const Item& it : items) max_chunk = std::max(max_chunk, it.kv1 - it.kv0);
    info.kv_chunk_tokens = fixed_chunk > 0 ? fixed_chunk : (d.num_split_units ? max_chunk : INT32_MAX);
    info.num_ctas_cuda = grid_cuda;
    info.num_ctas_tensor = grid_tensor;
    info.num_items_tensor = d.num_items_tensor;
    info.launches_append = T > 0 ? 1 : 0;
    // span tiles and decode rows share one fused launch when a step has both
    info.launches_attn = ((n_items_cuda > 0 || d.num_items_tensor > 0) ? 1 : 0) + (merge_blocks.empty() ? 0 : 1) + (joins.empty() ? 0 : 1);
    info.num_sms = n_sms;
    info.total_kv_tokens = total_kv;
    info.device_bytes_used = dev_need;
    info.host_bytes_used = host_need;

    if (!host_only) {
        // By kernel where the workspace is page-locked, so that kernels can read it, and the plan neither so small that the
        // copy engine is as fast nor so large that the bus is what takes the time.
        const void* by_kernel = L.blob_bytes >= kUploadMinBytes && L.blob_bytes <= kUploadMaxBytes ? page_locked_on_device(hb, L.blob_bytes) : nullptr;
        cudaError_t e = by_kernel ? upload_plan(db, by_kernel, L.blob_bytes, (cudaStream_t)stream)
                                  : cudaMemcpyAsync(db, hb, L.blob_bytes, cudaMemcpyHostToDevice, (cudaStream_t)stream);
        if (int rc = cuda_status(e)) return rc;
        // (no call may find anything but pages of the pool in the lists)
        if (sparse && T > 0) e = cudaMemsetAsync(db + off_error, 0, off_keys - off_error, (cudaStream_t)stream);
        if (int rc = cuda_status(e)) return rc;
        plan->fresh = by_kernel ? 1 : 0;
    }
    *out_plan = plan;
    return ASYNCLM_OK;
}

// The planner's lists grow with the batch; no exception passes a C entry.
template <typename... Args>
int plan_or_error(const Args&... args) {
    try {
        return make_plan(args...);
    } catch (const std::exception&) {      // (bad_alloc, or length_error: nothing else is thrown)
        return ASYNCLM_ERR_MEMORY;
    }
}

}  // namespace

extern "C" int asynclm_plan(const asynclm_shape* shape, const asynclm_plan_options* opts,
                            const asynclm_batch* batch, void* host_ws, size_t host_bytes,
                            void* dev_ws, size_t dev_bytes, void* stream,
                            asynclm_plan_t** out_plan) {
    return plan_or_error(shape, opts, batch, PlanExtra{}, host_ws, host_bytes, dev_ws, dev_bytes, stream, out_plan);
}

extern "C" int asynclm_plan_prefix(const asynclm_shape* shape, const asynclm_plan_options* opts, const asynclm_batch* batch,
                                   const asynclm_prefix_group* groups, int32_t n_groups, void* host_ws, size_t host_bytes, void* dev_ws,
                                   size_t dev_bytes, void* stream, asynclm_plan_t** out_plan) {
    if (n_groups < 0 || (n_groups > 0 && !groups)) return ASYNCLM_ERR_INVALID_ARG;
    PlanExtra extra;
    extra.groups = groups;
    extra.n_groups = n_groups;
    return plan_or_error(shape, opts, batch, extra, host_ws, host_bytes, dev_ws, dev_bytes, stream, out_plan);
}

extern "C" int asynclm_plan_sparse(const asynclm_shape* shape, const asynclm_plan_options* opts, const asynclm_batch* batch, const asynclm_sparse* sparse,
                                   void* host_ws, size_t host_bytes, void* dev_ws, size_t dev_bytes, void* stream, asynclm_plan_t** out_plan) {
    if (!sparse || sparse->first_pages < 0 || sparse->last_pages < 1 || sparse->reserved != 0 ||
        (int64_t)sparse->first_pages + sparse->last_pages > sparse->budget_pages || (opts && opts->kv_chunk_tokens != 0))
        return ASYNCLM_ERR_INVALID_ARG;
    PlanExtra extra;
    extra.sparse = sparse;
    return plan_or_error(shape, opts, batch, extra, host_ws, host_bytes, dev_ws, dev_bytes, stream, out_plan);
}

extern "C" int asynclm_plan_get_info(const asynclm_plan_t* plan, asynclm_plan_info* info) {
    if (!plan || !info || plan->magic != kPlanMagic) return ASYNCLM_ERR_INVALID_ARG;
    *info = plan->info;
    return ASYNCLM_OK;
}

extern "C" int asynclm_plan_get_shape(const asynclm_plan_t* plan, asynclm_shape* shape, int32_t* batch, int32_t* total_q) {
    if (!plan || !shape || !batch || !total_q || plan->magic != kPlanMagic) return ASYNCLM_ERR_INVALID_ARG;
    *shape = plan->shape;
    *batch = plan->dev.batch;
    *total_q = plan->dev.total_q;
    return ASYNCLM_OK;
}

extern "C" int asynclm_plan_get_sparse(const asynclm_plan_t* plan, asynclm_sparse* sparse) {
    if (!plan || !sparse || plan->magic != kPlanMagic || !plan->sparse) return ASYNCLM_ERR_INVALID_ARG;
    *sparse = asynclm_sparse{plan->dev.select_budget, plan->dev.select_first, plan->dev.select_last, 0};
    return ASYNCLM_OK;
}

extern "C" int asynclm_plan_get_items(const asynclm_plan_t* plan, asynclm_item_view* out,
                                      int32_t capacity) {
    if (!plan || plan->magic != kPlanMagic || capacity < 0 || (capacity > 0 && !out))
        return ASYNCLM_ERR_INVALID_ARG;
    const int n = plan->dev.num_items;
    for (int i = 0; i < n && i < capacity; ++i) {
        const Item& it = plan->h_items[i];
        const Unit& u = plan->h_units[it.unit];
        asynclm_item_view v;
        v.seq = u.seq;
        v.kv_head = u.kv_head;
        const int32_t shift = plan->h_unit_shift ? plan->h_unit_shift[it.unit] : 0;
        v.tok0 = u.q_row0 - plan->h_q_indptr[u.seq];
        v.ntok = u.ntok;
        v.kv0 = it.kv0 + std::max(shift, 0);
        v.kv1 = it.kv1 + std::max(shift, 0);
        v.path = i < plan->h_units_path_split ? kPathCuda : kPathTensor;
        v.cta = plan->h_item_cta[i];
        out[i] = v;
    }
    return n;
}
