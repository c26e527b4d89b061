// C-ABI layer of the latent-cache operators: contexts, plans (host integers and their device image), launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <string>
#include <vector>

#include "capi_util.h"
#include "latent_kernels.h"
#include "taper_internal.h"
#include "taper_plan.h"

using taper::align_up;
using taper::aligned;
using taper::guarded;
using taper::hip_error;
using taper::OnDevice;
using taper::set_error;

namespace {

// Memory of a plan: a pinned image and, on the device, that image followed by the calls' workspace.  Handed back to the context
// when the plan is freed, so that a steady decode loop allocates nothing.
struct Buffers {
    void *dev = nullptr, *staging = nullptr, *staging_dev = nullptr;
    size_t dev_bytes = 0, staging_bytes = 0;
    hipEvent_t uploaded = nullptr;
};

void destroy(Buffers& b) {
    if (b.uploaded) {
        (void)hipEventSynchronize(b.uploaded);
        (void)hipEventDestroy(b.uploaded);
    }
    if (b.dev) (void)hipFree(b.dev);
    if (b.staging) (void)hipHostFree(b.staging);
    b = Buffers();
}

}  // namespace

struct taper_latent_ctx {
    taper_latent_config cfg;
    int units = 256;  // compute units
    std::vector<Buffers> free_buffers;
};

struct taper_latent_plan {
    taper_latent_ctx* ctx = nullptr;
    bool prompt = false;
    taper::HostPlan batch;
    int64_t device_bytes = 0;
    // decode
    std::vector<taper_latent_item> items;
    std::vector<int32_t> piece_start, piece_row;
    int64_t n_partial_rows = 0;
    // prompt
    std::vector<taper::PromptTile> tiles, merges;
    std::vector<int32_t> e_page, e_valid, e_low;
    int32_t n_low = 0;
    int64_t n_rows = 0;
    int heads_at_once = 0;
    // device
    Buffers buf;
    taper::LatentDecodeArgs dargs;
    taper::PromptArgs pargs;
};

namespace {

taper::LatentShape shape_of(const taper_latent_config& c) { return {c.n_heads, c.latent_dim, c.head_dim, c.scale * 1.4426950408889634f}; }

int acquire(taper_latent_ctx* ctx, size_t image, size_t total, Buffers* out) {
    size_t best = ctx->free_buffers.size();
    for (size_t i = 0; i < ctx->free_buffers.size(); ++i) {
        const Buffers& b = ctx->free_buffers[i];
        if (b.staging_bytes >= image && b.dev_bytes >= total && (best == ctx->free_buffers.size() || b.dev_bytes < ctx->free_buffers[best].dev_bytes)) best = i;
    }
    if (best < ctx->free_buffers.size()) {
        const hipError_t e = hipEventSynchronize(ctx->free_buffers[best].uploaded);  // the pinned image is about to be overwritten
        if (e != hipSuccess) return hip_error(e, "hipEventSynchronize");
        *out = ctx->free_buffers[best];
        ctx->free_buffers.erase(ctx->free_buffers.begin() + best);
        return TAPER_OK;
    }
    Buffers b;
    b.staging_bytes = align_up(image + image / 2, 4096);
    b.dev_bytes = align_up(total + total / 4, 4096);  // (head-room: the next step's plan is a little larger)
    hipError_t e = hipHostMalloc(&b.staging, b.staging_bytes, hipHostMallocDefault);
    if (e == hipSuccess) e = hipHostGetDevicePointer(&b.staging_dev, b.staging, 0);
    if (e == hipSuccess) e = hipMalloc(&b.dev, b.dev_bytes);
    if (e == hipSuccess) e = hipEventCreateWithFlags(&b.uploaded, hipEventDisableTiming);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        destroy(b);
        return set_error(TAPER_ENOMEM, std::string("plan allocation of ") + std::to_string(total) + " bytes: " + hipGetErrorString(e));
    }
    *out = b;
    return TAPER_OK;
}

// The pieces of a plan's device memory, in order; those without a source are workspace.
class Layout {
  public:
    void add(const void* src, size_t bytes) {
        pieces_.push_back({src, bytes, total_});
        total_ = align_up(total_ + std::max<size_t>(bytes, 16), 256);
    }
    size_t total() const { return total_; }
    void* at(void* base, int i) const { return (char*)base + pieces_[i].off; }
    void write(void* staging) const {
        for (const Piece& p : pieces_)
            if (p.src && p.bytes) std::memcpy((char*)staging + p.off, p.src, p.bytes);
    }

  private:
    struct Piece {
        const void* src;
        size_t bytes, off;
    };
    std::vector<Piece> pieces_;
    size_t total_ = 0;
};

int upload(taper_latent_plan* plan, const Layout& lay, size_t image, hipStream_t s) {
    if (taper::recording(s)) return set_error(TAPER_EINVAL, "a plan cannot be built on a stream that is being recorded");
    const int st = acquire(plan->ctx, image, lay.total(), &plan->buf);
    if (st != TAPER_OK) return st;
    lay.write(plan->buf.staging);
    HIP_TRY(taper::launch_upload(plan->buf.dev, plan->buf.staging_dev, image, nullptr, 0, s));
    HIP_TRY(hipEventRecord(plan->buf.uploaded, s));
    return TAPER_OK;
}

constexpr size_t kMostBlocks = (size_t)1 << 22;  // of a launch (which has fewer than 2^32 threads)

// ---------------------------------------------------------------------------- decode plan
// What some tokens cost: their tiles, at the price of the rows they meet (measured: a tile of 16 rows takes 3.1 us when all units
// stream from memory, one of 64 rows 2.6 us where the L2 has it, a little more than the former where it has not).
constexpr int kTile = taper::kLatentTileTokens, kRows = taper::kLatentTileRows;
double tile_cost(int rows) { return rows <= 64 ? 1.0 : rows <= 96 ? 1.2 : 1.5; }
// of an item beside its tiles: its first tile's way from memory, its queries in, its partial rows out
double start_cost(int rows) { return 2.5 + rows * (2.0 / 128); }
constexpr int kMostPieces = 64;    // of a segment, about: a row's pieces are merged by some lanes of one workgroup

struct Span {
    int seq0, page0, n_tokens, row0, n_rows;
};

// How spans are cut: into stretches that take `big` of a unit's equal share, and the last `small_share` of each into ones 1 / small_part
// as long.  The long ones start first, and the short ones even out what is left.
struct CutRule {
    double big, small_share;
    int small_part;
};
// (of these the one that ends soonest: the first suits short spans, an item a unit, the second spans of all lengths, the others few
// long ones)
constexpr CutRule kCutRules[] = {{1.2, 0.0, 1}, {0.4, 0.0, 1}, {0.5, 0.3, 3}, {1.0, 0.4, 6}};
constexpr int kXcds = 8;

struct DecodeItems {
    std::vector<taper_latent_item> items;
    std::vector<int> list[kXcds];  // of each XCD, in the order in which its workgroups start
    int64_t rows = 0;
    double time = 0;  // when the last unit ends, in tiles
};

double item_cost(const taper_latent_item& it) { return (it.n_tokens + kTile - 1) / kTile * tile_cost(it.n_rows) + start_cost(it.n_rows); }

void cut_spans(const std::vector<Span>& spans, int page_size, int units, double total, const CutRule& rule, DecodeItems* out) {
    struct Unit {
        double cost;
        int first, n;
    };
    std::vector<Unit> stretches;
    const double share = total / units * rule.big;
    for (const Span& s : spans) {
        const int tiles = (s.n_tokens + kTile - 1) / kTile, least = std::max(1, tiles * 2 / kMostPieces);
        const int widest = std::min(s.n_rows, kRows), big = std::max({least, 2, (int)((share - start_cost(widest)) / tile_cost(widest))});
        int t = 0, n_small = 0;
        if (tiles > big && rule.small_part > 1) n_small = std::max(std::max(least, big / rule.small_part), (int)(tiles * rule.small_share));
        while (t < tiles) {
            const int left = tiles - n_small - t;  // before the short ones
            const int size = left > 0 ? big : std::max({least, big / rule.small_part, 2});
            const int n = left > 0 ? (left + size - 1) / size : (tiles - t + size - 1) / size;  // equal stretches
            const int t1 = t + ((left > 0 ? left : tiles - t) + n - 1) / n;
            const int tok0 = t * kTile, tok1 = std::min(s.n_tokens, t1 * kTile);
            // the row tiles of one stretch of tokens stay on one XCD, whose L2 then serves all but the first of them
            Unit u = {0, (int)out->items.size(), 0};
            for (int r = 0; r < s.n_rows; r += kRows) {
                out->items.push_back({s.seq0, s.page0 + tok0 / page_size, tok1 - tok0, s.row0 + r, std::min(kRows, s.n_rows - r), (int32_t)(out->rows + r)});
                u.cost += item_cost(out->items.back());
                ++u.n;
                if (u.cost > total / (2 * kXcds) || r + kRows >= s.n_rows) {
                    stretches.push_back(u);
                    u = {0, (int)out->items.size(), 0};
                }
            }
            out->rows += s.n_rows;
            t = t1;
        }
    }
    std::stable_sort(stretches.begin(), stretches.end(), [](const Unit& x, const Unit& y) { return x.cost * y.n > y.cost * x.n; });
    double load[kXcds] = {0};
    for (const Unit& u : stretches) {
        const int x = (int)(std::min_element(load, load + kXcds) - load);
        load[x] += u.cost;
        for (int i = 0; i < u.n; ++i) out->list[x].push_back(u.first + i);
    }
    std::vector<double> busy;
    for (const auto& l : out->list) {
        busy.assign(std::max(1, units / kXcds), 0.0);
        for (int i : l) {
            std::pop_heap(busy.begin(), busy.end(), std::greater<double>());
            busy.back() += item_cost(out->items[i]);
            std::push_heap(busy.begin(), busy.end(), std::greater<double>());
        }
        out->time = std::max(out->time, *std::max_element(busy.begin(), busy.end()));
    }
}

void make_decode_items(const taper_latent_config& cfg, int units, taper_latent_plan* plan) {
    const taper::HostPlan& b = plan->batch;
    const int H = cfg.n_heads;
    std::vector<Span> spans;
    for (int g = 0; g < b.n_groups; ++g) {
        const int s0 = b.group_start[g], s1 = b.group_start[g + 1];
        if (b.prefix_len[s0] > 0) spans.push_back({s0, 0, b.prefix_len[s0], s0 * H, (s1 - s0) * H});
        for (int s = s0; s < s1; ++s)
            for (int k = b.seg_start[s]; k < b.seg_start[s + 1]; ++k)
                if (b.seg_len[k] > 0) spans.push_back({s, b.seg_page0[k], b.seg_len[k], s * H, H});
    }
    double total = 0;
    for (const Span& s : spans) {
        const int full = s.n_rows / kRows, rest = s.n_rows % kRows;
        const double each = full * tile_cost(kRows) + (rest ? tile_cost(rest) : 0.0);
        total += (s.n_tokens + kTile - 1) / kTile * each + full * start_cost(kRows) + (rest ? start_cost(rest) : 0.0);
    }
    DecodeItems best;
    for (const CutRule& rule : kCutRules) {
        DecodeItems d;
        cut_spans(spans, cfg.page_size, units, total, rule, &d);
        if (best.items.empty() || d.time < 0.98 * best.time) std::swap(best, d);
    }
    // the pieces of each sequence's rows: one for every stretch that holds tokens of it
    plan->n_partial_rows = best.rows;
    plan->piece_start.assign(b.n_seqs + 1, 0);
    auto each_piece = [&](auto f) {
        for (const taper_latent_item& it : best.items)
            for (int q = (it.row0 + H - 1) / H; q * H < it.row0 + it.n_rows; ++q) f(q, it.part_row + q * H - it.row0);  // the item with head 0's row
    };
    each_piece([&](int q, int) { plan->piece_start[q + 1]++; });
    for (int s = 0; s < b.n_seqs; ++s) plan->piece_start[s + 1] += plan->piece_start[s];
    plan->piece_row.resize(plan->piece_start[b.n_seqs]);
    std::vector<int32_t> at(plan->piece_start.begin(), plan->piece_start.end() - 1);
    each_piece([&](int q, int row) { plan->piece_row[at[q]++] = row; });
    // workgroup i runs on XCD i mod 8
    size_t longest = 0;
    for (const auto& l : best.list) longest = std::max(longest, l.size());
    for (size_t i = 0; i < longest; ++i)
        for (int x = 0; x < kXcds; ++x) plan->items.push_back(i < best.list[x].size() ? best.items[best.list[x][i]] : taper_latent_item{0, 0, 0, 0, 0, 0});
}

int build_decode(taper_latent_ctx* ctx, int n_seqs, const int32_t* block_table, int stride, const int32_t* group, const int32_t* prefix,
                 const int32_t* seg_start, const int32_t* seg_len, int64_t n_pool_pages, int target_workgroups, hipStream_t s,
                 taper_latent_plan* plan) {
    const taper_latent_config& cfg = ctx->cfg;
    std::vector<int32_t> one;
    if (!seg_start && n_seqs > 0) {
        one.resize((size_t)n_seqs + 1);
        for (int i = 0; i <= n_seqs; ++i) one[i] = i;
        seg_start = one.data();
    }
    const int st = taper::resolve_batch(cfg.page_size, n_seqs, block_table, stride, group, prefix, seg_start, seg_len, n_pool_pages, &plan->batch);
    if (st != TAPER_OK) return st;
    // (32 threads a row, 16 sequences a workgroup of the grid's second axis: a launch takes less than 2^32 and 2^16)
    if ((int64_t)n_seqs * cfg.n_heads > (1 << 26) || n_seqs > 16 * 65535) return set_error(TAPER_EINVAL, "too many query rows");
    make_decode_items(cfg, target_workgroups > 0 ? std::min(target_workgroups, 1 << 16) : ctx->units, plan);
    if (plan->n_partial_rows > INT32_MAX || plan->items.size() > kMostBlocks) return set_error(TAPER_EINVAL, "too many query rows");
    const int KD = cfg.latent_dim + cfg.rope_dim;
    Layout lay;
    lay.add(plan->batch.block_table.data(), plan->batch.block_table.size() * 4);
    lay.add(plan->items.data(), plan->items.size() * sizeof(taper_latent_item));
    lay.add(plan->piece_start.data(), plan->piece_start.size() * 4);
    lay.add(plan->piece_row.data(), plan->piece_row.size() * 4);
    const size_t image = lay.total();
    lay.add(nullptr, (size_t)n_seqs * cfg.n_heads * KD * 2);
    lay.add(nullptr, (size_t)n_seqs * cfg.n_heads * cfg.latent_dim * 2);
    lay.add(nullptr, (size_t)plan->n_partial_rows * sizeof(taper::PartStats));
    lay.add(nullptr, (size_t)plan->n_partial_rows * cfg.latent_dim * 2);
    plan->device_bytes = (int64_t)lay.total();
    if (cfg.device < 0) return TAPER_OK;
    const int su = upload(plan, lay, image, s);
    if (su != TAPER_OK) return su;
    void* d = plan->buf.dev;
    taper::LatentDecodeArgs& a = plan->dargs;
    std::memset(&a, 0, sizeof a);
    a.bt = (const int32_t*)lay.at(d, 0);
    a.items = (const taper_latent_item*)lay.at(d, 1);
    a.piece_start = (const int32_t*)lay.at(d, 2);
    a.piece_row = (const int32_t*)lay.at(d, 3);
    a.q_lat = lay.at(d, 4);
    a.q_rest = lay.at(d, 5);
    a.stats = (taper::PartStats*)lay.at(d, 6);
    a.part = lay.at(d, 7);
    a.bt_stride = stride;
    a.n_seqs = n_seqs;
    a.n_items = (int32_t)plan->items.size();
    return TAPER_OK;
}

// ---------------------------------------------------------------------------- prompt plan
constexpr int kPromptRows = 256;
constexpr int64_t kMostExpandedBytes = (int64_t)4 << 30;  // of the heads expanded at a time

constexpr int kLeastPiecePages = 16;  // a piece's start and its partial rows cost about as much as so many pages
constexpr int kMostBundle = 8;        // items side by side: what an XCD's 32 compute units hold of four heads
constexpr double kBundleLeast = 0.75;  // the shortest of them, relative to the longest (shorter ones are better kept for the end)

// From the row tiles (in the order of their sequences' rows) to items: tiles with more than a unit's equal share of the keys are cut into
// pieces; items that meet the same keys at the same time are bundled; the longest bundles come first.
void make_prompt_items(int units, taper_latent_plan* plan) {
    std::vector<taper::PromptTile> rows;
    rows.swap(plan->tiles);
    int64_t pages = 0;
    for (const taper::PromptTile& t : rows) pages += t.page_end;
    const int64_t share = std::max<int64_t>(kLeastPiecePages, (pages * plan->heads_at_once + units - 1) / units);
    std::vector<std::vector<taper::PromptTile>> bundles;
    size_t e = rows.size();
    while (e > 0) {  // from the longest tile of a sequence down
        const int longest = rows[e - 1].page_end, n_pieces = (int)((longest + share - 1) / share);
        size_t i = e - 1;
        while (i > 0 && e - i < (size_t)kMostBundle && rows[i - 1].suffix_e == rows[e - 1].suffix_e && rows[i - 1].page_end > kBundleLeast * longest) --i;
        const int per = ((longest + n_pieces - 1) / n_pieces + 3) / 4 * 4;
        for (size_t j = i; j < e; ++j) {
            taper::PromptTile& t = rows[j];
            t.n_pieces = (t.page_end + per - 1) / per;
            if (t.n_pieces == 1) continue;
            t.part_row = (int32_t)plan->n_partial_rows;
            plan->n_partial_rows += (int64_t)t.n_pieces * t.n_rows;
            plan->merges.push_back(t);
        }
        for (int k = 0; k < n_pieces; ++k) {
            std::vector<taper::PromptTile> bundle;
            for (size_t j = i; j < e; ++j) {
                taper::PromptTile t = rows[j];
                if (k >= t.n_pieces) continue;
                if (t.n_pieces > 1) t.part_row += k * t.n_rows;
                t.page_begin = k * per;
                t.page_end = std::min(t.page_end, (k + 1) * per);
                bundle.push_back(t);
            }
            if (!bundle.empty()) bundles.push_back(bundle);
        }
        e = i;
    }
    std::stable_sort(bundles.begin(), bundles.end(), [](const std::vector<taper::PromptTile>& x, const std::vector<taper::PromptTile>& y) {
        return x.back().page_end - x.back().page_begin > y.back().page_end - y.back().page_begin;
    });
    for (const auto& bundle : bundles) {
        const int32_t first = (int32_t)plan->tiles.size();
        for (taper::PromptTile t : bundle) {
            t.bundle = first;
            t.n_bundle = (int32_t)bundle.size();
            plan->tiles.push_back(t);
        }
    }
}

int build_prompt(taper_latent_ctx* ctx, int n_seqs, const int32_t* block_table, int stride, const int32_t* group, const int32_t* prefix,
                 const int32_t* suffix, const int32_t* new_len, int64_t n_pool_pages, hipStream_t s, taper_latent_plan* plan) {
    const taper_latent_config& cfg = ctx->cfg;
    std::vector<int32_t> one((size_t)n_seqs + 1);
    for (int i = 0; i <= n_seqs; ++i) one[i] = i;
    const int st = taper::resolve_batch(cfg.page_size, n_seqs, block_table, stride, group, prefix, one.data(), suffix, n_pool_pages, &plan->batch);
    if (st != TAPER_OK) return st;
    const taper::HostPlan& b = plan->batch;
    const int P = cfg.page_size;
    plan->prompt = true;
    for (int q = 0; q < n_seqs; ++q) {
        if (new_len[q] < 0 || new_len[q] > suffix[q])
            return set_error(TAPER_ELEN, "sequence " + std::to_string(q) + ": new_len must lie between 0 and its private tokens");
        plan->n_rows += new_len[q];
    }
    if (plan->n_rows == 0) return set_error(TAPER_ELEN, "no sequence has a new token");
    if (plan->n_rows > INT32_MAX / cfg.n_heads) return set_error(TAPER_ELEN, "too many query rows");
    auto expand = [&](int seq, int entry0, int n_tokens, int position) {  // (of the first token)
        const int at = (int)plan->e_page.size();
        for (int j = 0; j * P < n_tokens; ++j) {
            plan->e_page.push_back(b.block_table[(size_t)seq * stride + entry0 + j]);
            plan->e_valid.push_back(std::min(P, n_tokens - j * P));
            plan->e_low.push_back(position + j * P < taper::kLowPositions ? plan->n_low++ : -1);
        }
        if (plan->e_page.size() % 2) {  // pages go in pairs: one without tokens
            plan->e_page.push_back(plan->e_page.back());
            plan->e_valid.push_back(0);
            plan->e_low.push_back(-1);
        }
        return at;
    };
    int row0 = 0;
    for (int g = 0; g < b.n_groups; ++g) {
        int prefix_e = -1;
        for (int q = b.group_start[g]; q < b.group_start[g + 1]; ++q) {
            const int pl = prefix[q], n = new_len[q], npre = b.n_prefix_pages[q];
            if (n == 0) continue;
            if (prefix_e < 0) prefix_e = expand(q, 0, pl, 0);
            const int suffix_e = expand(q, npre, suffix[q], pl);
            for (int r = 0; r < n; r += kPromptRows) {
                taper::PromptTile t;
                t.row0 = row0 + r;
                t.n_rows = std::min(kPromptRows, n - r);
                t.first_pos = pl + suffix[q] - n + r;
                t.prefix_len = pl;
                t.prefix_e = prefix_e;
                t.suffix_e = suffix_e;
                t.page_begin = 0;
                t.page_end = (npre + 1) / 2 * 2 + (t.first_pos + t.n_rows - pl + P - 1) / P;
                t.part_row = -1;
                t.n_pieces = 1;
                plan->tiles.push_back(t);
            }
            row0 += n;
        }
    }
    const int64_t head_bytes = (int64_t)plan->e_page.size() * P * 2 * cfg.head_dim * 2;
    plan->heads_at_once = (int)std::max<int64_t>(1, std::min<int64_t>(cfg.n_heads, kMostExpandedBytes / head_bytes));
    if (plan->heads_at_once > 8) plan->heads_at_once -= plan->heads_at_once % 8 && plan->heads_at_once < cfg.n_heads ? plan->heads_at_once % 8 : 0;
    make_prompt_items(ctx->units, plan);
    if ((int64_t)std::max(plan->tiles.size(), plan->e_page.size()) * plan->heads_at_once > (int64_t)kMostBlocks || plan->n_partial_rows * plan->heads_at_once > INT32_MAX) return set_error(TAPER_ELEN, "too many query rows");
    Layout lay;
    lay.add(plan->e_page.data(), plan->e_page.size() * 4);
    lay.add(plan->e_valid.data(), plan->e_valid.size() * 4);
    lay.add(plan->e_low.data(), plan->e_low.size() * 4);
    lay.add(plan->tiles.data(), plan->tiles.size() * sizeof(taper::PromptTile));
    lay.add(plan->merges.data(), plan->merges.size() * sizeof(taper::PromptTile));
    const size_t image = lay.total();
    const int64_t n_chunks = ((int64_t)plan->e_page.size() + 3) / 4;
    lay.add(nullptr, (size_t)head_bytes * plan->heads_at_once);
    lay.add(nullptr, (size_t)n_chunks * plan->heads_at_once * 8);
    lay.add(nullptr, (size_t)plan->n_low * plan->heads_at_once * P * cfg.head_dim * 2);
    lay.add(nullptr, (size_t)plan->n_partial_rows * plan->heads_at_once * sizeof(float2));
    lay.add(nullptr, (size_t)plan->n_partial_rows * plan->heads_at_once * cfg.head_dim * sizeof(float));
    plan->device_bytes = (int64_t)lay.total();
    if (cfg.device < 0) return TAPER_OK;
    const int su = upload(plan, lay, image, s);
    if (su != TAPER_OK) return su;
    void* d = plan->buf.dev;
    taper::PromptArgs& a = plan->pargs;
    std::memset(&a, 0, sizeof a);
    a.e_page = (const int32_t*)lay.at(d, 0);
    a.e_valid = (const int32_t*)lay.at(d, 1);
    a.e_low = (const int32_t*)lay.at(d, 2);
    a.tiles = (const taper::PromptTile*)lay.at(d, 3);
    a.merges = (const taper::PromptTile*)lay.at(d, 4);
    a.kv = lay.at(d, 5);
    a.format = (int32_t*)lay.at(d, 6);
    a.k_low = lay.at(d, 7);
    a.ml = (float2*)lay.at(d, 8);
    a.part = (float*)lay.at(d, 9);
    a.n_low = plan->n_low;
    a.n_chunks = (int32_t)n_chunks;
    a.units = ctx->units;
    a.n_expanded = (int32_t)plan->e_page.size();
    a.n_tiles = (int32_t)plan->tiles.size();
    a.n_merges = (int32_t)plan->merges.size();
    a.n_partial_rows = (int32_t)plan->n_partial_rows;
    a.heads_at_once = plan->heads_at_once;
    return TAPER_OK;
}

template <typename Build>
int build_plan(taper_latent_ctx* ctx, taper_latent_plan** out_plan, Build&& build) {
    if (!ctx || !out_plan) return set_error(TAPER_EINVAL, "null argument");
    return guarded([&] {
        taper_latent_plan* plan = new taper_latent_plan();
        plan->ctx = ctx;
        int st = TAPER_OK;
        try {
            if (ctx->cfg.device >= 0) {
                OnDevice on(ctx->cfg.device);
                st = on.error == hipSuccess ? build(plan) : hip_error(on.error, "hipSetDevice");
            } else {
                st = build(plan);
            }
        } catch (...) {
            taper_latent_plan_free(plan);
            throw;
        }
        if (st != TAPER_OK) {
            const std::string keep = taper_last_error();
            taper_latent_plan_free(plan);
            return set_error(st, keep);
        }
        *out_plan = plan;
        return (int)TAPER_OK;
    });
}

int check_call(const taper_latent_ctx* ctx, const taper_latent_plan* plan, bool prompt, const void* q, const void* w_up, const void* pages,
               const void* out, const float* lse) {
    if (!ctx || !plan) return set_error(TAPER_EINVAL, "null ctx or plan");
    if (plan->ctx != ctx) return set_error(TAPER_EINVAL, "plan was built on another context");
    if (plan->prompt != prompt) return set_error(TAPER_EINVAL, prompt ? "not a prompt plan" : "not a decode plan");
    if (ctx->cfg.device < 0 || !plan->buf.dev) return set_error(TAPER_EHIP, "host-only context: no device work possible");
    if (!q || !w_up || !pages || !out) return set_error(TAPER_EINVAL, "null tensor pointer");
    if (!aligned(q, 16) || !aligned(w_up, 16) || !aligned(pages, 16) || !aligned(out, 16) || !aligned(lse, 4))
        return set_error(TAPER_EINVAL, "tensors must be 16-byte aligned");
    return TAPER_OK;
}

}  // namespace

extern "C" {

int taper_latent_create(const taper_latent_config* cfg, taper_latent_ctx** out_ctx) {
    if (!cfg || !out_ctx) return set_error(TAPER_EINVAL, "null argument");
    if (cfg->n_heads < 1 || cfg->n_heads > 256) return set_error(TAPER_EINVAL, "n_heads must be 1 to 256");
    if (cfg->latent_dim != 256 && cfg->latent_dim != 512) return set_error(TAPER_EINVAL, "latent_dim must be 256 or 512");
    if (cfg->rope_dim != taper::kRopeDim) return set_error(TAPER_EINVAL, "rope_dim must be 64");
    if (cfg->head_dim != 64 && cfg->head_dim != 128) return set_error(TAPER_EINVAL, "head_dim must be 64 or 128");
    if (cfg->page_size != 16) return set_error(TAPER_EINVAL, "page_size must be 16");
    if (!(cfg->scale > 0.0f) || !(cfg->scale < 1e30f)) return set_error(TAPER_EINVAL, "scale must be positive and finite");
    return guarded([&] {
        int units = 256;
        if (cfg->device >= 0) {
            int n = 0;
            if (hipGetDeviceCount(&n) != hipSuccess || cfg->device >= n) return set_error(TAPER_EHIP, "no such HIP device");
            HIP_TRY(hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, cfg->device));
        }
        taper_latent_ctx* ctx = new taper_latent_ctx();
        ctx->cfg = *cfg;
        ctx->units = std::max(1, units);
        *out_ctx = ctx;
        return (int)TAPER_OK;
    });
}

void taper_latent_destroy(taper_latent_ctx* ctx) {
    if (!ctx) return;
    if (ctx->cfg.device >= 0) {
        OnDevice on(ctx->cfg.device);
        (void)hipDeviceSynchronize();
        for (Buffers& b : ctx->free_buffers) destroy(b);
    }
    delete ctx;
}

int taper_latent_plan_build(taper_latent_ctx* ctx, int n_seqs, const int32_t* block_table, int bt_row_stride, const int32_t* branch_group,
                            const int32_t* prefix_len, const int32_t* seg_start, const int32_t* seg_len, int64_t n_pool_pages,
                            int target_workgroups, void* hip_stream, taper_latent_plan** out_plan) {
    return build_plan(ctx, out_plan, [&](taper_latent_plan* plan) {
        return build_decode(ctx, n_seqs, block_table, bt_row_stride, branch_group, prefix_len, seg_start, seg_len, n_pool_pages,
                            target_workgroups, (hipStream_t)hip_stream, plan);
    });
}

int taper_latent_prompt_plan_build(taper_latent_ctx* ctx, int n_seqs, const int32_t* block_table, int bt_row_stride, const int32_t* branch_group,
                                   const int32_t* prefix_len, const int32_t* suffix_len, const int32_t* new_len, int64_t n_pool_pages,
                                   void* hip_stream, taper_latent_plan** out_plan) {
    if (n_seqs < 1 || !suffix_len || !new_len) return set_error(TAPER_EINVAL, "null argument");
    return build_plan(ctx, out_plan, [&](taper_latent_plan* plan) {
        return build_prompt(ctx, n_seqs, block_table, bt_row_stride, branch_group, prefix_len, suffix_len, new_len, n_pool_pages,
                            (hipStream_t)hip_stream, plan);
    });
}

void taper_latent_plan_free(taper_latent_plan* plan) {
    if (!plan) return;
    if (plan->buf.dev) {
        try {
            plan->ctx->free_buffers.push_back(plan->buf);
        } catch (...) {  // (no room to remember them: given back to the device instead)
            OnDevice on(plan->ctx->cfg.device);
            (void)hipDeviceSynchronize();
            destroy(plan->buf);
        }
    }
    delete plan;
}

int taper_latent_plan_export(const taper_latent_plan* plan, taper_latent_view* v) {
    if (!plan || !v) return set_error(TAPER_EINVAL, "null argument");
    if (plan->prompt) return set_error(TAPER_EINVAL, "not a decode plan");
    v->n_seqs = plan->batch.n_seqs;
    v->n_groups = plan->batch.n_groups;
    v->n_items = (int32_t)plan->items.size();
    v->items = plan->items.data();
    v->piece_start = plan->piece_start.data();
    v->piece_row = plan->piece_row.data();
    v->n_partial_rows = plan->n_partial_rows;
    v->tokens_unique = plan->batch.tokens_unique;
    v->tokens_logical = plan->batch.tokens_logical;
    v->device_bytes = plan->device_bytes;
    return TAPER_OK;
}

int taper_latent_decode_step_attention(taper_latent_ctx* ctx, const taper_latent_plan* plan, const void* q, const void* w_up, const void* pages,
                                       void* out, float* lse, void* hip_stream) {
    const int st = check_call(ctx, plan, false, q, w_up, pages, out, lse);
    if (st != TAPER_OK) return st;
    OnDevice on(ctx->cfg.device);
    HIP_TRY(on.error);
    taper::LatentDecodeArgs a = plan->dargs;
    a.q = q;
    a.w_up = w_up;
    a.pages = pages;
    a.out = out;
    a.lse = lse;
    HIP_TRY(taper::launch_latent_decode(shape_of(ctx->cfg), a, (hipStream_t)hip_stream));
    return TAPER_OK;
}

int taper_latent_prompt_attention(taper_latent_ctx* ctx, const taper_latent_plan* plan, const void* q, const void* w_up, const void* pages,
                                  void* out, float* lse, void* hip_stream) {
    const int st = check_call(ctx, plan, true, q, w_up, pages, out, lse);
    if (st != TAPER_OK) return st;
    OnDevice on(ctx->cfg.device);
    HIP_TRY(on.error);
    taper::PromptArgs a = plan->pargs;
    a.q = q;
    a.w_up = w_up;
    a.pages = pages;
    a.out = out;
    a.lse = lse;
    HIP_TRY(taper::launch_latent_prompt(shape_of(ctx->cfg), a, (hipStream_t)hip_stream));
    return TAPER_OK;
}

int taper_latent_append(taper_latent_ctx* ctx, int64_t n_tokens, const void* latent, int64_t latent_stride, const void* rope, int64_t rope_stride,
                        const int64_t* slots, void* pages, int64_t n_pool_pages, void* hip_stream) {
    if (!ctx) return set_error(TAPER_EINVAL, "null argument");
    if (n_tokens < 0 || n_tokens > ((int64_t)1 << 31) || n_pool_pages < 1 || n_pool_pages > ((int64_t)1 << 31)) return set_error(TAPER_EINVAL, "bad argument");
    if (latent_stride < ctx->cfg.latent_dim || rope_stride < ctx->cfg.rope_dim || latent_stride % 8 || rope_stride % 8)
        return set_error(TAPER_EINVAL, "row strides must be multiples of 8 and hold a row");
    if (ctx->cfg.device < 0) return set_error(TAPER_EHIP, "host-only context: no device work possible");
    if (n_tokens == 0) return TAPER_OK;
    if (!latent || !rope || !slots || !pages) return set_error(TAPER_EINVAL, "null tensor pointer");
    if (!aligned(latent, 16) || !aligned(rope, 16) || !aligned(pages, 16) || !aligned(slots, 8)) return set_error(TAPER_EINVAL, "tensors must be 16-byte aligned");
    OnDevice on(ctx->cfg.device);
    HIP_TRY(on.error);
    HIP_TRY(taper::launch_latent_append(ctx->cfg.latent_dim, n_tokens, latent, latent_stride, rope, rope_stride, slots, pages,
                                        n_pool_pages * ctx->cfg.page_size, (hipStream_t)hip_stream));
    return TAPER_OK;
}

}  // extern "C"
