// Page pool (host integers) and mover (argument checks, lists of calls, launches).
#include "taper_pages.h"

#include <algorithm>
#include <cstring>
#include <mutex>
#include <unordered_map>
#include <vector>

#include "capi_util.h"
#include "pages_kernels.h"
#include "taper_internal.h"
#include "taper_plan.h"

using taper::align_up;
using taper::aligned;
using taper::guarded;
using taper::hip_error;
using taper::OnDevice;
using taper::recording;
using taper::set_error;

struct taper_page_pool {
    std::vector<int32_t> users;
    int64_t n_free = 0;
    int64_t first_free = 0;  // no page below it is free
};

// Lists of one call on the device, and the pinned image they come from.
struct MoveLists {
    void *dev = nullptr, *staging = nullptr, *staging_dev = nullptr;
    size_t bytes = 0;
    hipEvent_t done = nullptr;  // behind the kernel that reads them
};
constexpr int kListsInFlight = 4;

struct taper_mover {
    taper_page_format format;
    int64_t page_bytes = 0;
    std::mutex lock;
    MoveLists lists[kListsInFlight];
    int next = 0;
    std::vector<uint32_t> seen;  // per page: 2 * call (read) or 2 * call + 1 (written) of the last call that named it
    uint32_t call = 0;
};

namespace {

std::string at_entry(const char* what, int64_t i) { return std::string(what) + " at entry " + std::to_string(i); }

bool in_pool(const taper_page_pool* p, int32_t page) { return page >= 0 && page < (int64_t)p->users.size(); }

int check_layers(int n_layers, void* const* pools, int64_t n_pool_pages) {
    if (n_layers < 1 || !pools) return set_error(TAPER_EINVAL, "no pools");
    for (int l = 0; l < n_layers; ++l) {
        if (!pools[l]) return set_error(TAPER_EINVAL, "null pool pointer");
        if (!aligned(pools[l], 16)) return set_error(TAPER_EINVAL, "pools must be 16-byte aligned");
    }
    if (n_pool_pages < 1 || n_pool_pages > (int64_t)1 << 31) return set_error(TAPER_EINVAL, "n_pool_pages outside the int32 page id range");
    return TAPER_OK;
}

// Pages of this call: what it reads and what it writes must not meet.
void begin_call(taper_mover* m, int64_t n_pool_pages) {
    if ((int64_t)m->seen.size() < n_pool_pages) m->seen.resize(n_pool_pages, 0);
    if (++m->call >= 0x7fffffffu) {
        std::fill(m->seen.begin(), m->seen.end(), 0u);
        m->call = 1;
    }
}
int note_written(taper_mover* m, int32_t page) {
    if (m->seen[page] == 2 * m->call + 1) return set_error(TAPER_EINVAL, "page " + std::to_string(page) + " is a destination twice");
    m->seen[page] = 2 * m->call + 1;
    return TAPER_OK;
}
int note_read(taper_mover* m, int32_t page) {  // (after all written ones)
    if (m->seen[page] == 2 * m->call + 1) return set_error(TAPER_EINVAL, "page " + std::to_string(page) + " is a source and a destination");
    return TAPER_OK;
}

// The next lists, once the call that used them last has been through, with room for `bytes`.
int next_lists(taper_mover* m, size_t bytes, MoveLists** out) {
    MoveLists& l = m->lists[m->next];
    m->next = (m->next + 1) % kListsInFlight;
    if (l.done) HIP_TRY(hipEventSynchronize(l.done));
    if (l.bytes < bytes) {
        if (l.dev) (void)hipFree(l.dev);
        if (l.staging) (void)hipHostFree(l.staging);
        l.dev = l.staging = nullptr;
        l.bytes = 0;
        const size_t room = align_up(bytes + bytes / 2, 4096);
        hipError_t e = l.done ? hipSuccess : hipEventCreateWithFlags(&l.done, hipEventDisableTiming);
        if (e == hipSuccess) e = hipHostMalloc(&l.staging, room, hipHostMallocDefault);
        if (e == hipSuccess) e = hipHostGetDevicePointer(&l.staging_dev, l.staging, 0);
        if (e == hipSuccess) e = hipMalloc(&l.dev, room);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            return set_error(TAPER_ENOMEM, std::string("lists of a page move: ") + hipGetErrorString(e));
        }
        l.bytes = room;
    }
    *out = &l;
    return TAPER_OK;
}

template <typename Launch>
int for_layers(int n_layers, void* const* pools, Launch&& launch) {
    for (int l0 = 0; l0 < n_layers; l0 += taper::kLayersPerLaunch) {
        taper::PoolPointers p;
        std::memset(&p, 0, sizeof p);
        const int n = std::min(taper::kLayersPerLaunch, n_layers - l0);
        for (int l = 0; l < n; ++l) p.base[l] = pools[l0 + l];
        HIP_TRY(launch(p, n));
    }
    return TAPER_OK;
}

}  // namespace

extern "C" {

int taper_page_pool_create(int64_t n_pages, taper_page_pool** out_pool) {
    if (!out_pool || n_pages < 1 || n_pages > (int64_t)1 << 31) return set_error(TAPER_EINVAL, "bad argument");
    return guarded([&] {
        taper_page_pool* p = new taper_page_pool();
        try {
            p->users.assign((size_t)n_pages, 0);
        } catch (...) {
            delete p;
            throw;
        }
        p->n_free = n_pages;
        *out_pool = p;
        return (int)TAPER_OK;
    });
}

void taper_page_pool_destroy(taper_page_pool* pool) { delete pool; }

int64_t taper_page_pool_free_pages(const taper_page_pool* pool) { return pool ? pool->n_free : -1; }

int32_t taper_page_pool_users(const taper_page_pool* pool, int32_t page) { return pool && in_pool(pool, page) ? pool->users[page] : -1; }

int taper_page_pool_alloc(taper_page_pool* pool, int64_t n, int32_t* pages) {
    if (!pool || n < 0 || (n > 0 && !pages)) return set_error(TAPER_EINVAL, "bad argument");
    if (n > pool->n_free) return guarded([&] { return set_error(TAPER_ENOMEM, std::to_string(n) + " pages wanted, " + std::to_string(pool->n_free) + " are free"); });
    for (int64_t i = 0; i < n; ++i) {
        while (pool->users[pool->first_free] != 0) ++pool->first_free;
        pages[i] = (int32_t)pool->first_free;
        pool->users[pool->first_free++] = 1;
    }
    pool->n_free -= n;
    return TAPER_OK;
}

int taper_page_pool_share(taper_page_pool* pool, int64_t n, const int32_t* pages) {
    if (!pool || n < 0 || (n > 0 && !pages)) return set_error(TAPER_EINVAL, "bad argument");
    return guarded([&] {
        for (int64_t i = 0; i < n; ++i)
            if (!in_pool(pool, pages[i]) || pool->users[pages[i]] == 0) return set_error(TAPER_EBLOCK, at_entry("no page in use", i));
        for (int64_t i = 0; i < n; ++i) ++pool->users[pages[i]];
        return (int)TAPER_OK;
    });
}

int taper_page_pool_release(taper_page_pool* pool, int64_t n, const int32_t* pages, int64_t* n_freed) {
    if (!pool || n < 0 || (n > 0 && !pages)) return set_error(TAPER_EINVAL, "bad argument");
    return guarded([&] {
        int64_t i = 0, freed = 0;
        for (; i < n; ++i) {
            if (!in_pool(pool, pages[i]) || pool->users[pages[i]] == 0) break;
            --pool->users[pages[i]];
        }
        if (i < n) {
            const int64_t bad = i;
            while (i-- > 0) ++pool->users[pages[i]];
            return set_error(TAPER_EBLOCK, at_entry("no page in use", bad));
        }
        for (i = 0; i < n; ++i)
            if (pool->users[pages[i]] == 0) {
                pool->users[pages[i]] = -1;  // (counted once if it occurs twice)
                ++freed;
                pool->first_free = std::min<int64_t>(pool->first_free, pages[i]);
            }
        for (i = 0; i < n; ++i)
            if (pool->users[pages[i]] == -1) pool->users[pages[i]] = 0;
        pool->n_free += freed;
        if (n_freed) *n_freed = freed;
        return (int)TAPER_OK;
    });
}

int taper_page_pool_fork(taper_page_pool* pool, const int32_t* parent_row, int64_t n_tokens, int page_size, int32_t* child_row,
                         int32_t* copy_src, int32_t* copy_dst) {
    if (!pool || n_tokens < 0 || page_size < 1 || !copy_src || !copy_dst || (n_tokens > 0 && (!parent_row || !child_row)))
        return set_error(TAPER_EINVAL, "bad argument");
    const int64_t full = n_tokens / page_size;
    const bool rest = n_tokens % page_size != 0;
    int32_t own = -1;
    if (rest) {
        if (!in_pool(pool, parent_row[full]) || pool->users[parent_row[full]] == 0) return guarded([&] { return set_error(TAPER_EBLOCK, at_entry("no page in use", full)); });
        const int st = taper_page_pool_alloc(pool, 1, &own);
        if (st != TAPER_OK) return st;
    }
    const int st = taper_page_pool_share(pool, full, parent_row);
    if (st != TAPER_OK) {
        if (rest) {
            pool->users[own] = 0;
            ++pool->n_free;
            pool->first_free = std::min<int64_t>(pool->first_free, own);
        }
        return st;
    }
    *copy_src = *copy_dst = -1;
    if (rest) {
        *copy_src = parent_row[full];
        *copy_dst = own;
    }
    std::memmove(child_row, parent_row, (size_t)full * sizeof(int32_t));
    if (rest) child_row[full] = own;
    return TAPER_OK;
}

int taper_page_pool_compact(taper_page_pool* pool, int64_t max_moves, int32_t* src, int32_t* dst, int64_t* n_moves) {
    if (!pool || max_moves < 0 || !n_moves || (max_moves > 0 && (!src || !dst))) return set_error(TAPER_EINVAL, "bad argument");
    int64_t lo = pool->first_free, hi = (int64_t)pool->users.size() - 1, n = 0;
    while (n < max_moves) {
        while (lo < hi && pool->users[lo] != 0) ++lo;
        while (lo < hi && pool->users[hi] == 0) --hi;
        if (lo >= hi) break;
        src[n] = (int32_t)hi;
        dst[n++] = (int32_t)lo;
        pool->users[lo++] = pool->users[hi];
        pool->users[hi--] = 0;
    }
    pool->first_free = std::min(lo, (int64_t)pool->users.size() - 1);
    *n_moves = n;
    return TAPER_OK;
}

int taper_pages_remap(int64_t n_entries, int32_t* entries, int64_t n_moves, const int32_t* src, const int32_t* dst) {
    if (n_entries < 0 || n_moves < 0 || (n_entries > 0 && !entries) || (n_moves > 0 && (!src || !dst))) return set_error(TAPER_EINVAL, "bad argument");
    return guarded([&] {
        std::unordered_map<int32_t, int32_t> to;
        to.reserve((size_t)n_moves);
        for (int64_t i = 0; i < n_moves; ++i)
            if (!to.emplace(src[i], dst[i]).second) return set_error(TAPER_EINVAL, at_entry("page moves twice", i));
        for (int64_t i = 0; i < n_entries; ++i) {
            const auto it = to.find(entries[i]);
            if (it != to.end()) entries[i] = it->second;
        }
        return (int)TAPER_OK;
    });
}

int taper_mover_create(const taper_page_format* f, taper_mover** out_mover) {
    if (!f || !out_mover) return set_error(TAPER_EINVAL, "null argument");
    if (f->page_size != 16) return set_error(TAPER_EINVAL, "page_size must be 16");
    if (f->kind == TAPER_PAGES_KV) {
        if (f->n_heads < 1 || f->n_heads > 4096 || (f->dim != 64 && f->dim != 128)) return set_error(TAPER_EINVAL, "a KV pool has KV heads of head_dim 64 or 128");
    } else if (f->kind == TAPER_PAGES_LATENT) {
        if (f->n_heads != 1 || (f->dim != 320 && f->dim != 576)) return set_error(TAPER_EINVAL, "a latent pool has one head of 320 or 576 values");
    } else {
        return set_error(TAPER_EINVAL, "unknown page kind");
    }
    return guarded([&] {
        if (f->device >= 0) {
            int n = 0;
            if (hipGetDeviceCount(&n) != hipSuccess || f->device >= n) return set_error(TAPER_EHIP, "no such HIP device");
        }
        taper_mover* m = new taper_mover();
        m->format = *f;
        m->page_bytes = (int64_t)f->n_heads * f->dim * 32 * (f->kind == TAPER_PAGES_KV ? 2 : 1);
        *out_mover = m;
        return (int)TAPER_OK;
    });
}

void taper_mover_destroy(taper_mover* m) {
    if (!m) return;
    if (m->format.device >= 0) {
        OnDevice on(m->format.device);
        (void)hipDeviceSynchronize();
        for (MoveLists& l : m->lists) {
            if (l.done) (void)hipEventDestroy(l.done);
            if (l.dev) (void)hipFree(l.dev);
            if (l.staging) (void)hipHostFree(l.staging);
        }
    }
    delete m;
}

int taper_pages_copy(taper_mover* m, int n_layers, void* const* pools, int64_t n_moves, const int32_t* src, const int32_t* dst,
                     int64_t n_pool_pages, void* hip_stream) {
    if (!m || n_moves < 0 || (n_moves > 0 && (!src || !dst))) return set_error(TAPER_EINVAL, "bad argument");
    int st = check_layers(n_layers, pools, n_pool_pages);
    if (st != TAPER_OK) return st;
    return guarded([&] {
        std::lock_guard<std::mutex> alone(m->lock);
        begin_call(m, n_pool_pages);
        for (int64_t i = 0; i < n_moves; ++i)
            if (src[i] < 0 || src[i] >= n_pool_pages || dst[i] < 0 || dst[i] >= n_pool_pages) return set_error(TAPER_EBLOCK, at_entry("page outside the pool", i));
        int st = TAPER_OK;
        for (int64_t i = 0; i < n_moves && st == TAPER_OK; ++i) st = note_written(m, dst[i]);
        for (int64_t i = 0; i < n_moves && st == TAPER_OK; ++i) st = note_read(m, src[i]);
        if (st != TAPER_OK) return st;
        if (m->format.device < 0) return set_error(TAPER_EHIP, "host-only mover: no device work possible");
        if (n_moves == 0) return (int)TAPER_OK;
        OnDevice on(m->format.device);
        HIP_TRY(on.error);
        hipStream_t s = (hipStream_t)hip_stream;
        // Short lists travel in the launch's own arguments; so do long ones that are recorded, some at a time (a replay must not find
        // another call's list in a shared buffer).
        if (n_moves <= taper::kMovesInArguments || recording(s)) {
            for (int64_t i0 = 0; i0 < n_moves; i0 += taper::kMovesInArguments) {
                const int n = (int)std::min<int64_t>(taper::kMovesInArguments, n_moves - i0);
                taper::MoveArguments args;
                std::memset(&args, 0, sizeof args);
                for (int i = 0; i < n; ++i) args.move[i] = {src[i0 + i], dst[i0 + i]};
                const int st = for_layers(n_layers, pools, [&](const taper::PoolPointers& p, int nl) {
                    return taper::launch_pages_copy(p, nl, nullptr, &args, n, m->page_bytes, s);
                });
                if (st != TAPER_OK) return st;
            }
            return (int)TAPER_OK;
        }
        MoveLists* l = nullptr;
        const size_t bytes = align_up((size_t)n_moves * sizeof(taper::PageMove), 16);
        st = next_lists(m, bytes, &l);
        if (st != TAPER_OK) return st;
        taper::PageMove* list = (taper::PageMove*)l->staging;
        for (int64_t i = 0; i < n_moves; ++i) list[i] = {src[i], dst[i]};
        HIP_TRY(taper::launch_upload(l->dev, l->staging_dev, bytes, nullptr, 0, s));
        st = for_layers(n_layers, pools, [&](const taper::PoolPointers& p, int nl) {
            return taper::launch_pages_copy(p, nl, (const taper::PageMove*)l->dev, nullptr, n_moves, m->page_bytes, s);
        });
        HIP_TRY(hipEventRecord(l->done, s));
        return st;
    });
}

int taper_pages_pack(taper_mover* m, int n_layers, void* const* pools, int n_seqs, const int32_t* block_table, int bt_row_stride,
                     const int32_t* prefix_len, const int32_t* seg_start, const int32_t* seg_len, const int32_t* first_token,
                     const int32_t* dst_table, int dst_row_stride, int64_t n_pool_pages, void* hip_stream) {
    if (!m || !dst_table || dst_row_stride < 1 || n_seqs < 1) return set_error(TAPER_EINVAL, "bad argument");
    int st = check_layers(n_layers, pools, n_pool_pages);
    if (st != TAPER_OK) return st;
    return guarded([&] {
        const int P = m->format.page_size;
        std::vector<int32_t> group((size_t)n_seqs);
        for (int q = 0; q < n_seqs; ++q) group[q] = q;  // every sequence for itself
        taper::HostPlan b;
        int st = taper::resolve_batch(P, n_seqs, block_table, bt_row_stride, group.data(), prefix_len, seg_start, seg_len, n_pool_pages, &b);
        if (st != TAPER_OK) return st;
        std::vector<taper::PackPage> pages;
        std::vector<int32_t> run_start(1, 0), run_token, run_entry;
        for (int q = 0; q < n_seqs; ++q) {
            const int first = first_token ? first_token[q] : 0;
            if (first < 0 || first % P != 0 || first > b.ctx_len[q])
                return set_error(TAPER_ELEN, "sequence " + std::to_string(q) + ": first_token must be a multiple of the page size within the context");
            if ((b.ctx_len[q] - first + P - 1) / P > dst_row_stride)
                return set_error(TAPER_ELEN, "sequence " + std::to_string(q) + ": the destination row is too short");
            for (int t = first, j = 0; t < b.ctx_len[q]; t += P, ++j) {
                const int32_t to = dst_table[(size_t)q * dst_row_stride + j];
                if (to < 0 || to >= n_pool_pages) return set_error(TAPER_EBLOCK, "sequence " + std::to_string(q) + ": destination outside the pool");
                pages.push_back({to, q, t, std::min(P, b.ctx_len[q] - t)});
            }
            int token = 0;
            auto run = [&](int entry, int n) {
                if (n == 0) return;
                run_token.push_back(token);
                run_entry.push_back(entry);
                token += n;
            };
            run(0, prefix_len[q]);
            for (int k = seg_start[q]; k < seg_start[q + 1]; ++k) run(b.seg_page0[k], seg_len[k]);
            run_start.push_back((int32_t)run_token.size());
        }
        std::lock_guard<std::mutex> alone(m->lock);
        begin_call(m, n_pool_pages);
        for (const taper::PackPage& p : pages)
            if ((st = note_written(m, p.dst)) != TAPER_OK) return st;
        for (int q = 0; q < n_seqs; ++q) {
            const int first = first_token ? first_token[q] : 0;
            for (int k = run_start[q]; k < run_start[q + 1]; ++k) {
                const int end = k + 1 < run_start[q + 1] ? run_token[k + 1] : b.ctx_len[q];
                for (int t = std::max(0, first - run_token[k]) / P * P; t < end - run_token[k]; t += P)
                    if ((st = note_read(m, b.block_table[(size_t)q * bt_row_stride + run_entry[k] + t / P])) != TAPER_OK) return st;
            }
        }
        if (m->format.device < 0) return set_error(TAPER_EHIP, "host-only mover: no device work possible");
        if (pages.empty()) return (int)TAPER_OK;
        OnDevice on(m->format.device);
        HIP_TRY(on.error);
        hipStream_t s = (hipStream_t)hip_stream;
        if (recording(s)) return set_error(TAPER_EINVAL, "a join cannot be recorded into a graph");
        struct Piece {
            const void* src;
            size_t bytes, off;
        } piece[5] = {{pages.data(), pages.size() * sizeof(taper::PackPage), 0},
                      {b.block_table.data(), b.block_table.size() * 4, 0},
                      {run_start.data(), run_start.size() * 4, 0},
                      {run_token.data(), run_token.size() * 4, 0},
                      {run_entry.data(), run_entry.size() * 4, 0}};
        size_t total = 0;
        for (Piece& p : piece) {
            p.off = total;
            total = align_up(total + p.bytes, 256);
        }
        MoveLists* l = nullptr;
        st = next_lists(m, total, &l);
        if (st != TAPER_OK) return st;
        for (const Piece& p : piece) std::memcpy((char*)l->staging + p.off, p.src, p.bytes);
        HIP_TRY(taper::launch_upload(l->dev, l->staging_dev, total, nullptr, 0, s));
        taper::PackArgs a;
        char* d = (char*)l->dev;
        a.pages = (const taper::PackPage*)(d + piece[0].off);
        a.bt = (const int32_t*)(d + piece[1].off);
        a.run_start = (const int32_t*)(d + piece[2].off);
        a.run_token = (const int32_t*)(d + piece[3].off);
        a.run_entry = (const int32_t*)(d + piece[4].off);
        a.bt_stride = bt_row_stride;
        a.n_pages = (int32_t)pages.size();
        a.kind = m->format.kind;
        a.n_heads = m->format.n_heads;
        a.dim = m->format.dim;
        st = for_layers(n_layers, pools, [&](const taper::PoolPointers& p, int nl) { return taper::launch_pages_pack(p, nl, a, s); });
        HIP_TRY(hipEventRecord(l->done, s));
        return st;
    });
}

}  // extern "C"
