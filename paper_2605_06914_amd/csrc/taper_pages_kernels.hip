// gfx950 kernels that move pages and tokens of paged caches, through all layers of a model at once.  Both are bound by memory:
// a byte moved is read once and written once.
#include "pages_kernels.h"

#include "taper_pages.h"

namespace taper {
namespace pages {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
#define DEV __device__ __forceinline__

// A page is a run of bytes: 256 threads copy pieces of 16 KiB, 64 bytes a thread and all loads ahead of the stores.
constexpr int kPiece = 16384;
DEV void copy_piece(const PoolPointers& pools, const PageMove mv, const int layer, const int64_t page_bytes, const int piece) {
    const char* from = (const char*)pools.base[layer] + mv.src * page_bytes;
    char* to = (char*)pools.base[layer] + mv.dst * page_bytes;
    u32x4 v[4];
    const int64_t at = (int64_t)piece * kPiece + threadIdx.x * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_bytes) v[i] = __builtin_nontemporal_load((const u32x4*)(from + at + i * 4096));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_bytes) __builtin_nontemporal_store(v[i], (u32x4*)(to + at + i * 4096));
}
__global__ __launch_bounds__(256) void pages_copy_kernel(const PoolPointers pools, const PageMove* list, const int64_t page_bytes) {
    copy_piece(pools, list[blockIdx.x], blockIdx.z, page_bytes, blockIdx.y);
}
__global__ __launch_bounds__(256) void pages_copy_few_kernel(const PoolPointers pools, const MoveArguments args, const int64_t page_bytes) {
    copy_piece(pools, args.move[blockIdx.x], blockIdx.z, page_bytes, blockIdx.y);
}

// Joins.  A workgroup has one destination page of one layer, or some heads of it.  16 lanes find where the page's tokens come from; K and
// latent tiles ([d / 8][16][8]) are then 16-byte pieces.  V tiles ([16 / 4][d][4]) hold 4 tokens of a d in 8 bytes: where a group of 4
// comes from consecutive tokens, also across a page's end, it is shifted out of the two groups it lies in (a token at a time, 2 bytes
// each, took 263 us for 0.46 GB moved, this 204); where a run of tokens ends in between, it is gathered.
struct Quarter {
    long long first, second;  // byte offsets of the two groups (in a tile of head 0)
    int shift;                // bits of the first that are not wanted, -1: gather, -2: no token
};
template <int KIND, int D>
__global__ __launch_bounds__(256) void pages_pack_kernel(const PoolPointers pools, const PackArgs a) {
    constexpr bool KV = KIND == TAPER_PAGES_KV;
    constexpr int TILE = D * 32, UN = 8;
    __shared__ int src_page[16], src_tok[16];
    __shared__ long long src_at[16];  // of a token in a K tile: its page and its place in a group of 8 dims
    __shared__ Quarter quarter[4];
    const PackPage pg = a.pages[blockIdx.x];
    const int t = threadIdx.x;
    const int heads = KV ? a.n_heads : 1;
    const long long page_bytes = (long long)TILE * heads * (KV ? 2 : 1);
    if (t < 16) {
        int page = -1, tok = 0;
        if (t < pg.n_tokens) {
            const int token = pg.token0 + t;
            int lo = a.run_start[pg.seq], hi = a.run_start[pg.seq + 1] - 1;  // the last run that begins at or before the token
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (a.run_token[mid] <= token) lo = mid;
                else hi = mid - 1;
            }
            const int at = token - a.run_token[lo];
            page = a.bt[(int64_t)pg.seq * a.bt_stride + a.run_entry[lo] + (at >> 4)];
            tok = at & 15;
        }
        src_page[t] = page;
        src_tok[t] = tok;
        src_at[t] = page < 0 ? -1 : page * page_bytes + tok * 16;
    }
    __syncthreads();
    if (KV && t < 4) {
        const int p0 = src_page[4 * t], p3 = src_page[4 * t + 3], t0 = src_tok[4 * t];
        bool in_row = p3 >= 0;
        for (int j = 1; j < 4; ++j) in_row = in_row && src_tok[4 * t + j] == ((t0 + j) & 15) && src_page[4 * t + j] == (t0 + j < 16 ? p0 : p3);
        const int q0 = t0 >> 2;
        Quarter q;
        q.shift = p0 < 0 ? -2 : (in_row ? (t0 & 3) * 16 : -1);
        q.first = p0 * page_bytes + q0 * (D * 8);
        q.second = (t0 & 3) == 0 ? q.first : (q0 < 3 ? p0 * page_bytes + (q0 + 1) * (D * 8) : p3 * page_bytes);
        quarter[t] = q;
    }
    __syncthreads();
    char* pool = (char*)pools.base[blockIdx.z];
    char* const to = pool + pg.dst * page_bytes;
    const int step = gridDim.y * 256;
    const int n_k = heads * (D * 2);  // 16-byte pieces of the K tiles
    for (int i0 = blockIdx.y * 256 + t; i0 < n_k; i0 += UN * step) {
        u32x4 v[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = i0 + u * step, head = i / (D * 2), d8 = i % (D * 2) >> 4;
            if (i < n_k && src_at[i & 15] >= 0) v[u] = __builtin_nontemporal_load((const u32x4*)(pool + src_at[i & 15] + (long long)head * TILE + d8 * 256));
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = i0 + u * step;
            if (i < n_k && src_at[i & 15] >= 0) __builtin_nontemporal_store(v[u], (u32x4*)(to + (long long)i * 16));
        }
    }
    if (!KV) return;
    pool += (long long)heads * TILE;  // (the V tiles)
    char* const to_v = to + (long long)heads * TILE;
    const int n_v = heads * (D * 4);  // groups of four tokens of a d
    for (int i0 = blockIdx.y * 256 + t; i0 < n_v; i0 += UN * step) {
        unsigned long long x[UN], y[UN];
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = i0 + u * step, head = i / (D * 4), d = i % D;
            if (i >= n_v) continue;
            const Quarter& q = quarter[i / D % 4];
            const long long at = (long long)head * TILE + d * 8;
            if (q.shift >= 0) {
                x[u] = *(const unsigned long long*)(pool + q.first + at);
                y[u] = *(const unsigned long long*)(pool + q.second + at);
            }
        }
#pragma unroll
        for (int u = 0; u < UN; ++u) {
            const int i = i0 + u * step, head = i / (D * 4), d = i % D, qi = i / D % 4;
            if (i >= n_v) continue;
            const int shift = quarter[qi].shift;
            if (shift >= 0) {
                __builtin_nontemporal_store(shift ? x[u] >> shift | y[u] << (64 - shift) : x[u], (unsigned long long*)(to_v + (long long)i * 8));
            } else if (shift == -1) {
                for (int j = 0; j < 4; ++j) {
                    const int k = 4 * qi + j;
                    if (src_page[k] < 0) break;
                    const char* from = pool + src_page[k] * page_bytes + (long long)head * TILE + (src_tok[k] >> 2) * (D * 8) + d * 8 + (src_tok[k] & 3) * 2;
                    *(unsigned short*)(to_v + (long long)i * 8 + j * 2) = *(const unsigned short*)from;
                }
            }
        }
    }
}

}  // namespace pages

using namespace pages;

constexpr int64_t kMostBlocks = 1 << 20;  // of a launch's first dimension (a launch has fewer than 2^32 threads)

hipError_t launch_pages_copy(const PoolPointers& pools, int n_layers, const PageMove* list, const MoveArguments* args, int64_t n_moves,
                             int64_t page_bytes, hipStream_t s) {
    for (int64_t i = 0; i < n_moves; i += kMostBlocks) {
        const dim3 grid((unsigned)(n_moves - i < kMostBlocks ? n_moves - i : kMostBlocks), (unsigned)((page_bytes + kPiece - 1) / kPiece), n_layers);
        if (list) hipLaunchKernelGGL(pages_copy_kernel, grid, dim3(256), 0, s, pools, list + i, page_bytes);
        else hipLaunchKernelGGL(pages_copy_few_kernel, grid, dim3(256), 0, s, pools, *args, page_bytes);
    }
    return hipGetLastError();
}

template <int KIND, int D>
static void launch_pack_as(const PoolPointers& pools, int n_layers, const PackArgs& a, hipStream_t s) {
    const int split = a.n_heads >= 4 && (int64_t)a.n_pages * n_layers < 1024 ? 4 : 1;  // (finding the tokens is done once a workgroup)
    for (int64_t i = 0; i < a.n_pages; i += kMostBlocks) {
        PackArgs b = a;
        b.pages += i;
        hipLaunchKernelGGL((pages_pack_kernel<KIND, D>), dim3((unsigned)(a.n_pages - i < kMostBlocks ? a.n_pages - i : kMostBlocks), split, n_layers), dim3(256), 0, s, pools, b);
    }
}

hipError_t launch_pages_pack(const PoolPointers& pools, int n_layers, const PackArgs& a, hipStream_t s) {
    if (a.kind == TAPER_PAGES_KV && a.dim == 128) launch_pack_as<TAPER_PAGES_KV, 128>(pools, n_layers, a, s);
    else if (a.kind == TAPER_PAGES_KV && a.dim == 64) launch_pack_as<TAPER_PAGES_KV, 64>(pools, n_layers, a, s);
    else if (a.kind == TAPER_PAGES_LATENT && a.dim == 576) launch_pack_as<TAPER_PAGES_LATENT, 576>(pools, n_layers, a, s);
    else if (a.kind == TAPER_PAGES_LATENT && a.dim == 320) launch_pack_as<TAPER_PAGES_LATENT, 320>(pools, n_layers, a, s);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace taper
