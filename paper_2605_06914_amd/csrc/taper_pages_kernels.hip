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

// One destination page (of one layer and tile group) a workgroup.  16 lanes find where the page's tokens come from; K and latent
// tiles ([d / 8][16][8]) are then 16-byte pieces, V tiles ([16 / 4][d][4]) four tokens of a d.
__global__ __launch_bounds__(256) void pages_pack_kernel(const PoolPointers pools, const PackArgs a) {
    __shared__ int src_page[16], src_tok[16];
    const PackPage pg = a.pages[blockIdx.x];
    const int t = threadIdx.x;
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
    }
    __syncthreads();
    char* pool = (char*)pools.base[blockIdx.z];
    const int D = a.dim, per_k = D * 2;  // 16-byte pieces of a K tile
    const int64_t tile = (int64_t)D * 32, page_bytes = tile * a.n_heads * (a.kind == TAPER_PAGES_KV ? 2 : 1);
    for (int i = blockIdx.y * 256 + t; i < a.n_heads * per_k; i += gridDim.y * 256) {
        const int head = i / per_k, d8 = i % per_k >> 4, tok = i & 15;
        if (src_page[tok] < 0) continue;
        const int64_t at = head * tile + d8 * 256;
        *(u32x4*)(pool + pg.dst * page_bytes + at + tok * 16) = *(const u32x4*)(pool + src_page[tok] * page_bytes + at + src_tok[tok] * 16);
    }
    if (a.kind != TAPER_PAGES_KV) return;
    const int per_v = D * 4;  // groups of four tokens of a d
    for (int i = blockIdx.y * 256 + t; i < a.n_heads * per_v; i += gridDim.y * 256) {
        const int head = i / per_v, q = i % per_v / D, d = i % D;
        const int64_t at = (a.n_heads + head) * tile + d * 8;
        unsigned short* to = (unsigned short*)(pool + pg.dst * page_bytes + at + q * D * 8);
        unsigned short v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (src_page[4 * q + j] >= 0)
                v[j] = *(const unsigned short*)(pool + src_page[4 * q + j] * page_bytes + at + (src_tok[4 * q + j] >> 2) * (D * 8) + (src_tok[4 * q + j] & 3) * 2);
        if (src_page[4 * q + 3] >= 0) {
            *(u32x2*)to = u32x2{v[0] | (unsigned)v[1] << 16, v[2] | (unsigned)v[3] << 16};
        } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
                if (src_page[4 * q + j] >= 0) to[j] = v[j];
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

hipError_t launch_pages_pack(const PoolPointers& pools, int n_layers, const PackArgs& a, hipStream_t s) {
    const int split = a.n_heads >= 4 ? 2 : 1;
    for (int64_t i = 0; i < a.n_pages; i += kMostBlocks) {
        PackArgs b = a;
        b.pages += i;
        hipLaunchKernelGGL(pages_pack_kernel, dim3((unsigned)(a.n_pages - i < kMostBlocks ? a.n_pages - i : kMostBlocks), split, n_layers), dim3(256), 0, s, pools, b);
    }
    return hipGetLastError();
}

}  // namespace taper
