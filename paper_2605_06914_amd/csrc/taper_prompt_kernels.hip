// gfx950 kernels of a prompt's attention over a latent cache, in expanded form.
//
// expand_kernel makes every head's keys without rotation and values of every cached token that a new token sees (a shared prefix
// once for all branches of its request), some heads at a time, in the tile layouts that the attention's matrix operands have: K
// [d / 8][16 tokens][8], V [16 / 4][d][4].  prompt_kernel is causal attention of tiles of 128 query rows over them; the rotated
// key parts come from the cache itself.  Where there are too few tiles for the chip their keys are cut into pieces, which
// prompt_merge_kernel brings together.
#include <cmath>

#include "latent_device.h"

namespace taper {
namespace latent {

// ---------------------------------------------------------------------------
// expand: a product of (tokens x R) and (R x 2 head_dim) for each head.  A workgroup takes 8 pages x 128 rows of W, 64 values of the
// contraction at a time, both sides through LDS; a wave 4 pages x 64 rows.  Keys come out as W C^T (a lane: 4 consecutive d of a
// token), values as C W^T (4 consecutive tokens of a d): both are 8 bytes of their tile.  A page's 64 values are 2 KiB in a row and
// in operand order as they are; W's rows are 128 bytes each, their 16-byte pieces swapped about by the row so that 16 rows' pieces
// lie in different banks.
// ---------------------------------------------------------------------------
struct ExpandSmem {
    __bf16 c[2][8][8 * 128];  // [page][8 groups of 8 values][16 tokens][8]
    __bf16 w[2][128][64];
};

template <int HD>
__global__ __launch_bounds__(256, 2) void expand_kernel(const LatentShape sh, const PromptArgs a, const int h0, const int n_heads) {
    __shared__ ExpandSmem sm;
    const int R = sh.latent_dim, KD = R + kRopeDim;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int e0 = blockIdx.x / n_heads * 8, hl = blockIdx.x % n_heads, part = blockIdx.y;
    const char* w = (const char*)((const __bf16*)a.w_up + ((int64_t)(h0 + hl) * 2 * HD + part * 128) * R);
    int64_t page[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) page[i] = (int64_t)uniform(a.e_page[min(e0 + 2 * wave + i, a.n_expanded - 1)]) * KD * 32;
    const int wrow = lane >> 3, wpiece = (lane & 7) ^ (wrow & 7);
    auto fetch = [&](int k, int b) {  // values 64 k .. of both sides
#pragma unroll
        for (int i = 0; i < 4; ++i)
            load_to_lds((const char*)a.pages + page[i >> 1] + k * 2048, (i & 1) * 1024 + lane * 16, uniform(lds_address(&sm.c[b][2 * wave + (i >> 1)][0])) + (i & 1) * 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            load_to_lds(w + k * 128, ((32 * wave + 8 * i + wrow) * R + wpiece * 8) * 2, uniform(lds_address(&sm.w[b][32 * wave + 8 * i][0])));
    };
    const int p0 = (wave & 1) * 4, r0 = (wave >> 1) * 64;
    const bool values = part * 128 + r0 >= HD;
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    fetch(0, 0);
    for (int k = 0; k < R / 64; ++k) {
        wait_loads_and_meet<0>();
        if (k + 1 < R / 64) fetch(k + 1, (k + 1) & 1);
        const int b = k & 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 cf[4], wf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) cf[i] = *(const bf16x8*)&sm.c[b][p0 + i][(4 * kk + g) * 128 + n * 8];
#pragma unroll
            for (int j = 0; j < 4; ++j) wf[j] = *(const bf16x8*)&sm.w[b][r0 + 16 * j + n][((4 * kk + g) ^ (n & 7)) * 8];
            if (values) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = mfma16(cf[i], wf[j], acc[i][j]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = mfma16(wf[j], cf[i], acc[i][j]);
            }
        }
    }
    const int d0 = (part * 128 + r0) % HD;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = e0 + p0 + i;
        if (e >= a.n_expanded) continue;
        const int valid = a.e_valid[e];
        __bf16* to = (__bf16*)a.kv + ((int64_t)hl * a.n_expanded + e) * (32 * HD);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4 v = acc[i][j];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = (values ? 4 * g + x : n) < valid ? v[x] : 0.f;  // (slots past a length may hold anything)
            const bf16x4 o = __builtin_convertvector(v, bf16x4);  // (the matrix operand's type)
            const int d = d0 + 16 * j;
            if (values) *(bf16x4*)(to + 16 * HD + g * 4 * HD + (d + n) * 4) = o;
            else *(bf16x4*)(to + ((d + 4 * g) >> 3) * 128 + n * 8 + (g & 1) * 4) = o;
        }
    }
}

// ---------------------------------------------------------------------------
// The attention: 4 waves of 32 query rows, 64 tokens (4 pages) at a time through LDS, everything transposed as in the decode kernels:
// S^T = K Q^T leaves the weights in the layout that O^T = V^T P^T takes them in.
// ---------------------------------------------------------------------------
template <int HD>
struct PromptSmem {
    __bf16 k[2][4][HD * 16];
    __bf16 r[2][4][kRopeDim * 16];
    __bf16 v[2][4][HD * 16];
};

template <int HD>
__global__ __launch_bounds__(256, 2) void prompt_kernel(const LatentShape sh, const PromptArgs a, const int h0, const int n_heads) {
    constexpr int KS = HD / 32, DT = HD / 16, NT = 2;
    __shared__ PromptSmem<HD> sm;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int hl = blockIdx.x % n_heads, h = h0 + hl, H = sh.n_heads;
    const PromptTile t = a.tiles[blockIdx.x / n_heads];
    const int npre = (t.prefix_len + 15) / 16;
    const float c = sh.scale_log2e;
    auto expanded = [&](int vp) { return vp < npre ? t.prefix_e + vp : t.suffix_e + (vp - npre); };
    const int64_t page_bytes = (sh.latent_dim + kRopeDim) * 32LL;
    auto fetch = [&](int vp0, int b) {
        const int e = uniform(expanded(min(vp0 + wave, t.page_end - 1)));
        const char* kv = (const char*)a.kv + ((int64_t)hl * a.n_expanded + e) * (64 * HD);
        const char* rope = (const char*)a.pages + (int64_t)uniform(a.e_page[e]) * page_bytes + sh.latent_dim * 32;
        const unsigned kl = uniform(lds_address(sm.k[b][wave])), vl = uniform(lds_address(sm.v[b][wave])), rl = uniform(lds_address(sm.r[b][wave]));
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) load_to_lds(kv, i * 1024 + lane * 16, kl + i * 1024);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_to_lds(rope, i * 1024 + lane * 16, rl + i * 1024);
#pragma unroll
        for (int i = 0; i < HD / 32; ++i) load_to_lds(kv + 32 * HD, i * 1024 + lane * 16, vl + i * 1024);
    };
    fetch(t.page_begin, 0);
    bf16x8 qf[NT][KS + 2];
    int pos[NT];  // of this lane's rows
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int r = min(32 * wave + 16 * k + n, t.n_rows - 1);
        pos[k] = t.first_pos + r;
        const __bf16* q = (const __bf16*)a.q + ((int64_t)(t.row0 + r) * H + h) * (HD + kRopeDim) + 8 * g;
#pragma unroll
        for (int j = 0; j < KS + 2; ++j) qf[k][j] = *(const bf16x8*)(q + 32 * j);
    }
    const int first_pos = t.first_pos + min(32 * wave, t.n_rows - 1);  // of this wave's rows
    f32x4 O[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) O[k][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int vp0 = t.page_begin, b = 0; vp0 < t.page_end; vp0 += 4, b ^= 1) {
        wait_loads_and_meet<0>();  // this tile is here for all, and all are done with the one before
        if (vp0 + 4 < t.page_end) fetch(vp0 + 4, b ^ 1);
        f32x4 s[4][NT];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
#pragma unroll
            for (int k = 0; k < NT; ++k) s[p][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < KS + 2; ++j) {
                const __bf16* from = j < KS ? sm.k[b][p] + (4 * j + g) * 128 : sm.r[b][p] + (4 * (j - KS) + g) * 128;
                const bf16x8 kf = *(const bf16x8*)(from + n * 8);
#pragma unroll
                for (int k = 0; k < NT; ++k) s[p][k] = mfma16(kf, qf[k][j], s[p][k]);
            }
        }
        // pages that hold tokens ahead of some row, none at all, or the end of a prefix
        const bool whole = vp0 + 4 <= t.page_end && (vp0 + 4 <= npre ? 16 * vp0 + 64 <= t.prefix_len : vp0 >= npre && t.prefix_len + 16 * (vp0 - npre) + 63 <= first_pos);
        if (!whole) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int vp = vp0 + p;
                // positions of the page begin at `from`; those of a prefix end with it, and a page that is not there has none
                const int from = vp < npre ? 16 * vp : t.prefix_len + 16 * (vp - npre);
                const int most = vp >= t.page_end ? -1 : vp < npre ? t.prefix_len - 1 : 0x7fffffff;
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[p][k][i] = from + 4 * g + i <= min(pos[k], most) ? s[p][k][i] : -INFINITY;
            }
        }
        bf16x4 pr[4][NT];
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            float mx = -INFINITY;
#pragma unroll
            for (int p = 0; p < 4; ++p) mx = fmaxf(fmaxf(mx, fmaxf(s[p][k][0], s[p][k][1])), fmaxf(s[p][k][2], s[p][k][3]));
            if (__any(mx * c > m[k])) {
                const float mn = fmaxf(m[k], max_lane_groups(mx) * c);
                const float alpha = fast_exp2(m[k] - (mn == -INFINITY ? 0.f : mn));
                l[k] *= alpha;
#pragma unroll
                for (int d = 0; d < DT; ++d) O[k][d] *= alpha;
                m[k] = mn;
            }
            const float ref = m[k] == -INFINITY ? 0.f : m[k];  // (a row may see nothing of these pages)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                f32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = fast_exp2(fmaf(s[p][k][i], c, -ref));
                l[k] += (w[0] + w[1]) + (w[2] + w[3]);
                pr[p][k] = __builtin_convertvector(w, bf16x4);  // (weights of at most 1, in 8 bits each)
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int at = g * 4 * HD + (16 * d + n) * 4;
                const bf16x8 vf = cat(*(const bf16x4*)(sm.v[b][2 * ks] + at), *(const bf16x4*)(sm.v[b][2 * ks + 1] + at));
#pragma unroll
                for (int k = 0; k < NT; ++k) O[k][d] = mfma16(vf, cat(pr[2 * ks][k], pr[2 * ks + 1][k]), O[k][d]);
            }
    }
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int r = 32 * wave + 16 * k + n;
        const float total = sum_lane_groups(l[k]);
        if (r >= t.n_rows) continue;
        const float inv = total > 0.f ? 1.0f / total : total;  // (NaN stays what it is)
        if (t.part_row >= 0) {
            const int64_t at = (int64_t)hl * a.n_partial_rows + t.part_row + r;
            if (g == 0) a.ml[at] = make_float2(m[k], total);
#pragma unroll
            for (int d = 0; d < DT; ++d) *(f32x4*)(a.part + at * HD + 16 * d + 4 * g) = O[k][d] * inv;
        } else {
            const int64_t at = (int64_t)(t.row0 + r) * H + h;
            if (g == 0 && a.lse) a.lse[at] = (m[k] + log2f(total)) * 0.6931471805599453f;
#pragma unroll
            for (int d = 0; d < DT; ++d) *(bf16x4*)((__bf16*)a.out + at * HD + 16 * d + 4 * g) = __builtin_convertvector(O[k][d] * inv, bf16x4);
        }
    }
}

// One wave a row: the pieces of a row lie n_rows of its tile apart.
template <int HD>
__global__ __launch_bounds__(256) void prompt_merge_kernel(const LatentShape sh, const PromptArgs a, const int h0, const int n_heads) {
    constexpr int PER = HD / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hl = blockIdx.x % n_heads, h = h0 + hl;
    const PromptTile t = a.merges[blockIdx.x / n_heads];
    for (int r = wave + 4 * blockIdx.y; r < t.n_rows; r += 4 * gridDim.y) {
        const int64_t first = (int64_t)hl * a.n_partial_rows + t.part_row + r;
        float M = -INFINITY, L = 0.f, acc[PER];
        for (int p = 0; p < t.n_pieces; ++p) M = fmaxf(M, a.ml[first + (int64_t)p * t.n_rows].x);
#pragma unroll
        for (int j = 0; j < PER; ++j) acc[j] = 0.f;
        for (int p = 0; p < t.n_pieces; ++p) {
            const int64_t at = first + (int64_t)p * t.n_rows;
            const float2 ml = a.ml[at];
            const float w = ml.y * fast_exp2(ml.x - M);
            L += w;
#pragma unroll
            for (int j = 0; j < PER; ++j) acc[j] = fmaf(w, a.part[at * HD + lane * PER + j], acc[j]);
        }
        const float inv = 1.0f / L;
        const int64_t to = (int64_t)(t.row0 + r) * sh.n_heads + h;
#pragma unroll
        for (int j = 0; j < PER; ++j) ((__bf16*)a.out)[to * HD + lane * PER + j] = (__bf16)(acc[j] * inv);
        if (lane == 0 && a.lse) a.lse[to] = (M + log2f(L)) * 0.6931471805599453f;
    }
}

template <int HD>
static hipError_t launch_prompt_as(const LatentShape& sh, const PromptArgs& a, hipStream_t s) {
    for (int h0 = 0; h0 < sh.n_heads; h0 += a.heads_at_once) {
        const int nh = sh.n_heads - h0 < a.heads_at_once ? sh.n_heads - h0 : a.heads_at_once;
        hipLaunchKernelGGL(expand_kernel<HD>, dim3((unsigned)((a.n_expanded + 7) / 8) * nh, HD / 64), dim3(256), 0, s, sh, a, h0, nh);
        hipLaunchKernelGGL(prompt_kernel<HD>, dim3((unsigned)a.n_tiles * nh), dim3(256), 0, s, sh, a, h0, nh);
        if (a.n_merges > 0) hipLaunchKernelGGL(prompt_merge_kernel<HD>, dim3((unsigned)a.n_merges * nh, 8), dim3(256), 0, s, sh, a, h0, nh);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace latent

hipError_t launch_latent_prompt(const LatentShape& sh, const PromptArgs& a, hipStream_t s) {
    return sh.head_dim == 128 ? latent::launch_prompt_as<128>(sh, a, s) : latent::launch_prompt_as<64>(sh, a, s);
}

}  // namespace taper
