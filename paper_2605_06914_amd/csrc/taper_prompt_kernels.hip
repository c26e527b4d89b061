// gfx950 kernels of a prompt's attention over a latent cache, in expanded form.
//
// expand_kernel makes every head's keys without rotation and values of every cached token that a new token sees (a shared prefix
// once for all branches of its request), some heads at a time, in the layouts that the attention's matrix operands have: pages in
// pairs, [K of the first: [d / 8][16 tokens][8]][K of the second][V: [4 lane groups][d][4 tokens of the first, 4 of the second]].
// prompt_kernel is causal attention of tiles of query rows over them; the rotated key parts come from the cache itself.  Where there
// are too few tiles for the chip their keys are cut into pieces, which prompt_merge_kernel brings together.
//
// Expanded keys and values are half precision, and so are the weights they meet: 11 bits of each instead of bf16's 8.  Four pages
// whose keys (or values) half precision does not hold, beyond 65504 or all of them below 2^-10, are bf16 instead; `format` says
// which.  A query's part without rotation is brought into half precision's range by a power of two of its own.
#include <cmath>
#include <type_traits>

#include "latent_device.h"

namespace taper {
namespace latent {

typedef std::true_type yes;
typedef std::false_type no;
DEV f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
DEV float max_wave(float v) {
#pragma unroll
    for (int x = 32; x; x >>= 1) v = fmaxf(v, __shfl_xor(v, x));
    return v;
}

// ---------------------------------------------------------------------------
// expand: a product of (tokens x R) and (R x 2 head_dim) for each head.  A workgroup keeps 128 rows of W in LDS (R = 512: 128 KiB,
// read 1 KiB an operand, each 16-byte piece moved by its row so that 16 rows' pieces lie in different banks) and its 8 waves go through
// the tokens 64 at a time, each by itself: a page's operands come straight from the cache, 1 KiB in a row each, and nothing but W is
// shared, so no wave waits for another.  Keys come out as W C^T (a lane: 4 consecutive d of a token), values as C W^T (4 consecutive
// tokens of a d).
// ---------------------------------------------------------------------------
template <int R, int HD, int KIND>  // KIND 0: keys, 1: values, 2: 64 rows of keys, then 64 of values
DEV void expand_chunk(const PromptArgs& a, const __bf16* w, const int hl, const int chunk) {
    constexpr int KD = R + kRopeDim, KSTEPS = R / 32, AHEAD = 2;
    int lane = opaque(threadIdx.x) & 63, n = lane & 15, g = lane >> 4;
    auto is_value = [](int j) { return KIND == 1 || (KIND == 2 && j >= 4); };
    const __bf16* page[4];
    const int at = g * 128 + n * 8;
    int valid[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = min(4 * chunk + i, a.n_expanded - 1);
        page[i] = (const __bf16*)a.pages + (int64_t)uniform(a.e_page[e]) * (KD * 16);
        valid[i] = uniform(a.e_valid[e]);
    }
    const __bf16* w_at[4][2];  // where this lane reads W in each of four steps, its first and its last 64 rows
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) w_at[x][y] = w + (64 * y + n) * R + ((4 * x + g) ^ n) * 8;
    f32x4 acc[4][8];
    bf16x8 cf[AHEAD][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) cf[k][i] = *(const bf16x8*)(page[i] + at + k * 512);
    }
#pragma unroll
    for (int k = 0; k < KSTEPS; ++k) {
        bf16x8 c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = cf[k % AHEAD][i];
            if (k + AHEAD < KSTEPS) cf[k % AHEAD][i] = *(const bf16x8*)(page[i] + at + (k + AHEAD) * 512);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bf16x8 wf = *(const bf16x8*)(w_at[k & 3][j / 4] + (16 * (j % 4)) * R + (k >> 2) * 128);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i][j] = is_value(j) ? mfma16(c[i], wf, acc[i][j]) : mfma16(wf, c[i], acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);  // (else more of W is read ahead than there are registers for)
    }
    lane = opaque(threadIdx.x) & 63, n = lane & 15, g = lane >> 4;  // (again: no registers for them in between)
    float most[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float v = (is_value(j) ? 4 * g + x : n) < valid[i] ? acc[i][j][x] : 0.f;  // (slots past a length may hold anything)
                acc[i][j][x] = v;
                most[is_value(j)] = fmaxf(most[is_value(j)], fabsf(v));
            }
    bool wide[2] = {false, false};  // not for half precision
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        if (KIND != 2 && KIND != v) continue;
        const float m = max_wave(most[v]);
        wide[v] = uniform(m > 65504.f || (m > 0.f && m < 0x1p-10f));
        if (lane == 0) a.format[((int64_t)hl * a.n_chunks + chunk) * 2 + v] = wide[v];
    }
    auto store = [&](auto kind, auto convert) {  // (the operands' types: every value is rounded once)
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {
            if (4 * chunk + 2 * pair >= a.n_expanded) return;
            uint16_t* to = (uint16_t*)a.kv + ((int64_t)hl * (a.n_expanded / 2) + 2 * chunk + pair) * (64 * HD);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (is_value(j) != decltype(kind)::value) continue;
                const int d = 16 * j - (KIND == 2 && is_value(j) ? 64 : 0);
                if constexpr (decltype(kind)::value) {
                    const uint2 x = convert(acc[2 * pair][j]), y = convert(acc[2 * pair + 1][j]);
                    *(uint4*)(to + 32 * HD + (g * HD + d + n) * 8) = make_uint4(x.x, x.y, y.x, y.y);
                } else {
#pragma unroll
                    for (int i = 0; i < 2; ++i) *(uint2*)(to + i * 16 * HD + ((d + 4 * g) >> 3) * 128 + n * 8 + (g & 1) * 4) = convert(acc[2 * pair + i][j]);
                }
            }
        }
    };
    if (KIND != 1 && a.lse) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int low = 4 * chunk + i < a.n_expanded ? uniform(a.e_low[4 * chunk + i]) : -1;
            if (low < 0) continue;
            uint16_t* to = (uint16_t*)a.k_low + ((int64_t)hl * a.n_low + low) * (16 * HD) + n * 8 + (g & 1) * 4;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (is_value(j)) continue;
                f32x4 rest;
#pragma unroll
                for (int x = 0; x < 4; ++x) rest[x] = wide[0] ? 0.f : (acc[i][j][x] - (float)(_Float16)acc[i][j][x]) * 0x1p11f;
                *(uint2*)(to + ((16 * j + 4 * g) >> 3) * 128) = __builtin_bit_cast(uint2, __builtin_convertvector(rest, f16x4));
            }
        }
    }
    auto half = [](f32x4 v) { return __builtin_bit_cast(uint2, __builtin_convertvector(v, f16x4)); };
    auto brain = [](f32x4 v) { return __builtin_bit_cast(uint2, __builtin_convertvector(v, bf16x4)); };
    if (KIND != 1) {
        if (wide[0]) store(no(), brain);
        else store(no(), half);
    }
    if (KIND != 0) {
        if (wide[1]) store(yes(), brain);
        else store(yes(), half);
    }
}

template <int R, int HD>
__global__ __launch_bounds__(512, 2) void expand_kernel(const PromptArgs a, const int h0, const int n_heads) {
    __shared__ __align__(16) __bf16 w[128 * R];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    const int hl = blockIdx.x % n_heads, split = blockIdx.x / n_heads, part = blockIdx.y;
    const char* from = (const char*)((const __bf16*)a.w_up + ((int64_t)(h0 + hl) * 2 * HD + part * 128) * R);
    constexpr int ROWS = 512 / R;  // rows of W in a KiB
#pragma unroll
    for (int i = 0; i < 16 / ROWS; ++i) {
        const int row = (i * 8 + wave) * ROWS, mine = row + lane * ROWS / 64;
        load_to_lds(from + row * R * 2, (mine - row) * R * 2 + ((lane % (64 / ROWS)) ^ (mine & 15)) * 16, uniform(lds_address(w + row * R)));
    }
    wait_loads_and_meet<0>();
    const int n_waves = gridDim.x / n_heads * 8;
    for (int c = split * 8 + wave; c < a.n_chunks; c += n_waves) {
        if constexpr (HD == 64) {
            expand_chunk<R, HD, 2>(a, w, hl, c);
        } else if (part == 0) {
            expand_chunk<R, HD, 0>(a, w, hl, c);
        } else {
            expand_chunk<R, HD, 1>(a, w, hl, c);
        }
    }
}

// ---------------------------------------------------------------------------
// The attention: 8 waves of 32 query rows, 64 tokens (4 pages) at a time through LDS, two such tiles on their way behind the one at
// hand (with one, half of the time went by in waits), everything transposed as in the decode kernels: S^T = K Q^T leaves the weights in
// the layout that O^T = V^T P^T takes them in.
// ---------------------------------------------------------------------------
constexpr int kStages = 3;
// Weights are made 2^10 times as large: half precision ends at 2^-24, and tokens whose weights are that far below the largest may still
// be so many that they matter (64000 of weight 2^-24 are a 256th).  At 2^10 those of 2^-34 are kept, and 2^6 is left to its upper end
// for the rounding of large scores.
constexpr float kWeightBits = 10.f;
template <int HD>
struct PromptSmem {
    _Float16 k[kStages][4][HD * 16];
    __bf16 r[kStages][4][kRopeDim * 16];
    _Float16 v[kStages][2][HD * 32];
};

// Which item and head a workgroup has.  Items that meet the same keys lie together (a bundle); of each head of a bundle the items
// become workgroups 8 apart, so that they run on one XCD (workgroup i runs on XCD i mod 8) at about the same time and share its L2.
DEV void tile_of_block(const PromptArgs& a, const int block, const int n_heads, int* tile, int* head) {
    const PromptTile& t = a.tiles[block / n_heads];
    const int b = t.bundle, n = t.n_bundle, u = block - b * n_heads, eights = n_heads / 8 * 8;
    if (u < eights * n) {
        *tile = b + u % (8 * n) / 8;
        *head = u / (8 * n) * 8 + u % 8;
    } else {
        const int v = u - eights * n, rest = n_heads - eights;
        *tile = b + v / rest;
        *head = eights + v % rest;
    }
}

template <int HD>
__global__ __launch_bounds__(512, 2) void prompt_kernel(const LatentShape sh, const PromptArgs a, const int h0, const int n_heads) {
    constexpr int KS = HD / 32, DT = HD / 16, NT = 2, LOADS = HD / 32 + 1;  // LOADS: KiB of half a page
    __shared__ PromptSmem<HD> sm;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    int hl, item;
    tile_of_block(a, blockIdx.x, n_heads, &item, &hl);
    const int h = h0 + hl, H = sh.n_heads;
    const PromptTile t = a.tiles[item];
    const int npre = (t.prefix_len + 31) / 32 * 2;  // (pages of the prefix, in pairs)
    const int64_t page_bytes = (sh.latent_dim + kRopeDim) * 32LL;
    const scalar_row e_page = (scalar_row)a.e_page;
    auto expanded = [&](int vp) { return vp < npre ? t.prefix_e + vp : t.suffix_e + (vp - npre); };
    // a wave brings half of a page: keys and half of its rotated part, or the other half and a half of a pair's values
    auto fetch = [&](int vp0, int b) {
        const int pg = wave >> 1, e = expanded(min(vp0 + pg, t.page_end - 1));
        const char* kv = (const char*)a.kv + ((int64_t)hl * (a.n_expanded / 2) + e / 2) * (128 * HD);
        const char* rope = (const char*)a.pages + (int64_t)e_page[e] * page_bytes + sh.latent_dim * 32;
        if ((wave & 1) == 0) {
            const unsigned to = uniform(lds_address(sm.k[b][pg]));
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) load_to_lds(kv + (e & 1) * (32 * HD) + i * 1024, lane * 16, to + i * 1024);
            load_to_lds(rope, lane * 16, uniform(lds_address(sm.r[b][pg])));
        } else {
            const unsigned to = uniform(lds_address(sm.v[b][pg >> 1])) + (pg & 1) * (32 * HD);
            load_to_lds(rope + 1024, lane * 16, uniform(lds_address(sm.r[b][pg])) + 1024);
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) load_to_lds(kv + 64 * HD + (pg & 1) * (32 * HD) + i * 1024, lane * 16, to + i * 1024);
        }
    };
    const int n_tiles = (t.page_end - t.page_begin + 3) / 4;
    fetch(t.page_begin, 0);
    if (n_tiles > 1) fetch(t.page_begin + 4, 1);
    f16x8 qf[NT][KS];
    bf16x8 qr[NT][2];
    int pos[NT];   // of this lane's rows
    float c[NT];   // scale * log2(e) * the power of two its query was divided by
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int r = min(32 * wave + 16 * k + n, t.n_rows - 1);
        pos[k] = t.first_pos + r;
        const __bf16* q = (const __bf16*)a.q + ((int64_t)(t.row0 + r) * H + h) * (HD + kRopeDim) + 8 * g;
        typedef float f32x8 __attribute__((ext_vector_type(8)));
        f32x8 v[KS];
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
            v[j] = __builtin_convertvector(*(const bf16x8*)(q + 32 * j), f32x8);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(v[j][i]));
        }
        // q_n in [0.5, 1), but q_r at most 2^20 (its products with r shall not overflow where q_n is all but nothing; q_n's last bit is
        // then below 2^-44 of the query), and c a normal number
        bf16x8 rot[2];
        float most_r = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            rot[j] = *(const bf16x8*)(q + HD + 32 * j);
#pragma unroll
            for (int i = 0; i < 8; ++i) most_r = fmaxf(most_r, fabsf((float)rot[j][i]));
        }
        const int e = max(max(exponent_of(max_lane_groups(most)), exponent_of(max_lane_groups(most_r)) - 20), -100);
        const float down = __uint_as_float((unsigned)(127 - e) << 23);
        c[k] = sh.scale_log2e * __uint_as_float((unsigned)(127 + e) << 23);
#pragma unroll
        for (int j = 0; j < KS; ++j) qf[k][j] = __builtin_convertvector(v[j] * down, f16x8);
#pragma unroll
        for (int j = 0; j < 2; ++j) qr[k][j] = __builtin_convertvector(__builtin_convertvector(rot[j], f32x8) * down, bf16x8);
    }
    const int first_pos = t.first_pos + min(32 * wave, t.n_rows - 1), last_pos = t.first_pos + min(32 * wave + 31, t.n_rows - 1);  // of this wave's rows
    const bool idle = 32 * wave >= t.n_rows, few = a.lse && first_pos < kLowPositions;
    int some = 0;  // pages in bf16 among those of this tile?
    {
        const int* format = a.format + (int64_t)hl * a.n_chunks * 2;
        const int p_end = (t.prefix_e + min(t.page_end, npre) + 3) / 4, s_end = (t.suffix_e + max(t.page_end - npre, 0) + 3) / 4;
        for (int i = t.prefix_e / 4 * 2 + lane; i < 2 * p_end; i += 64) some |= format[i];
        for (int i = t.suffix_e / 4 * 2 + lane; i < 2 * s_end; i += 64) some |= format[i];
    }
    f32x4 O[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; ++d) O[k][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto tile = [&](const int vp0, const int b, auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        int format[4] = {0, 0, 0, 0};  // per pair: keys, values
        if constexpr (!PLAIN)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                format[i] = ((scalar_row)a.format)[((int64_t)hl * a.n_chunks + expanded(min(vp0 + (i & 2), t.page_end - 1)) / 4) * 2 + (i & 1)];
        f32x4 s[4][NT];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
#pragma unroll
            for (int k = 0; k < NT; ++k) s[p][k] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (PLAIN || !format[p & 2]) {
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    const f16x8 kf = *(const f16x8*)(sm.k[b][p] + (4 * j + g) * 128 + n * 8);
#pragma unroll
                    for (int k = 0; k < NT; ++k) s[p][k] = mfma16(kf, qf[k][j], s[p][k]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    const bf16x8 kf = *(const bf16x8*)(sm.k[b][p] + (4 * j + g) * 128 + n * 8);
#pragma unroll
                    for (int k = 0; k < NT; ++k) {
                        u32x4 bits = __builtin_bit_cast(u32x4, qf[k][j]);
                        asm volatile("" : "+v"(bits));  // (converted here each time: there are no registers to keep the results)
                        const f16x8 h = __builtin_bit_cast(f16x8, bits);
                        bf16x8 q;
#pragma unroll
                        for (int i = 0; i < 8; ++i) q[i] = (__bf16)(float)h[i];  // (they were bf16)
                        s[p][k] = mfma16(kf, q, s[p][k]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const bf16x8 kf = *(const bf16x8*)(sm.r[b][p] + (4 * j + g) * 128 + n * 8);
#pragma unroll
                for (int k = 0; k < NT; ++k) s[p][k] = mfma16(kf, qr[k][j], s[p][k]);
            }
        }
        if (few && 16 * vp0 < kLowPositions + 16) {
#pragma unroll 1
            for (int p = 0; p < 4; ++p) {
                const int low = vp0 + p < t.page_end ? ((scalar_row)a.e_low)[expanded(vp0 + p)] : -1;
                if (low < 0) continue;
                const _Float16* from = (const _Float16*)a.k_low + ((int64_t)hl * a.n_low + low) * (16 * HD) + g * 128 + n * 8;
                f32x4 rest[NT];
#pragma unroll
                for (int k = 0; k < NT; ++k) rest[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < KS; ++j) {
                    const f16x8 kf = *(const f16x8*)(from + j * 512);
#pragma unroll
                    for (int k = 0; k < NT; ++k) rest[k] = mfma16(kf, qf[k][j], rest[k]);
                }
#pragma unroll
                for (int x = 0; x < 4; ++x)  // (s is indexed by the unrolled x)
                    if (x == p)
#pragma unroll
                        for (int k = 0; k < NT; ++k) s[x][k] += rest[k] * 0x1p-11f;
            }
        }
        // pages that hold tokens ahead of some row, none at all, or the end of a prefix
        const bool whole = vp0 + 4 <= t.page_end && (vp0 + 4 <= npre ? 16 * vp0 + 64 <= t.prefix_len : vp0 >= npre && t.prefix_len + 16 * (vp0 - npre) + 63 <= first_pos);
        if (!whole) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const int vp = vp0 + p;
                // positions of the page begin at `first`; those of a prefix end with it, and a page that is not there has none
                const int first = vp < npre ? 16 * vp : t.prefix_len + 16 * (vp - npre);
                const int most = vp >= t.page_end ? -1 : vp < npre ? t.prefix_len - 1 : 0x7fffffff;
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[p][k][i] = first + 4 * g + i <= min(pos[k], most) ? s[p][k][i] : -INFINITY;
            }
        }
        uint2 pr[4][NT];
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            const float mx = max2(max2(max4(s[0][k]), max4(s[1][k])), max2(max4(s[2][k]), max4(s[3][k])));
            if (__any(!(mx * c[k] <= m[k]))) {
                const float mn = max2(m[k], max_lane_groups(mx) * c[k]);
                const float alpha = fast_exp2(m[k] - (mn == -INFINITY ? 0.f : mn));
                l[k] *= alpha;
#pragma unroll
                for (int d = 0; d < DT; ++d) O[k][d] *= alpha;
                m[k] = mn;
            }
            const float ref = m[k] == -INFINITY ? 0.f : m[k] - kWeightBits;  // (a row may see nothing of these pages)
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                f32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = fast_exp2(fmaf(s[p][k][i], c[k], -ref));
                l[k] += (w[0] + w[1]) + (w[2] + w[3]);
                // (in the type of the values they meet)
                pr[p][k] = PLAIN || !format[(p & 2) + 1] ? __builtin_bit_cast(uint2, __builtin_convertvector(w, f16x4)) : __builtin_bit_cast(uint2, __builtin_convertvector(w, bf16x4));
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const uint4 vf = *(const uint4*)(sm.v[b][ks] + (g * HD + 16 * d + n) * 8);
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const uint4 pf = make_uint4(pr[2 * ks][k].x, pr[2 * ks][k].y, pr[2 * ks + 1][k].x, pr[2 * ks + 1][k].y);
                    if (PLAIN || !format[2 * ks + 1]) O[k][d] = mfma16(__builtin_bit_cast(f16x8, vf), __builtin_bit_cast(f16x8, pf), O[k][d]);
                    else O[k][d] = mfma16(__builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, pf), O[k][d]);
                }
            }
    };
    auto all_tiles = [&](auto plain) {
        for (int i = 0, b = 0; i < n_tiles; ++i, b = b == kStages - 1 ? 0 : b + 1) {
            // this tile is here for all (the next may be on its way), and all are done with the one before, where the one after the next goes
            if (i + 1 < n_tiles) wait_loads_and_meet<LOADS>();
            else wait_loads_and_meet<0>();
            const int vp0 = t.page_begin + 4 * i;
            if (i + 2 < n_tiles) fetch(vp0 + 8, b == 0 ? kStages - 1 : b - 1);
            const bool ahead = vp0 >= npre && t.prefix_len + 16 * (vp0 - npre) > last_pos;  // of all of this wave's rows
            if (!ahead && !idle) tile(vp0, b, plain);
        }
    };
    if (__any(some)) all_tiles(no());
    else all_tiles(yes());
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int r = 32 * wave + 16 * k + n;
        const float total = sum_lane_groups(l[k]);
        if (r >= t.n_rows) continue;
        const float inv = total > 0.f ? 1.0f / total : total;  // (NaN stays what it is)
        if (t.part_row >= 0) {
            const int64_t at = (int64_t)hl * a.n_partial_rows + t.part_row + r;
            if (g == 0) a.ml[at] = make_float2(m[k] - kWeightBits, total);
#pragma unroll
            for (int d = 0; d < DT; ++d) *(f32x4*)(a.part + at * HD + 16 * d + 4 * g) = O[k][d] * inv;
        } else {
            const int64_t at = (int64_t)(t.row0 + r) * H + h;
            if (g == 0 && a.lse) a.lse[at] = (m[k] - kWeightBits + log2f(total)) * 0.6931471805599453f;
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

template <int R, int HD>
static hipError_t launch_prompt_as(const LatentShape& sh, const PromptArgs& a, hipStream_t s) {
    for (int h0 = 0; h0 < sh.n_heads; h0 += a.heads_at_once) {
        const int nh = sh.n_heads - h0 < a.heads_at_once ? sh.n_heads - h0 : a.heads_at_once;
        // a workgroup a compute unit (two at R = 256), unless there are fewer tokens than that
        const int parts = nh * (HD / 64), most = (a.n_chunks + 7) / 8, wish = a.units * (512 / R) / parts;
        const int split = wish < 1 ? 1 : (wish > most ? most : wish);
        hipLaunchKernelGGL((expand_kernel<R, HD>), dim3((unsigned)nh * split, HD / 64), dim3(512), 0, s, a, h0, nh);
        hipLaunchKernelGGL(prompt_kernel<HD>, dim3((unsigned)a.n_tiles * nh), dim3(512), 0, s, sh, a, h0, nh);
        if (a.n_merges > 0) hipLaunchKernelGGL(prompt_merge_kernel<HD>, dim3((unsigned)a.n_merges * nh, 8), dim3(256), 0, s, sh, a, h0, nh);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace latent

hipError_t launch_latent_prompt(const LatentShape& sh, const PromptArgs& a, hipStream_t s) {
    using namespace latent;
    if (sh.latent_dim == 512) return sh.head_dim == 128 ? launch_prompt_as<512, 128>(sh, a, s) : launch_prompt_as<512, 64>(sh, a, s);
    return sh.head_dim == 128 ? launch_prompt_as<256, 128>(sh, a, s) : launch_prompt_as<256, 64>(sh, a, s);
}

}  // namespace taper
