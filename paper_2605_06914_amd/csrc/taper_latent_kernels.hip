// gfx950 kernels of the decode step over a latent cache: one vector c_t of R values and a rotated key part r_t of 64 values
// a token, read once for all heads.
//
// Three launches.  absorb_kernel rewrites the queries, q_lat = (W_k[h]^T q_n, q_r).  latent_decode_kernel computes
// softmax(scale q_lat . (c, r)) . c for items of up to 128 query rows and some tokens, as partial rows.  finish_kernel merges
// a row's partials through their (max, sum) and applies W_v[h].
#include <cmath>
#include <type_traits>

#include "latent_device.h"

namespace taper {
namespace latent {

// ---------------------------------------------------------------------------
// absorb: q_lat[s,h,r] = sum_n q[s,h,n] W_k[h][n][r].  The contraction runs over W's rows, so a matrix operand needs 8 rows of
// one column in a lane: a lane loads 16 bytes of each of 8 rows and transposes the 8 x 8 block in registers (a v_perm per
// register).  Its 8 columns go to 8 different products, whose results then hold 8 consecutive r of a query.  One wave a
// (head, 128 columns); W is read once and stays in registers for all sequences.
// ---------------------------------------------------------------------------
template <int KS>  // head_dim / 32
__global__ __launch_bounds__(64) void absorb_kernel(const LatentShape sh, const LatentDecodeArgs a, const int s_per_block) {
    const int lane = threadIdx.x, n = lane & 15, g = lane >> 4, h = blockIdx.x, r0 = blockIdx.y * 128;
    const int R = sh.latent_dim, KD = R + kRopeDim, HD = 32 * KS, H = sh.n_heads;
    // lane n's columns are block 4 (n mod 4) + n / 4 of eight: a query's results then leave as 64 bytes in a row from four lanes
    const __bf16* w = (const __bf16*)a.w_up + (int64_t)h * 2 * HD * R + r0 + 8 * ((n & 3) * 4 + (n >> 2));
    bf16x8 wf[KS][8];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        u32x4 row[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) row[j] = *(const u32x4*)(w + (int64_t)(32 * ks + 8 * g + j) * R);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u32x4 c;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[j] = __builtin_amdgcn_perm(row[2 * j + 1][i / 2], row[2 * j][i / 2], i & 1 ? 0x07060302u : 0x05040100u);
            wf[ks][i] = __builtin_bit_cast(bf16x8, c);
        }
    }
    const int s_end = min(a.n_seqs, (int)(blockIdx.z + 1) * s_per_block);
    for (int s0 = blockIdx.z * s_per_block; s0 < s_end; s0 += 16) {
        const int s = min(s0 + n, a.n_seqs - 1);
        const __bf16* q = (const __bf16*)a.q + ((int64_t)s * H + h) * (HD + kRopeDim);
        bf16x8 qf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(q + 32 * ks + 8 * g);
        __bf16* to = (__bf16*)a.q_lat + ((int64_t)s * H + h) * KD;
        f32x4 acc[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) acc[i] = mfma16(wf[ks][i], qf[ks], acc[i]);
        }
        if (s0 + n >= a.n_seqs) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // (bf16, as the products with the cache take it)
            bf16x8 v;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (__bf16)acc[i][j];
            *(bf16x8*)(to + r0 + 8 * (4 * j + g)) = v;
            if (a.lse) {  // what the rounding took away: finish_kernel puts its effect on the normaliser back
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (__bf16)(acc[i][j] - (float)v[i]);
                *(bf16x8*)((__bf16*)a.q_rest + ((int64_t)s * H + h) * R + r0 + 8 * (4 * j + g)) = v;
            }
        }
        if (r0 == 0) {
            *(bf16x8*)(to + R + 8 * g) = *(const bf16x8*)(q + HD + 8 * g);
            *(bf16x8*)(to + R + 32 + 8 * g) = *(const bf16x8*)(q + HD + 32 + 8 * g);
        }
    }
}

// ---------------------------------------------------------------------------
// The attention.  A workgroup of 8 waves, two on each SIMD, holds up to 128 query rows, 16 a wave, and takes 64 tokens (4 pages, 72 KiB)
// at a time through LDS.  A wave makes the scores of its rows, S^T = C Q^T, weighs them and adds the values, O^T = C^T P^T, by itself: its
// queries (16 rows x 576 values: 72 registers) and accumulators (16 rows x 512 values: 128) stay with it, the weights leave the score
// product in the layout that the value product takes them in, and waves meet once a tile.  K and V are the same bytes; V's operand is
// columns of a token-major page: ds_read_b64_tr_b16 reads 4 tokens x 16 columns transposed.
// What bounds it: every wave reads the whole tile from LDS, for K and for V, 1088 KiB a tile and workgroup, which at 128 bytes a clock
// is 8700 clocks against 4350 of products; the matrix units are busy for 0.40 of the time.  (32 rows a wave, 4 waves, would halve that,
// but 144 + 256 registers leave none for operands in flight: it spilled.  Two groups of 4 waves in turns, one at its products while the
// other weighs, took 884 us where one group of 8 took 793.)
// Bringing a tile to LDS blocks the waves that ask for it (1230 clocks for its 72 KiB from the L2, 2200 from memory), so many rows a
// tile matter (a workgroup of 64 rows, whose waves shared the work by pages and columns, took 6300 clocks a tile), and waves without
// rows bring the tiles of items that leave some.  At 8 requests x 16 branches over 32768 shared tokens each and 32 single sequences, 64
// heads: 660 us, 950 TF/s; 32 single sequences of 1024 to 4096 tokens at 16 heads: 38.5 us, of which the cache's bytes take 16.
// ---------------------------------------------------------------------------
// Weights are taken relative to a row's reference, the largest score of some earlier tile, so that a tile's weights do not wait for its
// maximum.  A score that is more than this above its reference (in log2; a first tile always is) makes the wave take new references.
// Weights are then at most 2^6: a bf16 weight has 8 bits whatever its size, sums and accumulators are fp32.
constexpr float kMostAbove = 6.f;

template <int R>
struct DecodeSmem {
    unsigned sink[64];  // nobody reads it (see touch)
    __bf16 tile[2][4][(R + kRopeDim) * 16];
};

template <int R, bool FULL>  // FULL: all waves have rows
DEV void decode_item(const LatentShape& sh, const LatentDecodeArgs& a, const taper_latent_item& it, DecodeSmem<R>& sm) {
    constexpr int KD = R + kRopeDim, JK = KD / 32, DT = R / 16, PAGE = KD * 16, NT = 1;
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int row0 = wave * 16 * NT, busy = (it.n_rows + 16 * NT - 1) / (16 * NT);  // this wave's first row; waves that have rows
    const scalar_row row = (scalar_row)(a.bt + (int64_t)it.seq0 * a.bt_stride + it.page0);
    const int last_page = (it.n_tokens + 15) / 16 - 1, n_tiles = (it.n_tokens + 63) / 64;
    const char* pages = (const char*)a.pages;
    const float c = sh.scale_log2e;

    auto page = [&](int t, int pg) { return pages + (int64_t)row[min(4 * t + pg, last_page)] * (PAGE * 2); };  // (past the end: the last one)
    auto place = [&](int t, int pg) { return uniform(lds_address(sm.tile[t & 1][pg])); };
    // In LDS every other row of 16 tokens has its fours of tokens in the opposite order: V's operand takes 8 tokens of two rows at a time,
    // which would lie in the same banks (a third of the LDS's time went by in such conflicts), and K's 16-byte reads, which meet eight tokens
    // of each of two rows as well, stay without any.  (Not where waves only bring tiles: that takes 2 % longer so, and conflicts do not matter.)
    constexpr int TURN = FULL ? 12 : 0;
    const int lane_from = (lane ^ (lane >> 4 & 1) * TURN) * 16;
    auto load = [&](const char* from, unsigned to, int i) { load_to_lds(from + i * 1024, lane_from, to + i * 1024); };  // (scalar sums: one lane offset for all)
    constexpr int LOADS = PAGE / 1024;  // of half a page
    if (!FULL && wave >= busy) {  // bring the tiles
        const int others = 8 - busy;
        auto bring = [&](int t) {
            for (int x = wave - busy; x < 8; x += others) {  // half pages
                const char* from = page(t, x & 3) + (x >> 2) * PAGE;
                const unsigned to = place(t, x & 3) + (x >> 2) * PAGE;
#pragma unroll
                for (int i = 0; i < LOADS; ++i) load(from, to, i);
            }
        };
        bring(0);
        for (int t = 0; t < n_tiles; ++t) {
            wait_loads_and_meet<0>();
            if (t + 1 < n_tiles) bring(t + 1);
        }
        return;
    }
    const int pg = wave & 3, half_bytes = (wave >> 2) * PAGE;  // where all waves have rows each brings half of a page
    // and its lines into the L2 two tiles before that: pages are scattered, and from memory a tile takes longer than another's work
    constexpr int LINES = PAGE / 128, TOUCHES = (LINES + 63) / 64;
    auto touch = [&](const char* from) {
#pragma unroll
        for (int i = 0; i < TOUCHES; ++i) word_to_lds(from, min(64 * i + lane, LINES - 1) * 128, uniform(lds_address(sm.sink)));
    };
    const char *next = page(1, pg) + half_bytes, *next2 = page(2, pg) + half_bytes;
    if (FULL) {
        const char* from = page(0, pg) + half_bytes;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(from, place(0, pg) + half_bytes, i);
        touch(next2);
    }
    bf16x8 qf[NT][JK];
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const __bf16* q = (const __bf16*)a.q_lat + (int64_t)(it.row0 + min(row0 + 16 * k + n, it.n_rows - 1)) * KD + 8 * g;
#pragma unroll
        for (int j = 0; j < JK; ++j) qf[k][j] = *(const bf16x8*)(q + 32 * j);
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
    auto step = [&](const int t, auto last) {
        if (FULL) wait_loads_and_meet<TOUCHES>();  // tile t is here for all, and all are done with tile t - 1
        else wait_loads_and_meet<0>();
        constexpr bool bring = !decltype(last)::value && FULL;
        const char* const from = next;
        const unsigned to = place(t + 1, pg) + half_bytes;
        next = next2;
        next2 = page(t + 3, pg) + half_bytes;
        const __bf16* const tile = sm.tile[t & 1][0];
        if (last && it.n_tokens - 64 * t < 64) {
            // What follows the last token may be anything: zeros, so that its zero weight meets no NaN.  (Every wave writes all of them before
            // it reads any: nobody need wait for another.)
            for (int pg = 0; pg < 4; ++pg) {
                const int valid = it.n_tokens - 64 * t - 16 * pg;
                if (valid >= 16) continue;
                for (int i = lane; i < KD / 8 * 16; i += 64)
                    if (((i ^ (i >> 4 & 1) * TURN) & 15) >= valid) *(u32x4*)(sm.tile[t & 1][pg] + i * 8) = u32x4{0, 0, 0, 0};
            }
        }
        f32x4 s[4][NT];
        constexpr int AHEAD = 2;  // steps of two pages' operands in flight
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // two pages at a time: twice as many chains of products
            const __bf16* const k_at = tile + half * 2 * PAGE + lane_from / 2;
            bf16x8 kf[AHEAD][2];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int x = 0; x < 2; ++x) kf[j][x] = *(const bf16x8*)(k_at + x * PAGE + j * 512);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int k = 0; k < NT; ++k) s[2 * half + x][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < JK; ++j) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
#pragma unroll
                    for (int k = 0; k < NT; ++k) s[2 * half + x][k] = mfma16(kf[j % AHEAD][x], qf[k][j], s[2 * half + x][k]);
                    if (j + AHEAD < JK) kf[j % AHEAD][x] = *(const bf16x8*)(k_at + x * PAGE + (j + AHEAD) * 512);
                }
                if (bring && j % 4 == 1 && half * (LOADS + 1) / 2 + j / 4 < (half ? LOADS : (LOADS + 1) / 2)) load(from, to, half * (LOADS + 1) / 2 + j / 4);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (bring) touch(next2);
        bool higher = false;
#pragma unroll
        for (int k = 0; k < NT; ++k) {
            if (last)
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[p][k][i] = 64 * t + 16 * p + 4 * g + i < it.n_tokens ? s[p][k][i] : -INFINITY;
            const float mx = max2(max2(max4(s[0][k]), max4(s[1][k])), max2(max4(s[2][k]), max4(s[3][k])));
            higher |= !(mx * c <= m[k] + kMostAbove);
        }
        if (__any(higher)) {
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const float mx = max2(max2(max4(s[0][k]), max4(s[1][k])), max2(max4(s[2][k]), max4(s[3][k])));
                const float mn = max2(m[k], max_lane_groups(mx) * c), alpha = fast_exp2(m[k] - mn);
                m[k] = mn;
                l[k] *= alpha;
#pragma unroll
                for (int d = 0; d < DT; ++d) O[k][d] *= alpha;
            }
        }
        bf16x4 pr[4][NT];
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                f32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = fast_exp2(fmaf(s[p][k][i], c, -m[k]));
                l[k] += (w[0] + w[1]) + (w[2] + w[3]);
                pr[p][k] = __builtin_convertvector(w, bf16x4);  // (8 bits of each weight)
            }
        const __bf16* const v_at = tile + (lane >> 1 & 1) * 128 + ((4 * g + (n >> 2)) ^ (lane >> 1 & 1) * TURN) * 8 + (lane & 1) * 4;
        auto columns = [&](int x) {  // 16 columns of 32 tokens; x: column group, then pair of pages
            typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
            const __bf16* at = v_at + x / DT * 2 * PAGE + x % DT * 256;
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at), v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + PAGE));
            return cat(__builtin_bit_cast(bf16x4, v0), __builtin_bit_cast(bf16x4, v1));
        };
        constexpr int V_AHEAD = 4;
        bf16x8 vf[V_AHEAD];
#pragma unroll
        for (int x = 0; x < V_AHEAD; ++x) vf[x] = columns(x);
#pragma unroll
        for (int x = 0; x < 2 * DT; ++x) {
#pragma unroll
            for (int k = 0; k < NT; ++k) O[k][x % DT] = mfma16(vf[x % V_AHEAD], cat(pr[x / DT * 2][k], pr[x / DT * 2 + 1][k]), O[k][x % DT]);
            if (x + V_AHEAD < 2 * DT) vf[x % V_AHEAD] = columns(x + V_AHEAD);
            if (x % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (else more is read ahead than there are registers for)
        }
    };
    for (int t = 0; t < n_tiles - 1; ++t) step(t, std::false_type());
    step(n_tiles - 1, std::true_type());
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (nothing on its way to LDS when the workgroup ends)
#pragma unroll
    for (int k = 0; k < NT; ++k) {
        const int r = row0 + 16 * k + n;
        const float total = sum_lane_groups(l[k]), inv = 1.0f / total;
        if (r >= it.n_rows) continue;
        const int64_t at = it.part_row + r;
        // the row travels divided by its own sum, in half precision after division by a power of two of each eighth of its columns that
        // brings their largest magnitude into [0.5, 1): off by 2^-12 of that, whatever the magnitude, and half the bytes of fp32 rows
        PartStats* const st = a.stats + at;
#pragma unroll
        for (int e8 = 0; e8 < 8; ++e8) {
            float most = 0.f;
            f32x4 v[DT / 8];
#pragma unroll
            for (int d = 0; d < DT / 8; ++d) {
                v[d] = O[k][e8 * (DT / 8) + d] * inv;
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(v[d][i]));
            }
            const int e = exponent_of(max_lane_groups(most));
            if (g == 0) st->exponent[e8] = (signed char)e;
            const float down = __uint_as_float((unsigned)(127 - e) << 23);
            _Float16* to = (_Float16*)a.part + at * R + e8 * (R / 8) + 4 * g;
#pragma unroll
            for (int d = 0; d < DT / 8; ++d) *(f16x4*)(to + 16 * d) = __builtin_convertvector(v[d] * down, f16x4);
        }
        if (g == 0) {
            st->m = m[k];
            st->l = total;
        }
    }
}

template <int R>
__global__ __launch_bounds__(512, 2) void latent_decode_kernel(const LatentShape sh, const LatentDecodeArgs a) {
    __shared__ DecodeSmem<R> sm;
    const taper_latent_item it = a.items[blockIdx.x];
    if (it.n_rows <= 0) return;
    if (it.n_rows <= 112) decode_item<R, false>(sh, a, it, sm);
    else decode_item<R, true>(sh, a, it, sm);
}

// ---------------------------------------------------------------------------
// finish: merges the pieces of SB sequences' rows of one head and applies W_v[h]: out^T = W_v O^T, W's rows straight from memory
// (a lane's 16 bytes are 8 consecutive values of one row; asked for before the merge, whose reads they overlap), the merged rows
// through LDS as a sum of two bf16 values each, so that they are not rounded to one.
// ---------------------------------------------------------------------------
template <int R, int HD, int SB>
__global__ __launch_bounds__(512) void finish_kernel(const LatentShape sh, const LatentDecodeArgs a) {
    constexpr int PITCH = R + 8, PER = R * SB / 512, UN = SB == 4 ? 8 : 4;  // PER: columns of a thread; UN: pieces in flight
    typedef _Float16 part_t __attribute__((ext_vector_type(PER)));
    __shared__ __align__(16) __bf16 o[2][SB][PITCH];
    __shared__ float dots[SB][2], norm[SB];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4, h = blockIdx.x, s0 = blockIdx.y * SB;
    const int H = sh.n_heads;
    constexpr int VT = HD / 16;  // waves with a tile of 16 values
    const __bf16* w = (const __bf16*)a.w_up + ((int64_t)h * 2 + 1) * HD * R + (int64_t)(wave * 16 + n) * R + 8 * g;
    constexpr int EARLY = R / 64;  // (half of them: with all, two workgroups would not fit a compute unit's registers)
    bf16x8 wf[R / 32];
    if (wave < VT)
#pragma unroll
        for (int j = 0; j < EARLY; ++j) wf[j] = *(const bf16x8*)(w + 32 * j);
    {
        constexpr int THREADS = 512 / SB, LANES = THREADS < 64 ? THREADS : 64;
        const int i = tid / THREADS, d0 = tid % THREADS * PER, s = s0 + i, chunk = d0 / (R / 8);
        float acc[PER], M = -INFINITY, L = 0.f;
#pragma unroll
        for (int j = 0; j < PER; ++j) acc[j] = 0.f;
        const int b = s < a.n_seqs ? a.piece_start[s] : 0, e = s < a.n_seqs ? a.piece_start[s + 1] : 0;
        // 32 pieces at a time: a lane finds one's row and statistics, all of them their common maximum; the rows follow, some in flight
        for (int p0 = b; p0 < e; p0 += 32) {
            const int here = min(32, e - p0), mine = min(lane & 31, here - 1);
            const int r = a.piece_row[p0 + mine] + h;
            const float2 ml = *(const float2*)&a.stats[r];
            float most = ml.x;
#pragma unroll
            for (int x = 16; x; x >>= 1) most = fmaxf(most, __shfl_xor(most, x, 32));
            most = fmaxf(most, M);
            const float old = fast_exp2(M - most), w = (lane & 31) < here ? ml.y * fast_exp2(ml.x - most) : 0.f;
            float total = w;
#pragma unroll
            for (int x = 16; x; x >>= 1) total += __shfl_xor(total, x, 32);
            L = fmaf(L, old, total);
            M = most;
#pragma unroll
            for (int j = 0; j < PER; ++j) acc[j] *= old;
            for (int p = 0; p < here; p += UN) {
                part_t v[UN];
                int ex[UN];
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const int64_t at = __shfl(r, min(p + u, here - 1), 32);
                    ex[u] = a.stats[at].exponent[chunk];
                    v[u] = *(const part_t*)((const _Float16*)a.part + at * R + d0);
                }
#pragma unroll
                for (int u = 0; u < UN; ++u) {
                    const float up = __shfl(w, min(p + u, here - 1), 32) * __uint_as_float((unsigned)(127 + ex[u]) << 23);
                    if (p + u < here)
#pragma unroll
                        for (int j = 0; j < PER; ++j) acc[j] = fmaf(up, (float)v[u][j], acc[j]);
                }
            }
        }
        if (s < a.n_seqs) {
            const float inv = 1.0f / L;
#pragma unroll
            for (int j = 0; j < PER; ++j) acc[j] *= inv;
            if (a.lse) {
                // The scores were made with rounded queries: to first order the normaliser is off by the weighted mean of the scores'
                // errors, scale (q - rounded q) . (sum_t p_t c_t).
                const __bf16* rest = (const __bf16*)a.q_rest + ((int64_t)s * H + h) * R + d0;
                float dot = 0.f;
#pragma unroll
                for (int j = 0; j < PER; ++j) dot = fmaf((float)rest[j], acc[j], dot);
#pragma unroll
                for (int x = LANES / 2; x; x >>= 1) dot += __shfl_xor(dot, x);
                if (lane % LANES == 0) dots[i][tid % THREADS / 64] = dot;
                if (d0 == 0) norm[i] = M + log2f(L);
            }
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const __bf16 hi = (__bf16)acc[j];
            o[0][i][d0 + j] = hi;
            o[1][i][d0 + j] = (__bf16)(acc[j] - (float)hi);
        }
    }
    __syncthreads();
    if (a.lse && tid < SB && s0 + tid < a.n_seqs) {
        float dot = 0.f;
        for (int x = 0; x < (512 / SB + 63) / 64; ++x) dot += dots[tid][x];
        a.lse[(int64_t)(s0 + tid) * H + h] = (norm[tid] + dot * sh.scale_log2e) * 0.6931471805599453f;
    }
    if (wave >= VT) return;
#pragma unroll
    for (int j = EARLY; j < R / 32; ++j) wf[j] = *(const bf16x8*)(w + 32 * j);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < R / 32; ++j) {
        acc = mfma16(wf[j], *(const bf16x8*)(&o[1][n % SB][32 * j + 8 * g]), acc);
        acc = mfma16(wf[j], *(const bf16x8*)(&o[0][n % SB][32 * j + 8 * g]), acc);
    }
    if (n < SB && s0 + n < a.n_seqs)
        *(bf16x4*)((__bf16*)a.out + ((int64_t)(s0 + n) * H + h) * HD + wave * 16 + 4 * g) = __builtin_convertvector(acc, bf16x4);
}

// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void latent_append_kernel(const __bf16* __restrict__ latent, const int64_t latent_stride,
                                                            const __bf16* __restrict__ rope, const int64_t rope_stride,
                                                            const int64_t* __restrict__ slots, __bf16* __restrict__ pages,
                                                            const int64_t n, const int64_t n_slots, const int R) {
    const int per = (R + kRopeDim) / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n * per; i += (int64_t)gridDim.x * 256) {
        const int64_t tok = i / per, slot = slots[tok];
        const int d8 = (int)(i - tok * per);
        if (slot < 0 || slot >= n_slots) continue;
        const __bf16* from = 8 * d8 < R ? latent + tok * latent_stride + 8 * d8 : rope + tok * rope_stride + (8 * d8 - R);
        *(bf16x8*)(pages + ((slot >> 4) * per + d8) * 128 + (slot & 15) * 8) = *(const bf16x8*)from;
    }
}

}  // namespace latent

using namespace latent;

hipError_t launch_latent_append(int latent_dim, int64_t n, const void* latent, int64_t latent_stride, const void* rope, int64_t rope_stride,
                                const int64_t* slots, void* pages, int64_t n_slots, hipStream_t s) {
    const int64_t threads = n * ((latent_dim + kRopeDim) / 8);
    const int64_t blocks = (threads + 255) / 256, most = 1 << 20;  // (a launch has fewer than 2^32 threads)
    hipLaunchKernelGGL(latent_append_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, (const __bf16*)latent, latent_stride,
                       (const __bf16*)rope, rope_stride, slots, (__bf16*)pages, n, n_slots, latent_dim);
    return hipGetLastError();
}

template <int R, int HD>
static void launch_finish(bool many, const LatentShape& sh, const LatentDecodeArgs& a, hipStream_t s) {
    if (many) hipLaunchKernelGGL((finish_kernel<R, HD, 16>), dim3(sh.n_heads, (a.n_seqs + 15) / 16), dim3(512), 0, s, sh, a);
    else hipLaunchKernelGGL((finish_kernel<R, HD, 4>), dim3(sh.n_heads, (a.n_seqs + 3) / 4), dim3(512), 0, s, sh, a);
}

hipError_t launch_latent_decode(const LatentShape& sh, const LatentDecodeArgs& a, hipStream_t s) {
    const int s_per_block = a.n_seqs <= 256 ? 16 : 64;  // (W is read again for each block of sequences; few sequences leave little else to do at once)
    const dim3 grid(sh.n_heads, sh.latent_dim / 128, (a.n_seqs + s_per_block - 1) / s_per_block);
    if (sh.head_dim == 128) hipLaunchKernelGGL((absorb_kernel<4>), grid, dim3(64), 0, s, sh, a, s_per_block);
    else hipLaunchKernelGGL((absorb_kernel<2>), grid, dim3(64), 0, s, sh, a, s_per_block);
    if (sh.latent_dim == 512) hipLaunchKernelGGL((latent_decode_kernel<512>), dim3(a.n_items), dim3(512), 0, s, sh, a);
    else hipLaunchKernelGGL((latent_decode_kernel<256>), dim3(a.n_items), dim3(512), 0, s, sh, a);
    // Sixteen sequences a workgroup read W_v once for all of them; where that leaves most of the chip idle, four.
    const bool many = (int64_t)sh.n_heads * ((a.n_seqs + 15) / 16) >= 256;
    if (sh.latent_dim == 512 && sh.head_dim == 128) launch_finish<512, 128>(many, sh, a, s);
    else if (sh.latent_dim == 512) launch_finish<512, 64>(many, sh, a, s);
    else if (sh.head_dim == 128) launch_finish<256, 128>(many, sh, a, s);
    else launch_finish<256, 64>(many, sh, a, s);
    return hipGetLastError();
}

}  // namespace taper
