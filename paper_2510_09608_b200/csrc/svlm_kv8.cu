// Key/value movement of the 8-bit cache (layout and rules: svlm_store8.h): writing appended tokens, and widening a layer to bf16 for
// the chunk kernels.  Both are streaming kernels, bound by latency and HBM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "svlm_dev.h"
#include "svlm_e4m3.cuh"
#include "svlm_launch.h"
#include "svlm_ptx.cuh"
#include "svlm_rope.cuh"
#include "svlm_store8.h"

namespace {

__device__ __forceinline__ int axis_of(const SvlmCacheDev& cd, int pair) {
    return cd.rope_mode == 0 ? 0 : (pair < cd.sec_t ? 0 : (pair < cd.sec_th ? 1 : 2));
}
__device__ __forceinline__ SvlmHead8* heads_of(const SvlmCacheDev& cd) {
    return reinterpret_cast<SvlmHead8*>(static_cast<unsigned char*>(cd.tmaps) + 512);
}
// Factors of pairs 8 g .. 8 g + 7 at positions p; a short loop, since this is code that runs once.
__device__ __forceinline__ void factors8(const SvlmCacheDev& cd, int g, const int (&p)[3], float2 (&cs)[8]) {
    const float2* tab = reinterpret_cast<const float2*>(cd.rope_tab);
    const int half = cd.head_dim / 2;
    bool far = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int axis = axis_of(cd, g * 8 + e), c = axis == 0 ? p[0] : (axis == 1 ? p[1] : p[2]);
        cs[e] = svlm_rope_cs_batched(tab, half, g * 8 + e, c);
        far |= c <= -65536 || c >= 65536;
    }
    if (far)
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const int axis = axis_of(cd, g * 8 + e);
            const float2 f = svlm_rope_cs(tab, half, g * 8 + e, axis == 0 ? p[0] : (axis == 1 ? p[1] : p[2]), cd.theta[g * 8 + e]);
#pragma unroll
            for (int q = 0; q < 8; ++q) if (q == e) cs[q] = f;
        }
}

// One thread block per (16 appended tokens, share of the [layer][kv_head] rows).  A block of the cache has one exponent for all its new
// tokens, so it belongs to the first of them: the thread block serves the cache's blocks that begin with one of its tokens, normally
// one or two (a token is first where its slot is the block's first or the slot before it holds no token of this append); two thread blocks share them, the
// second has all but the first one.  (One after another the two in which an append begins were everybody's wait: 12 tokens of 4 heads of 128 10.4 us,
// 7.1 now.)  A thread has 8 pairs (i, i + D/2) of one slot.  early: the caller vouches that the kernel before this one writes none of this cache's metadata; the chain up to the
// factors is then walked while it still runs.  Bound by latency: slots, ordinals, positions, factors one after another, then the rows; one warp per block with its 16
// tokens one after another in unrolled code took 10 us for one token and 24 for nine, which was the fetching of that code.
template <int D, bool ANYWHERE>
__global__ void __launch_bounds__(SVLM_BLOCK8 * D / 16) kv_write8_kernel(SvlmCacheDev cd, SvlmStore8 st, int layer, const uint16_t* K, const uint16_t* V,
                                                                        const int* pos, int n, int rows_per_block, int early) {
    using namespace svlm_ptx;
    constexpr int T = SVLM_BLOCK8, HALF = D / 2, GROUPS = HALF / 8, THREADS = T * GROUPS, WARPS = THREADS / 32;
    __shared__ unsigned s_first, s_most[2][WARPS];
    __shared__ int s_slot[T];
    bool entered = false;                                            // (every thread block waits: who starts behind this kernel finds all work before it done)
    auto enter = [&] {
        if (entered) return;
        entered = true;
        pdl_wait();
        pdl_launch_dependents();
    };
    if (!early) enter();
    const int tid = threadIdx.x, lane = tid & 31, j = tid / GROUPS, g = tid % GROUPS;
    if (ld_l2(&cd.ctrl->append_n) != n) {                            // the metadata append was dropped (capacity)
        enter();
        return;
    }
    const long long first = ld_l2(&cd.ctrl->n_total) - n;            // ordinal of the append's first token
    if (tid < 32) {
        const int i = (blockIdx.x >> 1) * T + lane;
        bool mine = lane < T && i < n;
        const int slot = mine ? ld_l2(cd.new_slot + i) : 0;
        if (mine) {
            mine = ld_l2(cd.slot_gid + slot) == first + i;           // (an eviction may have dropped it since)
            if (slot % T) mine = mine && ld_l2(cd.slot_gid + slot - 1) < first;
        }
        const unsigned all = __ballot_sync(0xffffffffu, mine);
        if (lane < T) s_slot[lane] = slot;
        if (lane == 0) s_first = all;
    }
    __syncthreads();
    const int n_rows = layer < 0 ? cd.layers * cd.kv_heads : cd.kv_heads;
    const int row0 = blockIdx.y * rows_per_block, row1 = min(n_rows, row0 + rows_per_block);
    const int first_row = layer < 0 ? 0 : layer * cd.kv_heads;
    for (unsigned left = blockIdx.x & 1 ? s_first & (s_first - 1) : s_first & (0u - s_first); left; left &= left - 1) {
        const int base = s_slot[__ffs(left) - 1] & ~(T - 1), slot = base + j;
        const long long gid = ld_l2(cd.slot_gid + slot);
        const bool fresh = gid >= first, old = gid >= 0 && gid < first;      // old: holds the block to its exponent
        const int any_old = __syncthreads_or(old);
        float2 cs[8];
        if (fresh) {
            int p[3];
            if (layer <= 0) {
                const int* at = pos + (gid - first) * (cd.rope_mode == 0 ? 1 : 3);
#pragma unroll
                for (int k = 0; k < 3; ++k) p[k] = ld_in(at + (cd.rope_mode == 0 ? 0 : k));
                if (blockIdx.y == 0) {
                    if (g == 0) st.native[slot] = p[0];
                    const int before = any_old ? st.apart[base / T] : 0;
                    if (before != 0)                                 // beside tokens that are to be turned: this one by nothing
#pragma unroll
                        for (int k = 0; k < D / 4 / GROUPS; ++k) st.turn[(size_t)slot * (D / 4) + g * (D / 4 / GROUPS) + k] = make_uint2(0x3c003c00u, 0u);
                }
            } else {
                const int c0 = ld_l2(cd.slot_c + slot), shift = ld_l2(st.native + slot) - c0;
                p[0] = c0 + shift;
#pragma unroll
                for (int k = 1; k < 3; ++k) p[k] = ld_l2(cd.slot_c + (size_t)k * cd.n_slots + slot) + shift;
            }
#pragma unroll 4
            for (int e = 0; e < 8; ++e) {
                const int axis = axis_of(cd, g * 8 + e);
                const float2 f = rope_cs_exact(st.rope64, HALF, g * 8 + e, axis == 0 ? p[0] : (axis == 1 ? p[1] : p[2]), cd.theta[g * 8 + e]);
#pragma unroll
                for (int q = 0; q < 8; ++q) if (q == e) cs[q] = f;
            }
        }
        if (layer <= 0 && blockIdx.y == 0) {
            const int before = any_old ? st.apart[base / T] : 0;
            __syncthreads();                                         // everybody has read it
            if (tid == 0) st.apart[base / T] = before == 0 ? 0 : MIXED8;
        }
        enter();
        // A block that begins: the layers that are still to come have nothing in it yet.  (An eviction behind layer 0's append looks at their exponents,
        // and what a page's earlier tokens have left there may be 2^100 above everything.)
        if (layer == 0 && blockIdx.y == 0 && !any_old)
            for (int r = cd.kv_heads + tid; r < cd.layers * cd.kv_heads; r += THREADS) st.exps[((size_t)r * cd.n_slots + base) / T] = NO_EXPONENTS;
        for (int r = row0; r < row1; ++r) {
            const int l = r / cd.kv_heads, h = r - l * cd.kv_heads;
            const size_t row = (size_t)(first_row + r) * cd.n_slots, src = (((size_t)l * n + (fresh ? gid - first : 0)) * cd.kv_heads + h) * D + g * 8;
            float x[2][2][8];                                        // [keys, values][half]
            unsigned most[2] = {0, 0};
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const uint16_t* at = (which ? V : K) + src + hf * HALF;
                    uint4 raw = make_uint4(0, 0, 0, 0);
                    if (fresh) {
                        if (ANYWHERE) {
                            unsigned w[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) w[k] = (unsigned)ld_in(at + 2 * k) | (unsigned)ld_in(at + 2 * k + 1) << 16;
                            raw = make_uint4(w[0], w[1], w[2], w[3]);
                        } else {
                            raw = ld_in(reinterpret_cast<const uint4*>(at));
                        }
                    }
                    const unsigned w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        x[which][hf][2 * k] = __uint_as_float(w[k] << 16);
                        x[which][hf][2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                    }
                }
            if (fresh)
#pragma unroll
                for (int e = 0; e < 8; ++e) rotate_exact(x[0][0][e], x[0][1][e], cs[e]);
#pragma unroll
            for (int which = 0; which < 2; ++which) {
#pragma unroll
                for (int e = 0; e < 8; ++e) most[which] = max(most[which], max(finite_bits(x[which][0][e]), finite_bits(x[which][1][e])));
                most[which] = __reduce_max_sync(0xffffffffu, most[which]);
                if (lane == 0) s_most[which][tid >> 5] = most[which];
            }
            unsigned* exp_at = st.exps + (row + base) / T;
            const unsigned held = any_old ? ld_l2(exp_at) : 0;
            unsigned exps = 0;
            __syncthreads();                                         // (the exponents are read, too)
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                unsigned char* dst = (which ? st.V : st.K) + (row + slot) * D + g * 8;
                unsigned top = 0;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) top = max(top, s_most[which][w]);
                int ex = block_exponent(top);
                if (any_old) {
                    const int before = exponent_of(held, which);
                    if (ex > before && old) {                        // the block's earlier values in the new unit
                        const float f = ex - before > 126 ? 0.f : pow2i(before - ex);
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf) {
                            uint2* at = reinterpret_cast<uint2*>(dst + hf * HALF);
                            const uint2 v = *at;
                            unsigned w[2] = {v.x, v.y};
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const float2 a = e4m3x2_to_float2((uint16_t)w[k]), b = e4m3x2_to_float2((uint16_t)(w[k] >> 16));
                                w[k] = to_e4m3x2(a.x * f, a.y * f) | (unsigned)to_e4m3x2(b.x * f, b.y * f) << 16;
                            }
                            *at = make_uint2(w[0], w[1]);
                        }
                    }
                    ex = max(ex, before);
                }
                const float unit = pow2i(-ex), limit = ex == E8_MAX ? E8_TOP : 448.f;      // (256 * 2^120 would be infinite)
                if (fresh)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        unsigned w[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float* y = &x[which][hf][4 * k];
                            w[k] = to_e4m3x2(y[0] * unit, y[1] * unit, limit) | (unsigned)to_e4m3x2(y[2] * unit, y[3] * unit, limit) << 16;
                        }
                        *reinterpret_cast<uint2*>(dst + hf * HALF) = make_uint2(w[0], w[1]);
                    }
                exps |= (unsigned)(ex & 255) << (8 * which);
            }
            if (tid == 0) {
                *exp_at = exps;
                atomicMax(st.most + first_row + r, exponent_of(exps, 0) + MOST8_BIAS);
            }
            __syncthreads();                                         // the maxima are read
        }
    }
    enter();
}

// One thread block per page of the list, a warp per block of 16 slots; blockIdx.y: the cache.  The thread blocks behind the pages' each take a
// [layer][kv_head] row's largest exponent of its keys (SvlmStore8::most) anew: over the blocks that have lost nothing, and over those that
// have, whose exponent may be a lost token's, as far as that is not more than 2^20 above.
template <int D>
__global__ void __launch_bounds__(256) shift8_kernel(SvlmCacheList list, SvlmStore8List stores) {
    using namespace svlm_ptx;
    __shared__ SvlmCacheDev cd;
    svlm_load_desc(&cd, list.cd[blockIdx.y]);
    pdl_wait();
    pdl_launch_dependents();
    const int n_tiles = ld_l2(&cd.ctrl->n_tiles);
    if ((int)blockIdx.x >= cd.n_pages) {
        __shared__ int s_all, s_whole;
        if (threadIdx.x == 0) s_all = s_whole = E8_MIN;
        __syncthreads();
        const int row = blockIdx.x - cd.n_pages;
        const unsigned* exps = stores.at[blockIdx.y].exps + (size_t)row * (cd.n_slots / SVLM_BLOCK8);
        int all = E8_MIN, whole = E8_MIN;
#pragma unroll 4
        for (int u = threadIdx.x; u < 8 * n_tiles; u += 256) {
            const int4 tl = ld_l2(reinterpret_cast<const int4*>(cd.tiles + (u >> 3)));
            const int k0 = (u & 7) * SVLM_BLOCK8, lo = max(tl.y - k0, 0), hi = min(tl.z - k0, SVLM_BLOCK8);
            if (lo >= hi) continue;
            const int e = exponent_of(ld_l2(exps + (tl.x * SVLM_PAGE + k0) / SVLM_BLOCK8), 0);
            all = max(all, e);
            if (lo == 0) whole = max(whole, e);
        }
        all = __reduce_max_sync(0xffffffffu, all);
        whole = __reduce_max_sync(0xffffffffu, whole);
        if ((threadIdx.x & 31) == 0) { atomicMax(&s_all, all); atomicMax(&s_whole, whole); }
        __syncthreads();
        if (threadIdx.x == 0) {
            stores.at[blockIdx.y].most[row] = (s_whole == E8_MIN ? s_all : min(s_all, s_whole + 20)) + MOST8_BIAS;
            if (row < cd.kv_heads) heads_of(cd)[row].late = 0;
        }
        return;
    }
    if ((int)blockIdx.x >= n_tiles) return;
    const SvlmStore8& st = stores.at[blockIdx.y];
    const int4 tile = ld_l2(reinterpret_cast<const int4*>(cd.tiles + blockIdx.x));       // page, lo, hi, pad
    const int lane = threadIdx.x & 31, k0 = (threadIdx.x >> 5) * SVLM_BLOCK8, off = k0 + (lane & 15), base = tile.x * SVLM_PAGE + k0;
    const int S = (int)ld_l2(&cd.ctrl->shift_total);
    const bool live = off >= tile.y && off < tile.z;
    const unsigned tokens = __ballot_sync(0xffffffffu, live) & 0xffffu;
    if (tokens == 0) return;
    const int apart = live ? S - (ld_l2(st.native + base + (lane & 15)) - ld_l2(cd.slot_c + base + (lane & 15))) : 0;
    const int one = __shfl_sync(0xffffffffu, apart, __ffs(tokens) - 1);
    const bool same = __all_sync(0xffffffffu, !live || apart == one);
    if (lane == 0) st.apart[base / SVLM_BLOCK8] = same ? one : MIXED8;
    if (same && one == 0) return;
    const float2* tab = reinterpret_cast<const float2*>(cd.rope_tab);
#pragma unroll 4
    for (int i = 0; i < SVLM_BLOCK8; ++i) {
        const int by = __shfl_sync(0xffffffffu, apart, i);
        if (lane >= D / 4) continue;
        float2 f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) f[e] = svlm_rope_cs_batched(tab, D / 2, 2 * lane + e, by);
        if (by <= -65536 || by >= 65536)
#pragma unroll
            for (int e = 0; e < 2; ++e) f[e] = svlm_rope_cs(tab, D / 2, 2 * lane + e, by, cd.theta[2 * lane + e]);
        const __half2 c = __floats2half2_rn(f[0].x, f[1].x), s = __floats2half2_rn(f[0].y, f[1].y);
        st.turn[(size_t)(base + i) * (D / 4) + lane] = make_uint2(*reinterpret_cast<const unsigned*>(&c), *reinterpret_cast<const unsigned*>(&s));
    }
}

// One thread block per (page, KV head); a thread has 8 pairs of four tokens, which usually share their rotation (what follows the last
// evicted token shares one shift), so its factors are looked up once.  early: as above, the kernel before this one writes none of the cache's metadata (but
// may write this layer's bytes).  half: the unit of a head's keys is kept with the bytes (SvlmStore8::most).  Where a block that has lost tokens
// owes its unit to one of them, it may be 2^20 above that (see shift8_kernel); what is more than 2^6 above then (448 sqrt(2) 2^6 is a half) is held as
// 2^6 above: a key that is 2^26 times all other blocks' decides its rows' softmax either way, by the sign of its score, which its direction gives.
// One layer of 10,000 tokens of 4 heads of 128: 9 us, 31 MB; 20 with a thread's four heads one after another and the unit found by each thread block for itself.
template <int D, bool HALF_KEYS>
__device__ __forceinline__ void widen8(const SvlmCacheDev& cd, const SvlmStore8& st, int layer, int n_q, int early) {
    using namespace svlm_ptx;
    constexpr int HALF = D / 2, GROUPS = HALF / 8, TOKENS = 4;
    if (!early) {
        pdl_wait();
        pdl_launch_dependents();
    }
    const int n_tiles = ld_l2(&cd.ctrl->n_tiles);
    const int4 tile = ld_l2(reinterpret_cast<const int4*>(cd.tiles + blockIdx.x));      // page, lo, hi, pad (left over from earlier behind the list's end)
    const int off = threadIdx.x / GROUPS, g = threadIdx.x % GROUPS, h = blockIdx.y;
    int by[TOKENS], turned = 0;
    bool live[TOKENS];
    float2 cs[8];
    auto factors = [&](int c) {
        const int p[3] = {c, c, c};
        factors8(cd, g, p, cs);
        turned = c;
    };
    const bool here = (int)blockIdx.x < n_tiles;
    if (here) {
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const int o = off + 32 * i, slot = tile.x * SVLM_PAGE + o;
            live[i] = o >= tile.y && o < tile.z;
            by[i] = live[i] ? ld_l2(cd.slot_c + slot) - ld_l2(st.native + slot) : 0;
        }
        factors(live[0] ? by[0] : (live[1] ? by[1] : (live[2] ? by[2] : by[3])));
    }
    if (early) {
        pdl_wait();
        pdl_launch_dependents();
    }
    if (!here) return;
    const int unit = HALF_KEYS ? ld_l2(st.most + layer * cd.kv_heads + h) - MOST8_BIAS : 0;
    if (HALF_KEYS && blockIdx.x == 0 && threadIdx.x == 0) heads_of(cd)[h].unit = unit;
    const size_t row0 = ((size_t)layer * cd.kv_heads + h) * cd.n_slots + (size_t)tile.x * SVLM_PAGE + off;
    uint2 raw[TOKENS][4];                                    // low and high halves of the key, of the value
    unsigned exps[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
        const unsigned char* k = st.K + (row0 + 32 * i) * D + g * 8;
        const unsigned char* v = st.V + (row0 + 32 * i) * D + g * 8;
        auto two = [&](const unsigned char* p) { return live[i] ? *reinterpret_cast<const uint2*>(p) : make_uint2(0, 0); };
        raw[i][0] = two(k); raw[i][1] = two(k + HALF);
        raw[i][2] = two(v); raw[i][3] = two(v + HALF);
        exps[i] = live[i] ? ld_l2(st.exps + (row0 + 32 * i) / SVLM_BLOCK8) : 0;
    }
    if (HALF_KEYS) {                                         // values that are not finite: see svlm_store8.h
        unsigned any = 0;
#pragma unroll
        for (int i = 0; i < TOKENS; ++i)
#pragma unroll
            for (int q = 2; q < 4; ++q) any |= nan_bytes(raw[i][q].x) | nan_bytes(raw[i][q].y);
        if (__builtin_expect(any != 0, 0)) {
            const long long first = ld_l2(&cd.ctrl->n_total) - n_q;
#pragma unroll
            for (int i = 0; i < TOKENS; ++i)
                if (live[i] && ld_l2(cd.slot_gid + tile.x * SVLM_PAGE + off + 32 * i) > first)
#pragma unroll
                    for (int q = 2; q < 4; ++q)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            unsigned& w = k ? raw[i][q].y : raw[i][q].x;
                            const unsigned nan = nan_bytes(w);
                            w &= ~(nan * 0xffu);
                            if (nan) heads_of(cd)[h].late = 1;
                        }
        }
    }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) {
        if (live[i] && by[i] != turned) factors(by[i]);
        const int up = exponent_of(exps[i], 0) - unit;       // (f16: 0 at most, but for the case above)
        const float ku = pow2i(max(-126, min(HALF_KEYS ? 6 : 127, up))), vu = pow2i(exponent_of(exps[i], 1));
        auto key = [&](float p, float q) {
            if (HALF_KEYS) {
                const __half2 y = __floats2half2_rn(p, q);
                return *reinterpret_cast<const unsigned*>(&y);
            }
            const __nv_bfloat162 y = __floats2bfloat162_rn(p, q);
            return *reinterpret_cast<const unsigned*>(&y);
        };
        auto value = [&](const float2& w) {
            const __nv_bfloat162 y = __floats2bfloat162_rn(w.x * vu, w.y * vu);
            return *reinterpret_cast<const unsigned*>(&y);
        };
        unsigned w[4][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            auto two = [&](const uint2& r) { return e4m3x2_to_float2((uint16_t)((e < 2 ? r.x : r.y) >> (16 * (e & 1)))); };
            const float2 x0 = two(raw[i][0]), y0 = two(raw[i][1]), f = cs[2 * e], f1 = cs[2 * e + 1];
            w[0][e] = key((x0.x * f.x - y0.x * f.y) * ku, (x0.y * f1.x - y0.y * f1.y) * ku);
            w[1][e] = key((y0.x * f.x + x0.x * f.y) * ku, (y0.y * f1.x + x0.y * f1.y) * ku);
            w[2][e] = value(two(raw[i][2]));
            w[3][e] = value(two(raw[i][3]));
        }
        const size_t out = ((size_t)h * cd.n_slots + (size_t)tile.x * SVLM_PAGE + off + 32 * i) * D + g * 8;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<uint4*>((q < 2 ? cd.K : cd.V) + out + (q & 1) * HALF) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
    }
}

template <int D, bool HALF_KEYS>
__global__ void __launch_bounds__(2 * D) widen8_kernel(SvlmCacheDev cd, SvlmStore8 st, int layer, int n_q, int early) {
    widen8<D, HALF_KEYS>(cd, st, layer, n_q, early);
}
// blockIdx.z: the cache (sixteen streams, 32/8 heads of 128 over 2,900 keys: 74 tokens each, append and attention 322 us a layer, 370 with a launch for each).
template <int D, bool HALF_KEYS>
__global__ void __launch_bounds__(2 * D) widen8_batch_kernel(SvlmCacheList list, SvlmStore8List stores, int layer, int early) {
    __shared__ SvlmCacheDev cd;
    svlm_load_desc(&cd, list.cd[blockIdx.z]);
    widen8<D, HALF_KEYS>(cd, stores.at[blockIdx.z], layer, stores.n_q[blockIdx.z], early);
}

}  // namespace

cudaError_t svlm_launch_kv_write8(const SvlmCacheDev& cd, const SvlmStore8& st8, int layer, const void* K, const void* V, const int* pos, int n,
                                  bool early, cudaStream_t st) {
    const int x = 2 * ((n + SVLM_BLOCK8 - 1) / SVLM_BLOCK8);
    const int rows = layer < 0 ? cd.layers * cd.kv_heads : cd.kv_heads;
    // one row per thread block while that leaves the grid at a few of them per SM, then up to eight
    int per = 1;
    while (per < 8 && (long long)x * ((rows + per - 1) / per) > 8 * svlm_sm_count()) per *= 2;
    const dim3 grid(x, (rows + per - 1) / per);
    const uint16_t* k = static_cast<const uint16_t*>(K);
    const uint16_t* v = static_cast<const uint16_t*>(V);
    const bool anywhere = (((uintptr_t)K | (uintptr_t)V) & 15) != 0;
    const auto kernel = cd.head_dim == 128 ? (anywhere ? kv_write8_kernel<128, true> : kv_write8_kernel<128, false>)
                                           : (anywhere ? kv_write8_kernel<64, true> : kv_write8_kernel<64, false>);
    return svlm_launch_chained(kernel, grid, dim3(SVLM_BLOCK8 * cd.head_dim / 16), 0, 1, st, cd, st8, layer, k, v, pos, n, per, (int)early);
}

cudaError_t svlm_launch_shift8(const SvlmCacheList& list, const SvlmStore8List& stores, const SvlmCacheDev& geom, cudaStream_t st) {
    return svlm_launch_chained(geom.head_dim == 128 ? shift8_kernel<128> : shift8_kernel<64>, dim3(geom.n_pages + geom.layers * geom.kv_heads, list.n), dim3(256), 0, 1, st, list, stores);
}

cudaError_t svlm_launch_widen8(const SvlmCacheDev& cd, const SvlmStore8& st8, int layer, int n_q, bool half, bool early, cudaStream_t st) {
    const auto kernel = cd.head_dim == 128 ? (half ? widen8_kernel<128, true> : widen8_kernel<128, false>) : (half ? widen8_kernel<64, true> : widen8_kernel<64, false>);
    return svlm_launch_chained(kernel, dim3(cd.n_pages, cd.kv_heads), dim3(2 * cd.head_dim), 0, 1, st, cd, st8, layer, n_q, (int)early);
}

cudaError_t svlm_launch_widen8_batch(const SvlmCacheList& list, const SvlmStore8List& stores, const SvlmCacheDev& geom, int layer, bool half, bool early, cudaStream_t st) {
    const auto kernel = geom.head_dim == 128 ? (half ? widen8_batch_kernel<128, true> : widen8_batch_kernel<128, false>)
                                             : (half ? widen8_batch_kernel<64, true> : widen8_batch_kernel<64, false>);
    return svlm_launch_chained(kernel, dim3(geom.n_pages, geom.kv_heads, list.n), dim3(2 * geom.head_dim), 0, 1, st, list, stores, layer, (int)early);
}
