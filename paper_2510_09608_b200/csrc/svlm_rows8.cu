// Attention of few query rows over a cache that holds its keys and values in 8 bits: one generated token, whose own key and value the
// launch may append as well, or a short chunk.
//
//   score[m, j] = <R(p_m - S) q_m, R(-s_j) k'_j> 2^ke / sqrt(D) = <R(p_m) q_m, R(S - s_j) k'_j> 2^ke / sqrt(D)
//
// k' is the key as stored (rotated at its native position), s_j its token's shift, S the shift of the newest tokens and p_m the
// query's native position.  For tokens with s = S (whatever follows the last evicted one in stream order) the turned query is the same; where all
// tokens of a unit share another shift, as those of a second of video do once text behind them is gone, a warp turns its queries once
// more, by factors that the eviction has left (SvlmStore8::turn), and keeps them for the next unit; where they do not, it turns the unit's keys.
// (Tried when a generated token over 9216 keys of 28/4 heads of 128 took 19 us: turning the queries for each shift of such a unit, 16 units with sixteen
// shifts each, 22 us; one warp's work is everybody's wait.  When it took 9.2: turning the keys of every unit with s other than S and 0, 10.6 where no
// unit is one of those.)
//
// Work.  A unit is one block of 16 tokens of a KV head, 16 D bytes of keys and as many of values, each contiguous, with one exponent each.
// Each warp takes a run of units, two at a time (their chains of steps are independent).  It copies them asynchronously into slots of its own, so that
// nothing is handed over between warps, the next pair's keys as soon as this one's are read; room for two pairs changed nothing (30.2 and 30.6 us for 9 rows
// over 9216 keys).  The bytes become MMA fragments without being rearranged, since a product does not care in which order it sums: lane (g, t) = (lane / 4, lane % 4) takes for the scores
// S^T = K Q^T a quarter of the rows g and g + 8 (D / 4 consecutive bytes), and for the outputs O^T += V^T P^T an eighth of the dims of tokens
// 2t, 2t + 1, 2t + 8, 2t + 9, paired by byte permutes.  e4m3 is exact in f16, so the MMAs are m16n8k16 in f16 with fp32 sums.
// Roundings on the way: the turned query, in units of a power of two of its row, to f16 (2^-12), and a turned key; the weights to f16,
// relative to the largest weight times unit that the row has met: w = 2^(s + ve - R), R the running maximum of s + ve (s in powers of
// two), so that values far apart in different blocks neither overflow nor vanish.  The sum of the weights has its own running maximum m, in
// fp32, and R is kept as R - m: the sum of a score of thousands and a unit would be rounded, and with it the size of the output (scores of 2^32
// gave outputs 2^7 and 2^14 times too large).  A split's partial result goes to those that merge it as bf16, its maximum and sum as fp32.
// A thread block has 8 columns, query rows of a KV head; the others are other blocks', which read the units again out of L2.
// Instances: one query token of up to 8 heads (ONE), with and without its append, for one layer of one cache (LAYER) and for several; anything else.
//
// A layer-step's chain (one token, one layer of one stream, about one thread block per SM).  Programmatic dependent launch lets a layer's
// kernel read the page list and its units while the layer before still runs (early: the caller vouches that nothing in between writes them);
// behind the wait there are the query, scores and outputs of units that are there already, and the meeting of the splits, as tagged words
// that the first thread blocks of a KV head poll for, each combining a share (see combine_tagged).
//
// What bounds it: the latency of a unit's steps one after another (conversions, MMAs, maxima, exponentials: some 520 instructions, of which a warp issues
// one in six cycles), with sixteen warps an SM at most to hide it.  No unit of the SM is full: sixteen streams have the issue slots 33 % busy, the
// integer pipe 45 %, the tensor pipe 12 % and DRAM 35 %, and 256 blocks on 296 places, so that some SMs have one and wait for those with two.  With fewer keys the chain's
// length is all that counts.  Measured, 28/4 heads of 128, us a layer-step in a
// graph: 7.1 over 9216 keys with 28 layers in a row (1.4 at the copy rate; the 16-bit cache's kernel, which has nothing to convert, 6.0), 6.2 over 512, 18.2 over
// 44512; sixteen streams of 9216 keys 45 (23); 32/8 heads over
// 44512 keys 32 (14); nine tokens' chunk over 9216 keys 27.  A stream that has just moved on, most of whose units have shifts of their own, 8.5.
// Tried: keys made into fragments before the wait (10 us), runs of 4 units dealt out in turn (sixteen streams 52, nine rows over 44512 keys 84 instead of 118).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "svlm_e4m3.cuh"
#include "svlm_launch.h"
#include "svlm_ptx.cuh"
#include "svlm_rope.cuh"
#include "svlm_store8.h"

namespace {

using namespace svlm_ptx;

constexpr int R8_WARPS = 8;
constexpr int R8_THREADS = R8_WARPS * 32;
// Tiles of 8 columns (query rows of a KV head) that a warp takes at once.  Two turn a unit's bytes into fragments once for both, in 213 registers and so one thread
// block to an SM: 9 rows of 28/4 heads over 9216 keys 30.5 us instead of 30.0, over 336 keys 13.5 instead of 10.3; 44512 keys 110 instead of 118.
constexpr int R8_TILES = 1;
constexpr int R8_SLOTS = 2;                        // units of a warp worked on together, and on their way
constexpr size_t R8_TWO_FIT = 113 * 1024;          // shared memory of which an SM has room for two
constexpr int R8_GROUPS = 7;                       // groups of 8 output elements of a thread block that combines, about
constexpr int R8_PAD = 4;                          // floats behind a row of the merge buffer: its stores fall into different banks

__device__ __forceinline__ unsigned movmatrix_trans(unsigned a) {
    unsigned d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ unsigned pack_half2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ unsigned pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, uint2 b) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A word of a record that meets its readers without a fence, a counter or a second round trip: { payload, tag }, 64 bits and so single-copy
// atomic.  Nothing else is ever written to the area, the tag of a launch is its KV head's epoch + 1, and the epoch goes up by one per launch: with the
// last of the head's blocks to ask for it, so that no block of a launch, however late it begins and whoever has given up waiting for it, takes the
// next launch's tag.  (It went up with the first block's last poll: a block that began after a wait had run out left records which
// the next launch took for its own.)
// (The answer is looked at when it is wanted, behind the outputs: looked at as soon as it has been asked for, it held up thread 0's queries by 0.13 us.)
__device__ __forceinline__ unsigned long long ask_tag(unsigned long long* epoch) { return atomicAdd(epoch, 1ull); }      // { epoch, blocks that have asked }
__device__ __forceinline__ unsigned tag_of(unsigned long long asked) { return (unsigned)(asked >> 32) + 1; }
__device__ __forceinline__ void move_on(unsigned long long asked, unsigned long long* epoch, int splits) {      // nobody else asks before this launch has ended
    if ((unsigned)asked == (unsigned)splits - 1) __stcg(epoch, (unsigned long long)tag_of(asked) << 32);
}
__device__ __forceinline__ void st_tagged2(void* p, unsigned a, unsigned b, unsigned tag) {
    const unsigned long long hi = (unsigned long long)tag << 32;
    asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(hi | a), "l"(hi | b) : "memory");
}
__device__ __forceinline__ void ld_tagged2(const void* p, unsigned long long& a, unsigned long long& b) {
    asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "l"(p) : "memory");
}
template <int D>
__host__ __device__ constexpr int tagged_rec_bytes() { return 8 * D * 4 + 8 * 16; }      // 8 columns of bf16 pairs, then (m, l) of each
__host__ __device__ inline size_t tagged_head_bytes(int kv_heads) { return ((size_t)kv_heads * 8 + 127) & ~(size_t)127; }

template <int D>
struct R8 {
    static constexpr int KS = D / 16;              // k-steps of the scores; blocks of 16 dims of the outputs
    static constexpr int KW = D / 16, VW = D / 32; // words of a lane: of a key row, of a token's values
    static constexpr int COLS = 8 * R8_TILES, HALF = D / 2, PPL = D / 64;
    static constexpr int REC = COLS * D * 2 + COLS * 8;             // a partial result: o bf16, then (m, l) per column
    static constexpr int ITEM = SVLM_BLOCK8 * D;                    // bytes of a unit's keys
    static constexpr int SLOT = 2 * ITEM + 32 + 128 + 2 * D;        // keys, values, four blocks' exponents and distances, ordinals, a token's rotation
    // One turned copy of the queries, in fragment order [tile][k-step][lane][4 dims]; a k-step is followed by 16 bytes, so that a column's stores, a
    // k-step apart, fall into different banks.
    static constexpr int STEP = 34;                                 // of uint2
    static constexpr size_t frag_bytes = (size_t)R8_TILES * KS * STEP * 8;
    static constexpr size_t ring_bytes = (size_t)R8_WARPS * R8_SLOTS * SLOT;
    static constexpr size_t work_bytes = ring_bytes;
    struct Small {
        float q_unit[COLS];                        // power of two of a column's query, times log2(e) / sqrt(D)
        int q_tok[COLS];                           // its token of the chunk
        float m[R8_WARPS][COLS], r[R8_WARPS][COLS], l[R8_WARPS][COLS];      // maxima of s; of s + ve, less those; sums
        float2 cs[HALF];                           // the appended token's rotation
        int last, tag;
        unsigned wait_limit;
    };
    static constexpr int COPIES = 2 + R8_WARPS * R8_SLOTS;          // of the queries: for s = S, for the middle of the block's units, and each warp's latest ones
    static constexpr size_t smem(int n_pages) { return work_bytes + COPIES * frag_bytes + (sizeof(Small) + 15) / 16 * 16 + (size_t)n_pages * 4; }
};
// What a product of a query in its units and a key in its own is to be multiplied by.  The two units first: either may be large and the other
// small.  Above 0, however small (a query of zeros, keys next to nothing): what hides a token is a score of -inf, which stays one.  Finite.
__device__ __forceinline__ float score_unit(float q_unit, float k_unit) { return fminf(fmaxf(q_unit * k_unit, 1.2e-38f), 3.0e38f); }
// Where a row's 16-byte chunk lies in a slot: so that eight lanes' 16 bytes fall into different banks.
template <int D>
__device__ __forceinline__ int chunk_at(int row, int chunk) { return row * D + ((chunk ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4); }

// One query token's outputs from the splits' tagged records: the first `shares` splits of a KV head take groups of eight output elements each.
// Eight lanes cover eight groups, which lie side by side in a record; the lane groups of all warps take 32 records at a time, two rounds in
// flight.  A word that does not carry the tag yet is read again, wait_limit times at most; then the status word says so and what there is
// is written.  All thread blocks of the launch have places together (one wave of them, and a dependent launch enters only when
// all of them have passed their trigger), so the wait is for stragglers; beside other streams' launches it is for those to end, too: only these first
// splits of a launch ever wait, and the others leave their places by themselves.
template <int D>
__device__ __forceinline__ void combine_tagged(int share, int shares, int splits, const unsigned char* parts, unsigned tag, float* buf, int G,
                                               uint16_t* out_row0, unsigned wait_limit, int* status) {
    constexpr int REC = tagged_rec_bytes<D>();
    const int groups = G * (D / 8), per = (groups + shares - 1) / shares;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gl = lane & 7, rl = lane >> 3;
    float* slab = buf + (size_t)(warp * 8 + gl) * 12;        // [warp][group of the round][M, L, acc[8], pad]
    bool timed_out = false;
#pragma unroll 1
    for (int g0 = 0; g0 < per; g0 += 8) {
        const int grp = share * per + g0 + gl;
        const bool valid = g0 + gl < per && grp < groups;
        const int h = valid ? grp / (D / 8) : 0, d0 = valid ? (grp % (D / 8)) * 8 : 0;
        const unsigned char* ml = parts + 8 * D * 4 + h * 16;
        const unsigned char* ov = parts + (size_t)(h * D + d0) * 4;
        float M = -INFINITY, L = 0.f, acc[8] = {};
#pragma unroll 1
        for (int r0 = warp * 4 + rl; r0 < splits; r0 += 2 * R8_WARPS * 4) {
            unsigned long long w[2][6];
            bool want[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) want[k] = valid && r0 + k * R8_WARPS * 4 < splits;
            for (unsigned polls = 0;; ++polls) {
                if (__builtin_expect(polls >= wait_limit, 0)) { timed_out = true; break; }
                bool ok = true;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (!want[k]) continue;
                    const size_t off = (size_t)(r0 + k * R8_WARPS * 4) * REC;
                    ld_tagged2(ov + off, w[k][0], w[k][1]);
                    ld_tagged2(ov + off + 16, w[k][2], w[k][3]);
                    ld_tagged2(ml + off, w[k][4], w[k][5]);
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (!want[k]) continue;
#pragma unroll
                    for (int i = 0; i < 6; ++i) ok = ok && (unsigned)(w[k][i] >> 32) == tag;
                }
                if (ok) break;
            }
            float mr[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                want[k] = want[k] && !timed_out;
                mr[k] = want[k] ? __uint_as_float((unsigned)w[k][4]) : -INFINITY;
            }
            const float Mn = fmaxf(M, fmaxf(mr[0], mr[1])), resc = M == -INFINITY ? 1.f : exp2f(M - Mn);      // (nothing but a NaN is in L while M is -inf)
            L *= resc;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= resc;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!want[k]) continue;
                if (mr[k] == -INFINITY) {
                    L += __uint_as_float((unsigned)w[k][5]);
                    continue;
                }
                const float wt = exp2f(mr[k] - Mn);
                L += __uint_as_float((unsigned)w[k][5]) * wt;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const unsigned pr = (unsigned)w[k][i];
                    acc[2 * i] += __uint_as_float(pr << 16) * wt;
                    acc[2 * i + 1] += __uint_as_float(pr & 0xffff0000u) * wt;
                }
            }
            M = Mn;
        }
        const float Mw = fmaxf(fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 8)),
                               fmaxf(__shfl_xor_sync(0xffffffffu, M, 16), __shfl_xor_sync(0xffffffffu, M, 24)));
        const float f = M > -INFINITY ? exp2f(M - Mw) : 1.f;
        L *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= f;
#pragma unroll
        for (int sft = 8; sft < 32; sft <<= 1) {
            L += __shfl_xor_sync(0xffffffffu, L, sft);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], sft);
        }
        if (rl == 0) {
            *reinterpret_cast<float4*>(slab) = make_float4(Mw, L, acc[0], acc[1]);
            *reinterpret_cast<float4*>(slab + 4) = make_float4(acc[2], acc[3], acc[4], acc[5]);
            *reinterpret_cast<float2*>(slab + 8) = make_float2(acc[6], acc[7]);
        }
        __syncthreads();
        if (threadIdx.x < 32) {                              // four threads per group, two output elements each
            const int fg = lane >> 2, e2 = lane & 3, fgrp = share * per + g0 + fg;
            const float* sl = buf + (size_t)fg * 12;
            float Ma = -INFINITY, La = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
            for (int wp = 0; wp < R8_WARPS; ++wp) Ma = fmaxf(Ma, sl[wp * 96]);
#pragma unroll
            for (int wp = 0; wp < R8_WARPS; ++wp) {
                const float wt = sl[wp * 96] == -INFINITY ? 1.f : exp2f(sl[wp * 96] - Ma);
                const float2 a = *reinterpret_cast<const float2*>(sl + wp * 96 + 2 + 2 * e2);
                La += sl[wp * 96 + 1] * wt;
                a0 += a.x * wt;
                a1 += a.y * wt;
            }
            if (g0 + fg < per && fgrp < groups) {
                const float inv = La > 0.f ? 1.f / La : (La == 0.f ? 0.f : La);
                *reinterpret_cast<uint32_t*>(out_row0 + (size_t)(fgrp / (D / 8)) * D + (fgrp % (D / 8)) * 8 + 2 * e2) = pack_bf16x2(a0 * inv, a1 * inv);
            }
        }
        if (g0 + 8 < per) __syncthreads();                   // the slabs are read before the next round writes them
    }
    if (__builtin_expect(timed_out, 0)) atomicCAS(status, 0, -5);   // SVLM_ERR_TIMEOUT
}

template <int D, bool ONE, bool APPEND, bool LAYER>
__global__ void __launch_bounds__(R8_THREADS, 2)
rows8_kernel(SvlmAttend8 a, int layer0, int n_layers, const uint16_t* Q, const int* q_pos, int n_q_arg, int q_heads, uint16_t* out, int splits, int col_groups,
             const uint16_t* Knew, const uint16_t* Vnew, int early) {
    using C = R8<D>;
    constexpr int PPL = C::PPL;
    extern __shared__ __align__(128) unsigned char smem[];
    unsigned char* ring = smem;                                                      // [warp][slot]
    float* merge = reinterpret_cast<float*>(smem);                                   // the same memory, later
    uint2* frags = reinterpret_cast<uint2*>(smem + C::work_bytes);                   // [copies][R8_TILES][KS][STEP]
    typename C::Small& sh = *reinterpret_cast<typename C::Small*>(smem + C::work_bytes + C::COPIES * C::frag_bytes);
    unsigned* tile_pk = reinterpret_cast<unsigned*>(smem + C::work_bytes + C::COPIES * C::frag_bytes + (sizeof(sh) + 15) / 16 * 16);   // page | lo << 16 | hi << 24

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x, hk = blockIdx.y / col_groups, cg = blockIdx.y % col_groups;
    const int ci = blockIdx.z / n_layers, li = blockIdx.z % n_layers, layer = layer0 + li;
    const SvlmView8& vw = a.view[ci];
    const int G = q_heads / a.kv_heads, n_q = ONE ? 1 : (a.q_varlen ? a.q_cnt[ci] : n_q_arg);
    const int m0 = cg * C::COLS, m_total = n_q * G;
    const size_t q_row0 = a.q_varlen ? (size_t)a.q_off[ci] : ((size_t)ci * n_layers + li) * n_q;
    const size_t p_row0 = a.q_varlen ? (size_t)a.q_off[ci] : (size_t)ci * n_q;
    const int pw = a.rope_mode == 0 ? 0 : 1;                                         // a position's stride per axis

    // ---- the queries: warp w takes columns w, w + 8, ...; a lane PPL neighbouring pairs (i, i + D/2) ----
    uint16_t q_lo[R8_TILES][PPL], q_hi[R8_TILES][PPL];
    int q_at[R8_TILES][PPL];
    uint16_t new_lo[2][PPL], new_hi[2][PPL];       // of the appended token's key, of its value
    unsigned long long asked = 0;                  // thread 0's
    unsigned long long* const epoch = reinterpret_cast<unsigned long long*>(vw.tagged) + hk;
    auto axis_of = [&](int pair) { return a.rope_mode == 0 ? 0 : (pair < a.sec_t ? 0 : (pair < a.sec_th ? 1 : 2)); };
    auto load_queries = [&] {
        if (LAYER && threadIdx.x == 0) asked = ask_tag(epoch);
#pragma unroll
        for (int c = 0; c < R8_TILES; ++c) {
            const int m = m0 + c * R8_WARPS + warp, r = m < m_total ? m / G : 0, h = m < m_total ? m - r * G : 0;
            const uint16_t* row = Q + ((q_row0 + r) * q_heads + hk * G + h) * D + lane * PPL;
            const int* qp = q_pos + (p_row0 + r) * (2 * pw + 1);
#pragma unroll
            for (int e = 0; e < PPL; ++e) {
                q_lo[c][e] = ld_in(row + e);
                q_hi[c][e] = ld_in(row + C::HALF + e);
                if (!APPEND) q_at[c][e] = ld_in(qp + pw * axis_of(lane * PPL + e));
            }
        }
    };

    if (!early) pdl_wait();
    pdl_launch_dependents();
    if (m0 >= m_total) return;                                                       // (streams with shorter chunks)
    if (!early) load_queries();
    if (LAYER && threadIdx.x == 32) sh.wait_limit = ld_l2(&vw.ctrl->wait_limit);
    const int n_tiles = ld_l2(&vw.ctrl->n_tiles);
    const int S = (int)ld_l2(&vw.ctrl->shift_total);
    const long long gid_q0 = ONE ? 0 : ld_l2(&vw.ctrl->n_total) - n_q;
    for (int i = threadIdx.x; i < a.n_slots / SVLM_PAGE; i += R8_THREADS) {          // (without waiting for their number)
        const int4 tl = ld_l2(reinterpret_cast<const int4*>(vw.tiles + i));          // page, lo, hi, pad
        tile_pk[i] = (unsigned)tl.x | ((unsigned)tl.y << 16) | ((unsigned)tl.z << 24);
    }
    // the appended token: where it lives and whether it is still stored there
    int new_slot = -1;
    if (APPEND) {
        const int s = ld_l2(vw.new_slot);
        if (ld_l2(&vw.ctrl->append_n) == 1 && ld_l2(vw.slot_gid + s) == ld_l2(&vw.ctrl->n_total) - 1) new_slot = s;
        // its position is in the metadata already, so the factors do not wait for the previous kernel
#pragma unroll
        for (int e = 0; e < PPL; ++e) q_at[0][e] = ld_l2(vw.slot_c + (size_t)axis_of(lane * PPL + e) * a.n_slots + s) + S;
    }
    __syncthreads();

    // ---- the units ----
    const size_t head_row0 = ((size_t)layer * a.kv_heads + hk) * a.n_slots;
    // (Of a layer-step neighbouring runs go to neighbouring thread blocks, one further at each warp: units that take longer are neighbours, the
    // newest and those of a second's end, and with fewer units than warps every block has the same number of them.)
    const int total = 8 * n_tiles, runs = splits * R8_WARPS, run = LAYER ? warp * splits + (split + warp) % splits : split * R8_WARPS + warp;
    const int u0 = (int)((long long)total * run / runs), u1 = (int)((long long)total * (run + 1) / runs);
    unsigned char* const mine = ring + (size_t)warp * R8_SLOTS * C::SLOT;
    auto tokens_of = [&](int u, int& first) {                                        // a bit each; 0: nothing here
        const unsigned pk = tile_pk[u >> 3];
        const int k0 = (u & 7) * SVLM_BLOCK8, lo = max((int)((pk >> 16) & 0xFF) - k0, 0), hi = min((int)(pk >> 24) - k0, SVLM_BLOCK8);
        first = (int)(pk & 0xFFFF) * SVLM_PAGE + k0;
        return lo < hi ? ((1u << hi) - 1) & ~((1u << lo) - 1) : 0u;
    };
    auto copy16 = [&](unsigned char* dst, const unsigned char* src) {                // 16 rows of D bytes
#pragma unroll
        for (int i = 0; i < C::ITEM / 512; ++i) cp_async16(dst + chunk_at<D>((lane + 32 * i) / (D / 16), lane % (D / 16)), src + (lane + 32 * i) * 16);
    };
    auto load_keys = [&](int u) {                                                    // of units u, u + 1, and what else belongs to them
#pragma unroll
        for (int k = 0; k < R8_SLOTS; ++k) {
            int first;
            const unsigned tokens = u + k < u1 ? tokens_of(u + k, first) : 0u;
            if (!tokens) continue;
            unsigned char* dst = mine + k * C::SLOT;
            const size_t at = head_row0 + first;
            copy16(dst, vw.K + at * D);
            if (lane == 0) cp_async16(dst + 2 * C::ITEM, vw.exps + (at / SVLM_BLOCK8 & ~(size_t)3));
            if (lane == 1) cp_async16(dst + 2 * C::ITEM + 16, vw.apart + (first / SVLM_BLOCK8 & ~3));
            // (a few units a warp: fetched ahead, needed or not; many, of which most need none or their predecessor's: when it is wanted)
            if (LAYER && lane < D / 8) cp_async16(dst + 2 * C::ITEM + 160 + lane * 16, vw.turn + (size_t)(first + __ffs(tokens) - 1) * (D / 4) + lane * 2);
            if (!ONE && lane >= 24) cp_async16(dst + 2 * C::ITEM + 32 + (lane - 24) * 16, vw.slot_gid + first + (lane - 24) * 2);
        }
        cp_async_commit();
    };
    auto load_values = [&](int u) {
#pragma unroll
        for (int k = 0; k < R8_SLOTS; ++k) {
            int first;
            if (u + k < u1 && tokens_of(u + k, first)) copy16(mine + k * C::SLOT + C::ITEM, vw.V + (head_row0 + first) * D);
        }
        cp_async_commit();
    };
    load_keys(u0);
    load_values(u0);
    // How far the middle of this thread block's units is from S: it has a copy of the queries of its own, the others turn theirs when they get there.
    // All threads have to see one value (each warp puts its column into that copy, and all read it), so the block that the appended token joins
    // has none: its word is the one that somebody may be writing meanwhile, another head's block of this launch or, with early, layer 0's.
    int apart0 = 0;
    if (!LAYER && total > 0) {
        int first;
        const unsigned tokens = tokens_of((int)((long long)total * (2 * split + 1) / (2 * splits)), first);
        const bool joined = APPEND && new_slot >= 0 && (new_slot & ~(SVLM_BLOCK8 - 1)) == first;
        if (tokens && !joined) apart0 = max(0, ld_l2(vw.apart + first / SVLM_BLOCK8));
    }
    // the appended token's rows come in with the queries, to the warp whose unit they join
    bool joins = false;
    if (APPEND && new_slot >= 0)
        for (int u = u0 + lane; u < u1; u += 32) {
            int first;
            if (tokens_of(u, first) && (new_slot & ~(SVLM_BLOCK8 - 1)) == first) joins = true;
        }
    joins = APPEND && __any_sync(0xffffffffu, joins);

    // ---- what is known of a pair of units ----
    unsigned valid[R8_SLOTS], exps[R8_SLOTS];
    int first[R8_SLOTS], apart[R8_SLOTS], fresh = -1;                                // fresh: the appended token's row of its unit, + 16 in the second one
    auto know = [&](int u) {
#pragma unroll
        for (int i = 0; i < R8_SLOTS; ++i) {
            unsigned char* slot = mine + i * C::SLOT;
            first[i] = 0;
            valid[i] = u + i < u1 ? tokens_of(u + i, first[i]) : 0u;
            const int which4 = (first[i] / SVLM_BLOCK8) & 3;
            exps[i] = valid[i] ? reinterpret_cast<const unsigned*>(slot + 2 * C::ITEM)[which4] : 0u;
            apart[i] = valid[i] ? reinterpret_cast<const int*>(slot + 2 * C::ITEM + 16)[which4] : 0;
            if (APPEND && new_slot >= 0 && valid[i] && (new_slot & ~(SVLM_BLOCK8 - 1)) == first[i]) fresh = new_slot - first[i] + 16 * i;
        }
    };
    auto key_words = [&](int i, int c, unsigned (&k)[2][4]) {                         // chunk c of the lane's share of rows g and g + 8
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 x = *reinterpret_cast<const uint4*>(mine + i * C::SLOT + chunk_at<D>(g + 8 * h, t * (C::KW / 4) + c));
            k[h][0] = x.x; k[h][1] = x.y; k[h][2] = x.z; k[h][3] = x.w;
        }
    };
    // A key's pair of dims turned: the halves of a pair (i, i + D/2) are D / 2 dims and so two lanes of the row's four apart.
    auto turn_key = [&](unsigned& y, unsigned c, unsigned sn) {
        const unsigned other = __shfl_xor_sync(0xffffffffu, y, 2);
        if (t < 2) sn ^= 0x80008000u;
        const __half2 z = __hfma2(*reinterpret_cast<const __half2*>(&y), *reinterpret_cast<const __half2*>(&c),
                                  __hmul2(*reinterpret_cast<const __half2*>(&other), *reinterpret_cast<const __half2*>(&sn)));
        y = *reinterpret_cast<const unsigned*>(&z);
    };
    const uint4 as_it_is = make_uint4(0x3c003c00u, 0u, 0x3c003c00u, 0u);

    // ---- the queries again: turned, in fragment order ----
    float2 cs[R8_TILES][PPL], cs0[R8_TILES][PPL];
    auto factors = [&] {
        const float2* tab = reinterpret_cast<const float2*>(a.rope_tab);
#pragma unroll
        for (int c = 0; c < R8_TILES; ++c)
#pragma unroll
            for (int e = 0; e < PPL; ++e) {
                const int pair = lane * PPL + e;
                // (the appended token's key is turned by its query's factors)
                if (!LAYER && apart0) cs0[c][e] = svlm_rope_cs(tab, C::HALF, pair, (long long)q_at[c][e] - apart0, a.theta[pair]);
                cs[c][e] = APPEND ? rope_cs_exact(vw.rope64, C::HALF, pair, q_at[c][e], a.theta[pair]) : svlm_rope_cs(tab, C::HALF, pair, q_at[c][e], a.theta[pair]);
            }
    };
    if (APPEND) {
        factors();
        if (warp == 0)
#pragma unroll
            for (int e = 0; e < PPL; ++e) sh.cs[lane * PPL + e] = cs[0][e];
    }
    if (early) {
        pdl_wait();
        load_queries();
    }
    if (joins) {
        const size_t src = (((size_t)ci * n_layers + li) * a.kv_heads + hk) * D + lane * PPL;
#pragma unroll
        for (int e = 0; e < PPL; ++e) {
            new_lo[0][e] = ld_in(Knew + src + e); new_hi[0][e] = ld_in(Knew + src + C::HALF + e);
            new_lo[1][e] = ld_in(Vnew + src + e); new_hi[1][e] = ld_in(Vnew + src + C::HALF + e);
        }
    }
    if (APPEND && __builtin_expect(new_slot < 0, 0)) {                               // dropped, or evicted since: its position as given
        const int* qp = q_pos + p_row0 * (2 * pw + 1);
#pragma unroll
        for (int e = 0; e < PPL; ++e) q_at[0][e] = ld_in(qp + pw * axis_of(lane * PPL + e));
    }
    if (!APPEND || new_slot < 0) factors();
    auto half_at = [&](int copy, int col, int d) {                                   // where element d of a column's query lies
        const int e = d % (D / 4);
        return reinterpret_cast<__half*>(frags) + copy * (C::frag_bytes / 2) + ((((col >> 3) * C::KS + e / 4) * C::STEP + (col & 7) * 4 + d / (D / 4)) * 4 + (e & 3));
    };
#pragma unroll
    for (int c = 0; c < R8_TILES; ++c) {
        const int col = c * R8_WARPS + warp, m = m0 + col;
        const bool live = m < m_total;
        float lo[PPL], hi[PPL];
        unsigned most = 0;
#pragma unroll
        for (int e = 0; e < PPL; ++e) {
            lo[e] = live ? __uint_as_float((unsigned)q_lo[c][e] << 16) : 0.f;
            hi[e] = live ? __uint_as_float((unsigned)q_hi[c][e] << 16) : 0.f;
            most = max(most, max(__float_as_uint(lo[e]) & 0x7fffffffu, __float_as_uint(hi[e]) & 0x7fffffffu));
        }
        // units: the row's largest magnitude is in [1, 2) of them (a smaller row's, zeros among them, of 2^-120: q_unit is a normal number)
        const int ex = max(-120, min(126, (int)(__reduce_max_sync(0xffffffffu, most) >> 23) - 127));
        const float f = pow2i(-ex);
        float put_lo[PPL], put_hi[PPL];
#pragma unroll
        for (int e = 0; e < PPL; ++e) {
            const float x = lo[e] * f, y = hi[e] * f;
            lo[e] = x * cs[c][e].x - y * cs[c][e].y;
            hi[e] = y * cs[c][e].x + x * cs[c][e].y;
            if (!LAYER) {
                put_lo[e] = x * cs0[c][e].x - y * cs0[c][e].y;
                put_hi[e] = y * cs0[c][e].x + x * cs0[c][e].y;
            }
        }
        auto put = [&](int copy, const float (&l)[PPL], const float (&h)[PPL]) {
            if (PPL == 2) {
                *reinterpret_cast<unsigned*>(half_at(copy, col, lane * PPL)) = pack_half2(l[0], l[PPL - 1]);
                *reinterpret_cast<unsigned*>(half_at(copy, col, C::HALF + lane * PPL)) = pack_half2(h[0], h[PPL - 1]);
            } else {
                *half_at(copy, col, lane) = __float2half_rn(l[0]);
                *half_at(copy, col, C::HALF + lane) = __float2half_rn(h[0]);
            }
        };
        put(0, lo, hi);
        if (!LAYER && apart0) put(1, put_lo, put_hi);
        if (lane == 0) {
            sh.q_unit[col] = pow2i(ex) * (1.4426950408889634f * rsqrtf((float)D));
            sh.q_tok[col] = live ? m / G : -1;
        }
    }
    __syncthreads();

    float o[R8_TILES][C::KS][4];
    float m[R8_TILES][2], r[R8_TILES][2], l[R8_TILES][2];            // of columns 2t, 2t + 1: maximum of s; of s + ve, less that; this lane's share of the sum
#pragma unroll
    for (int n = 0; n < R8_TILES; ++n) {
#pragma unroll
        for (int k = 0; k < C::KS; ++k) o[n][k][0] = o[n][k][1] = o[n][k][2] = o[n][k][3] = 0.f;
        m[n][0] = m[n][1] = r[n][0] = r[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
    }

    // The appended token's key and value into its row of the unit, here and in the cache; the rules are svlm_store8.h's.  Returns the
    // unit's exponents and says how far apart its tokens' shifts are from S.
    auto append_here = [&](unsigned char* slot, unsigned valid, int first, unsigned exps, int& apart) {
        const int off = new_slot - first;
        const unsigned held = valid & ((1u << off) - 1);
        const size_t at = head_row0 + first;
        unsigned result = 0;
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            unsigned char* here = slot + which * C::ITEM;
            unsigned char* there = (which ? vw.V : vw.K) + at * D;
            float lo[PPL], hi[PPL];
            unsigned most = 0;
#pragma unroll
            for (int e = 0; e < PPL; ++e) {
                lo[e] = __uint_as_float((unsigned)(which ? new_lo[1][e] : new_lo[0][e]) << 16);
                hi[e] = __uint_as_float((unsigned)(which ? new_hi[1][e] : new_hi[0][e]) << 16);
                if (which == 0) rotate_exact(lo[e], hi[e], sh.cs[lane * PPL + e]);
                most = max(most, max(finite_bits(lo[e]), finite_bits(hi[e])));
            }
            int ex = block_exponent(__reduce_max_sync(0xffffffffu, most));
            if (held) {
                const int before = exponent_of(exps, which);
                if (ex > before) {                 // the block's earlier values in the new unit
                    const float f = ex - before > 126 ? 0.f : pow2i(before - ex);
#pragma unroll 1
                    for (int i = lane; i < C::ITEM / 4; i += 32) {
                        const int tok = i / (D / 4), w = i % (D / 4);
                        if (!((held >> tok) & 1)) continue;
                        unsigned* x = reinterpret_cast<unsigned*>(here + chunk_at<D>(tok, w >> 2)) + (w & 3);
                        const float2 y = e4m3x2_to_float2((uint16_t)*x), z = e4m3x2_to_float2((uint16_t)(*x >> 16));
                        *x = to_e4m3x2(y.x * f, y.y * f) | (unsigned)to_e4m3x2(z.x * f, z.y * f) << 16;
                        reinterpret_cast<unsigned*>(there)[i] = *x;
                    }
                }
                ex = max(ex, before);
            }
            const float unit = pow2i(-ex), limit = ex == E8_MAX ? E8_TOP : 448.f;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int d = hf * C::HALF + lane * PPL;
                const float* y = hf ? hi : lo;
                const uint16_t b = to_e4m3x2(y[0] * unit, y[PPL - 1] * unit, limit);
                unsigned char* x = here + chunk_at<D>(off, d >> 4) + (d & 15);
                if (PPL == 2) {
                    *reinterpret_cast<uint16_t*>(x) = b;
                    *reinterpret_cast<uint16_t*>(there + off * D + d) = b;
                } else {
                    *x = (unsigned char)b;
                    there[off * D + d] = (unsigned char)b;
                }
            }
            result |= (unsigned)(ex & 255) << (8 * which);
        }
        // (other thread blocks' copies of this word may be of before or of behind this: the warp whose unit it is comes to the same here, nobody else
        // uses it)
        apart = held && apart != 0 ? MIXED8 : 0;
        if (lane == 0) {
            vw.exps[at / SVLM_BLOCK8] = result;
            atomicMax(vw.most + layer * a.kv_heads + hk, exponent_of(result, 0) + MOST8_BIAS);
        }
        if (layer == 0 && hk == 0) {
            if (lane == 0) {
                vw.apart[first / SVLM_BLOCK8] = apart;
                vw.native[new_slot] = ld_l2(vw.slot_c + new_slot) + S;
            }
            if (apart != 0 && lane < D / 4) vw.turn[(size_t)new_slot * (D / 4) + lane] = make_uint2(0x3c003c00u, 0u);
            if (held == 0 && n_layers == 1)        // the block begins: later layers have nothing in it yet (kv_write8_kernel)
#pragma unroll 1
                for (int row = a.kv_heads + lane; row < a.layers * a.kv_heads; row += 32) vw.exps[((size_t)row * a.n_slots + first) / SVLM_BLOCK8] = NO_EXPONENTS;
        }
        __syncwarp();
        return result;
    };

    int own_apart[R8_SLOTS] = {0, 0};              // what this warp's copies of the queries are turned for
    auto join = [&](int i) {                       // the appended token, where its unit is the pair's i-th
        if (!APPEND || fresh < 0 || (fresh >> 4) != i) return;
        cp_async_wait<0>();
        __syncwarp();
        exps[i] = append_here(mine + i * C::SLOT, valid[i], first[i], exps[i], apart[i]);
    };
    // Of a unit that holds tokens which come after some of the rows': the tokens (a bit each) that columns 2t and 2t + 1 see.
    bool later[R8_SLOTS] = {};
    unsigned seen[R8_SLOTS][R8_TILES][2];
    // a pair's values by its weights
    auto outputs = [&](int u, const uint2 (&p)[R8_SLOTS][R8_TILES]) {
        cp_async_wait<1>();
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R8_SLOTS; ++i) {
            unsigned v[4][C::VW];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int tok = 2 * t + (k & 1) + 8 * (k >> 1);
                if constexpr (D == 128) {
                    const uint4 x = *reinterpret_cast<const uint4*>(mine + i * C::SLOT + C::ITEM + chunk_at<D>(tok, g));
                    v[k][0] = x.x; v[k][1] = x.y; v[k][2] = x.z; v[k][3] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(mine + i * C::SLOT + C::ITEM + chunk_at<D>(tok, g >> 1) + (g & 1) * 8);
                    v[k][0] = x.x; v[k][1] = x.y;
                }
            }
            if (!ONE && __builtin_expect(later[i], 0)) {
                // 0 times a value that is not a number must be 0 in the rows that do not see it: it goes into the others' sums here, and out of the product
                bool any = false;
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int w = 0; w < C::VW; ++w) {
                        const unsigned nan = nan_bytes(v[k][w]);
                        any |= nan != 0;
                        v[k][w] &= ~(nan * 0xffu);
                    }
                if (__any_sync(0xffffffffu, any))
#pragma unroll 1
                    for (int tok = 0; tok < SVLM_BLOCK8; ++tok)
#pragma unroll
                        for (int k = 0; k < C::KS; ++k) {
                            const int d = g * (D / 8) + 2 * k;
                            const unsigned two = *reinterpret_cast<const uint16_t*>(mine + i * C::SLOT + C::ITEM + chunk_at<D>(tok, d >> 4) + (d & 15));
#pragma unroll
                            for (int n = 0; n < R8_TILES; ++n)
#pragma unroll
                                for (int c = 0; c < 2; ++c)
                                    if ((seen[i][n][c] >> tok) & 1) {
                                        if ((two & 0x7fu) == 0x7fu) o[n][k][c] = NAN;
                                        if ((two & 0x7f00u) == 0x7f00u) o[n][k][2 + c] = NAN;
                                    }
                        }
            }
            if (valid[i] != 0xffffu) {             // (0 times what lies there must be 0)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (!((valid[i] >> (2 * t + (k & 1) + 8 * (k >> 1))) & 1))
#pragma unroll
                        for (int w = 0; w < C::VW; ++w) v[k][w] = 0;
            }
#pragma unroll
            for (int w = 0; w < C::VW; ++w)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const unsigned sel = half ? 0x7362 : 0x5140;    // bytes 2, 3 or 0, 1 of both tokens, by dim
                    const unsigned x01 = __byte_perm(v[0][w], v[1][w], sel), x23 = __byte_perm(v[2][w], v[3][w], sel);
                    const unsigned a0 = e4m3x2_to_half2((uint16_t)x01), a1 = e4m3x2_to_half2((uint16_t)(x01 >> 16));
                    const unsigned a2 = e4m3x2_to_half2((uint16_t)x23), a3 = e4m3x2_to_half2((uint16_t)(x23 >> 16));
#pragma unroll
                    for (int n = 0; n < R8_TILES; ++n) mma_f16(o[n][2 * w + half], a0, a1, a2, a3, p[i][n]);
                }
        }
        __syncwarp();
        load_values(u + R8_SLOTS);
    };
    // from a pair's scores to its share of the outputs; asks for the next pair's bytes on the way
    auto finish = [&](int u, float (&s)[R8_SLOTS][R8_TILES][4]) {
        // scale, hide what is not there or not yet, column maxima of each unit
        float mx[R8_SLOTS][R8_TILES][2];
#pragma unroll
        for (int i = 0; i < R8_SLOTS; ++i) {
            const float ku = pow2i(exponent_of(exps[i], 0));
            float f[R8_TILES][2];
#pragma unroll
            for (int n = 0; n < R8_TILES; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) f[n][c] = score_unit(sh.q_unit[n * 8 + 2 * t + c], ku);
            int rel[2] = {0, 0};
            bool causal = false;
            if (!ONE) {
                const long long* gids = reinterpret_cast<const long long*>(mine + i * C::SLOT + 2 * C::ITEM + 32);
#pragma unroll
                for (int h = 0; h < 2; ++h) rel[h] = valid[i] ? (int)max(gids[g + 8 * h] - gid_q0, -0x40000000ll) : 0;
                causal = __any_sync(0xffffffffu, max(rel[0], rel[1]) > 0);
                later[i] = causal;
            }
#pragma unroll
            for (int n = 0; n < R8_TILES; ++n) {
                mx[i][n][0] = mx[i][n][1] = -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int col = n * 8 + 2 * t + (e & 1);
                    const bool in = ((valid[i] >> (g + 8 * (e >> 1))) & 1) && (!causal || rel[e >> 1] <= sh.q_tok[col]);
                    s[i][n][e] = in ? s[i][n][e] * f[n][e & 1] : -INFINITY;
                    mx[i][n][e & 1] = fmaxf(mx[i][n][e & 1], s[i][n][e]);
                    if (!ONE && causal) {          // lane 4 g + t knows of token g + 8 (e / 2) and column 2 t + e % 2
                        const unsigned they = __ballot_sync(0xffffffffu, in) >> t;
                        if (e < 2) seen[i][n][e] = 0;
#pragma unroll 1
                        for (int r = 0; r < 8; ++r) seen[i][n][e & 1] |= ((they >> (4 * r)) & 1u) << (r + 8 * (e >> 1));
                    }
                }
            }
        }
        __syncwarp();
        load_keys(u + R8_SLOTS);                   // into the place of these
#pragma unroll
        for (int sft = 4; sft < 32; sft <<= 1)
#pragma unroll
            for (int i = 0; i < R8_SLOTS; ++i)
#pragma unroll
                for (int n = 0; n < R8_TILES; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) mx[i][n][c] = fmaxf(mx[i][n][c], __shfl_xor_sync(0xffffffffu, mx[i][n][c], sft));
        uint2 p[R8_SLOTS][R8_TILES];
        bool grows = false;
        float corr[R8_TILES][2];
        const float ve[R8_SLOTS] = {(float)exponent_of(exps[0], 1), (float)exponent_of(exps[1], 1)};
#pragma unroll
        for (int n = 0; n < R8_TILES; ++n) {
            float mu[2], ru[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float mn = fmaxf(m[n][c], fmaxf(mx[0][n][c], mx[1][n][c]));
                mu[c] = mn == -INFINITY ? 0.f : mn;
                const float down = m[n][c] - mu[c], was = r[n][c] + down;          // -inf where there was nothing
                const float rn = fmaxf(was, fmaxf((mx[0][n][c] - mu[c]) + ve[0], (mx[1][n][c] - mu[c]) + ve[1]));
                ru[c] = rn == -INFINITY ? 0.f : rn;
                l[n][c] *= exp2f(down);
                corr[n][c] = exp2f(was - ru[c]);
                grows |= rn != was;
                m[n][c] = mn;
                r[n][c] = rn;
            }
#pragma unroll
            for (int i = 0; i < R8_SLOTS; ++i) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = s[i][n][e] - mu[e & 1];
                    l[n][e & 1] += exp2f(x);
                    w[e] = exp2f(x + (ve[i] - ru[e & 1]));
                }
                p[i][n].x = movmatrix_trans(pack_half2(w[0], w[1]));
                p[i][n].y = movmatrix_trans(pack_half2(w[2], w[3]));
            }
        }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int n = 0; n < R8_TILES; ++n)
#pragma unroll
                for (int i = 0; i < C::KS; ++i) {
                    o[n][i][0] *= corr[n][0]; o[n][i][2] *= corr[n][0];
                    o[n][i][1] *= corr[n][1]; o[n][i][3] *= corr[n][1];
                }
        }

        outputs(u, p);
    };
    // a pair's scores
    auto scores = [&](int u, float (&s)[R8_SLOTS][R8_TILES][4]) {
        // keys of this pair of units; their values, asked for behind them, may still be on the way
        cp_async_wait<1>();
        __syncwarp();
        fresh = -1;
        know(u);
        const uint2* q[R8_SLOTS];
#pragma unroll
        for (int i = 0; i < R8_SLOTS; ++i) {
            join(i);
            const bool as_first = i > 0 && apart[i] == apart[0];
            if (apart[i] > 0 && apart[i] != apart0 && apart[i] != own_apart[i] && !as_first) {      // <q, R(a) k> = <R(-a) q, k>
                own_apart[i] = apart[i];
                // in fragment order, so that a warp's accesses lie side by side (by pairs, eight lanes of a store met in one bank, and
                // sixteen units of an SM took 2 us)
                uint4* f = reinterpret_cast<uint4*>(mine + i * C::SLOT + 2 * C::ITEM + 160);
                if (!LAYER && lane < D / 8) f[lane] = ld_l2(reinterpret_cast<const uint4*>(vw.turn + (size_t)(first[i] + __ffs(valid[i]) - 1) * (D / 4)) + lane);
                uint2* to = frags + (2 + warp * R8_SLOTS + i) * (C::frag_bytes / 8);
                __syncwarp();
#pragma unroll 4
                for (int k = 0; k < R8_TILES * C::KS; ++k) {
                    const uint2 x = frags[k * C::STEP + lane], y = frags[k * C::STEP + (lane ^ 2)];      // a column's four dims; their partners
                    const uint4 w = f[(t & 1) * (D / 16) + k % C::KS];
                    const unsigned sign = t < 2 ? 0u : 0x80008000u;
                    auto turned = [&](unsigned u, unsigned v, unsigned c, unsigned sn) {
                        sn ^= sign;
                        const __half2 z = __hfma2(*reinterpret_cast<const __half2*>(&u), *reinterpret_cast<const __half2*>(&c),
                                                  __hmul2(*reinterpret_cast<const __half2*>(&v), *reinterpret_cast<const __half2*>(&sn)));
                        return *reinterpret_cast<const unsigned*>(&z);
                    };
                    to[k * C::STEP + lane] = make_uint2(turned(x.x, y.x, w.x, w.y), turned(x.y, y.y, w.z, w.w));
                }
                __syncwarp();
            }
            const int copy = apart[i] <= 0 ? 0 : apart[i] == apart0 ? 1 : 2 + warp * R8_SLOTS + (as_first ? 0 : i);
            q[i] = frags + copy * (C::frag_bytes / 8) + lane;
        }
        // scores: both units' chains side by side
        if (apart[0] != MIXED8 && apart[1] != MIXED8) {
#pragma unroll
            for (int c = 0; c < C::KW / 4; ++c) {
                unsigned k[R8_SLOTS][2][4];
#pragma unroll
                for (int i = 0; i < R8_SLOTS; ++i) key_words(i, c, k[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < R8_SLOTS; ++i) {
                        const unsigned a0 = e4m3x2_to_half2((uint16_t)k[i][0][j]), a2 = e4m3x2_to_half2((uint16_t)(k[i][0][j] >> 16));
                        const unsigned a1 = e4m3x2_to_half2((uint16_t)k[i][1][j]), a3 = e4m3x2_to_half2((uint16_t)(k[i][1][j] >> 16));
#pragma unroll
                        for (int n = 0; n < R8_TILES; ++n) mma_f16(s[i][n], a0, a1, a2, a3, q[i][(n * C::KS + 4 * c + j) * C::STEP]);
                    }
            }
        } else {                               // one of them has its keys turned
#pragma unroll
            for (int i = 0; i < R8_SLOTS; ++i) {
                if (!valid[i]) continue;
                const uint4* f = reinterpret_cast<const uint4*>(vw.turn + (size_t)(first[i] + g) * (D / 4)) + (t & 1) * (D / 16);
#pragma unroll 1
                for (int c = 0; c < C::KW / 4; ++c) {
                    unsigned k[2][4];
                    key_words(i, c, k);
                    uint4 fs[4][2];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            fs[j][h] = as_it_is;
                            if (apart[i] == MIXED8 && !(APPEND && fresh == g + 8 * h + 16 * i)) fs[j][h] = ld_l2(f + 8 * h * (D / 8) + 4 * c + j);
                        }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        unsigned a0 = e4m3x2_to_half2((uint16_t)k[0][j]), a2 = e4m3x2_to_half2((uint16_t)(k[0][j] >> 16));
                        unsigned a1 = e4m3x2_to_half2((uint16_t)k[1][j]), a3 = e4m3x2_to_half2((uint16_t)(k[1][j] >> 16));
                        turn_key(a0, fs[j][0].x, fs[j][0].y);
                        turn_key(a2, fs[j][0].z, fs[j][0].w);
                        turn_key(a1, fs[j][1].x, fs[j][1].y);
                        turn_key(a3, fs[j][1].z, fs[j][1].w);
#pragma unroll
                        for (int n = 0; n < R8_TILES; ++n) mma_f16(s[i][n], a0, a1, a2, a3, q[i][(n * C::KS + 4 * c + j) * C::STEP]);
                    }
                }
            }
        }
    };
    if constexpr (LAYER) {
        if (u0 < u1) {                             // the first pair, usually the only one
            float s[R8_SLOTS][R8_TILES][4] = {};
            scores(u0, s);
            // Nothing has gone before, so there is nothing to rescale, and the two units' weights share a reference where their values' units are not
            // far apart: w = 2^(s - m) 2^(ve - vmax + 8), R - m = vmax - 8.  (What is behind the wait is paid by the instruction: code that runs once in a
            // launch runs at the pace of its fetching, 4 to 8 cycles each.)
            const int vmax = max(exponent_of(exps[0], 1), valid[1] ? exponent_of(exps[1], 1) : -127);
            const int below[R8_SLOTS] = {vmax - exponent_of(exps[0], 1), valid[1] ? vmax - exponent_of(exps[1], 1) : 0};
            if (max(below[0], below[1]) > 8 || !valid[0]) {
                finish(u0, s);
            } else {
                if ((valid[0] & valid[1]) != 0xffffu) {
#pragma unroll
                    for (int i = 0; i < R8_SLOTS; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!((valid[i] >> (g + 8 * (e >> 1))) & 1)) s[i][0][e] = -INFINITY;
                }
                float mx[2] = {-INFINITY, -INFINITY};
                const float qu[2] = {sh.q_unit[2 * t], sh.q_unit[2 * t + 1]};
#pragma unroll
                for (int i = 0; i < R8_SLOTS; ++i) {
                    const float ku = pow2i(exponent_of(exps[i], 0)), f[2] = {score_unit(qu[0], ku), score_unit(qu[1], ku)};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        s[i][0][e] *= f[e & 1];
                        mx[e & 1] = fmaxf(mx[e & 1], s[i][0][e]);
                    }
                }
                __syncwarp();
                load_keys(u0 + R8_SLOTS);
#pragma unroll
                for (int sft = 4; sft < 32; sft <<= 1) {
                    mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], sft));
                    mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], sft));
                }
                const float mu[2] = {mx[0] == -INFINITY ? 0.f : mx[0], mx[1] == -INFINITY ? 0.f : mx[1]};
                uint2 p[R8_SLOTS][R8_TILES];
#pragma unroll
                for (int i = 0; i < R8_SLOTS; ++i) {
                    const float f = pow2i(8 - below[i]);
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = exp2f(s[i][0][e] - mu[e & 1]);
                        l[0][e & 1] += w[e];
                        w[e] *= f;
                    }
                    p[i][0].x = movmatrix_trans(pack_half2(w[0], w[1]));
                    p[i][0].y = movmatrix_trans(pack_half2(w[2], w[3]));
                }
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    m[0][c] = mx[c];
                    r[0][c] = (float)(vmax - 8);
                }
                outputs(u0, p);
            }
        }
    }
#pragma unroll 1
    for (int u = LAYER ? u0 + R8_SLOTS : u0; u < u1; u += R8_SLOTS) {
        float s[R8_SLOTS][R8_TILES][4] = {};
        scores(u, s);
        finish(u, s);
    }
    cp_async_wait<0>();

    // ---- the warps' results meet ----
#pragma unroll
    for (int n = 0; n < R8_TILES; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int sft = 4; sft < 32; sft <<= 1) l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], sft);
    __syncwarp();                                  // the warp's slots are read: its result goes there
    constexpr int ROW = D + R8_PAD;
    static_assert(C::COLS * ROW * 4 <= R8_SLOTS * C::SLOT, "");
    auto result_of = [&](int w) { return reinterpret_cast<float*>(ring + (size_t)w * R8_SLOTS * C::SLOT); };
#pragma unroll
    for (int n = 0; n < R8_TILES; ++n) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int col = n * 8 + 2 * t + c;
            float* base = result_of(warp) + col * ROW + g * (D / 8);
#pragma unroll
            for (int k = 0; k < C::KS; ++k) *reinterpret_cast<float2*>(base + 2 * k) = make_float2(o[n][k][c], o[n][k][2 + c]);
            if (g == 0) {
                sh.m[warp][col] = m[n][c];
                sh.r[warp][col] = r[n][c];
                sh.l[warp][col] = l[n][c];
            }
        }
    }
    if (LAYER && threadIdx.x == 0) sh.tag = (int)tag_of(asked);
    __syncthreads();
    const int n_cols = min(C::COLS, m_total - m0);
    // (token r, head h) of column m lies at row r * q_heads + h = r * (q_heads - G) + m
    auto out_at = [&](int col) { return out + (q_row0 * q_heads + hk * G + (size_t)sh.q_tok[col] * (q_heads - G) + m0 + col) * D; };
    const int record = ((blockIdx.z * gridDim.y + blockIdx.y) * splits) + split;
    unsigned char* const rec = reinterpret_cast<unsigned char*>(a.scratch) + R8_COUNTERS * 4 + (size_t)record * C::REC;
    unsigned char* const parts = vw.tagged + tagged_head_bytes(a.kv_heads) + (size_t)hk * splits * tagged_rec_bytes<D>();
    unsigned char* const part = parts + (size_t)split * tagged_rec_bytes<D>();
    constexpr int CH = D / 8;                      // chunks of 8 dims of a column
    for (int i = threadIdx.x; i < n_cols * (D / 4); i += R8_THREADS) {      // four dims a thread
        const int col = i / (D / 4), d0 = i % (D / 4) * 4;
        float M = -INFINITY, L = 0.f, acc[4] = {};
#pragma unroll
        for (int w = 0; w < R8_WARPS; ++w) M = fmaxf(M, sh.m[w][col]);
#pragma unroll 4
        for (int w = 0; w < R8_WARPS; ++w) {
            const float mw = sh.m[w][col];
            const bool none = mw == -INFINITY;                      // no score, or none that is a number
            const float f = none ? 0.f : exp2f((mw - M) + sh.r[w][col]);         // back from s + ve to s
            const float4 x = *reinterpret_cast<const float4*>(result_of(w) + col * ROW + d0);
            acc[0] += x.x * f; acc[1] += x.y * f; acc[2] += x.z * f; acc[3] += x.w * f;
            if (d0 == 0 || splits == 1) L += sh.l[w][col] * (none ? 1.f : exp2f(mw - M));
        }
        if (splits == 1) {
            const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] *= inv;
        }
        const unsigned pk[2] = {pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
        if (LAYER) {
            const unsigned tag = (unsigned)sh.tag;
            st_tagged2(part + (size_t)(col * D + d0) * 4, pk[0], pk[1], tag);
            if (d0 == 0) st_tagged2(part + 8 * D * 4 + col * 16, __float_as_uint(M), __float_as_uint(L), tag);
        } else {
            if (splits > 1 && d0 == 0) *reinterpret_cast<float2*>(rec + C::COLS * D * 2 + col * 8) = make_float2(M, L);
            unsigned* dst = reinterpret_cast<unsigned*>(splits == 1 ? reinterpret_cast<unsigned char*>(out_at(col) + d0) : rec + (col * D + d0) * 2);
            dst[0] = pk[0];                                         // (out need only be 4-byte aligned)
            dst[1] = pk[1];
        }
    }
    if (splits == 1) return;
    __syncthreads();                               // the merge buffer is read, the records are on their way
    if (LAYER) {
        if (threadIdx.x == 0) move_on(asked, epoch, splits);
        const int groups = G * CH, shares = min((groups + R8_GROUPS - 1) / R8_GROUPS, splits);
        if (split < shares)
            combine_tagged<D>(split, shares, splits, parts, (unsigned)sh.tag, merge, G, out + (q_row0 * q_heads + hk * G) * D, sh.wait_limit,
                              const_cast<int*>(&vw.ctrl->status));
        return;
    }

    // ---- the last block of these columns merges the splits' results ----
    unsigned* counter = reinterpret_cast<unsigned*>(a.scratch) + blockIdx.z * gridDim.y + blockIdx.y;
    if (threadIdx.x == 0) {
        unsigned before;
        __threadfence();
        asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
        sh.last = before == (unsigned)splits - 1;
        if (sh.last) *counter = 0;                 // ready for the next launch
    }
    __syncthreads();
    if (!sh.last) return;
    const unsigned char* recs = reinterpret_cast<const unsigned char*>(a.scratch) + R8_COUNTERS * 4 + (size_t)(record - split) * C::REC;
    for (int i = threadIdx.x; i < n_cols * CH; i += R8_THREADS) {
        const int col = i / CH, d0 = i % CH * 8;
        float M = -INFINITY, L = 0.f, acc[8] = {};
#pragma unroll 1
        for (int k0 = 0; k0 < splits; k0 += 8) {
            float2 ml[8];
            uint4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const unsigned char* at = recs + (size_t)min(k0 + k, splits - 1) * C::REC;
                ml[k] = ld_l2(reinterpret_cast<const float2*>(at + C::COLS * D * 2 + col * 8));
                v[k] = ld_l2(reinterpret_cast<const uint4*>(at + (col * D + d0) * 2));
            }
            float Mn = M;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k < splits) Mn = fmaxf(Mn, ml[k].x);
            const float f0 = M == -INFINITY ? 1.f : exp2f(M - Mn);  // (there is nothing but a NaN in L then)
            L *= f0;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] *= f0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k0 + k >= splits) continue;
                if (ml[k].x == -INFINITY) {
                    L += ml[k].y;
                    continue;
                }
                const float f = exp2f(ml[k].x - Mn);
                const unsigned w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
                L += ml[k].y * f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[2 * e] += __uint_as_float(w[e] << 16) * f;
                    acc[2 * e + 1] += __uint_as_float(w[e] & 0xffff0000u) * f;
                }
            }
            M = Mn;
        }
        const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);
        unsigned* dst = reinterpret_cast<unsigned*>(out_at(col) + d0);
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    }
}

template <int D, bool ONE, bool APPEND, bool LAYER>
cudaError_t launch_as(const SvlmAttend8& a, const SvlmRows8& x, int splits, int col_groups, cudaStream_t st) {
    using C = R8<D>;
    const int n_pages = a.n_slots / SVLM_PAGE;
    const cudaError_t e = svlm_allow_smem<rows8_kernel<D, ONE, APPEND, LAYER>>(C::smem(R8_MAX_PAGES));
    if (e != cudaSuccess) return e;
    return svlm_launch_chained(rows8_kernel<D, ONE, APPEND, LAYER>, dim3(splits, a.kv_heads * col_groups, a.n_caches * x.n_layers), dim3(R8_THREADS),
                               C::smem(n_pages), 1, st, a, x.layer0, x.n_layers, static_cast<const uint16_t*>(x.Q), x.q_pos, x.n_q, x.q_heads,
                               static_cast<uint16_t*>(x.out), splits, col_groups, static_cast<const uint16_t*>(x.Knew), static_cast<const uint16_t*>(x.Vnew),
                               x.early);
}

template <int D, bool ONE, bool APPEND>
cudaError_t launch(const SvlmAttend8& a, const SvlmRows8& x, cudaStream_t st) {
    using C = R8<D>;
    const int G = x.q_heads / a.kv_heads, problems = a.n_caches * x.n_layers, n_pages = a.n_slots / SVLM_PAGE;
    const int col_groups = (x.n_q * G + 8 * R8_TILES - 1) / (8 * R8_TILES), rows = a.kv_heads * col_groups * problems;
    // One wave of blocks, no more than the units keep busy.  Two to an SM, where a warp of one would have many units: what hides a unit's chain of dependent steps
    // then is other warps.  Fewer units are done sooner by one, whose blocks have less to meet about (28/4 heads over 9216 keys, 2 rows a block's
    // worth: 18.5 us, 20.3 with two to an SM; 4, 8 units a warp: 25.3 and 22.0), and from layer to layer it leaves room for the next launch to begin (one
    // token over 44512 keys, 9 units: 18.2 us a layer-step, 19.6 with two; 32/8 heads, 19 units: 36.6 and 32.3).  Shorter shares for several waves cost
    // more than they balance (sixteen streams: 45 us a layer-step, 53 in two waves).
    const bool chained = ONE && problems == 1;
    const bool two = x.pages * rows / svlm_sm_count() >= (chained ? 16 : 6) && C::smem(n_pages) <= R8_TWO_FIT;      // (a chained launch's are resident together)
    const int per_sm = two ? 2 : 1;
    // No more splits than there are units to go round: two a warp, or, where their results meet in as many blocks as there are (combine_tagged), one a warp
    // but enough of them to share that work (28/4 heads, 28 layers in a row, splits by four a page and this way: 200 keys 7.1 and 6.6 us, 700 7.0
    // and 6.6, 2100 7.5 and 6.8, 3300 7.5 and 7.8; the smallest stream's, 4/1 heads of 64 over 200 keys, in one split 5.8, in several 4.9).
    const int useful = chained ? std::max(x.pages, (G * (D / 8) + R8_GROUPS - 1) / R8_GROUPS) : x.pages * (SVLM_PAGE / SVLM_BLOCK8 / 2);
    const int most = std::min({per_sm * svlm_sm_count() / rows, useful, R8_MAX_RECORDS / rows});
    const int splits = rows > R8_COUNTERS ? 1 : std::max(1, most);
    // the splits of one layer of one cache poll for one another's results: all of them are resident
    if (chained && splits > 1) return launch_as<D, ONE, APPEND, ONE>(a, x, splits, col_groups, st);
    return launch_as<D, ONE, APPEND, false>(a, x, splits, col_groups, st);
}

}  // namespace

size_t svlm_rows8_scratch_bytes(int head_dim) {
    return R8_COUNTERS * 4 + (size_t)R8_MAX_RECORDS * (head_dim == 128 ? R8<128>::REC : R8<64>::REC);
}
size_t svlm_rows8_tagged_bytes(int kv_heads, int head_dim) {
    return tagged_head_bytes(kv_heads) + (size_t)std::max(kv_heads, 2 * svlm_sm_count()) * (head_dim == 128 ? tagged_rec_bytes<128>() : tagged_rec_bytes<64>());
}

bool svlm_rows8_supported(int n_pages) { return n_pages <= R8_MAX_PAGES; }

cudaError_t svlm_launch_rows8(const SvlmAttend8& a, const SvlmRows8& x, cudaStream_t st) {
    const bool one = !a.q_varlen && x.n_q == 1 && x.q_heads / a.kv_heads <= 8;
    if (x.Knew && !one) return cudaErrorInvalidValue;
    auto go = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (!one) return launch<D, false, false>(a, x, st);
        return x.Knew ? launch<D, true, true>(a, x, st) : launch<D, true, false>(a, x, st);
    };
    return a.head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}
