// Projections with 4-bit weights: Y[t][o] = sum over k of X[t][k] * s[o][k / group] * (q[o][k] - 8).  For a few tokens the work is reading the
// weights once, half a byte each, and turning them into operands.
//
// A thread block owns 16 output features at a time, the M side of mma.sync.m16n8k16 in bf16; the tokens are its N side in tiles of 8.  Its eight warps share K in
// blocks of 128: lane (g, t) takes of rows g and g + 8 four words of eight weights each, a quarter of what a group spans, so that every MMA stays within
// one group and a group's sum is scaled once, in fp32.  A nibble becomes a bf16 in place: q + 128 is exact in seven mantissa bits, q + 128 - 136
// as well.  Shifting a word by 0, 4, 8, 12 yields the pairs (k, k + 4) of its eight weights, and a product does not care in which order k is
// summed: the activations are paired the same way.  The weights depend on nothing earlier in the stream: while the predecessor still runs
// (programmatic dependent launch) a warp asks for its first four blocks; behind the wait come the activations.  The warps' sums meet in
// shared memory and are added in their order: the same bits every time.
//
// Of 8192 -> 24576 the turning of nibbles is 17 us of the integer pipe (some 72 operations for 1 KB of weights) and the loads alone take 19; together they take 27, with
// neither full (the pipe 52 % busy, DRAM 40 %): a warp's loads and its products take turns, and sixteen warps an SM do not hide that.
// Measured (inputs -> outputs, group 128 unless said, back to back in a graph; in brackets the bytes at the copy rate; a matrix of up to 126 MB may be in L2 in
// part when it is read again): one token 3584 -> 4608 3.7 us (1.3), group 32 6.7; two 8192 -> 24576 27 us, 3.9 TB/s (16); sixteen 3584 -> 3584, group 64, 5.1 us (1.1); thirty-two 3584 -> 4608 11.2 us
// (1.4).  From sixteen tokens on each 16 features read all activations again, and that is what bounds it.  Tried: a cluster of eight blocks for 128
// features, each with an eighth of K and its share of the activations in shared memory: 9.0 us, 52 us, 8.7 us, 16.7 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "svlm_launch.h"
#include "svlm_ptx.cuh"
#include "svlm_store8.h"

namespace {

using namespace svlm_ptx;

constexpr int W4_WARPS = 8;
constexpr int W4_AHEAD = 4;      // blocks of 128 of K that a warp has in flight
constexpr int W4_ROWS = 16;
constexpr size_t W4_SMEM = 113 * 1024;      // two thread blocks to an SM

__device__ __forceinline__ void mma_bf16_tile(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// N consecutive words of weights (read once per pass over the layers: the first to make room in L2)
template <int N>
__device__ __forceinline__ void ld_weights(unsigned* w, const uint8_t* p, unsigned long long policy) {
    if constexpr (N == 4)
        asm volatile("ld.global.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], %5;" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p), "l"(policy));
    else if constexpr (N == 2)
        asm volatile("ld.global.L2::cache_hint.v2.u32 {%0, %1}, [%2], %3;" : "=r"(w[0]), "=r"(w[1]) : "l"(p), "l"(policy));
    else
        asm volatile("ld.global.L2::cache_hint.u32 %0, [%1], %2;" : "=r"(w[0]) : "l"(p), "l"(policy));
}
// Weights k + J and k + J + 4 of a word's eight, less 8, as a pair of bf16 (exact).
template <int J>
__device__ __forceinline__ unsigned pair_of(unsigned w) {
    unsigned x;
    const unsigned eight = 0x43084308u;                          // 136
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(x) : "r"(w >> (4 * J)), "r"(0x000f000fu), "r"(0x43004300u));     // 128 + q, in one operation
    const __nv_bfloat162 y = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&eight));
    return *reinterpret_cast<const unsigned*>(&y);
}

template <int NT>
struct W4 {
    static constexpr int COLS = 8 * NT;
    static constexpr int PART = W4_WARPS * W4_ROWS * (COLS + 1);        // floats: the warps' sums of a tile
    static constexpr int fixed = 2 * PART * 4;
};

// NT: tiles of 8 tokens, blockIdx.y: which NT of them.
// ONCE: a thread block has one set of features and a warp one round of blocks, so there is nothing to run ahead to (eight tokens 3584 -> 4608: 4.5 us, 5.8 by the
//   other instance; one, group 32: 6.7 and 8.5).
// STAGED: the activations lie in shared memory, as operands, for all the features a thread block gets to (four tokens 8192 -> 24576: 29 us, 40 without).  With one
//   set of features it is worth it for the fewest tokens only (one 3584 -> 4608: 3.7 and 3.8 us; eight: 5.8 and 4.4).  What does not fit next to a second
//   thread block comes from the L1 cache (eight 8192 -> 24576: 46 us; one thread block to an SM: 41, but sixteen 3584 -> 4608 7.7 instead of 6.6).
// TAIL: K is not a multiple of 128.
template <int GROUP, int NT, bool STAGED, bool ONCE, bool TAIL>
__global__ void __launch_bounds__(W4_WARPS * 32, 2) w4_kernel(const uint16_t* X, const uint8_t* W, const uint16_t* scales, uint16_t* Y, int n, int in_dim, int out_dim) {
    using C = W4<NT>;
    constexpr int WPG = GROUP / 32, GROUPS = 4 / WPG;            // words of a lane per group; groups in a block of 128
    extern __shared__ __align__(128) unsigned char smem[];
    float* const part = reinterpret_cast<float*>(smem);          // [tile's parity][warp][row][column, pad]
    uint4* const xs = reinterpret_cast<uint4*>(smem + C::fixed); // [block][token][16 pieces]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int t0 = blockIdx.y * C::COLS, here = min(n - t0, C::COLS);
    const int n_blocks = (in_dim + 127) / 128, n_groups = in_dim / GROUP, n_tiles = (out_dim + W4_ROWS - 1) / W4_ROWS, step = gridDim.x;
    const unsigned long long once = l2_read_once();
    unsigned w[W4_AHEAD][2][4];
    uint16_t sc[W4_AHEAD][2][GROUPS];
    // Word j of a block belongs to group j / WPG of it and holds k = k_of(j), ..., + 7 of the block.
    auto k_of = [&](int j) { return j / WPG * GROUP + t * (GROUP / 4) + j % WPG * 8; };

    // The weights run ahead of the products, from tile to tile.  An address is the tile's, the same for all lanes, and a lane's 32-bit distance from it.  (A load
    // that there is no use for goes to the tile's, or the matrix's, first weights: with a branch around it the loads were waited for as soon as they had been
    // issued, and the loads alone of 8192 -> 24576 took 36 us instead of 19.)
    int ld_tile = blockIdx.x;
    const uint8_t* ld_w;
    const uint16_t* ld_s;
    unsigned at_w[2], at_s[2];
    bool any;
    auto enter = [&] {
        any = ld_tile < n_tiles;
        const size_t r0 = any ? (size_t)ld_tile * W4_ROWS : 0;
        ld_w = W + r0 * (in_dim / 2);
        ld_s = scales + r0 * n_groups;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned row = any ? min(g + 8 * h, out_dim - 1 - (int)r0) : 0;    // (rows past the end repeat the last one: nobody reads their sums)
            at_w[h] = row * (in_dim / 2) + k_of(0) / 2;
            at_s[h] = row * n_groups;
        }
    };
    auto load_block = [&](int i, int b0) {
        const unsigned b = any && b0 < n_blocks ? b0 : 0;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) {
                const bool in = !TAIL || b * 128 + q * GROUP < in_dim;
                ld_weights<WPG>(&w[i][h][q * WPG], ld_w + (at_w[h] + b * 64 + (in ? q * (GROUP / 2) : 0)), once);
                sc[i][h][q] = ld_in(ld_s + (at_s[h] + b * GROUPS + (in ? q : 0)));
            }
    };
    pdl_launch_dependents();
    enter();
#pragma unroll
    for (int i = 0; i < W4_AHEAD; ++i) load_block(i, warp + i * W4_WARPS);
    pdl_wait();
    if (STAGED) {
        // Piece (j, t) of a token's 16 lies at j ^ (token & 1), t: eight lanes' pieces, two tokens', fall into different banks
        for (int i = threadIdx.x; i < here * n_blocks * 16; i += W4_WARPS * 32) {
            const int tok = i / (n_blocks * 16), at = i - tok * (n_blocks * 16), ch = at & 15, b = at >> 4;
            const uint4 x = at * 8 < in_dim ? ld_in(reinterpret_cast<const uint4*>(X + (size_t)(t0 + tok) * in_dim + at * 8)) : make_uint4(0, 0, 0, 0);
            const int rem = ch * 8 % GROUP, j = ch * 8 / GROUP * WPG + rem % (GROUP / 4) / 8;
            xs[((size_t)b * here + tok) * 16 + (j ^ (tok & 1)) * 4 + rem / (GROUP / 4)] =
                make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
        }
        __syncthreads();
    }

    // where a lane's pieces of its columns' tokens lie, of even words and of odd ones (columns past the last token repeat it: nobody reads their sums)
    int at_x[NT][2];
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int tok = min(c * 8 + g, here - 1);
            at_x[c][j] = (tok * 16 + (j ^ (tok & 1)) * 4 + t) * 16;
        }
    int parity = 0;
#pragma unroll 1
    for (int tile = blockIdx.x; tile < n_tiles; tile += step) {
        float sum[NT][4];
#pragma unroll
        for (int c = 0; c < NT; ++c) sum[c][0] = sum[c][1] = sum[c][2] = sum[c][3] = 0.f;
#pragma unroll 1
        for (int b0 = warp; b0 < n_blocks; b0 += W4_AHEAD * W4_WARPS) {
            int ld_b = b0 + W4_AHEAD * W4_WARPS;
            if (!ONCE && ld_b >= n_blocks) {
                ld_b = warp;
                ld_tile += step;
                enter();
            }
#pragma unroll
            for (int i = 0; i < W4_AHEAD; ++i) {
                const int b = b0 + i * W4_WARPS;
                if (b < n_blocks) {
                    const unsigned char* const xb = reinterpret_cast<const unsigned char*>(xs) + b * here * 256;
#pragma unroll
                    for (int q = 0; q < GROUPS; ++q) {
                        if (TAIL && b * 128 + q * GROUP >= in_dim) break;
                        // (the first tile's sums in two halves: an MMA does not wait for the one before)
                        float acc[NT][4], acc2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int c = 0; c < NT; ++c) acc[c][0] = acc[c][1] = acc[c][2] = acc[c][3] = 0.f;
#pragma unroll
                        for (int j = q * WPG; j < (q + 1) * WPG; ++j) {
                            const unsigned u = w[i][0][j], v = w[i][1][j];
                            const unsigned a[2][4] = {{pair_of<0>(u), pair_of<0>(v), pair_of<1>(u), pair_of<1>(v)}, {pair_of<2>(u), pair_of<2>(v), pair_of<3>(u), pair_of<3>(v)}};
#pragma unroll
                            for (int c = 0; c < NT; ++c) {
                                uint4 y;
                                if (STAGED) {
                                    y = *reinterpret_cast<const uint4*>(xb + at_x[c][j & 1] + (j >> 1) * 128);
                                } else {
                                    const int tok = min(t0 + c * 8 + g, n - 1), k = b * 128 + k_of(j);
                                    const uint4 x = !TAIL || k < in_dim ? ld_in(reinterpret_cast<const uint4*>(X + (size_t)tok * in_dim + k)) : make_uint4(0, 0, 0, 0);
                                    y = make_uint4(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632), __byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
                                }
                                mma_bf16_tile(acc[c], a[0][0], a[0][1], a[0][2], a[0][3], y.x, y.y);
                                mma_bf16_tile(NT == 1 ? acc2 : acc[c], a[1][0], a[1][1], a[1][2], a[1][3], y.z, y.w);
                            }
                        }
                        const float s0 = __uint_as_float((unsigned)sc[i][0][q] << 16), s1 = __uint_as_float((unsigned)sc[i][1][q] << 16);
#pragma unroll
                        for (int c = 0; c < NT; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[c][e] += (e < 2 ? s0 : s1) * (NT == 1 ? acc[c][e] + acc2[e] : acc[c][e]);
                    }
                }
                if (!ONCE) load_block(i, ld_b + i * W4_WARPS);
            }
            if (ONCE) break;
        }
        // the warps' sums meet; two buffers, so that one barrier a tile will do
        float* const mine = part + parity * C::PART + warp * (W4_ROWS * (C::COLS + 1));
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(g + 8 * (e >> 1)) * (C::COLS + 1) + c * 8 + 2 * t + (e & 1)] = sum[c][e];
        __syncthreads();
        for (int i = threadIdx.x; i < W4_ROWS * here; i += W4_WARPS * 32) {
            const int r = i % W4_ROWS, c = i / W4_ROWS;
            const float* p = part + parity * C::PART + r * (C::COLS + 1) + c;
            float y = 0.f;
#pragma unroll
            for (int k = 0; k < W4_WARPS; ++k) y += p[k * (W4_ROWS * (C::COLS + 1))];
            if (tile * W4_ROWS + r < out_dim) Y[(size_t)(t0 + c) * out_dim + tile * W4_ROWS + r] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
        }
        if (ONCE) break;
        parity ^= 1;
    }
}

template <int GROUP, int NT>
cudaError_t launch_as(const uint16_t* x, const uint8_t* w, const uint16_t* s, uint16_t* y, int n, int in_dim, int out_dim, cudaStream_t st) {
    const int tiles = (out_dim + W4_ROWS - 1) / W4_ROWS, y_blocks = (n + 8 * NT - 1) / (8 * NT), grid = std::min(tiles, std::max(1, 2 * svlm_sm_count() / y_blocks));
    const size_t staged = W4<NT>::fixed + (size_t)std::min(n, 8 * NT) * ((in_dim + 127) / 128) * 256;
    const dim3 g(grid, y_blocks), b(W4_WARPS * 32);
    auto go = [&](auto staged_, auto once_, auto tail_) {
        constexpr bool STAGED = decltype(staged_)::value, ONCE = decltype(once_)::value, TAIL = decltype(tail_)::value;
        constexpr auto kernel = w4_kernel<GROUP, NT, STAGED, ONCE, TAIL>;
        const cudaError_t e = STAGED ? svlm_allow_smem<kernel>(W4_SMEM) : cudaSuccess;
        return e != cudaSuccess ? e : svlm_launch_chained(kernel, g, b, STAGED ? staged : W4<NT>::fixed, 1, st, x, w, s, y, n, in_dim, out_dim);
    };
    const std::true_type yes;
    const std::false_type no;
    const bool fits = staged <= W4_SMEM;
    if constexpr (GROUP < 128)
        if (in_dim % 128) return fits ? go(yes, no, yes) : go(no, no, yes);
    if (tiles == grid && in_dim <= 128 * W4_AHEAD * W4_WARPS) {
        if constexpr (NT == 1)
            if (n < 4) return go(yes, yes, no);
        return go(no, yes, no);
    }
    return fits ? go(yes, no, no) : go(no, no, no);
}
template <int GROUP>
cudaError_t launch(const uint16_t* x, const uint8_t* w, const uint16_t* s, uint16_t* y, int n, int in_dim, int out_dim, cudaStream_t st) {
    const int nt = std::min(4, (n + 7) / 8);
    const auto go = nt == 1 ? launch_as<GROUP, 1> : nt == 2 ? launch_as<GROUP, 2> : nt == 3 ? launch_as<GROUP, 3> : launch_as<GROUP, 4>;
    return go(x, w, s, y, n, in_dim, out_dim, st);
}

}  // namespace

cudaError_t svlm_launch_w4(const void* X, const void* W4, const void* scales, void* Y, int n, int in_dim, int out_dim, int group, cudaStream_t st) {
    const auto go = group == 128 ? launch<128> : group == 64 ? launch<64> : launch<32>;
    return go(static_cast<const uint16_t*>(X), static_cast<const uint8_t*>(W4), static_cast<const uint16_t*>(scales), static_cast<uint16_t*>(Y), n, in_dim, out_dim, st);
}
