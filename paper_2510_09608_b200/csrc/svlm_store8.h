// Device-side layout of a cache that holds its keys and values in 8 bits, and the launchers of its kernels.
//
// Pages, slots and per-token metadata are those of svlm_dev.h.  Of every [layer][kv_head] row of slots, 16 consecutive slots of a
// page are one BLOCK: their values are 8-bit floats (e4m3: 1 sign, 4 exponent, 3 mantissa bits, largest 448) in units of 2^e, one e
// for the block's keys and one for its values, the least that brings the block's largest finite value to 448 or less.  A float's
// relative precision does not depend on its unit, so e only has to keep the block in range; as a power of two it scales exactly,
// and a token that joins a block and raises e moves the exponents of those before it (exact above e4m3's subnormals, i.e. for
// whatever is not 2^15 times smaller than the block's largest).  NaN and infinities are stored as NaN and do not count for e.
//
// Keys are stored rotated at their NATIVE position and never again: an eviction lowers the contiguous position of a token by a shift
// that is the same on all its axes, R(c) k = R(-s) R(c + s) k, so what changes is one integer per token, s = native - contiguous,
// and attention turns the query by it instead of the key.  (Rotating a stored key in place, as the 16-bit cache does, would round it
// to three mantissa bits each time.)
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "svlm_dev.h"

#define SVLM_BLOCK8 16

struct SvlmStore8 {
    unsigned char* K;        // [layers][kv_heads][n_slots][head_dim] e4m3, rotated at the native position
    unsigned char* V;        // same shape
    unsigned* exps;          // [layers][kv_heads][n_slots / 16] the blocks' exponents: keys' in bits 0-7, values' in bits 8-15, signed
    int* most;               // [layers][kv_heads] the largest exponent of a row's stored keys + MOST8_BIAS (0: none yet), or a little more
    int* native;             // [n_slots] the token's native position on the first axis
    // What an eviction leaves for the attention (svlm_launch_shift8): S the total shift, s a token's.
    int* apart;              // [n_slots / 16] S - s where it is the same for all of a block's tokens, MIXED8 where it is not
    const double2* rope64;   // [3][256][head_dim / 2] (cos, sin) as SvlmCacheDev::rope_tab, not rounded
    uint2* turn;             // [n_slots][head_dim / 4] where apart is not 0, the tokens' rotation by S - s: { cos, sin } of the
                             // pairs 2i, 2i + 1 as two halves each
};
constexpr int MOST8_BIAS = 128;
constexpr int MIXED8 = -1;   // (S >= s: a shift only grows along the stream)
struct SvlmStore8List {
    SvlmStore8 at[SVLM_MAX_BATCH];
    int n_q[SVLM_MAX_BATCH]; // query rows of the attention over what is widened
};

// Behind an eviction's metadata: apart and turn of every active page's blocks.
cudaError_t svlm_launch_shift8(const SvlmCacheList& list, const SvlmStore8List& stores, const SvlmCacheDev& geom, cudaStream_t st);

// The appended tokens' keys and values into their slots (the counterpart of svlm_launch_kv_write).  pos: the native positions, for
// layer <= 0 (null otherwise: they are kept per slot).  early, here and below: the caller vouches that the launch just before writes none of
// the cache's metadata.
cudaError_t svlm_launch_kv_write8(const SvlmCacheDev& cd, const SvlmStore8& st8, int layer, const void* K, const void* V, const int* pos, int n,
                                  bool early, cudaStream_t st);
// One layer's stored keys, rotated at their contiguous positions, and values in 16 bits in cd.K and cd.V ([kv_heads][n_slots][head_dim]):
// all slots of the active pages, those without a token as zeros.  Values are bf16 (exact).  Keys are bf16, or (half) f16 in units of a power
// of two of their KV head.  Its exponent goes into SvlmHead8; and there, values that are not finite of tokens that come behind the first of the latest n_q are
// zeros, since the rows before them must not have them, and late says so: the chunk kernel puts them into the others (from the bytes).
struct SvlmHead8 { int unit, late; };    // per KV head, 512 bytes behind cd.tmaps; late stays until an eviction
cudaError_t svlm_launch_widen8(const SvlmCacheDev& cd, const SvlmStore8& st8, int layer, int n_q, bool half, bool early, cudaStream_t st);
cudaError_t svlm_launch_widen8_batch(const SvlmCacheList& list, const SvlmStore8List& stores, const SvlmCacheDev& geom, int layer, bool half, bool early,
                                     cudaStream_t st);

// Few query rows straight from the 8-bit cache (svlm_rows8.cu).
struct SvlmView8 {           // what attention needs of one cache
    unsigned char* K;
    unsigned char* V;
    unsigned* exps;
    int* apart;
    uint2* turn;
    int* most;
    int* native;
    const double2* rope64;
    const SvlmCtrl* ctrl;
    const SvlmTile* tiles;
    const long long* slot_gid;
    const int* slot_c;
    const int* new_slot;
    unsigned char* tagged;   // epochs and tagged records (svlm_rows8_tagged_bytes, zero before the first launch)
};
struct SvlmAttend8 {         // kernel parameter: up to 32 caches share one launch
    int n_caches;
    int layers, kv_heads, head_dim, n_slots;
    int rope_mode, sec_t, sec_th;
    int q_varlen;            // as in SvlmAttendBatch
    int q_off[SVLM_MAX_BATCH];
    int q_cnt[SVLM_MAX_BATCH];
    SvlmView8 view[SVLM_MAX_BATCH];
    void* scratch;           // of the first cache: svlm_rows8_scratch_bytes, the counters in front zero before the first launch
    const float* rope_tab;
    double theta[SVLM_MAX_HALF];
};
constexpr int R8_COUNTERS = 4096;          // (problem, KV head, column group)s of a launch whose keys are divided
constexpr int R8_MAX_RECORDS = 512;        // splits of all of them
constexpr int R8_MAX_PAGES = 8192;         // the kernel keeps the list of active pages in shared memory
struct SvlmRows8 {           // a call
    int layer0, n_layers, n_q, q_heads;
    const void* Q;           // and out: [n_caches][n_layers][n_q][q_heads][d]; q_pos [n_caches][n_q](x3)
    const int* q_pos;
    void* out;
    int pages;               // about how many a cache holds: the division of the work depends on it, the result in the order of its sums
    // A decode step (n_q 1, at most 8 heads per KV head): the latest appended token's key and value, [n_caches][n_layers][kv_heads][d], are
    // written by this launch.  Null: nothing is.
    const void* Knew;
    const void* Vnew;
    // The caller vouches that nothing enqueued behind the launch before the previous one writes these caches' metadata or these layers'
    // keys and values: they are read while the previous kernel may still run.
    int early;
};
size_t svlm_rows8_scratch_bytes(int head_dim);
size_t svlm_rows8_tagged_bytes(int kv_heads, int head_dim);
bool svlm_rows8_supported(int n_pages);
cudaError_t svlm_launch_rows8(const SvlmAttend8& a, const SvlmRows8& x, cudaStream_t st);

// Y = X W^T with 4-bit weights and a scale per group (svlm_w4.cu)
cudaError_t svlm_launch_w4(const void* X, const void* W4, const void* scales, void* Y, int n, int in_dim, int out_dim, int group, cudaStream_t st);
