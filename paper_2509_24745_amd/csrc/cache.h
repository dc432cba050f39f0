// Host-side declarations of the rotation and paged-cache entry points and
// their launchers.  Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pa {

// Sequences of a batch at most: found by two looks of 64 lanes at new_start.
constexpr int kMaxSeqs = 4096;

// A norm and rotation with every default resolved (see proxyattn_rotary).
struct RotaryArgs {
    int rot;          // rotary_dim
    int interleaved;
    int table_len;
    double eps;
    const float* cos;
    const float* sin;
    const void* qw;
    const void* kw;
};

// A validated cache and batch.  Passed to kernels by value.
struct CacheShape {
    int b;           // sequences
    int t;           // rows of the token arrays
    int max_new, max_len;
    int hq, hkv, d, rep;
    int page_shift;  // log2(page_size)
    int num_pages, width;
    int dtype, fp4;
    int past;        // the attention reads the pages past the caches
    // softmax scale times log2(e): the fp32 below it, and what that leaves, above 0
    float scale2, scale2_rest;
    int64_t q_tok, q_head, kv_tok, kv_head, o_tok, o_head;  // element strides
};

struct PagePtrs {
    void *k, *v, *ks, *vs;
};

// Rows that proxyattn_norm_rotate works on: Q rows, then K rows.
struct RotateRows {
    const void *q, *k;   // NULL: no such rows
    void *qo, *ko;
    const int* positions;
    int first;
    int n, hq, hkv, d, dtype;
    int64_t q_tok, q_head, k_tok, k_head, qo_tok, qo_head, ko_tok, ko_head;
};
hipError_t launch_norm_rotate(const RotateRows& w, const RotaryArgs& r, hipStream_t st);

struct AppendArgs {
    const void *q, *k, *v;   // q NULL: keys and values alone
    void* qo;
    int64_t qo_tok, qo_head;
    int norm_rotate;         // 0: r is not used
};
hipError_t launch_cache_append(const CacheShape& s, const RotaryArgs& r, const AppendArgs& a,
                               const int* table, const int* lens, const int* starts,
                               const PagePtrs& pg, hipStream_t st);
hipError_t launch_cache_read(const CacheShape& s, const int* table, const int* lens,
                             const int* starts, const PagePtrs& pg, void* ko, void* vo,
                             hipStream_t st);

// Workspace of the cache attention: 256-byte aligned offsets.
struct CacheWs {
    size_t plan;   // first unit of each sequence [B + 1] int32
    size_t stat;   // partial rows' (reference, sum) [2 W][rows] float2
    size_t part;   // partial outputs [2 W][rows][d] fp32
    size_t total;
    int groups;    // workgroups W
    int tiles;     // 16-row tiles of a workgroup's rows: 1 to 4
    int joined;    // whether runs of units are cut between workgroups (else one to each)
};
// False: more units of work than an int counts.
bool cache_ws(const CacheShape& s, CacheWs* w);
hipError_t launch_cache_attention(const CacheShape& s, const void* q, const int* table,
                                  const int* lens, const int* starts, const PagePtrs& pg,
                                  void* out, float* lse, char* ws, const CacheWs& w,
                                  hipStream_t st);

}  // namespace pa
