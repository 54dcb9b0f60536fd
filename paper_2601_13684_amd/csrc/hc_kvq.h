// hc_kvq.h -- the cache held in 4 bits: its rows' format, and what its kernels share (not part of the C ABI).
//
// A row of 128 values is 64 bytes of codes and 4 scale bytes, one per 32 values.  Element i is bits 4 (i % 8) .. of dword i / 8: a sign and
// one of 0 .5 1 1.5 2 3 4 6, which stands for itself times 2^(s - 127), s the scale byte of its 32 values.  s is the smallest of which no
// value is more than 7 units (7 is taken to 6, as far off as 5 is from 4 or 6), at least 2: what a code stands for is then a normal number of 32 bits
// and of bf16 in every case, and exact in both.  s = 255: the 32 values are not numbers (one of them was not finite).
// Values of 1.75 * 2^127 and more may stand for 2^128, which reads as an infinity.
#pragma once
#include "hc_internal.h"

struct hc_kvq {
    uint32_t magic;
    hc_ctx* ctx;
    int n;                         // heads: B * Hkv
    int32_t max_cap;
    int64_t bytes, rows;           // that the cache and the tables of a number a row have to have room for
    int64_t units;                 // tiles of KQ_TILE rows of all heads at their caps
    std::vector<hc_kvq_head> host;
    hc_kvq_head* heads = nullptr;  // the same on the device
    int2* room = nullptr;          // [n]: cap, and tiles of the heads before it
    int2* chunks = nullptr;        // (head, first row) of every KQ_CHUNK rows of a head's cap
    int n_chunks = 0;
    int2* spans = nullptr;         // the same of every KQ_SPAN rows
    int n_spans = 0;
};
constexpr uint32_t HC_KVQ_MAGIC = 0x4843344bu;
constexpr int KQ_TILE = 32;                  // rows that a wave of the attention pass takes at a time
constexpr int KQ_CHUNK = 1024;               // rows of accumulated weights that a workgroup takes
constexpr int KQ_SHORT = 8 * 1024;           // longest head of a table whose evictions are done a workgroup to a head
constexpr int KQ_SPAN = 4096;                // rows that a workgroup of an eviction takes
constexpr int KQ_BINS = 2048;                // of an eviction's histograms: 11 bits of a key
constexpr int KQ_WG_PER_CU = 2;              // workgroups of the attention pass to a compute unit
constexpr int KQ_MOST_WG = 1024;             // of them, on any device
inline int hc_kvq_workgroups(const hc_ctx* ctx) { return ctx->n_cu * KQ_WG_PER_CU < KQ_MOST_WG ? ctx->n_cu * KQ_WG_PER_CU : KQ_MOST_WG; }

// Work buffer (byte offsets): what hc_kvq_attn and hc_kvq_evict leave there, one after the other.
struct hc_kvq_layout {
    size_t plan, part_ml, part_o, logits, list, hist, found, counts, bytes;
    int slots;
};
inline hc_kvq_layout hc_kvq_plan(const hc_kvq* k)
{
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const int G = k->ctx->G;
    hc_kvq_layout l;
    l.slots = hc_kvq_workgroups(k->ctx) + k->n;
    l.plan = 0;
    l.part_ml = up((size_t)k->n * sizeof(int2));
    l.part_o = l.part_ml + up((size_t)l.slots * G * 2 * sizeof(float));
    l.logits = l.part_o + up((size_t)l.slots * G * HC_D * sizeof(float));
    const size_t attn = l.logits + up((size_t)k->units * KQ_TILE * G * sizeof(float));
    l.list = 0;
    l.hist = up((size_t)k->rows * sizeof(int32_t));
    const bool spans = k->max_cap > KQ_SHORT;
    l.found = l.hist + (spans ? up((size_t)k->n * 3 * KQ_BINS * sizeof(uint32_t)) : 0);
    l.counts = l.found + (spans ? up((size_t)k->n * 3 * sizeof(uint2)) : 0);
    const size_t evict = l.counts + (spans ? up((size_t)k->n_spans * sizeof(uint2)) : 0);
    l.bytes = attn > evict ? attn : evict;
    return l;
}

hc_status hc_launch_kvq_attn(hc_ctx* ctx, const hc_kvq* kvq, const void* arena, const int32_t* state, const void* q, float* out, float* lse, float* acc,
                             float decay, void* work, hipStream_t st);

#if defined(__HIPCC__)
typedef __bf16 kq_bf16x2 __attribute__((ext_vector_type(2)));
// Two elements of a dword of codes (BYTE: which), times 2^(s - 127), bf16.
template <int BYTE>
__device__ __forceinline__ uint32_t kq_pair(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
// The scale byte as the factor that the conversions take (they make no number of an infinite one, as s = 255 stands for).
__device__ __forceinline__ float kq_scale(uint32_t s) { return __uint_as_float(s << 23); }
__device__ __forceinline__ int kq_rows(const int2* __restrict__ state, const int2* __restrict__ room, int i)
{
    return min(max(state[i].x, 0), room[i].x);
}
#endif
