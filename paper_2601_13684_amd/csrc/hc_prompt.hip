// hc_prompt.hip -- attention of a prompt's tokens, or of a chunk of them, over the prompt's K and V: causal, packed sequences, query
// heads in groups of G to a KV head.  For the token at position p of a sequence and query head a of KV head h
//     s_j = q . K_h[j] / sqrt(128),  j = 0 .. p;   out = sum_j exp(s_j - lse) V_h[j],   lse = log sum_j exp(s_j)
//
// Work is cut into tiles of PA_ROWS query rows of one KV head, the group's G heads of a token side by side: a tile spans PA_ROWS / G
// tokens, the group shares its K and V, and the diagonal is met in fine steps.  A wave holds 32 rows.  It forms the transposed
// product S^T = K Q^T on the matrix cores (v_mfma_f32_32x32x16_bf16), keys along the registers and a query to each lane, so that a
// row's maximum and sum stay inside a lane but for one exchange between the halves of the wave; and the registers that hold P^T
// are, rounded to bf16, the second product's operand as they are: O^T = V^T P^T may take the keys of a step in any order as long
// as both operands do, and V is read from LDS transposed (ds_read_b64_tr_b16) in the order that S^T leaves.  One pass with running
// maximum and sum; the reference moves only when a logit exceeds it by more than 2^PA_SLACK, so that the accumulators are seldom rescaled.
//
// P is rounded to bf16 for the matrix cores, to the nearest: the error of an output is that of its 2^-9 per weight, independent
// from key to key, about what the output's own rounding to bf16 adds.  Sum, maximum, lse and accumulators are 32-bit, the sum
// from the unrounded weights.
//
// K and V tiles of 64 keys go straight to LDS (buffer loads of 16 bytes a lane), two buffers, the next tile's loads in flight
// under the present one's arithmetic.  A tile lies in blocks of 16 rows by 4 chunks of 16 bytes (a load instruction's kilobyte), chunk c of
// row r at place c ^ (r / 4 mod 4) of its 64 bytes: the reads of K (16 rows, one chunk) and the transposed reads of V (4 rows, 4 chunks) then
// both go over all banks once, and all of a wave's reads of a tile are two addresses a lane and an offset that the instruction holds.
#include <algorithm>
#include <type_traits>

#include "hc_internal.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int PA_BLK = 256, PA_ROWS = 128;        // four waves of 32 query rows
constexpr int PA_PER_CU = 2;                      // workgroups that a compute unit holds
constexpr int PA_KEYS = 64;                       // keys of a tile in LDS
constexpr int PA_TILE = PA_KEYS * HC_D * 2;       // its bytes
constexpr float PA_SCALE = 1.4426950408889634f * 0.08838834764831845f;     // log2(e) / sqrt(128)
constexpr float PA_LN2 = 0.6931471805599453f;
constexpr float PA_SLACK = 8.0f;                  // log2 units: a weight is at most 2^8 before the reference moves

struct PromptSeq {
    int unit_end;          // of the launch's work units, sequence by sequence
    int first, count;      // positions before the chunk, tokens of the chunk
    int tok0;              // its first token among the packed ones
    int tiles, splits;     // tiles of query rows of a KV head; pieces of the keys
};
struct PromptArgs {
    const uint16_t *q, *kv;
    uint16_t* out;
    float *lse, *part_acc, *part_ml;
    int Hkv, n_seq, chunk, tokens;                // chunk: keys of a piece
    PromptSeq seq[HC_PROMPT_SEQS];
    int64_t k_off[HC_PROMPT_HEADS], v_off[HC_PROMPT_HEADS];
};

__device__ __forceinline__ void swap_halves32(uint32_t& x, uint32_t& y)
{
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
}
__device__ __forceinline__ float other_half(float x)
{
    uint32_t a = __float_as_uint(x), b = a;
    swap_halves32(a, b);                          // a: upper lanes hold the lower half's, b: lower lanes the upper half's
    return __uint_as_float((threadIdx.x & 32) ? a : b);
}
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}

// Every wave's loads to LDS have arrived, and every wave is through with the tile before.  (The barrier alone does not wait for them.)
__device__ __forceinline__ void tile_ready()
{
    __builtin_amdgcn_s_waitcnt(0x0f70);           // vmcnt(0)
    __syncthreads();
}

// How a step's instructions are to follow each other: behind each product operand reads for the next eight and a share of the weights'
// arithmetic.
__device__ __forceinline__ void interleave_half()
{
    constexpr int PRODUCT = 0x8, READ = 0x100, VALU = 0x2, TRANS = 0x400;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
        __builtin_amdgcn_sched_group_barrier(PRODUCT, 1, 0);
        __builtin_amdgcn_sched_group_barrier(VALU, 4, 0);
        __builtin_amdgcn_sched_group_barrier(TRANS, 2, 0);
    }
}
__device__ __forceinline__ void interleave()
{
    constexpr int PRODUCT = 0x8, READ = 0x100, VALU = 0x2, TRANS = 0x400;
    interleave_half();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_group_barrier(READ, 1, 0);
        __builtin_amdgcn_sched_group_barrier(PRODUCT, 1, 0);
        __builtin_amdgcn_sched_group_barrier(VALU, 4, 0);
        __builtin_amdgcn_sched_group_barrier(TRANS, 1, 0);
    }
}

// The reference and the sum of a lane's row.  ref is a whole number, so that what was weighed against an older one is rescaled exactly,
// bf16 weights included; lim = ref + PA_SLACK, -inf while the row has seen nothing.
struct RowState {
    float ref, lim, l;
};

// Four waves of 32 rows.
template <int G>
__global__ __launch_bounds__(PA_BLK, 2) void prompt_attn_kernel(PromptArgs a)
{
    // (arrays of their own, so that the compiler sees that a buffer's loads in flight are not what the reads of the other wait for)
    __shared__ __attribute__((aligned(1024))) char sm_k0[PA_TILE], sm_k1[PA_TILE], sm_v0[PA_TILE], sm_v1[PA_TILE];
    __shared__ unsigned long long sm_bad;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n = lane & 31, hh = lane >> 5;

    // which tile, which piece of its keys, which head: the longest sequence's last tiles first, heads fastest, so that the workgroups
    // that stream the same K and V land on the same die
    const int unit = blockIdx.x;
    const int si = __popcll(__builtin_amdgcn_ballot_w64(lane < a.n_seq && a.seq[lane].unit_end <= unit));
    const PromptSeq sq = a.seq[si];
    int u = unit - (si > 0 ? a.seq[si - 1].unit_end : 0);
    const int h = u % a.Hkv;
    u /= a.Hkv;
    const int split = u % sq.splits, tile = sq.tiles - 1 - u / sq.splits;
    const int m0 = tile * PA_ROWS;
    const int last_tok = min((m0 + PA_ROWS - 1) / G, sq.count - 1);
    const int key_begin = split * a.chunk;
    const int key_end = min(sq.first + last_tok + 1, key_begin + a.chunk);        // one behind the last key of this unit
    if (key_begin >= key_end) return;
    const int n_tiles = (key_end - key_begin + PA_KEYS - 1) / PA_KEYS;
    const int n_full = max(0, min(key_end, sq.first + m0 / G + 1) - key_begin) / PA_KEYS;      // tiles that every row sees whole

    // this wave's rows and how far each sees
    const int w0 = m0 + w * 32;
    const int wtok0 = w0 / G;
    const bool idle = wtok0 >= sq.count;
    const int wave_end = sq.first + min((w0 + 31) / G, sq.count - 1) + 1;
    const int limit = sq.first + min((w0 + n) / G, sq.count - 1);
    auto row_of = [&](int r) { return ((size_t)(sq.tok0 + min(r / G, sq.count - 1)) * a.Hkv + h) * G + r % G; };       // of q, out and lse
    bf16x8 Q[8];
    {
        const uint16_t* from = a.q + row_of(w0 + n) * HC_D + hh * 8;
#pragma unroll
        for (int d = 0; d < 8; ++d) Q[d] = *reinterpret_cast<const bf16x8*>(from + 16 * d);
    }
    const int head = si * a.Hkv + h;
    const char* kb = (const char*)(a.kv + a.k_off[head]) + (size_t)key_begin * (HC_D * 2);
    const char* vb = (const char*)(a.kv + a.v_off[head]) + (size_t)key_begin * (HC_D * 2);

    // loads: instruction i of wave w takes chunks 4 i .. 4 i + 3 of rows 16 w .. 16 w + 15, a lane one of them
    const int ld_row = 16 * w + (lane >> 2), ld_off = ld_row * 256 + ((lane & 3) ^ (lane >> 4)) * 16;
    auto load = [&](const char* from, int t, char* to) {
        const int rows = key_end - key_begin - t * PA_KEYS;
        const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(from + (size_t)t * PA_TILE), 0, PA_TILE, 0x00027000);
        const int off = rows >= PA_KEYS ? ld_off : ld_off + (min(ld_row, rows - 1) - ld_row) * 256;      // rows past the last key repeat it; they are masked
#pragma unroll
        for (int i = 0; i < 4; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)((lds_char*)to + (4 * w + i) * 1024), 16, off, 64 * i, 0, 0);
    };
    auto load_k = [&](int t, auto buf) { load(kb, t, buf() ? sm_k1 : sm_k0); };
    auto load_v = [&](int t, auto buf) { load(vb, t, buf() ? sm_v1 : sm_v0); };

    // operand reads: a lane's places in a tile, the same in every buffer
    const int n16 = lane & 15;
    uint32_t k_at[2], v_at[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        k_at[p] = n / 16 * 4096 + n16 * 64 + (((2 * p + hh) ^ (n16 >> 2)) * 16);
        v_at[p] = (8 * p + 4 * hh + (n16 >> 2)) * 64 + (((2 * (n / 16) + ((n16 & 3) >> 1)) ^ (2 * p + hh)) * 16) + (n16 & 1) * 8;
        asm("" : "+v"(k_at[p]), "+v"(v_at[p]));      // (opaque, so that a buffer goes into an instruction's offset and not into registers of its own)
    }

    f32x16 O[4];
    RowState row;
    // operands of 32 keys, half k of a tile
    auto read_k = [&](const char* tile_k, int k, bf16x8 (&F)[8]) {
#pragma unroll
        for (int d = 0; d < 8; ++d) F[d] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>((lds_char*)tile_k + k * 8192 + d / 2 * 1024 + k_at[d & 1]);
    };
    auto read_v = [&](const char* tile_v, int k, bf16x8 (&F)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const lds_char* at = (lds_char*)tile_v + k * 8192 + i / 4 * 4096 + i % 4 * 1024;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + v_at[0]));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + v_at[1]));
            F[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    };
    // S^T = K Q^T
    auto logits = [&](const bf16x8 (&F)[8], f32x16& S) {
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = 0.f;
#pragma unroll
        for (int d = 0; d < 8; ++d) S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(F[d], Q[d], S, 0, 0, 0);
    };
    // O^T += V^T P^T
    auto values = [&](const bf16x8 (&F)[8], const bf16x8 (&P)[2]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) O[i % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(F[i], P[i / 4], O[i % 4], 0, 0, 0);
    };
    auto largest = [&](const f32x16& S) {
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, S[i]);
        return fmaxf(top, other_half(top)) * PA_SCALE;
    };
    auto weights = [&](f32x16& S, bf16x8 (&P)[2]) {
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = __builtin_amdgcn_exp2f(fmaf(S[i], PA_SCALE, -row.ref));
        float sum[2] = {S[0], S[1]};
#pragma unroll
        for (int i = 2; i < 16; ++i) sum[i & 1] += S[i];
        row.l += sum[0] + sum[1];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = pack2(S[8 * s + 2 * e], S[8 * s + 2 * e + 1]);
            P[s] = __builtin_bit_cast(bf16x8, x);
        }
    };
    // Before weights are taken of logits up to `top`; P: weights against the reference so far that O does not hold yet.
    auto settle = [&](float top, bf16x8 (&P)[2]) {
        if (!__builtin_amdgcn_ballot_w64(top > row.lim)) return;
        const float ref = row.lim == -INFINITY ? ceilf(top) : fmaxf(row.ref, ceilf(top));
        const bool none = top == -INFINITY && row.lim == -INFINITY;
        const float f = row.lim == -INFINITY ? 0.f : ref == row.ref ? 1.f : __builtin_amdgcn_exp2f(row.ref - ref);
        if (!none) {
            row.ref = ref;
            row.lim = ref + PA_SLACK;
        }
        row.l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[d][i] *= f;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            u32x4 x = __builtin_bit_cast(u32x4, P[s]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = pack2(__uint_as_float(x[e] << 16) * f, __uint_as_float(x[e] & 0xffff0000u) * f);
            P[s] = __builtin_bit_cast(bf16x8, x);
        }
    };

    auto clear = [&] {
        row = RowState{0.f, -INFINITY, 0.f};
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[d][i] = 0.f;
    };
    // The logits of half a tile, -inf where a row does not see the key, and what follows from them.
    auto masked = [&](const char* tile_k, const char* tile_v, int key, int k) {
        f32x16 S;
        bf16x8 P[2]{}, F[8];
        read_k(tile_k, k, F);
        logits(F, S);
        read_v(tile_v, k, F);
        const int see = min(limit, key_end - 1) - key - 32 * k - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i / 4) + i % 4 > see) S[i] = -INFINITY;
        settle(largest(S), P);
        weights(S, P);
        values(F, P);
    };
    {
        clear();
        using B0 = std::integral_constant<int, 0>;
        using B1 = std::integral_constant<int, 1>;
        load_k(0, B0{});
        load_v(0, B0{});
        int k_next = 1;                              // first tile of K whose loads are not under way
        if (n_full > 0) {
            // Tiles that every row sees whole, in steps of 32 keys, three of them at a time: the logits of step i + 1 and the sums of step
            // i - 1 on the matrix cores, between them the weights of step i, which wait for neither.  Operands are read from LDS one
            // product ahead (eight reads' worth of registers for K, as many for V): a read takes longer than the few products that
            // could be put between it and its use.  K runs a tile ahead of V.  The one barrier of a tile stands where the wave has read
            // all that it will read of both buffers, before their last product, which then covers the first reads of the next tile.
            f32x16 S0, S1;
            bf16x8 P0[2]{}, P1[2], K[8], V[8];
            if (n_tiles > 1) load_k(1, B1{});
            tile_ready();
            read_k(sm_k0, 0, K);
            logits(K, S0);
            read_k(sm_k0, 1, K);
            settle(largest(S0), P0);
            logits(K, S1);
            weights(S0, P0);
            settle(largest(S1), P0);
            tile_ready();
            if (n_tiles > 1) load_v(1, B1{});
            if (n_tiles > 2) load_k(2, B0{});
            read_k(sm_k1, 0, K);                     // (of tile 1; nothing comes of it where there is none)
            // tile t's sums and tile t + 1's logits; vbuf: where V of tile t is, and where K of t + 1 is not
            auto body = [&](int t, auto vbuf) {
                char* const tile_k = vbuf() ? sm_k0 : sm_k1;
                char* const next_k = vbuf() ? sm_k1 : sm_k0;
                char* const tile_v = vbuf() ? sm_v1 : sm_v0;
                read_v(tile_v, 0, V);
                logits(K, S0);
                weights(S1, P1);
                read_k(tile_k, 1, K);
                values(V, P0);
                const float top0 = largest(S0);
                interleave();
                settle(top0, P1);
                read_v(tile_v, 1, V);
                logits(K, S1);
                weights(S0, P0);
                interleave_half();
                tile_ready();
                if (t + 3 < n_tiles) load(kb, t + 3, tile_k);
                if (t + 2 < n_tiles) load(vb, t + 2, tile_v);
                read_k(next_k, 0, K);
                values(V, P1);
                settle(largest(S1), P0);
            };
            int t = 0;
            for (; t + 2 < n_full; t += 2) {
                body(t, B0{});
                body(t + 1, B1{});
            }
            if (t + 1 < n_full) {
                body(t, B0{});
                ++t;
            }
            const char* tile_v = t & 1 ? sm_v1 : sm_v0;
            read_v(tile_v, 0, V);
            weights(S1, P1);
            values(V, P0);
            read_v(tile_v, 1, V);
            values(V, P1);
            k_next = n_full + 2;
        }
        tile_ready();
        // The tiles behind them, in which some row sees only the first keys.
        auto step = [&](int t, auto buf) {
            const int key = key_begin + t * PA_KEYS;
            if (t + 1 < n_tiles) {
                if (t + 1 >= k_next) load_k(t + 1, std::integral_constant<int, 1 - buf()>{});
                load_v(t + 1, std::integral_constant<int, 1 - buf()>{});
            }
            if (!idle && key < wave_end) {
                masked(buf() ? sm_k1 : sm_k0, buf() ? sm_v1 : sm_v0, key, 0);
                masked(buf() ? sm_k1 : sm_k0, buf() ? sm_v1 : sm_v0, key, 1);
            }
            tile_ready();
        };
        int t = n_full;
        if (t & 1 && t < n_tiles) step(t++, B1{});
        for (; t < n_tiles; t += 2) {
            step(t, B0{});
            if (t + 1 < n_tiles) step(t + 1, B1{});
        }
        float z = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = fmaf(O[d][i], 0.f, z);
        if (n_full < n_tiles && __syncthreads_or(z != 0.f)) {
            // Some sum is not finite: what a masked weight of zero makes of an infinity or a NaN in V must not count.  Once more, tile
            // by tile: such values leave the tile, and are added by hand to the rows that see them.
            clear();
            for (t = 0; t < n_tiles; ++t) {
                const int key = key_begin + t * PA_KEYS;
                load_k(t, B0{});
                load_v(t, B0{});
                if (tid == 0) sm_bad = 0;
                tile_ready();
                for (int i = tid; i < PA_TILE / 16; i += PA_BLK) {
                    u32x4* p = reinterpret_cast<u32x4*>(sm_v0 + i * 16);
                    u32x4 x = *p;
                    bool hit = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((x[e] & 0x7f80u) == 0x7f80u) { x[e] &= 0xffff0000u; hit = true; }
                        if ((x[e] & 0x7f800000u) == 0x7f800000u) { x[e] &= 0x0000ffffu; hit = true; }
                    }
                    if (hit) {
                        *p = x;
                        atomicOr(&sm_bad, 1ull << (i / 256 * 16 + i / 4 % 16));
                    }
                }
                __syncthreads();
                if (!idle && key < wave_end) {
#pragma unroll 1
                    for (int k = 0; k < 2; ++k) masked(sm_k0, sm_v0, key, k);
                    for (unsigned long long bad = sm_bad; bad; bad &= bad - 1) {
                        const int j = __builtin_ctzll(bad), at = min(key + j, key_end - 1);
                        const uint16_t* from = (const uint16_t*)(vb + (size_t)(at - key_begin) * (HC_D * 2)) + 4 * hh;
                        const bool sees = key + j == at && at <= limit;
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t x = from[32 * d + 8 * (i / 4) + i % 4];
                                if (sees && (x & 0x7f80u) == 0x7f80u) O[d][i] += __uint_as_float(x << 16);
                            }
                        }
                    }
                }
                __syncthreads();
            }
        }
    }

    float l = row.l;
    l += other_half(l);
    int late = tid;                                  // (opaque: what follows is not worked out before the loops and kept through them)
    asm volatile("" : "+v"(late));
    const int r = w * 32 + (late & 31), half = (late >> 5) & 1;
    if (m0 + r >= sq.count * G) return;
    if (sq.splits == 1) {
        const float f = 1.0f / l;
        const size_t row_out = row_of(m0 + r);
        uint16_t* to = a.out + row_out * HC_D + 8 * half;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i) {            // 16 dimensions: after the exchange a lane holds eight in a row
                uint32_t x0 = pack2(O[d][8 * i] * f, O[d][8 * i + 1] * f), x1 = pack2(O[d][8 * i + 2] * f, O[d][8 * i + 3] * f);
                uint32_t y0 = pack2(O[d][8 * i + 4] * f, O[d][8 * i + 5] * f), y1 = pack2(O[d][8 * i + 6] * f, O[d][8 * i + 7] * f);
                swap_halves32(x0, y0);
                swap_halves32(x1, y1);
                *reinterpret_cast<u32x4*>(to + 32 * d + 16 * i) = u32x4{x0, x1, y0, y1};
            }
        if (a.lse && half == 0) a.lse[row_out] = (row.ref + __builtin_amdgcn_logf(l)) * PA_LN2;
    } else {
        const size_t at = (size_t)unit * PA_ROWS + r;
        float* to = a.part_acc + at * HC_D + 4 * half;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(to + 32 * d + 8 * i) = f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
        if (half == 0) *reinterpret_cast<f32x2*>(a.part_ml + at * 2) = f32x2{row.lim == -INFINITY ? -INFINITY : row.ref, l};
    }
}

// The pieces of a row's keys together: a wave per row of (token, query head), two dimensions a lane.
template <int G>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a)
{
    const int lane = threadIdx.x & 63;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int token = row / (a.Hkv * G), x = row - token * (a.Hkv * G), h = x / G, g = x - h * G;
    if (token >= a.tokens) return;
    const int si = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.n_seq && token >= a.seq[lane].tok0 && token < a.seq[lane].tok0 + a.seq[lane].count));
    const PromptSeq sq = a.seq[si];
    if (sq.splits == 1) return;
    const int r = (token - sq.tok0) * G + g, tile = r / PA_ROWS;
    const int last_tok = min((tile * PA_ROWS + PA_ROWS - 1) / G, sq.count - 1);
    const int pieces = (sq.first + last_tok + a.chunk) / a.chunk;          // those that have a key of the tile
    const int unit0 = (si > 0 ? a.seq[si - 1].unit_end : 0) + (sq.tiles - 1 - tile) * sq.splits * a.Hkv + h;
    const size_t step = (size_t)a.Hkv * PA_ROWS, at = (size_t)unit0 * PA_ROWS + r % PA_ROWS;
    float M = -INFINITY;
    for (int s = lane; s < pieces; s += 64) M = fmaxf(M, a.part_ml[(at + s * step) * 2]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    const float ref = M == -INFINITY ? 0.f : M;
    float l = 0.f;
    f32x2 o{0.f, 0.f};
    for (int s = 0; s < pieces; ++s) {
        const size_t p = at + s * step;
        const f32x2 ml = *reinterpret_cast<const f32x2*>(a.part_ml + p * 2);
        const f32x2 v = *reinterpret_cast<const f32x2*>(a.part_acc + p * HC_D + 2 * lane);
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(v.x, f, o.x);
        o.y = fmaf(v.y, f, o.y);
    }
    const float f = 1.0f / l;
    reinterpret_cast<uint32_t*>(a.out + (size_t)row * HC_D)[lane] = pack2(o.x * f, o.y * f);
    if (a.lse && lane == 0) a.lse[row] = (ref + __builtin_amdgcn_logf(l)) * PA_LN2;
}

template <int G>
void launch(const PromptArgs& a, int units, bool join, hipStream_t st)
{
    prompt_attn_kernel<G><<<dim3(units), dim3(PA_BLK), 0, st>>>(a);
    if (join) prompt_join_kernel<G><<<dim3((a.tokens * a.Hkv * G + 3) / 4), dim3(256), 0, st>>>(a);
}

}   // namespace

// Partial results of the keys' pieces: at most two tiles for every workgroup that the GPU holds at a time.
size_t hc_prompt_work_bytes(const hc_ctx* ctx) { return (size_t)2 * PA_PER_CU * ctx->n_cu * PA_ROWS * (HC_D + 2) * sizeof(float); }

hc_status hc_launch_prefill_attn(hc_ctx* ctx, const void* q, const void* kv, const int64_t* k_off, const int64_t* v_off, const int32_t* first,
                                 const int32_t* count, void* out, float* lse, void* work, hipStream_t st)
{
    const hc_config& c = ctx->cfg;
    const int G = ctx->G, slots = PA_PER_CU * ctx->n_cu;
    const int most = std::min(HC_PROMPT_SEQS, HC_PROMPT_HEADS / c.Hkv);
    long long tok_done = 0;
    for (int b0 = 0; b0 < c.B; b0 += most) {
        const int nb = std::min(most, c.B - b0);
        PromptArgs a{};
        int order[HC_PROMPT_SEQS], tok0[HC_PROMPT_SEQS], n = 0;
        long long tokens = 0, tiles = 0, keys = 0;
        for (int i = 0; i < nb; ++i) {
            const int b = b0 + i;
            tok0[i] = (int)tokens;
            tokens += count[b];
            if (count[b] == 0) continue;
            order[n++] = i;
            const long long t = ((long long)count[b] * G + PA_ROWS - 1) / PA_ROWS * c.Hkv;
            tiles += t;
            keys += t * (first[b] + count[b]);
        }
        if (n == 0) continue;
        std::stable_sort(order, order + n, [&](int x, int y) { return first[b0 + x] + count[b0 + x] > first[b0 + y] + count[b0 + y]; });
        // fewer tiles than the GPU holds: the keys are cut into pieces, about as many in all as it holds
        long long chunk = 1 << 30;
        if (tiles < slots) chunk = std::max<long long>(256, (keys + slots - 1) / slots);
        a.chunk = (int)((chunk + PA_KEYS - 1) / PA_KEYS * PA_KEYS);
        long long units = 0;
        bool join = false;
        for (int i = 0; i < n; ++i) {
            const int b = b0 + order[i];
            PromptSeq& s = a.seq[i];
            s.first = first[b];
            s.count = count[b];
            s.tok0 = tok0[order[i]];
            s.tiles = (int)(((long long)count[b] * G + PA_ROWS - 1) / PA_ROWS);
            s.splits = (int)(((long long)first[b] + count[b] + a.chunk - 1) / a.chunk);
            join |= s.splits > 1;
            units += (long long)s.tiles * s.splits * c.Hkv;
            s.unit_end = (int)units;
            for (int h = 0; h < c.Hkv; ++h) {
                a.k_off[i * c.Hkv + h] = k_off[b * c.Hkv + h];
                a.v_off[i * c.Hkv + h] = v_off[b * c.Hkv + h];
            }
        }
        a.q = (const uint16_t*)q + (size_t)tok_done * c.Hq * HC_D;
        a.out = (uint16_t*)out + (size_t)tok_done * c.Hq * HC_D;
        a.lse = lse ? lse + (size_t)tok_done * c.Hq : nullptr;
        a.kv = (const uint16_t*)kv;
        a.Hkv = c.Hkv;
        a.n_seq = n;
        a.tokens = (int)tokens;
        a.part_acc = (float*)work;
        a.part_ml = (float*)work + (size_t)2 * slots * PA_ROWS * HC_D;
        switch (G) {
        case 1: launch<1>(a, (int)units, join, st); break;
        case 2: launch<2>(a, (int)units, join, st); break;
        case 4: launch<4>(a, (int)units, join, st); break;
        default: launch<8>(a, (int)units, join, st); break;
        }
        HC_HIP(ctx, hipGetLastError());
        tok_done += tokens;
    }
    return HC_OK;
}
