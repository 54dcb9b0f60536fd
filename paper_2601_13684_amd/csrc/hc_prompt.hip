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
// under the present one's arithmetic.  A row is 16 chunks of 16 bytes; chunk c of row r lies at c ^ swz(r), which spreads both the
// reads of K (16 rows, one chunk) and the transposed reads of V (4 rows, 4 chunks) over all banks.
#include <algorithm>
#include <numeric>

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
__device__ __forceinline__ int swz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }

// Every wave's loads to LDS have arrived, and every wave is through with the tile before.  (The barrier alone does not wait for them.)
__device__ __forceinline__ void tile_ready()
{
    __builtin_amdgcn_s_waitcnt(0x0f70);           // vmcnt(0)
    __syncthreads();
}

// NW waves of QT times 32 rows.
template <int G, int NW, int QT>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attn_kernel(PromptArgs a)
{
    constexpr int ROWS = NW * 32 * QT;
    __shared__ __attribute__((aligned(1024))) char sm[4 * PA_TILE];        // K, K, V, V
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
    const int m0 = tile * ROWS;
    const int last_tok = min((m0 + ROWS - 1) / G, sq.count - 1);
    const int key_end = min(sq.first + last_tok + 1, (split + 1) * a.chunk);      // one behind the last key of this unit
    const int key_begin = split * a.chunk;
    if (key_begin >= key_end) return;

    // this wave's rows and how far each sees
    const int w0 = m0 + w * 32 * QT;
    const int wtok0 = w0 / G, wtok1 = min((w0 + 32 * QT - 1) / G, sq.count - 1);
    const bool idle = wtok0 >= sq.count;
    const int wave_end = sq.first + wtok1 + 1;
    int limit[QT];
    bf16x8 Q[QT][8];
    size_t qrow[QT];                 // row of q, out and lse
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = w0 + 32 * t + n, tok = min(r / G, sq.count - 1);
        limit[t] = sq.first + tok;
        qrow[t] = ((size_t)(sq.tok0 + tok) * a.Hkv + h) * G + r % G;
        const uint16_t* src = a.q + qrow[t] * HC_D + hh * 8;
#pragma unroll
        for (int d = 0; d < 8; ++d) Q[t][d] = *reinterpret_cast<const bf16x8*>(src + 16 * d);
    }
    const int head = si * a.Hkv + h;
    const char* kb = (const char*)(a.kv + a.k_off[head]);
    const char* vb = (const char*)(a.kv + a.v_off[head]);

    // loads: instruction i of a wave takes rows 4 (NW i + w) .. + 3 of the tile, a lane 16 bytes of one of them
    constexpr int LOADS = PA_KEYS / 4 / NW;
    const int ld_row = 4 * w + (lane >> 4), ld_chunk = ((lane & 15) ^ swz(ld_row)) * 16;
    lds_char* const base = (lds_char*)sm;
    auto load = [&](int key, int buf) {
        const int rows = key_end - key;                              // rows past the last key repeat it; they are masked
        const auto rk = __builtin_amdgcn_make_buffer_rsrc((void*)(kb + (size_t)key * (HC_D * 2)), 0, PA_TILE, 0x00027000);
        const auto rv = __builtin_amdgcn_make_buffer_rsrc((void*)(vb + (size_t)key * (HC_D * 2)), 0, PA_TILE, 0x00027000);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int off = min(ld_row + 4 * NW * i, rows - 1) * (HC_D * 2) + ld_chunk;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (__attribute__((address_space(3))) void*)(base + buf * PA_TILE + (NW * i + w) * 1024), 16, off, 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (__attribute__((address_space(3))) void*)(base + (2 + buf) * PA_TILE + (NW * i + w) * 1024), 16, off, 0, 0, 0);
        }
    };
    // operand reads
    const int k_row = n * 256, k_x = (hh ^ swz(n)) * 16;
    const int n16 = lane & 15, g2 = (lane >> 4) & 1;
    int v_at[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
        v_at[p] = (8 * p + 4 * hh + (n16 >> 2)) * 256 + (((2 * g2 + ((n16 & 3) >> 1)) ^ (2 * p + hh)) * 16) + (n16 & 1) * 8;
    const int v_x = (n16 >> 2) * 64;

    f32x16 O[QT][4];
    float m[QT], l[QT];
    for (int safe = 0;; ++safe) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            m[t] = -INFINITY;
            l[t] = 0.f;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[t][d][i] = 0.f;
        }
        load(key_begin, 0);
        tile_ready();
        int buf = 0;
        for (int key = key_begin; key < key_end; key += PA_KEYS, buf ^= 1) {
            if (key + PA_KEYS < key_end) load(key + PA_KEYS, buf ^ 1);
            const bool masked = key + PA_KEYS > sq.first + m0 / G + 1 || key + PA_KEYS > key_end;      // for some row of the workgroup
            unsigned long long bad = 0;
            if (safe && masked) {
                // some result was not finite: what a masked weight of zero makes of an infinity or a NaN in V must not count.  Such values
                // leave the tile, and are added by hand to the rows that see them.
                if (tid == 0) sm_bad = 0;
                __syncthreads();
                for (int i = tid; i < PA_TILE / 16; i += NW * 64) {
                    u32x4* p = reinterpret_cast<u32x4*>(sm + (2 + buf) * PA_TILE + i * 16);
                    u32x4 x = *p;
                    bool hit = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((x[e] & 0x7f80u) == 0x7f80u) { x[e] &= 0xffff0000u; hit = true; }
                        if ((x[e] & 0x7f800000u) == 0x7f800000u) { x[e] &= 0x0000ffffu; hit = true; }
                    }
                    if (hit) {
                        *p = x;
                        atomicOr(&sm_bad, 1ull << (i / 16));
                    }
                }
                __syncthreads();
                bad = sm_bad;
            }
            if (!idle && key < wave_end) {
                const lds_char* kt = base + buf * PA_TILE + k_row;
                const lds_char* vt = base + (2 + buf) * PA_TILE;
                f32x16 S[QT][2];
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 16; ++i) S[t][k][i] = 0.f;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int d = 0; d < 8; ++d) {
                        const bf16x8 f = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(kt + k * 8192 + (k_x ^ (d * 32)));
#pragma unroll
                        for (int t = 0; t < QT; ++t) S[t][k] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, Q[t][d], S[t][k], 0, 0, 0);
                    }
                bf16x8 P[QT][4];
                const bool cut = key + PA_KEYS > sq.first + wtok0 + 1 || key + PA_KEYS > key_end;
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    if (cut) {
                        const int see = min(limit[t], key_end - 1) - key - 4 * hh;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (32 * k + 8 * (i / 4) + i % 4 > see) S[t][k][i] = -INFINITY;
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = fmaxf(top, S[t][k][i]);
                    top = fmaxf(top, other_half(top)) * PA_SCALE;
                    if (__builtin_amdgcn_ballot_w64(top > m[t] + PA_SLACK)) {
                        const float mn = fmaxf(m[t], top);
                        const float f = mn == m[t] ? 1.0f : __builtin_amdgcn_exp2f(m[t] - mn);
                        m[t] = mn;
                        l[t] *= f;
#pragma unroll
                        for (int d = 0; d < 4; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) O[t][d][i] *= f;
                    }
                    const float ref = m[t] == -INFINITY ? 0.f : m[t];
                    float sum = 0.f;
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            S[t][k][i] = __builtin_amdgcn_exp2f(fmaf(S[t][k][i], PA_SCALE, -ref));
                            sum += S[t][k][i];
                        }
                    l[t] += sum;
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        u32x4 x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = pack2(S[t][s / 2][8 * (s % 2) + 2 * e], S[t][s / 2][8 * (s % 2) + 2 * e + 1]);
                        P[t][s] = __builtin_bit_cast(bf16x8, x);
                    }
                }
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        typedef __attribute__((address_space(3))) s16x4* lds4;
                        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vt + v_at[0] + s * 4096 + (v_x ^ (d * 64))));
                        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(vt + v_at[1] + s * 4096 + (v_x ^ (d * 64))));
                        const bf16x8 f = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                        for (int t = 0; t < QT; ++t) O[t][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, P[t][s], O[t][d], 0, 0, 0);
                    }
                while (bad) {
                    const int j = __builtin_ctzll(bad);
                    bad &= bad - 1;
                    const int at = min(key + j, key_end - 1);
                    const uint16_t* row = (const uint16_t*)(vb + (size_t)at * (HC_D * 2)) + 4 * hh;
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        const bool sees = key + j == at && at <= limit[t];
#pragma unroll
                        for (int d = 0; d < 4; ++d)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint32_t x = row[32 * d + 8 * (i / 4) + i % 4];
                                if (sees && (x & 0x7f80u) == 0x7f80u) O[t][d][i] += __uint_as_float(x << 16);
                            }
                    }
                }
            }
            tile_ready();
        }
        float z = 0.f;
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) z = fmaf(O[t][d][i], 0.f, z);
        if (safe || !__syncthreads_or(z != 0.f)) break;
    }

#pragma unroll
    for (int t = 0; t < QT; ++t) {
        l[t] += other_half(l[t]);
        if (w0 + 32 * t + n >= sq.count * G) continue;
        if (sq.splits == 1) {
            const float f = 1.0f / l[t];
            uint16_t* to = a.out + qrow[t] * HC_D + 8 * hh;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 2; ++i) {            // 16 dimensions: after the exchange a lane holds eight in a row
                    uint32_t x0 = pack2(O[t][d][8 * i] * f, O[t][d][8 * i + 1] * f), x1 = pack2(O[t][d][8 * i + 2] * f, O[t][d][8 * i + 3] * f);
                    uint32_t y0 = pack2(O[t][d][8 * i + 4] * f, O[t][d][8 * i + 5] * f), y1 = pack2(O[t][d][8 * i + 6] * f, O[t][d][8 * i + 7] * f);
                    swap_halves32(x0, y0);
                    swap_halves32(x1, y1);
                    *reinterpret_cast<u32x4*>(to + 32 * d + 16 * i) = u32x4{x0, x1, y0, y1};
                }
            if (a.lse && hh == 0) a.lse[qrow[t]] = (m[t] + __builtin_amdgcn_logf(l[t])) * PA_LN2;
        } else {
            const size_t row = (size_t)unit * ROWS + w * 32 * QT + 32 * t + n;
            float* to = a.part_acc + row * HC_D + 4 * hh;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(to + 32 * d + 8 * i) = f32x4{O[t][d][4 * i], O[t][d][4 * i + 1], O[t][d][4 * i + 2], O[t][d][4 * i + 3]};
            if (hh == 0) *reinterpret_cast<f32x2*>(a.part_ml + row * 2) = f32x2{m[t], l[t]};
        }
    }
}

// The pieces of a row's keys together: a wave per row of (token, query head), two dimensions a lane.
template <int G>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptArgs a, int rows)
{
    const int lane = threadIdx.x & 63;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int token = row / (a.Hkv * G), x = row - token * (a.Hkv * G), h = x / G, g = x - h * G;
    if (token >= a.tokens) return;
    const int si = __builtin_ctzll(__builtin_amdgcn_ballot_w64(lane < a.n_seq && token >= a.seq[lane].tok0 && token < a.seq[lane].tok0 + a.seq[lane].count));
    const PromptSeq sq = a.seq[si];
    if (sq.splits == 1) return;
    const int r = (token - sq.tok0) * G + g, tile = r / rows;
    const int last_tok = min((tile * rows + rows - 1) / G, sq.count - 1);
    const int pieces = (sq.first + last_tok + a.chunk) / a.chunk;          // those that have a key of the tile
    const int unit0 = (si > 0 ? a.seq[si - 1].unit_end : 0) + (sq.tiles - 1 - tile) * sq.splits * a.Hkv + h;
    const size_t step = (size_t)a.Hkv * rows, at = (size_t)unit0 * rows + r % rows;
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

constexpr int PA_WAVES = 4, PA_QT = 1, PA_ROWS = PA_WAVES * 32 * PA_QT, PA_PER_CU = 2;

template <int G>
void launch(const PromptArgs& a, int units, bool join, hipStream_t st)
{
    prompt_attn_kernel<G, PA_WAVES, PA_QT><<<dim3(units), dim3(PA_WAVES * 64), 0, st>>>(a);
    if (join) prompt_join_kernel<G><<<dim3((a.tokens * a.Hkv * G + 3) / 4), dim3(256), 0, st>>>(a, PA_ROWS);
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
