// hc_prompt.hip -- attention of a prompt's tokens, or of a chunk of them, over the prompt's K and V: causal, packed sequences, query
// heads in groups of G to a KV head.  For the token at position p of a sequence and query head a of KV head h
//     s_j = q . K_h[j] / sqrt(128),  j = 0 .. p;   out = sum_j exp(s_j - lse) V_h[j],   lse = log sum_j exp(s_j)
//
// Work is cut into tiles of PA_ROWS query rows of one KV head, the group's G heads of a token side by side: a tile spans PA_ROWS / G
// tokens, the group shares its K and V, and the diagonal is met in fine steps.  A wave holds 32 rows.  It forms the transposed product
// S^T = K Q^T on the matrix cores (v_mfma_f32_32x32x16_bf16), keys along the registers and a query to each lane, so that a row's
// maximum and sum stay inside a lane but for one exchange between the halves of the wave; and the registers that hold P^T are, rounded
// to bf16, the second product's operand as they are: O^T = V^T P^T may take the keys of a step in any order as long as both operands
// do, and V is read from LDS transposed (ds_read_b64_tr_b16) in the order that S^T leaves.  One pass over the keys.
// A row's weights are 2^(t - ref), t the scaled logit, ref the largest of its first 32 keys rounded up to a whole number: weights,
// sums and bf16 are floating point, so that ref need not be the row's maximum to the end, only within a hundred binary orders of it.
// A workgroup that finds a row outside of that, a sum that is not finite or logits beyond 2^29, starts again with a running maximum (and in a form that
// keeps masked infinities and NaNs of V out): what that costs, 2.1 to 2.3 times a call's time where every workgroup does, is paid by
// inputs that need it; all others save the running maximum's 2 %.
//
// Bound: the matrix cores at the clock that their power leaves.  32,003 tokens (eight KV heads, groups of four) take 7.1 ms, 1.18
// PFLOP/s, 86 % of what a bf16 product of 16384^3 reaches on the same card (1.37; from card to card 6.9 to 7.4 ms); in the loop the
// clock falls from 2.4 to 1.7 GHz, and changes of the schedule that leave the matrix cores idle less let it fall further.  8,192 tokens
// 494 us, 1.11 PFLOP/s (476 to 502).  Few rows behind many keys are bound by memory: 17 tokens behind four contexts of 20K to 90K 166
// us, 5.5 TB/s.  Prompts of a few hundred to about 6,000 tokens are two to eight times above either bound: the loads before the first product, units
// too few or of unequal length, and a second launch where keys are cut (200 tokens 8 us, 1,024 18.5).
//
// P is rounded to bf16 for the matrix cores, to the nearest: the error of an output is that of at most 2^-8 per weight, independent
// from key to key, about what the output's own rounding to bf16 adds.  Sum, maximum, lse and accumulators are 32-bit, the sum
// from the unrounded weights.
//
// K and V tiles of 64 keys go straight to LDS (buffer loads of 16 bytes a lane), two buffers, the next tile's loads in flight
// under the present one's arithmetic.  A tile lies in blocks of 16 rows by 4 chunks of 16 bytes (a load instruction's kilobyte), chunk c of
// row r at place c ^ (r / 4 mod 4) of its 64 bytes: the reads of K (16 rows, one chunk) and the transposed reads of V (4 rows, 4 chunks) then
// both go over all banks once, and all of a wave's reads of a tile are two addresses a lane and an offset that the instruction holds.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "hc_internal.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int PA_BLK = 256;                       // four waves, 32 query rows to each
constexpr int PA_PER_CU = 2;                      // workgroups that a compute unit holds
constexpr int PA_DIES = 8;                        // with an L2 each; workgroups go to them in turn
constexpr int PA_ROOM = 4;                        // tiles of 128 rows of partial results to each of these workgroups
constexpr int PA_KEYS = 64;                       // keys of a tile in LDS
constexpr int PA_TILE = PA_KEYS * HC_D * 2;       // its bytes
constexpr float PA_SCALE = 1.4426950408889634f * 0.08838834764831845f;     // log2(e) / sqrt(128)
constexpr float PA_LN2 = 0.6931471805599453f;
constexpr float PA_SLACK = 8.0f;                  // log2 units: where there is a running maximum, a weight is at most 2^8 before the reference moves
// Where there is none: what a row's sum of weights lies between (below 2^-60 weights that are lost as denormals might count: 2^24 of
// 2^-126), and what the magnitudes of a lane's 64 sums add up to (the join adds up to 2^11 of them, of at most 2^24 weights).
constexpr float PA_LEAST = 0x1p-60f, PA_MOST = 0x1p100f, PA_LARGEST = 0x1p112f;

// A weight's fused product and difference has only the difference's rounding, but its reference comes from a rounded product, and may lie up to half a step
// of that from the product that it was made from.  As far as here that is 16 binary orders, and a row's largest weight 2^16 at most before slack; from 2^31 on
// it is more than the exponents hold.  Beyond (only in the second try) references are logits as they leave the first product, not scaled: their steps are at least
// 32 binary orders, so that logits are equal or nothing to each other.  A logit is larger than its scaled value, so that references of both kinds have one order, and
// whenever two of them differ and one is of the second kind, by more than the exponents hold: f = exp2(difference) serves both.
constexpr float PA_FAR = 0x1p29f;

constexpr int PA_SEQS = HC_PROMPT_SEQS, PA_HEADS = HC_PROMPT_HEADS;
struct PromptSeq {
    int unit_end;          // of the launch's work units, sequence by sequence
    int first, count;      // positions before the chunk, tokens of the chunk
    int tok0;              // its first token among the packed ones
    int tiles;             // tiles of query rows of a KV head
    int tile_end;          // tiles of all heads up to here
    uint32_t cut;          // pieces of the keys (low bits), tiles of 64 keys of a piece
    __host__ __device__ int splits() const { return cut & 0xfff; }
    __host__ __device__ int chunk() const { return (cut >> 12) * 64; }
};
struct PromptArgs {
    const uint16_t *q, *kv;
    uint16_t* out;
    float *lse, *part_acc, *part_ml;
    int Hkv, n_seq;
    // pieces whose tiles alternate, so that one piece of one head stays with one of the dies (52 tokens behind 115,286, one KV head of eight
    // query heads: 42 us; with the seven tiles of every piece on seven dies 70)
    int together;
    int n_cu, mirror;                             // compute units; units of the second round, which is dealt out backwards (0: it is not)
    // what is to be done, and where K and V are: here, or, of more sequences and heads than there is room for here, in the work buffer
    const PromptSeq* table;
    const int64_t* table_off;                     // K's, then V's, table_rows of each
    int table_rows;
    PromptSeq seq[PA_SEQS];
    int64_t k_off[PA_HEADS], v_off[PA_HEADS];
};
static_assert(sizeof(PromptArgs) <= 4096, "what a launch's arguments have room for");
// (what comes from the table is the same for all lanes; told so, the compiler keeps it, and what follows from it, in scalar registers)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}
__device__ __forceinline__ PromptSeq seq_of(const PromptArgs& a, int i)
{
    if (!a.table) return a.seq[i];
    const PromptSeq s = a.table[i];
    return PromptSeq{uniform(s.unit_end), uniform(s.first), uniform(s.count), uniform(s.tok0), uniform(s.tiles), uniform(s.tile_end), (uint32_t)uniform((int)s.cut)};
}
// First sequence whose `end` is past x, 64 of them looked at at a time.
template <class End>
__device__ __forceinline__ int find_seq(const PromptArgs& a, int x, int lane, End end)
{
    if (a.n_seq == 1) return 0;
    int lo = 0, n = a.n_seq;
    for (;;) {
        const int step = (n + 63) / 64, last = min((lane + 1) * step, n) - 1;
        const int skip = __popcll(__builtin_amdgcn_ballot_w64(lane * step < n && end(lo + last) <= x));
        lo += skip * step;
        if (step == 1) return lo;
        n = min(step, n - skip * step);
    }
}
// Entries of the table from a launch's arguments (seq and the offsets hold up to PA_SEQS and PA_HEADS of them).
__global__ __launch_bounds__(PA_HEADS) void prompt_table_kernel(PromptArgs a, PromptSeq* seq, int n_seq, int64_t* off, int n_off)
{
    const int i = threadIdx.x;
    if (i < n_seq) seq[i] = a.seq[i];
    if (i < n_off) {
        off[i] = a.k_off[i];
        off[a.table_rows + i] = a.v_off[i];
    }
}

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

// What a row's weights are taken against, of its largest logit.
__device__ __forceinline__ float reference(float s)
{
    const float t = s * PA_SCALE;
    return fabsf(t) < PA_FAR ? ceilf(t) : s;
}
__device__ __forceinline__ float lse_of(float ref, float l)
{
    return ((fabsf(ref) < PA_FAR ? ref : ref * PA_SCALE) + __builtin_amdgcn_logf(l)) * PA_LN2;
}

// Every wave's loads to LDS have arrived, and every wave is through with the tile before.  (The barrier alone does not wait for them.)
// `later`: loads issued after these, which are not waited for.
template <int later = 0>
__device__ __forceinline__ void tile_ready()
{
    static_assert(later < 16, "the low bits of vmcnt");
    __builtin_amdgcn_s_waitcnt(0x0f70 | later);   // vmcnt(later)
    __syncthreads();
}

// How the instructions of eight products are to follow each other: behind each of them operand reads for later ones and a share of the
// weights' arithmetic.
template <int products, int reads, int valu, int exps>
__device__ __forceinline__ void interleave()
{
    constexpr int PRODUCT = 0x8, READ = 0x100, VALU = 0x2, TRANS = 0x400;
#pragma unroll
    for (int i = 0; i < products; ++i) {
        if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(READ, reads, 0);
        __builtin_amdgcn_sched_group_barrier(PRODUCT, 1, 0);
        if constexpr (valu > 0) __builtin_amdgcn_sched_group_barrier(VALU, valu, 0);
        if constexpr (exps > 0) __builtin_amdgcn_sched_group_barrier(TRANS, exps, 0);
    }
}

// The reference and the sum of a lane's row.  ref is a whole number; lim = ref + PA_SLACK where there is a running maximum, -inf while
// the row has seen nothing.
struct RowState {
    float ref, lim, l;
};

// A unit is the work of a workgroup.  The first n_cu workgroups go to a compute unit each, the next n_cu beside them: these are dealt
// out backwards, the lightest beside the heaviest (head by head, so that a head stays with its die): 2,048 tokens of eight heads 42.9
// us against 44.7, 4,096 132.5 against 136, 8,192 no difference.
__device__ __forceinline__ int mirrored(int block, int n_cu, int second, int Hkv)
{
    const int r = block - n_cu;
    return r >= second ? block : n_cu + (second / Hkv - 1 - r / Hkv) * Hkv + r % Hkv;
}

// KS = 1: a tile has 128 rows, a wave takes all keys of its 32.  KS = 2: a tile has 64 rows, two waves share 32 of them, one half of
// every 64 keys to each, and what they have comes together in LDS at the end: twice the workgroups of half the length, for twice the
// traffic into LDS.  Eight KV heads, groups of four, KS = 1 against 2: 512 tokens 13.4 us against 11.4, 1,024 22.3 against 18.6, 2,048
// 42.9 against 47.5, 8,192 490 against 565.
template <int KS>
constexpr int pa_rows = 128 / KS;
template <int G, int KS>
__global__ __launch_bounds__(PA_BLK, 2) void prompt_attn_kernel(PromptArgs a)
{
    constexpr int PA_ROWS = pa_rows<KS>;
    // (arrays of their own, so that the compiler sees that a buffer's loads in flight are not what the reads of the other wait for)
    __shared__ __attribute__((aligned(1024))) char sm_k0[PA_TILE], sm_k1[PA_TILE], sm_v0[PA_TILE], sm_v1[PA_TILE];
    __shared__ unsigned long long sm_bad;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int n = lane & 31, hh = lane >> 5;

    // which piece of the keys, which tile, which head: the longest sequence first, its whole pieces and then the last ones of its
    // tiles, heads fastest, so that the workgroups that stream the same K and V do so at the same time on the same die
    const int unit = a.mirror > 0 && (int)blockIdx.x >= a.n_cu ? mirrored(blockIdx.x, a.n_cu, a.mirror, a.Hkv) : blockIdx.x;
    const int si = find_seq(a, unit, lane, [&](int i) { return a.table ? a.table[i].unit_end : a.seq[i].unit_end; });
    const PromptSeq sq = seq_of(a, si);
    const int unit0 = sq.unit_end - sq.tiles * sq.splits() * a.Hkv;
    int u = (unit - unit0) / a.Hkv;
    const int h = unit - unit0 - u * a.Hkv;
    int split = 0;
    bool whole = false;
    if (sq.splits() > 1) {
        const int left = u - (sq.splits() - 1) * sq.tiles;
        whole = left < 0;
        if (whole) {
            // `together` pieces at a time, their tiles in turn; one, where the tiles have different numbers of pieces
            // (dies would get more than others)
            const int some = sq.tiles * PA_ROWS <= sq.chunk() * G ? a.together : 1, at = u / (sq.tiles * some) * some, n_at = min(some, sq.splits() - 1 - at);
            u -= at * sq.tiles;
            split = at + u % n_at;
            u /= n_at;
        } else {
            u = left;
        }
    }
    const int tile = sq.tiles - 1 - u;
    const int m0 = tile * PA_ROWS;
    const int last_tok = min((m0 + PA_ROWS - 1) / G, sq.count - 1);
    if (sq.splits() > 1) {
        const int ends_in = (sq.first + last_tok) / sq.chunk();
        if (whole && split >= ends_in) return;
        if (!whole) split = ends_in;
    }
    const int place = unit0 + (split * sq.tiles + sq.tiles - 1 - tile) * a.Hkv + h;         // of partial results
    const int key_begin = split * sq.chunk();
    const int key_end = min(sq.first + last_tok + 1, key_begin + sq.chunk());     // one behind the last key of this unit
    const int n_tiles = (key_end - key_begin + PA_KEYS - 1) / PA_KEYS;
    const int n_full = max(0, min(key_end, sq.first + m0 / G + 1) - key_begin) / PA_KEYS;      // tiles that every row sees whole

    // this wave's rows and how far each sees; its half of the keys
    const int wr = w % (4 / KS), wk = w / (4 / KS);
    const int w0 = m0 + wr * 32;
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
    const int64_t k_off = a.table ? uniform(a.table_off[head]) : a.k_off[head], v_off = a.table ? uniform(a.table_off[a.table_rows + head]) : a.v_off[head];
    const char* kb = (const char*)(a.kv + k_off) + (size_t)key_begin * (HC_D * 2);
    const char* vb = (const char*)(a.kv + v_off) + (size_t)key_begin * (HC_D * 2);

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
        k_at[p] = wk * 8192 + n / 16 * 4096 + n16 * 64 + (((2 * p + hh) ^ (n16 >> 2)) * 16);
        v_at[p] = wk * 8192 + (8 * p + 4 * hh + (n16 >> 2)) * 64 + (((2 * (n / 16) + ((n16 & 3) >> 1)) ^ (2 * p + hh)) * 16) + (n16 & 1) * 8;
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
        return fmaxf(top, other_half(top));
    };
    // keys 8 s .. 8 s + 7 of a lane's 16
    auto weigh = [&](f32x16& S, bf16x8 (&P)[2], int s, auto careful) {
        u32x4 x;
#pragma unroll
        for (int i = 8 * s; i < 8 * s + 8; ++i) {
            float t = fmaf(S[i], PA_SCALE, -row.ref);
            if constexpr (careful()) t = fabsf(row.ref) < PA_FAR ? t : S[i] - row.ref;
            S[i] = __builtin_amdgcn_exp2f(t);
        }
        float sum[2] = {S[8 * s], S[8 * s + 1]};
#pragma unroll
        for (int i = 8 * s + 2; i < 8 * s + 8; ++i) sum[i & 1] += S[i];
        row.l += sum[0] + sum[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = pack2(S[8 * s + 2 * e], S[8 * s + 2 * e + 1]);
        P[s] = __builtin_bit_cast(bf16x8, x);
    };
    auto weights = [&](f32x16& S, bf16x8 (&P)[2], auto careful) {
        weigh(S, P, 0, careful);
        weigh(S, P, 1, careful);
    };
    // (Nothing but minus infinities: there is nothing to take weights against.  No weight is then larger than zero, and where the row sees other keys that
    // sum sends it to the second try: with a reference made up here, what these keys' sum comes to might lie too far from it for the sums of other parts.)
    auto start = [&](float top) { row.ref = top == -INFINITY ? INFINITY : ceilf(top * PA_SCALE); };
    // The running maximum of the second try, before weights are taken of logits up to `top`.
    auto settle = [&](float top) {
        const float next = reference(top);
        if (!__builtin_amdgcn_ballot_w64(next > row.lim)) return;
        const float ref = row.lim == -INFINITY ? next : fmaxf(row.ref, next);
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
    };

    auto clear = [&] {
        row = RowState{0.f, -INFINITY, 0.f};
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[d][i] = 0.f;
    };
    // The logits of half a tile, -inf where a row does not see the key, and what follows from them; careful: with the running maximum;
    // otherwise `first` says whether these are the unit's first keys.
    auto masked = [&](const char* tile_k, const char* tile_v, int key, int k, bool first, auto careful) {
        f32x16 S;
        bf16x8 P[2]{}, F[8];
        read_k(tile_k, k, F);
        logits(F, S);
        read_v(tile_v, k, F);
        const int see = min(limit, key_end - 1) - key - 32 * (k + wk) - 4 * hh;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (8 * (i / 4) + i % 4 > see) S[i] = -INFINITY;
        if constexpr (careful()) settle(largest(S));
        else if (first) start(largest(S));
        weights(S, P, careful);
        values(F, P);
    };
    {
        clear();
        using B0 = std::integral_constant<int, 0>;
        using B1 = std::integral_constant<int, 1>;
        load_k(0, B0{});
        load_v(0, B0{});
        int k_next = 1, v_next = 1;                  // first tiles of K and V whose loads are not under way
        if (n_full > 0) {
            // Tiles that every row sees whole, in steps of 32 keys, three of them at a time: the logits of step i + 1 and the sums of step
            // i - 1 on the matrix cores, between them the weights of step i, which wait for neither.  Operands are read from LDS one
            // product ahead (eight reads' worth of registers for K, as many for V): a read takes longer than the few products that
            // could be put between it and its use.  K runs a tile ahead of V.  The one barrier of a tile stands where the wave has read
            // all that it will read of both buffers, before their last product, which then covers the first reads of the next tile.
            f32x16 S0, S1;
            bf16x8 P0[2]{}, P1[2], K[8], V[8];
            if (n_tiles > 1) load_k(1, B1{});
            if constexpr (KS == 1) {
                if (n_tiles > 1) tile_ready<8>();
                else tile_ready<4>();
                read_k(sm_k0, 0, K);
                logits(K, S0);
                read_k(sm_k0, 1, K);
                start(largest(S0));
                logits(K, S1);
                weights(S0, P0, std::false_type{});
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
                    weights(S1, P1, std::false_type{});
                    read_k(tile_k, 1, K);
                    values(V, P0);
                    interleave<8, 2, 4, 2>();
                    interleave<8, 1, 4, 0>();
                    __builtin_amdgcn_sched_barrier(0);
                    read_v(tile_v, 1, V);
                    logits(K, S1);
                    weigh(S0, P0, 0, std::false_type{});
                    interleave<8, 2, 3, 1>();
                    tile_ready();
                    if (t + 3 < n_tiles) load(kb, t + 3, tile_k);
                    if (t + 2 < n_tiles) load(vb, t + 2, tile_v);
                    read_k(next_k, 0, K);
                    values(V, P1);
                    weigh(S0, P0, 1, std::false_type{});
                    interleave<8, 1, 3, 1>();
                    __builtin_amdgcn_sched_barrier(0);
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
                weights(S1, P1, std::false_type{});
                values(V, P0);
                read_v(tile_v, 1, V);
                values(V, P1);
                k_next = n_full + 2;
                v_next = n_full + 1;
            } else {
                // the same with a step a tile: logits of tile t + 1, sums of tile t - 1, weights of tile t
                if (n_tiles > 1) {
                    load_v(1, B1{});
                    tile_ready<12>();
                } else {
                    tile_ready<4>();
                }
                read_k(sm_k0, 0, K);
                logits(K, S0);
                start(largest(S0));
                tile_ready();
                if (n_tiles > 2) load_k(2, B0{});
                read_k(sm_k1, 0, K);
                auto body = [&](int t, auto odd, auto begin) {
                    f32x16 &S_now = odd() ? S1 : S0, &S_next = odd() ? S0 : S1;
                    bf16x8(&P_now)[2] = odd() ? P1 : P0;
                    bf16x8(&P_last)[2] = odd() ? P0 : P1;
                    char* const tile_k = odd() ? sm_k1 : sm_k0;          // of K t + 2
                    char* const spent_k = odd() ? sm_k0 : sm_k1;
                    char* const tile_v = odd() ? sm_v0 : sm_v1;          // of V t - 1
                    if (!begin()) read_v(tile_v, 0, V);
                    logits(K, S_next);
                    weigh(S_now, P_now, 0, std::false_type{});
                    interleave<8, 2, 3, 1>();
                    tile_ready();
                    if (t + 3 < n_tiles) load(kb, t + 3, spent_k);
                    if (!begin() && t + 1 < n_tiles) load(vb, t + 1, tile_v);
                    read_k(tile_k, 0, K);
                    if (!begin()) values(V, P_last);
                    weigh(S_now, P_now, 1, std::false_type{});
                    interleave<8, 1, 3, 1>();
                    __builtin_amdgcn_sched_barrier(0);
                };
                int t = 0;
                if (n_full > 1) body(t++, B0{}, std::true_type{});
                for (; t + 2 < n_full; t += 2) {
                    body(t, B1{}, std::false_type{});
                    body(t + 1, B0{}, std::false_type{});
                }
                if (t + 1 < n_full) {
                    body(t, B1{}, std::false_type{});
                    ++t;
                }
                // t == n_full - 1: its logits are there, and the weights of tile t - 1 if there is one
                char *const tile_v = t & 1 ? sm_v1 : sm_v0, *const other_v = t & 1 ? sm_v0 : sm_v1;
                if (t > 0) {
                    read_v(other_v, 0, V);
                    if (t & 1) values(V, P0);
                    else values(V, P1);
                }
                if (t & 1) weights(S1, P1, std::false_type{});
                else weights(S0, P1, std::false_type{});
                tile_ready();
                if (t > 0 && t + 1 < n_tiles) load(vb, t + 1, other_v);
                read_v(tile_v, 0, V);
                values(V, P1);
                k_next = n_full + 2;
                v_next = n_full + 1;
            }
            tile_ready();
        } else if (n_tiles > 1) {
            load_k(1, B1{});
            load_v(1, B1{});
            k_next = v_next = 2;
            tile_ready<8>();
        } else {
            tile_ready();
        }
        // The tiles behind them, in which some row sees only the first keys.
        auto step = [&](int t, auto buf) {
            const int key = key_begin + t * PA_KEYS;
            if (t + 1 < n_tiles) {
                if (t + 1 >= k_next) load_k(t + 1, std::integral_constant<int, 1 - buf()>{});
                if (t + 1 >= v_next) load_v(t + 1, std::integral_constant<int, 1 - buf()>{});
            }
            if (!idle && key < wave_end) {
#pragma unroll
                for (int k = 0; k < 2 / KS; ++k) masked(buf() ? sm_k1 : sm_k0, buf() ? sm_v1 : sm_v0, key, k, t == 0 && k == 0, std::false_type{});
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
            for (int i = 0; i < 16; ++i) z += fabsf(O[d][i]);
        const float sum = row.l + other_half(row.l);
        const bool sees = !idle && limit >= key_begin + 32 * wk;                 // any of its wave's keys
        if (__syncthreads_or(sees && !(z < PA_LARGEST && sum > PA_LEAST && sum < PA_MOST && fabsf(row.ref) < PA_FAR))) {
            // Once more, tile by tile, with a running maximum.  What a masked weight of zero makes of an infinity or a NaN
            // in V must not count: such values leave the tile, and are added by hand to the rows that see them.
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
                    for (int k = 0; k < 2 / KS; ++k) masked(sm_k0, sm_v0, key, k, false, std::true_type{});
                    for (unsigned long long bad = KS == 1 ? sm_bad : sm_bad & (0xffffffffull << (32 * wk)); bad; bad &= bad - 1) {
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
    if constexpr (KS == 2) {
        // the upper half's sums to the wave that has the lower half (the tiles' places are free: a barrier ended the last of them)
        f32x4* const o = reinterpret_cast<f32x4*>(wr ? sm_k1 : sm_k0) + lane;
        RowState* const other = reinterpret_cast<RowState*>(sm_v0) + wr * 64 + lane;
        if (wk) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i * 64] = f32x4{O[i / 4][4 * (i % 4)], O[i / 4][4 * (i % 4) + 1], O[i / 4][4 * (i % 4) + 2], O[i / 4][4 * (i % 4) + 3]};
            *other = RowState{row.ref, row.lim, l};
        }
        __syncthreads();
        if (wk) return;
        const RowState x = *other;
        const bool mine = l != 0.f, has = x.l != 0.f;
        const float ref = mine && has ? fmaxf(row.ref, x.ref) : mine ? row.ref : x.ref;
        const float f = mine ? __builtin_amdgcn_exp2f(row.ref - ref) : 0.f, g = has ? __builtin_amdgcn_exp2f(x.ref - ref) : 0.f;
        l = l * f + x.l * g;
        row.ref = ref;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const f32x4 y = o[i * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) O[i / 4][4 * (i % 4) + e] = O[i / 4][4 * (i % 4) + e] * f + y[e] * g;
        }
    }
    int late = tid;                                  // (opaque: what follows is not worked out before the loops and kept through them)
    asm volatile("" : "+v"(late));
    const int r = wr * 32 + (late & 31), half = (late >> 5) & 1;
    if (m0 + r >= sq.count * G) return;
    if (sq.splits() == 1) {
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
        if (a.lse && half == 0) a.lse[row_out] = lse_of(row.ref, l);
    } else {
        // as the registers lie: 1 KB to a store
        f32x4* to = reinterpret_cast<f32x4*>(a.part_acc) + ((size_t)place * (PA_ROWS / 32) + wr) * 1024 + (late & 63);
#pragma unroll
        for (int i = 0; i < 16; ++i) to[i * 64] = f32x4{O[i / 4][4 * (i % 4)], O[i / 4][4 * (i % 4) + 1], O[i / 4][4 * (i % 4) + 2], O[i / 4][4 * (i % 4) + 3]};
        if (half == 0) *reinterpret_cast<f32x2*>(a.part_ml + ((size_t)place * PA_ROWS + r) * 2) = f32x2{l == 0.f ? -INFINITY : row.ref, l};
    }
}

// The pieces of the keys together, for 32 rows of a tile and 32 of their dimensions: wave v takes pieces v, v + PJ_WAVES, ...,
// PJ_AHEAD of them at a time (what bounds this kernel is how long a read takes, not how much there is to read), a lane what the same
// lane of the attention kernel's wave left: row lane % 32, four times four dimensions.  The waves' sums meet in LDS.
constexpr int PJ_WAVES = 8, PJ_AHEAD = 4;
template <int G, int KS>
__global__ __launch_bounds__(PJ_WAVES * 64) void prompt_join_kernel(PromptArgs a)
{
    constexpr int PA_ROWS = pa_rows<KS>;
    __shared__ f32x4 sm_o[PJ_WAVES][4][64];
    __shared__ f32x2 sm_ml[PJ_WAVES][32];
    const int tid = threadIdx.x, v = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;
    const int dims = blockIdx.x % 4, block = blockIdx.x / 4 % (PA_ROWS / 32);
    int u = blockIdx.x / 4 / (PA_ROWS / 32);                 // tile by tile, as the units but for the pieces
    const PromptSeq sq = seq_of(a, find_seq(a, u, lane, [&](int i) { return a.table ? a.table[i].tile_end : a.seq[i].tile_end; }));
    u -= sq.tile_end - sq.tiles * a.Hkv;
    int unit0 = sq.unit_end - sq.tiles * sq.splits() * a.Hkv;
    const int h = u % a.Hkv, tile = u / a.Hkv, w0 = tile * PA_ROWS + block * 32;
    if (w0 >= sq.count * G) return;
    const int last_tok = min((tile * PA_ROWS + PA_ROWS - 1) / G, sq.count - 1);
    const int pieces = (sq.first + last_tok + sq.chunk()) / sq.chunk();    // those that have a key of the tile
    unit0 += (sq.tiles - 1 - tile) * a.Hkv + h;
    const bool row = w0 + n < sq.count * G;
    float ref = -INFINITY, l = 0.f;
    f32x4 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (row)
        for (int s0 = v; s0 < pieces; s0 += PJ_WAVES * PJ_AHEAD) {
            f32x2 ml[PJ_AHEAD];
            f32x4 x[PJ_AHEAD][4];
#pragma unroll
            for (int k = 0; k < PJ_AHEAD; ++k) {
                const int s = s0 + k * PJ_WAVES;
                const size_t unit = unit0 + (size_t)min(s, pieces - 1) * sq.tiles * a.Hkv;
                ml[k] = *reinterpret_cast<const f32x2*>(a.part_ml + (unit * PA_ROWS + block * 32 + n) * 2);
                if (s >= pieces) ml[k] = f32x2{-INFINITY, 0.f};
                const f32x4* from = reinterpret_cast<const f32x4*>(a.part_acc) + (unit * (PA_ROWS / 32) + block) * 1024 + dims * 256 + lane;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[k][i] = from[i * 64];
            }
            float next = ref;
#pragma unroll
            for (int k = 0; k < PJ_AHEAD; ++k) next = fmaxf(next, ml[k].x);
            const float zero = next == -INFINITY ? 0.f : next, f = __builtin_amdgcn_exp2f(ref - zero);
            ref = next;
            l *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] *= f;
#pragma unroll
            for (int k = 0; k < PJ_AHEAD; ++k) {
                if (s0 + k * PJ_WAVES >= pieces) break;      // (the last piece once more: an infinity times nothing must not count)
                const float g = __builtin_amdgcn_exp2f(ml[k].x - zero);
                l = fmaf(ml[k].y, g, l);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] = fmaf(x[k][i][e], g, o[i][e]);
            }
        }
    if (half == 0) sm_ml[v][n] = f32x2{ref, l};
#pragma unroll
    for (int i = 0; i < 4; ++i) sm_o[v][i][lane] = o[i];
    __syncthreads();
    if (v >= 4 || !row) return;                              // wave v: the v-th four dimensions
    float top = -INFINITY;
    for (int p = 0; p < PJ_WAVES; ++p) top = fmaxf(top, sm_ml[p][n].x);
    const float zero = top == -INFINITY ? 0.f : top;
    l = 0.f;
    f32x4 x{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < PJ_WAVES; ++p) {
        const float f = __builtin_amdgcn_exp2f(sm_ml[p][n].x - zero);
        l = fmaf(sm_ml[p][n].y, f, l);
        x += sm_o[p][v][lane] * f;
    }
    const float inv = 1.0f / l;
    const size_t at = ((size_t)(sq.tok0 + (w0 + n) / G) * a.Hkv + h) * G + (w0 + n) % G;
    *reinterpret_cast<u32x2*>(a.out + at * HC_D + dims * 32 + v * 8 + 4 * half) = u32x2{pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv)};
    if (a.lse && half == 0 && v == 0 && dims == 0) a.lse[at] = lse_of(zero, l);
}

template <int G, int KS>
void launch(const PromptArgs& a, int units, int tiles, hipStream_t st)
{
    prompt_attn_kernel<G, KS><<<dim3(units), dim3(PA_BLK), 0, st>>>(a);
    if (tiles) prompt_join_kernel<G, KS><<<dim3(tiles * (pa_rows<KS> / 32) * 4), dim3(PJ_WAVES * 64), 0, st>>>(a);
}

// Keys of a sequence's pieces: about `chunk`, all of one length but for the last.
struct Cut {
    int pieces, tiles;     // and tiles of 64 keys of a piece
};
Cut cut_of(int keys, int chunk)
{
    const int s = (keys + chunk - 1) / chunk, t = ((keys + s - 1) / s + PA_KEYS - 1) / PA_KEYS;
    return Cut{(keys + t * PA_KEYS - 1) / (t * PA_KEYS), t};
}
struct PromptPlan {
    int ks, chunk;         // waves to 32 rows; keys beyond which a sequence is cut, and about as many to a piece
};
// How long a call takes, in microseconds; < 0: the partial results have no room.  The constants are a fit on one card to 640 drawn
// batches (1 to 12 sequences of 1 to 16K tokens behind up to 128K, 1 to 8 KV heads, groups of 1 to 8) under 5 to 28 plans each.  Over 780
// batches measured with the plans made from it, the plan with the least was 3 % slower than the fastest of them on average, at worst 1.6
// times; times come out 11 % off on average, a third of them more than 12 %, and calls below 10 us too short.  Pieces against none: one token behind
// 131,072 102 us against 2185, 512 behind 120,001 900 against 1650 (eight KV heads, groups of four), 2,199 behind 59,264 of four heads
// 1007 against 1429; and where there are units enough, two pieces against none: 9,038 tokens of four single heads 124 against 109.
float plan_cost(int n, const int* order, const int32_t* first, const int32_t* count, int G, int Hkv, int ks, int chunk, int slots)
{
    const int rows = 128 / ks;
    const float tile_us = ks == 1 ? 0.93f : 0.60f;       // 64 keys: of a compute unit with two workgroups, and of a workgroup that has one for itself
    float work = 0.f, equal = 0.f, units = 0.f, longest = 0.f, kv = 0.f, parts = 0.f;
    long long room = 0;
    int pieces = 0;
    for (int i = 0; i < n; ++i) {
        const int b = order[i];
        const float f = (float)first[b], c = (float)count[b], mean = f + 0.5f * c;
        const long long t = ((long long)count[b] * G + rows - 1) / rows * Hkv;
        const Cut cut = cut_of(first[b] + count[b], chunk);
        work += t * (mean / PA_KEYS + 0.5f);
        float active = (float)t;
        if (cut.pieces > 1) {
            room += t * cut.pieces;
            active *= std::min((float)cut.pieces, std::max(1.f, mean / (cut.tiles * PA_KEYS) + 0.5f));
            parts += active * std::min(rows, count[b] * G) * 520.f;
        }
        equal += t * (mean - 0.5f * std::min(c, (float)cut.tiles * PA_KEYS)) / PA_KEYS;
        pieces = std::max(pieces, cut.pieces);
        units += active;
        longest = std::max(longest, (float)cut.tiles);
        kv += (f + c) * Hkv * 512.f;
    }
    if (room * rows > (long long)PA_ROOM * slots * 128) return -1.f;
    // units of one length (whole pieces, tiles of a chunk behind many keys) leave some compute units one more than others; a
    // prompt's tiles and last pieces are of all lengths and even out, the pieces less well.  The longest unit shares its compute
    // unit as long as there are others; and what comes beyond what the GPU holds at a time finds an otherwise idle one.
    const float cus = 0.5f * slots, more = units > slots ? 1.f - slots / units : 0.f, last = units - floorf((units - 1.f) / slots) * slots;
    const float uneven = units > cus || room > 0 ? 1.f + (ceilf(units / cus) / (units / cus) - 1.f) * equal / work : 1.f;
    const float ragged = room > 0 ? 0.25f * std::min(1.f, 3.f * (1.f - equal / work)) : 0.f;
    const float alone = longest * tile_us, shared = work * tile_us / cus;
    const float arithmetic = std::max(shared * uneven * (units <= cus ? 1.2f : 1.f) + ragged * alone, alone + 0.45f * more * shared);
    const float read = kv / 5.4e6f * (1.f + 0.12f * (uneven - 1.f));
    const float memory = units > slots ? read * (1.f - last / units) + std::max(read * last / units, longest * 0.45f * equal / work)
                                       : read / std::min(1.f, powf(units / cus, 0.3f));
    return std::max(arithmetic, memory) + (units > slots ? 5.5f : 3.5f) + (room > 0 ? 4.5f + 0.03f * pieces + parts / 3.0e6f : 0.f);
}
PromptPlan make_plan(int n, const int* order, const int32_t* first, const int32_t* count, int G, int Hkv, int slots)
{
    PromptPlan best{1, 1 << 30};
    float cost = plan_cost(n, order, first, count, G, Hkv, 1, 1 << 30, slots);
    const int longest = first[order[0]] + count[order[0]];
    for (int ks = 1; ks <= 2; ++ks)
        for (int pieces = 1; pieces <= 1024 && longest / pieces >= 128; pieces += 1 + pieces / 12) {
            const int chunk = pieces == 1 ? 1 << 30 : (longest + pieces - 1) / pieces;
            const float c = plan_cost(n, order, first, count, G, Hkv, ks, chunk, slots);
            if (c < 0.f) break;
            if (c < cost) {
                cost = c;
                best = PromptPlan{ks, chunk};
            }
        }
    return best;
}

// Rows of partial results that there is room for: PA_ROOM tiles of 128 for every workgroup that the GPU holds at a time.
size_t part_rows(const hc_ctx* ctx) { return (size_t)PA_ROOM * PA_PER_CU * ctx->n_cu * 128; }

}   // namespace

// The work buffer: partial results, then the table.
struct PromptWork {
    size_t ml, seq, off, bytes;
};
static PromptWork work_of(const hc_ctx* ctx)
{
    const size_t rows = part_rows(ctx), B = (size_t)ctx->cfg.B;
    PromptWork w{};
    w.ml = rows * HC_D * sizeof(float);
    w.seq = w.ml + rows * 2 * sizeof(float);
    w.off = w.seq + (B * sizeof(PromptSeq) + 255) / 256 * 256;
    w.bytes = w.off + B * ctx->cfg.Hkv * 2 * sizeof(int64_t);
    return w;
}
size_t hc_prompt_work_bytes(const hc_ctx* ctx) { return work_of(ctx).bytes; }
size_t hc_prompt_scratch_bytes(const hc_config& c) { return (size_t)c.B * (sizeof(PromptSeq) + 2 * sizeof(int)); }

hc_status hc_launch_prefill_attn(hc_ctx* ctx, const void* q, const void* kv, const int64_t* k_off, const int64_t* v_off, const int32_t* first,
                                 const int32_t* count, void* out, float* lse, void* work, hipStream_t st)
{
    const hc_config& c = ctx->cfg;
    const int G = ctx->G, slots = PA_PER_CU * ctx->n_cu;
    const PromptWork lay = work_of(ctx);
    // the sequences that bring tokens, the longest first
    PromptSeq* const seq = (PromptSeq*)ctx->prompt_scratch;
    int *const order = (int*)(seq + c.B), *const tok0 = order + c.B;
    int n = 0;
    long long tokens = 0;
    for (int b = 0; b < c.B; ++b) {
        tok0[b] = (int)tokens;
        tokens += count[b];
        if (count[b] > 0) order[n++] = b;
    }
    std::sort(order, order + n, [&](int x, int y) { return first[x] + count[x] != first[y] + count[y] ? first[x] + count[x] > first[y] + count[y] : x < y; });
    const PromptPlan plan = make_plan(n, order, first, count, G, c.Hkv, slots);
    const int rows = 128 / plan.ks;
    long long units = 0, tiles = 0, joined = 0, joined_tiles = 0;          // joined: those that leave partial results; they come first
    for (int i = 0; i < n; ++i) {
        const int b = order[i];
        PromptSeq& s = seq[i];
        s.first = first[b];
        s.count = count[b];
        s.tok0 = tok0[b];
        s.tiles = (int)(((long long)count[b] * G + rows - 1) / rows);
        const Cut cut = cut_of(first[b] + count[b], plan.chunk);
        s.cut = (uint32_t)cut.tiles << 12 | (uint32_t)cut.pieces;
        tiles += (long long)s.tiles * c.Hkv;
        units += (long long)s.tiles * cut.pieces * c.Hkv;
        if (cut.pieces > 1) {
            joined = units;
            joined_tiles = tiles;
        }
        s.unit_end = (int)units;
        s.tile_end = (int)tiles;
    }
    if (joined * rows > (long long)part_rows(ctx)) return hc_fail(ctx, HC_EINVAL, "hc_prefill_attn: partial results without room");       // (the plan sees to it)
    PromptArgs a{};
    a.q = (const uint16_t*)q;
    a.kv = (const uint16_t*)kv;
    a.out = (uint16_t*)out;
    a.lse = lse;
    a.part_acc = (float*)work;
    a.part_ml = (float*)((char*)work + lay.ml);
    a.Hkv = c.Hkv;
    a.n_seq = n;
    a.together = std::max(1, PA_DIES / c.Hkv);
    a.n_cu = ctx->n_cu;
    a.mirror = joined == 0 && ctx->n_cu % c.Hkv == 0 && units > ctx->n_cu ? (int)std::min<long long>(units - ctx->n_cu, ctx->n_cu) : 0;
    a.table_rows = n * c.Hkv;
    const bool in_table = n > PA_SEQS || a.table_rows > PA_HEADS;
    const int most = std::max(1, std::min(PA_SEQS, PA_HEADS / c.Hkv));          // sequences of an upload
    for (int i0 = 0; i0 < n; i0 += most) {
        const int m = std::min(most, n - i0);
        std::copy(seq + i0, seq + i0 + m, a.seq);
        for (int i = 0; i < m * c.Hkv; ++i) {
            const size_t from = (size_t)order[i0 + i / c.Hkv] * c.Hkv + i % c.Hkv;
            a.k_off[i] = k_off[from];
            a.v_off[i] = v_off[from];
        }
        if (in_table) {
            prompt_table_kernel<<<dim3(1), dim3(PA_HEADS), 0, st>>>(a, (PromptSeq*)((char*)work + lay.seq) + i0, m,
                                                                   (int64_t*)((char*)work + lay.off) + (size_t)i0 * c.Hkv, m * c.Hkv);
            HC_HIP(ctx, hipGetLastError());
        }
    }
    if (in_table) {
        a.table = (const PromptSeq*)((char*)work + lay.seq);
        a.table_off = (const int64_t*)((char*)work + lay.off);
    }
    switch (G * 4 + plan.ks) {
    case 5: launch<1, 1>(a, (int)units, (int)joined_tiles, st); break;
    case 6: launch<1, 2>(a, (int)units, (int)joined_tiles, st); break;
    case 9: launch<2, 1>(a, (int)units, (int)joined_tiles, st); break;
    case 10: launch<2, 2>(a, (int)units, (int)joined_tiles, st); break;
    case 17: launch<4, 1>(a, (int)units, (int)joined_tiles, st); break;
    case 18: launch<4, 2>(a, (int)units, (int)joined_tiles, st); break;
    case 33: launch<8, 1>(a, (int)units, (int)joined_tiles, st); break;
    default: launch<8, 2>(a, (int)units, (int)joined_tiles, st); break;
    }
    HC_HIP(ctx, hipGetLastError());
    return HC_OK;
}
