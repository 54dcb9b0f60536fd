// hc_kvq.hip -- the cache held in 4 bits (its format: hc_kvq.h): rows into it (a prompt's, the decode token's), back to bf16, and eviction by
// accumulated weight.  Attention over it: hc_kvq_attn.hip.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <new>

#include "hc_kvq.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}

// Eight elements of a row (bf16) as a dword of codes; scale: the byte of the 32 values that this lane and the three beside it hold.
__device__ __forceinline__ uint32_t encode(const u32x4 x, uint32_t& scale)
{
    uint32_t top = 0;                                            // largest magnitude, as the bits of a float: they order as the numbers do, with
#pragma unroll                                                   // infinities and NaNs behind them
    for (int i = 0; i < 4; ++i) top = max(top, max((x[i] << 16) & 0x7fffffffu, x[i] & 0x7fff0000u));
    top = max(top, dpp<0xB1>(top));                              // quad_perm [1,0,3,2]
    top = max(top, dpp<0x4E>(top));                              // quad_perm [2,3,0,1]
    if (top >= 0x7f800000u) {
        scale = 255u;
        return 0u;
    }
    // 2^x (1 + m) <= 7 2^e = 2^(e + 2) 1.75:  e = x - 2, and one more where m > 0.75
    scale = (uint32_t)max(((int)((top + 0x1fffffu) >> 23)) - 2, 2);
    const float unit = kq_scale(scale);
    const uint32_t a = x[0], b = x[1], c = x[2], d = x[3];
    uint32_t codes = 0;                                          // (the conversion rounds to the nearest, ties to the even code, and 7 down to 6)
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(kq_bf16x2, a), unit, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(kq_bf16x2, b), unit, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(kq_bf16x2, c), unit, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(kq_bf16x2, d), unit, 3);
    return codes;
}

// Codes and scale bytes of a row, 16 lanes a row.  The four scale bytes are stored by one lane.
__device__ __forceinline__ void put_row(uint8_t* __restrict__ codes_at, uint8_t* __restrict__ scales_at, int lane16, uint32_t codes, uint32_t scale)
{
    *reinterpret_cast<uint32_t*>(codes_at + lane16 * 4) = codes;
    uint32_t s = scale << (lane16 & 12) * 2;                     // bytes of the groups of four lanes
    s |= dpp<0x128>(s);                                          // rotate by 8
    s |= dpp<0x124>(s);                                          // rotate by 4
    if (lane16 == 0) *reinterpret_cast<uint32_t*>(scales_at) = s;
}

// ---- rows in and out --------------------------------------------------------------------------------------------------------------------
//
// A row is 16 lanes' work: a lane has 16 bytes of bf16 and a dword of codes, the largest of 32 values takes two moves between neighbours, and the conversions are the
// hardware's.  Bound by memory: a workgroup has all rows of its 64 tokens (of one head, K and V) on their way at once.  32,003 tokens of eight heads: in 33 us
// (166 MB, 5.0 TB/s, where a copy of 1 GiB reaches 5.2) and 4.8 for the counts behind them, out 26.5 (6.3, what was just written lies in the caches); 1.97 million
// rows out 296 us, 1.28 GB, 4.3 TB/s.  17 tokens of two heads 4.2 and 3.7 us: the launch and a chain of three loads.

constexpr int RW_BLK = 256;
constexpr int RW_TOKENS = 64;                 // of a workgroup
constexpr int RW_SEQS = HC_PROMPT_SEQS, RW_HEADS = HC_PROMPT_HEADS;
static_assert(4 * RW_SEQS == 2 * RW_HEADS, "either form of the offsets");

// Packed tokens of a launch, sequence by sequence, as hc_prefill_rope has them.
struct RowsArgs {
    uint8_t* arena;
    uint16_t* kv;
    const hc_kvq_head* heads;                 // of the launch's first sequence
    int2* state;
    float* acc;
    int Hkv, n_seq, tokens, whole, even;
    int end[RW_SEQS], first[RW_SEQS];
    // Where the heads' blocks of kv are: a K and a V offset to a head; or (even), where those of every sequence lie evenly apart, as they do but for heads of
    // different room, first K offset, step, first V offset, step to a sequence, so that a launch has room for 64 sequences of any number of heads.  Four
    // launches in place of one cost 64 decode tokens of eight heads 13 us, rows of 64 sequences their loading 485 us in place of 346 (then).
    int64_t off[2 * RW_HEADS];
};
// Where the K rows of a workgroup's tokens are (codes -1: nowhere); V's, 68 cap bytes and v_kv elements further on.
struct RowPlaces {
    int64_t codes[RW_TOKENS], scales[RW_TOKENS], kv[RW_TOKENS], v_kv[RW_TOKENS];
    int32_t cap[RW_TOKENS];
};

// Which tokens a workgroup takes: RW_TOKENS packed ones from blockIdx.x * RW_TOKENS on, or (whole) all of sequence blockIdx.x, which are no more; of head
// blockIdx.y.  row_of: (the sequence's first, number in it, rows that the head has) -> its row in the cache, or -1; at: the element that a token's row has in its block of kv.
template <typename R, typename A>
__device__ __forceinline__ int row_places(const RowsArgs& a, RowPlaces& x, R row_of, A at)
{
    const int tid = threadIdx.x, lane = tid & 63, h = blockIdx.y;
    const int t0 = a.whole ? (blockIdx.x > 0 ? a.end[blockIdx.x - 1] : 0) : blockIdx.x * RW_TOKENS;
    const int n = a.whole ? a.end[blockIdx.x] - t0 : min(RW_TOKENS, a.tokens - t0);
    if (tid < RW_TOKENS) {
        int i, f, bh;
        int64_t k, v;
        if (a.whole || a.n_seq == 1) {                           // one sequence: its arguments are the same for all lanes
            const int seq = a.whole ? blockIdx.x : 0;
            i = a.whole ? tid : t0 + tid;
            f = a.first[seq];
            bh = seq * a.Hkv + h;
            k = a.even ? a.off[4 * seq] + h * a.off[4 * seq + 1] : a.off[2 * bh];
            v = a.even ? a.off[4 * seq + 2] + h * a.off[4 * seq + 3] : a.off[2 * bh + 1];
        } else {
            // The launch's arguments may lie in the host's memory, microseconds away: a lane takes those of one sequence, and gets others' from its
            // neighbours.  (A search that read them step by step cost 1.97 million rows of 64 sequences 346 us in place of 294.)
            const int end = lane < a.n_seq ? a.end[lane] : INT_MAX, first = a.first[lane];
            int64_t off[4] = {0, 0, 0, 0};
            if (a.even)
#pragma unroll
                for (int e = 0; e < 4; ++e) off[e] = a.off[4 * lane + e];
            const int t = t0 + min(tid, n - 1);
            int seq = 0;                                         // sequences that end before this token
#pragma unroll
            for (int step = RW_SEQS / 2; step > 0; step >>= 1)
                if (__shfl(end, seq + step - 1) <= t) seq += step;
            const int before = __shfl(end, max(seq - 1, 0));
            i = t - (seq > 0 ? before : 0);
            f = __shfl(first, seq);
            bh = seq * a.Hkv + h;
            if (a.even) {
                k = __shfl(off[0], seq) + h * __shfl(off[1], seq);
                v = __shfl(off[2], seq) + h * __shfl(off[3], seq);
            } else {
                k = a.off[2 * bh];
                v = a.off[2 * bh + 1];
            }
        }
        const hc_kvq_head hd = a.heads[bh];
        const int rows = min(max(a.state[bh].x, 0), hd.cap);
        const int64_t row = tid < n ? row_of(f, i, rows, hd) : -1;
        x.codes[tid] = row < 0 ? -1 : hd.off + row * 64;
        x.scales[tid] = hd.off + (int64_t)64 * hd.cap + row * 4;
        x.cap[tid] = hd.cap;
        x.kv[tid] = k + at(f, i);
        x.v_kv[tid] = v - k;
    }
    __syncthreads();
    return n;
}
constexpr int RW_STEPS = RW_TOKENS / (RW_BLK / 16);              // rows that 16 lanes take of K, and of V

__global__ __launch_bounds__(RW_BLK) void kvq_store_kernel(RowsArgs a)
{
    __shared__ RowPlaces sm;
    const int n = row_places(a, sm,
                             [&](int, int i, int rows, const hc_kvq_head& hd) -> int64_t {
                                 const int64_t row = (int64_t)rows + i;
                                 if (row >= hd.cap) return -1;
                                 if (a.acc) a.acc[hd.row_off + row] = 0.f;
                                 return row;
                             },
                             [](int f, int i) { return ((int64_t)f + i) * HC_D; });
    const int tid = threadIdx.x, lane16 = tid & 15;
    u32x4 x[2 * RW_STEPS];
#pragma unroll
    for (int k = 0; k < 2 * RW_STEPS; ++k) {
        const int t = (tid >> 4) + RW_BLK / 16 * (k % RW_STEPS);
        if (sm.codes[t] >= 0) x[k] = *reinterpret_cast<const u32x4*>(a.kv + sm.kv[t] + (k < RW_STEPS ? 0 : sm.v_kv[t]) + lane16 * 8);
    }
#pragma unroll
    for (int k = 0; k < 2 * RW_STEPS; ++k) {
        const int t = (tid >> 4) + RW_BLK / 16 * (k % RW_STEPS);
        if (sm.codes[t] >= 0) {                                  // (the 16 lanes of a row go together)
            const int64_t v = k < RW_STEPS ? 0 : (int64_t)68 * sm.cap[t];
            uint32_t scale;
            const uint32_t codes = encode(x[k], scale);
            put_row(a.arena + v + sm.codes[t], a.arena + v + sm.scales[t], lane16, codes, scale);
        }
    }
    if (!a.whole || n == 0) return;
    __syncthreads();                                             // (everyone has read the state)
    if (tid == 0) {
        const int bh = blockIdx.x * a.Hkv + blockIdx.y, cap = a.heads[bh].cap;
        const int rows = min(max(a.state[bh].x, 0), cap);
        a.state[bh] = make_int2(min(n, cap - rows) + rows, a.first[blockIdx.x] + n);
    }
}

// Rows and positions of the heads after a store of several workgroups to a sequence.
__global__ __launch_bounds__(RW_BLK) void kvq_count_kernel(RowsArgs a)
{
    for (int bh = threadIdx.x; bh < a.n_seq * a.Hkv; bh += RW_BLK) {
        const int b = bh / a.Hkv, n = a.end[b] - (b > 0 ? a.end[b - 1] : 0), cap = a.heads[bh].cap;
        if (n == 0) continue;
        const int rows = min(max(a.state[bh].x, 0), cap);
        a.state[bh] = make_int2(min(n, cap - rows) + rows, a.first[b] + n);
    }
}

// (Heads of the same tokens side by side in the grid: 64 sequences of equal heads 281 us in place of 294, but a long head among short ones then runs on one die of
// the eight, 41 us in place of 18.)
__global__ __launch_bounds__(RW_BLK) void kvq_load_kernel(RowsArgs a)
{
    __shared__ RowPlaces sm;
    row_places(a, sm, [](int f, int i, int rows, const hc_kvq_head&) -> int64_t { return f + (int64_t)i < rows ? f + i : -1; },
               [](int, int i) { return (int64_t)i * HC_D; });
    const int tid = threadIdx.x, lane16 = tid & 15;
    uint32_t codes[2 * RW_STEPS], scale[2 * RW_STEPS];
#pragma unroll
    for (int k = 0; k < 2 * RW_STEPS; ++k) {
        const int t = (tid >> 4) + RW_BLK / 16 * (k % RW_STEPS);
        if (sm.codes[t] >= 0) {
            const uint8_t* const at = a.arena + (k < RW_STEPS ? 0 : (int64_t)68 * sm.cap[t]);
            codes[k] = *reinterpret_cast<const uint32_t*>(at + sm.codes[t] + lane16 * 4);
            scale[k] = at[sm.scales[t] + (lane16 >> 2)];
        }
    }
#pragma unroll
    for (int k = 0; k < 2 * RW_STEPS; ++k) {
        const int t = (tid >> 4) + RW_BLK / 16 * (k % RW_STEPS);
        if (sm.codes[t] >= 0) {
            const float f = kq_scale(scale[k]);
            const u32x4 x{kq_pair<0>(codes[k], f), kq_pair<1>(codes[k], f), kq_pair<2>(codes[k], f), kq_pair<3>(codes[k], f)};
            *reinterpret_cast<u32x4*>(a.kv + sm.kv[t] + (k < RW_STEPS ? 0 : sm.v_kv[t]) + lane16 * 8) = x;
        }
    }
}

// ---- the decode token ---------------------------------------------------------------------------------------------------------------------

struct TokenArgs {
    double turns[HC_D / 2];                   // frequencies in full turns a position
    const float *q_norm, *k_norm;
    float eps, gain;
    int rot, half;
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    uint16_t* q_out;
    uint8_t* arena;
    const hc_kvq_head* heads;
    int2* state;
    float* acc;
    int Hkv, G;
};

__host__ __device__ constexpr int token_threads(int G) { return (16 * (G + 2) + 63) / 64 * 64; }

__device__ __forceinline__ double sum16(double x)
{
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) x += __shfl_xor(x, d, 16);
    return x;
}

// One workgroup per KV head and sequence: the token's K row, its V row and the G query rows of the group, 16 lanes a row, eight elements in a row to
// each.  y = x (mean(x^2) + eps)^(-1/2) w, then pairs (u, v) -> gain (u cos a - v sin a, v cos a + u sin a), a = position * frequency; rounded to bf16, then to codes.
// Norm and rotation in 64 bits: next to the border between two codes the step from one to the other is a third of the value, and whoever computes in more
// bits than the row's own has the same row.  Bound by latency: 4.7 us for one sequence of two heads, 5.8 for 64 of eight (the angles' sine and cosine in 64
// bits are 1.2 of it, the norm 0.3).
template <bool F32>
__global__ __launch_bounds__(token_threads(HC_MAX_G)) void kvq_append_kernel(TokenArgs a)
{
    __shared__ double2 sm_turn[HC_D / 2];
    __shared__ double sm_x[HC_MAX_G + 1][HC_D];
    const int bh = blockIdx.x, b = bh / a.Hkv, h = bh - b * a.Hkv, tid = threadIdx.x;
    const hc_kvq_head hd = a.heads[bh];
    const int2 st = a.state[bh];
    const int lane16 = tid & 15, row = tid >> 4;                 // 0: V, 1: K, 2 + g: query head g of the group
    const int e0 = lane16 * 8;
    double x[8];
    u32x4 raw{};
    const bool mine = row < a.G + 2;
    if (mine) {
        const void* src = row == 0 ? a.v : row == 1 ? a.k : a.q;
        const size_t from = (row == 0   ? (size_t)b * a.v_stride + (size_t)h * HC_D
                             : row == 1 ? (size_t)b * a.k_stride + (size_t)h * HC_D
                                        : (size_t)b * a.q_stride + (size_t)(h * a.G + row - 2) * HC_D) + e0;
        if (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = ((const float*)src)[from + e];
        } else {
            raw = *reinterpret_cast<const u32x4*>((const uint16_t*)src + from);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e & 1 ? raw[e / 2] & 0xffff0000u : raw[e / 2] << 16);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0;
    }
    const float* const weight = row == 0 || !mine ? nullptr : row == 1 ? a.k_norm : a.q_norm;
    f32x4 w0{1.f, 1.f, 1.f, 1.f}, w1 = w0;                       // (on their way with the rest)
    if (weight) {
        w0 = *reinterpret_cast<const f32x4*>(weight + e0);
        w1 = *reinterpret_cast<const f32x4*>(weight + e0 + 4);
    }
    if (2 * tid < a.rot) {
        const double t = (double)st.y * a.turns[tid];
        double s, c;
        sincospi(2.0 * (t - rint(t)), &s, &c);
        sm_turn[tid] = make_double2(c * a.gain, s * a.gain);
    }
    double q = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) q = fma(x[e], x[e], q);
    q = sum16(q);
    if (weight) {
        const double f = 1.0 / sqrt(q * (1.0 / HC_D) + (double)a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= f * (double)(e < 4 ? w0[e & 3] : w1[e & 3]);
    }
    if (mine && row > 0)
#pragma unroll
        for (int e = 0; e < 8; ++e) sm_x[row - 1][e0 + e] = x[e];
    __syncthreads();                                             // (and everyone has read the state)
    if (mine && row > 0) {
        const int half = a.rot / 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = e0 + e;
            if (i >= a.rot) continue;
            const bool second = a.half ? i >= half : (i & 1);
            const int pair = a.half ? (second ? i - half : i) : i >> 1;
            const double other = sm_x[row - 1][a.half ? (second ? i - half : i + half) : i ^ 1];
            const double2 t = sm_turn[pair];
            x[e] = second ? fma(x[e], t.x, other * t.y) : fma(x[e], t.x, -other * t.y);
        }
    }
    // one rounding to bf16 (through 32 bits rounded to odd, so that the two steps round as one)
    u32x4 w{};
    if (row == 0 && !F32) w = raw;
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float f = (float)x[e];
            uint32_t u = __float_as_uint(f);
            if ((double)f != x[e] && !(u & 1) && (u & 0x7fffffffu) < 0x7f800000u) u += fabs((double)f) > fabs(x[e]) ? -1 : 1;
            u = (u & 0x7fffffffu) > 0x7f800000u ? u | 0x400000u : u + 0x7fffu + ((u >> 16) & 1);
            w[e / 2] |= e & 1 ? u & 0xffff0000u : u >> 16;
        }
    uint32_t scale;
    const uint32_t codes = encode(w, scale);
    const int at = min(max(st.x, 0), hd.cap);
    if (mine && row >= 2) *reinterpret_cast<u32x4*>(a.q_out + ((size_t)bh * a.G + row - 2) * HC_D + e0) = w;
    else if (row < 2 && at < hd.cap) {
        uint8_t* const block = a.arena + hd.off + (row == 0 ? (int64_t)68 * hd.cap : 0);
        put_row(block + (int64_t)at * 64, block + (int64_t)64 * hd.cap + (int64_t)at * 4, lane16, codes, scale);
        if (a.acc && row == 0 && lane16 == 1) a.acc[hd.row_off + at] = 0.f;
    }
    if (tid == 0) a.state[bh] = make_int2(min(at + 1, hd.cap), st.y + 1);
}

// ---- eviction -------------------------------------------------------------------------------------------------------------------------------
//
// What stays is what sorting by (weight descending, row ascending) would leave: the k-th largest key is found exactly, every larger one stays, and of its
// equals the first.  Tables of heads of up to KQ_SHORT rows: one workgroup a head, keys in LDS, then a launch that moves rows: 2,304 rows of two heads 7.7 and
// 2.8 us, mostly barriers and the chain of loads.  Longer: six launches over spans of KQ_SPAN rows, each bound by its own latency: 224K rows of eight
// heads 4.0 (clear), 3 x 5.1 (digits), 5.0 (count), 15.1 us (place); 512 heads of up to 32K rows 5.7, 3 x 13.7, 14 and 183 us.  The last is bound by memory: of
// rows of 64 bytes, a quarter of which stay, the memory reads lines of 128 (784 MB moved, 4.3 TB/s); with all rows staying it runs at 4.7 TB/s.
// Measured against that: one workgroup to a long head, 330 us in place of 44 at 224K rows and 78 in place of 60 for the 512 heads; spans of 2,048 and 8,192 rows, 256
// and 1,024 threads to a span: none better in both cases.

// Keys order as the weights do (hc_score_key), larger ones first; the k-th largest is found digit by digit, 11, 11 and 10 bits from the top, with a histogram of
// the keys that have the digits found so far.
__device__ __forceinline__ int digit_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t digit(uint32_t key, int pass) { return (key >> digit_shift(pass)) & (pass == 2 ? 1023u : 2047u); }
__device__ __forceinline__ uint32_t known_bits(int pass) { return pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u; }

// The bin, from the largest on, in which the k-th key is (k >= 1), and its number there.  BLK threads, KQ_BINS / BLK bins of `mine` each, largest first.
template <int BLK>
__device__ __forceinline__ uint2 find_bin(const uint32_t (&mine)[KQ_BINS / BLK], uint32_t k, uint32_t* sm_wave, uint32_t* sm_found)
{
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < KQ_BINS / BLK; ++i) all += mine[i];
    uint32_t upto = all;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) sm_wave[w] = upto;
    __syncthreads();
    uint32_t before = upto - all;
    for (int i = 0; i < w; ++i) before += sm_wave[i];
    if (before < k && k <= before + all) {
        uint32_t at = 0, n = before;
#pragma unroll
        for (int i = 0; i < KQ_BINS / BLK; ++i)
            if (n < k) {                                         // (the last bin that begins before the k-th key)
                at = i;
                before = n;
                n += mine[i];
            }
        sm_found[0] = KQ_BINS - 1 - tid * (KQ_BINS / BLK) - at;
        sm_found[1] = k - before;
    }
    __syncthreads();
    const uint2 r = make_uint2(sm_found[0], sm_found[1]);
    __syncthreads();
    return r;
}

struct EvictArgs {
    const hc_kvq_head *heads, *to;
    const int2* state;
    int2* to_state;
    const float* acc;
    float* to_acc;
    const uint8_t* arena;
    uint8_t* to_arena;
    int32_t* list;                            // rows that stay
    int list_is_to;                           // it is indexed as the target's tables, not the source's
    const int2* spans;
    uint32_t* hist;                           // [n][3][KQ_BINS]
    uint2* found;                             // [n][3]: after a digit, the key's digits so far, and its number among the keys that have them
    uint2* counts;                            // [spans]: rows that stay for certain, and keys equal to the k-th
};

// What a head is to keep: the first `lo` of n rows, those from `hi` on, and k of those between them; all, where m == n.
struct Keep {
    int n, m, lo, hi, k;
};
__device__ __forceinline__ Keep keep_of(const hc_kvq_head& from, const hc_kvq_head& to, int2 state)
{
    Keep x;
    x.n = min(max(state.x, 0), from.cap);
    x.m = min(x.n, to.budget);
    x.lo = to.sink;
    x.hi = x.n - to.recent;
    x.k = x.m - to.sink - to.recent;
    return x;
}

// A row of a head's block, as the four lanes that move it hold it: 16 bytes of codes of K and V each, and of lane 0 K's scales, of lane 1 V's, of lane 2 the
// weight.
struct MovedRow {
    u32x4 k, v;
    uint32_t more;
};
__device__ __forceinline__ MovedRow take_row(const uint8_t* src, const hc_kvq_head& from, int64_t i, int part, const float* acc)
{
    MovedRow r;
    r.k = *reinterpret_cast<const u32x4*>(src + i * 64 + part * 16);
    r.v = *reinterpret_cast<const u32x4*>(src + (int64_t)68 * from.cap + i * 64 + part * 16);
    r.more = 0;
    if (part < 3)
        r.more = *reinterpret_cast<const uint32_t*>(part < 2 ? src + (int64_t)(part == 0 ? 64 : 132) * from.cap + i * 4 : (const uint8_t*)(acc + from.row_off + i));
    return r;
}
__device__ __forceinline__ void put_row(const MovedRow& r, uint8_t* dst, const hc_kvq_head& to, int64_t j, int part, float* to_acc)
{
    *reinterpret_cast<u32x4*>(dst + j * 64 + part * 16) = r.k;
    *reinterpret_cast<u32x4*>(dst + (int64_t)68 * to.cap + j * 64 + part * 16) = r.v;
    if (part < 3) *reinterpret_cast<uint32_t*>(part < 2 ? dst + (int64_t)(part == 0 ? 64 : 132) * to.cap + j * 4 : (uint8_t*)(to_acc + to.row_off + j)) = r.more;
}

constexpr int EV_BLK = 1024, EV_WAVES = EV_BLK / 64;

// One workgroup per head: the rows that stay, in order.  Keys in LDS.
__global__ __launch_bounds__(EV_BLK) void kvq_select_kernel(EvictArgs a)
{
    __shared__ uint32_t sm_hist[KQ_BINS];
    __shared__ uint32_t sm_wave[EV_WAVES], sm_more[EV_WAVES];
    __shared__ uint32_t sm_found[2];
    __shared__ uint32_t sm_key[KQ_SHORT];
    const int bh = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const hc_kvq_head from = a.heads[bh], to = a.to[bh];
    const int2 st = a.state[bh];
    const Keep x = keep_of(from, to, st);
    int32_t* const list = a.list + (a.list_is_to ? to.row_off : from.row_off);
    if (tid == 0) a.to_state[bh] = make_int2(x.m, st.y);
    if (x.m == x.n) {
        for (int i = tid; i < x.n; i += EV_BLK) list[i] = i;
        return;
    }
    const float* const acc = a.acc + from.row_off;
    for (int i = tid; i < x.n; i += EV_BLK) sm_key[i] = hc_score_key(acc[i]);
    uint32_t found = ~0u, left = x.k;                            // (no key is larger, where none stays by its weight)
    if (x.k > 0) {
        found = 0;
        for (int pass = 0; pass < 3; ++pass) {
            for (int i = tid; i < KQ_BINS; i += EV_BLK) sm_hist[i] = 0;
            __syncthreads();
            for (int i = x.lo + tid; i < x.hi; i += EV_BLK) {
                const uint32_t u = sm_key[i];
                if ((u & known_bits(pass)) == found) atomicAdd(&sm_hist[digit(u, pass)], 1u);
            }
            __syncthreads();
            const uint32_t mine[2] = {sm_hist[KQ_BINS - 1 - 2 * tid], sm_hist[KQ_BINS - 2 - 2 * tid]};
            const uint2 r = find_bin<EV_BLK>(mine, left, sm_wave, sm_found);
            found |= r.x << digit_shift(pass);
            left = r.y;
        }
    }
    __syncthreads();
    // every wave a run of rows: how many of its keys are larger, and equal; then, knowing what is before it, which rows stay
    const int run = ((x.n + EV_WAVES - 1) / EV_WAVES + 63) / 64 * 64, r0 = min(x.n, w * run), r1 = min(x.n, r0 + run);
    uint32_t larger = 0, equal = 0;
    for (int i = r0 + lane; i - lane < r1; i += 64) {
        const bool in = i < r1 && i >= x.lo && i < x.hi;
        const uint32_t u = in ? sm_key[i] : 0u;
        larger += __popcll(__builtin_amdgcn_ballot_w64((i < r1 && !in) || (in && u > found)));
        equal += __popcll(__builtin_amdgcn_ballot_w64(in && u == found));
    }
    if (lane == 0) {
        sm_wave[w] = larger;
        sm_more[w] = equal;
    }
    __syncthreads();
    uint32_t ties = 0, at = 0;                                   // equal keys before; rows that stay before
    for (int i = 0; i < w; ++i) {
        at += sm_wave[i];
        ties += sm_more[i];
    }
    at += min(ties, left);
    const uint64_t below = (1ull << lane) - 1;
    for (int i = r0 + lane; i - lane < r1; i += 64) {
        const bool in = i < r1 && i >= x.lo && i < x.hi;
        const uint32_t u = in ? sm_key[i] : 0u;
        const uint64_t eq = __builtin_amdgcn_ballot_w64(in && u == found);
        const bool stays = i < r1 && (!in || u > found || (u == found && ties + __popcll(eq & below) < left));
        const uint64_t all = __builtin_amdgcn_ballot_w64(stays);
        if (stays) list[at + __popcll(all & below)] = i;
        at += __popcll(all);
        ties += __popcll(eq);
    }
}

// ---- the same of longer heads: a workgroup to KQ_SPAN rows, a launch to a digit ----

constexpr int SP_BLK = 512, SP_WAVES = SP_BLK / 64, SP_EACH = KQ_SPAN / SP_BLK;

__global__ __launch_bounds__(SP_BLK) void kvq_evict_clear_kernel(EvictArgs a)
{
    const int bh = blockIdx.x;
    const Keep x = keep_of(a.heads[bh], a.to[bh], a.state[bh]);
    if (x.m == x.n || x.k == 0) return;
    uint32_t* const hist = a.hist + (size_t)bh * 3 * KQ_BINS;
    for (int i = threadIdx.x; i < 3 * KQ_BINS; i += SP_BLK) hist[i] = 0;
}

// The keys of a span that are to be told apart, wave by wave in runs of 64 SP_EACH rows; others: 0 with `in` false.
struct SpanKeys {
    uint32_t u[SP_EACH];
    bool in[SP_EACH];
};
__device__ __forceinline__ void span_keys(const EvictArgs& a, const hc_kvq_head& from, const Keep& x, int first, SpanKeys& s)
{
    const int r0 = first + (threadIdx.x >> 6) * 64 * SP_EACH + (threadIdx.x & 63);
    const float* const acc = a.acc + from.row_off;
#pragma unroll
    for (int k = 0; k < SP_EACH; ++k) {
        const int r = r0 + 64 * k;
        s.in[k] = r >= x.lo && r < x.hi;
        s.u[k] = s.in[k] ? __float_as_uint(acc[r]) : 0u;
    }
#pragma unroll
    for (int k = 0; k < SP_EACH; ++k) s.u[k] = s.in[k] ? hc_score_key(__uint_as_float(s.u[k])) : 0u;
}
__device__ __forceinline__ uint2 span_find(const EvictArgs& a, int bh, int pass, uint32_t k, uint32_t* sm_wave, uint32_t* sm_found)
{
    const u32x4 h = *reinterpret_cast<const u32x4*>(a.hist + ((size_t)bh * 3 + pass) * KQ_BINS + KQ_BINS - 4 - 4 * threadIdx.x);
    const uint32_t mine[4] = {h[3], h[2], h[1], h[0]};
    return find_bin<SP_BLK>(mine, k, sm_wave, sm_found);
}
static_assert(KQ_BINS / SP_BLK == 4, "bins of a thread");

// Digit PASS of the keys that have the digits before it; the digit before it is found first.
template <int PASS>
__global__ __launch_bounds__(SP_BLK) void kvq_evict_digit_kernel(EvictArgs a)
{
    __shared__ uint32_t sm_hist[KQ_BINS], sm_wave[SP_WAVES], sm_found[2];
    const int2 span = a.spans[blockIdx.x];
    const int bh = span.x, tid = threadIdx.x;
    const hc_kvq_head from = a.heads[bh];
    const Keep x = keep_of(from, a.to[bh], a.state[bh]);
    if (x.m == x.n || x.k == 0 || span.y >= x.hi || span.y + KQ_SPAN <= x.lo) return;
    SpanKeys s;
    span_keys(a, from, x, span.y, s);
    for (int i = tid; i < KQ_BINS; i += SP_BLK) sm_hist[i] = 0;
    uint32_t found = 0;
    if (PASS > 0) {
        const uint2 last = PASS == 1 ? make_uint2(0u, (uint32_t)x.k) : a.found[(size_t)bh * 3 + PASS - 2];
        const uint2 r = span_find(a, bh, PASS - 1, last.y, sm_wave, sm_found);
        found = last.x | r.x << digit_shift(PASS - 1);
        if (tid == 0) a.found[(size_t)bh * 3 + PASS - 1] = make_uint2(found, r.y);       // (every span of the head writes the same)
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SP_EACH; ++k)
        if (s.in[k] && (s.u[k] & known_bits(PASS)) == found) atomicAdd(&sm_hist[digit(s.u[k], PASS)], 1u);
    __syncthreads();
    uint32_t* const hist = a.hist + ((size_t)bh * 3 + PASS) * KQ_BINS;
    for (int i = tid; i < KQ_BINS; i += SP_BLK)
        if (sm_hist[i]) atomicAdd(&hist[i], sm_hist[i]);
}

// How many rows of a span stay for certain, and how many keys are the k-th's equals.
__global__ __launch_bounds__(SP_BLK) void kvq_evict_count_kernel(EvictArgs a)
{
    __shared__ uint32_t sm_wave[SP_WAVES], sm_found[2], sm_more[SP_WAVES];
    const int2 span = a.spans[blockIdx.x];
    const int bh = span.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const hc_kvq_head from = a.heads[bh];
    const Keep x = keep_of(from, a.to[bh], a.state[bh]);
    if (x.m == x.n || span.y >= x.n) return;
    SpanKeys s;
    span_keys(a, from, x, span.y, s);
    uint32_t key = ~0u;
    if (x.k > 0) {
        const uint2 last = a.found[(size_t)bh * 3 + 1];
        const uint2 r = span_find(a, bh, 2, last.y, sm_wave, sm_found);
        key = last.x | r.x;
        if (tid == 0) a.found[(size_t)bh * 3 + 2] = make_uint2(key, r.y);
    }
    uint32_t larger = 0, equal = 0;
#pragma unroll
    for (int k = 0; k < SP_EACH; ++k) {
        const int r = span.y + w * 64 * SP_EACH + 64 * k + lane;
        larger += __popcll(__builtin_amdgcn_ballot_w64(r < x.n && (!s.in[k] || s.u[k] > key)));
        equal += __popcll(__builtin_amdgcn_ballot_w64(s.in[k] && s.u[k] == key));
    }
    __syncthreads();
    if (lane == 0) {
        sm_wave[w] = larger;
        sm_more[w] = equal;
    }
    __syncthreads();
    if (tid == 0) {
        for (int i = 1; i < SP_WAVES; ++i) {
            larger += sm_wave[i];
            equal += sm_more[i];
        }
        a.counts[blockIdx.x] = make_uint2(larger, equal);
    }
}

// The rows of a span that stay, to their places.
__global__ __launch_bounds__(SP_BLK) void kvq_evict_place_kernel(EvictArgs a)
{
    __shared__ uint32_t sm_wave[SP_WAVES], sm_more[SP_WAVES];
    __shared__ uint16_t sm_list[KQ_SPAN];
    const int2 span = a.spans[blockIdx.x];
    const int bh = span.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const hc_kvq_head from = a.heads[bh], to = a.to[bh];
    const int2 st = a.state[bh];
    const Keep x = keep_of(from, to, st);
    if (span.y >= x.n) {
        if (span.y == 0 && tid == 0) a.to_state[bh] = make_int2(x.m, st.y);
        return;
    }
    int count, at;                                               // rows of this span that stay; the first one's place
    if (x.m == x.n) {
        count = min(KQ_SPAN, x.n - span.y);
        at = span.y;
        for (int i = tid; i < count; i += SP_BLK) sm_list[i] = (uint16_t)i;
    } else {
        // what the head's spans before this one keep
        const int index = span.y / KQ_SPAN;
        const uint2 last = x.k > 0 ? a.found[(size_t)bh * 3 + 2] : make_uint2(~0u, 0u);
        const uint2 mine = tid < index ? a.counts[blockIdx.x - index + tid] : make_uint2(0u, 0u);
        SpanKeys s;
        span_keys(a, from, x, span.y, s);
        uint32_t larger = mine.x, equal = mine.y;
        for (int i = tid + SP_BLK; i < index; i += SP_BLK) {
            const uint2 c = a.counts[blockIdx.x - index + i];
            larger += c.x;
            equal += c.y;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            larger += __shfl_xor(larger, d);
            equal += __shfl_xor(equal, d);
        }
        if (lane == 0) {
            sm_wave[w] = larger;
            sm_more[w] = equal;
        }
        __syncthreads();
        uint32_t ties = 0, before = 0;
        for (int i = 0; i < SP_WAVES; ++i) {
            before += sm_wave[i];
            ties += sm_more[i];
        }
        before += min(ties, last.y);
        __syncthreads();
        larger = equal = 0;
#pragma unroll
        for (int k = 0; k < SP_EACH; ++k) {
            const int r = span.y + w * 64 * SP_EACH + 64 * k + lane;
            larger += __popcll(__builtin_amdgcn_ballot_w64(r < x.n && (!s.in[k] || s.u[k] > last.x)));
            equal += __popcll(__builtin_amdgcn_ballot_w64(s.in[k] && s.u[k] == last.x));
        }
        if (lane == 0) {
            sm_wave[w] = larger;
            sm_more[w] = equal;
        }
        __syncthreads();
        const uint32_t ties0 = ties;
        uint32_t here = 0, all = 0, all_ties = ties;
        for (int i = 0; i < SP_WAVES; ++i) {
            if (i < w) {
                here += sm_wave[i];
                ties += sm_more[i];
            }
            all += sm_wave[i];
            all_ties += sm_more[i];
        }
        const uint32_t kept0 = min(ties0, last.y);
        here += min(ties, last.y) - kept0;
        count = (int)(all + min(all_ties, last.y) - kept0);
        at = (int)before;
        const uint64_t below = (1ull << lane) - 1;
#pragma unroll
        for (int k = 0; k < SP_EACH; ++k) {
            const int i = w * 64 * SP_EACH + 64 * k + lane, r = span.y + i;
            const uint64_t eq = __builtin_amdgcn_ballot_w64(s.in[k] && s.u[k] == last.x);
            const bool stays = r < x.n && (!s.in[k] || s.u[k] > last.x || (s.u[k] == last.x && ties + __popcll(eq & below) < last.y));
            const uint64_t some = __builtin_amdgcn_ballot_w64(stays);
            if (stays) sm_list[here + __popcll(some & below)] = (uint16_t)i;
            here += __popcll(some);
            ties += __popcll(eq);
        }
    }
    __syncthreads();
    if (span.y == 0 && tid == 0) a.to_state[bh] = make_int2(x.m, st.y);
    if (a.list)
        for (int i = tid; i < count; i += SP_BLK) a.list[to.row_off + at + i] = span.y + sm_list[i];
    const uint8_t* const src = a.arena + from.off;
    uint8_t* const dst = a.to_arena + to.off;
    const int part = tid & 3;
    constexpr int AT_ONCE = 4;
    for (int q0 = 0; q0 < count; q0 += AT_ONCE * SP_BLK / 4) {
        MovedRow r[AT_ONCE];
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int q = q0 + e * SP_BLK / 4 + (tid >> 2);
            if (q < count) r[e] = take_row(src, from, span.y + sm_list[q], part, a.acc);
        }
#pragma unroll
        for (int e = 0; e < AT_ONCE; ++e) {
            const int q = q0 + e * SP_BLK / 4 + (tid >> 2);
            if (q < count) put_row(r[e], dst, to, at + q, part, a.to_acc);
        }
    }
}

constexpr int MV_BLK = 256, MV_ROWS = 64;

// The rows that stay, to their places.
__global__ __launch_bounds__(MV_BLK) void kvq_move_kernel(EvictArgs a)
{
    const int bh = blockIdx.y, tid = threadIdx.x;
    const int m = a.to_state[bh].x, j = blockIdx.x * MV_ROWS + (tid >> 2);
    if (j >= m) return;
    const hc_kvq_head from = a.heads[bh], to = a.to[bh];
    const MovedRow r = take_row(a.arena + from.off, from, a.list[(a.list_is_to ? to.row_off : from.row_off) + j], tid & 3, a.acc);
    put_row(r, a.to_arena + to.off, to, j, tid & 3, a.to_acc);
}

// ---- host ---------------------------------------------------------------------------------------------------------------------------------

bool kvq_ok(const hc_kvq* k) { return k && k->magic == HC_KVQ_MAGIC; }

// Kernels run on the current device, and what they are handed is the context's.
hc_status device_check(hc_ctx* ctx, const char* who)
{
    int now = -1;
    HC_HIP(ctx, hipGetDevice(&now));
    return now == ctx->device ? HC_OK : hc_fail(ctx, HC_ESTATE, "%s: the context is device %d's, the current one is %d", who, ctx->device, now);
}

// The cache, its state and its tables as a call is handed them.
hc_status cache_check(hc_ctx* ctx, const char* who, const hc_kvq* kvq, const void* arena, const int32_t* state, const float* acc, bool need_acc)
{
    if (!kvq_ok(kvq) || kvq->ctx != ctx) return hc_fail(ctx, HC_ESTATE, "%s: not a cache of this context", who);
    if (!arena || !state || (need_acc && !acc)) return hc_fail(ctx, HC_EINVAL, "%s: null pointer", who);
    if ((uintptr_t)arena & 63) return hc_fail(ctx, HC_EINVAL, "%s: the cache must be 64-byte aligned", who);
    if (((uintptr_t)state & 7) || ((uintptr_t)acc & 3)) return hc_fail(ctx, HC_EINVAL, "%s: misaligned state or weights", who);
    return device_check(ctx, who);
}

bool overlap(const void* a, size_t na, const void* b, size_t nb)
{
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

// Calls `launch` with the tokens of as many sequences at a time as a launch's arguments have room for.
template <typename F>
hc_status rows_launches(const hc_kvq* kvq, RowsArgs& a, const int32_t* first, const int32_t* count, const int64_t* k_off, const int64_t* v_off, void* state, F launch)
{
    const hc_config& c = kvq->ctx->cfg;
    a.Hkv = c.Hkv;
    a.even = 1;
    for (int i = 0; i < kvq->n && a.even; ++i) {
        const int h = i % c.Hkv, i0 = i - h;
        a.even = h < 2 || (k_off[i] - k_off[i0] == h * (k_off[i0 + 1] - k_off[i0]) && v_off[i] - v_off[i0] == h * (v_off[i0 + 1] - v_off[i0]));
    }
    const int most = a.even ? RW_SEQS : std::min(RW_SEQS, RW_HEADS / c.Hkv);
    for (int b0 = 0; b0 < c.B; b0 += most) {
        a.n_seq = std::min(most, c.B - b0);
        long long tokens = 0;
        int longest = 0;
        for (int i = 0; i < a.n_seq; ++i) {
            tokens += count[b0 + i];
            longest = std::max(longest, count[b0 + i]);
            a.end[i] = (int)tokens;
            a.first[i] = first[b0 + i];
        }
        if (tokens == 0) continue;
        for (int i = 0; i < a.n_seq * (a.even ? 1 : c.Hkv); ++i) {
            const int at = b0 * c.Hkv + (a.even ? i * c.Hkv : i);
            if (!a.even) {
                a.off[2 * i] = k_off[at];
                a.off[2 * i + 1] = v_off[at];
                continue;
            }
            a.off[4 * i] = k_off[at];
            a.off[4 * i + 2] = v_off[at];
            a.off[4 * i + 1] = c.Hkv > 1 ? k_off[at + 1] - k_off[at] : 0;
            a.off[4 * i + 3] = c.Hkv > 1 ? v_off[at + 1] - v_off[at] : 0;
        }
        a.heads = kvq->heads + (size_t)b0 * c.Hkv;
        a.state = (int2*)state + (size_t)b0 * c.Hkv;
        a.tokens = (int)tokens;
        a.whole = longest <= RW_TOKENS;
        const hc_status s = launch(dim3((unsigned)(a.whole ? a.n_seq : (tokens + RW_TOKENS - 1) / RW_TOKENS), (unsigned)c.Hkv));
        if (s != HC_OK) return s;
    }
    return HC_OK;
}

}   // namespace

extern "C" hc_status hc_kvq_create(hc_ctx* ctx, const hc_kvq_head* heads, hc_kvq** out)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    if (!heads || !out) return hc_fail(ctx, HC_EINVAL, "hc_kvq_create: null argument");
    *out = nullptr;
    const hc_status here = device_check(ctx, "hc_kvq_create");
    if (here != HC_OK) return here;
    const int n = ctx->cfg.B * ctx->cfg.Hkv;
    int64_t bytes = 0, rows = 0, units = 0;
    int32_t most = 0;
    for (int i = 0; i < n; ++i) {
        const hc_kvq_head& h = heads[i];
        if (h.cap < 16 || h.cap % 16 != 0 || h.cap > ctx->cfg.max_ctx)
            return hc_fail(ctx, HC_ESHAPE, "hc_kvq_create: head %d: cap %d must be a multiple of 16, 16 .. max_ctx", i, (int)h.cap);
        if (h.off < 0 || (h.off & 63) || h.off > ((int64_t)1 << 50) || h.row_off < 0 || h.row_off > ((int64_t)1 << 45))
            return hc_fail(ctx, HC_EINVAL, "hc_kvq_create: head %d: off must be a multiple of 64 bytes, and neither it nor row_off negative", i);
        // (sink and recent may be more than a head has rows: then all stay.  Rows less both of them are a number of 32 bits.)
        if (h.sink < 0 || h.sink > 1 << 30 || h.recent < 0 || h.recent > 1 << 30 || h.budget < 1 || h.budget > h.cap)
            return hc_fail(ctx, HC_EINVAL, "hc_kvq_create: head %d: budget %d of %d rows, sink %d, recent %d", i, (int)h.budget, (int)h.cap, (int)h.sink, (int)h.recent);
        bytes = std::max(bytes, h.off + (int64_t)136 * h.cap);
        rows = std::max(rows, h.row_off + h.cap);
        units += (h.cap + KQ_TILE - 1) / KQ_TILE;
        most = std::max(most, h.cap);
    }
    if (units + (int64_t)n * 64 > INT_MAX) return hc_fail(ctx, HC_ESHAPE, "hc_kvq_create: more rows than one call takes");
    hc_kvq* k = new (std::nothrow) hc_kvq();
    if (!k) return hc_fail(ctx, HC_ENOMEM, "host allocation failed");
    std::vector<int> order;
    std::vector<int2> chunks, spans;
    std::vector<int2> room;
    int bad = -1;
    try {
        k->host.assign(heads, heads + n);
        for (int i = 0; i < n; ++i) {
            order.push_back(i);
            room.push_back(make_int2(heads[i].cap, i == 0 ? 0 : room[i - 1].y + (heads[i - 1].cap + KQ_TILE - 1) / KQ_TILE));
            for (int r = 0; r < heads[i].cap; r += KQ_CHUNK) chunks.push_back(make_int2(i, r));
            for (int r = 0; r < heads[i].cap; r += KQ_SPAN) spans.push_back(make_int2(i, r));
        }
    } catch (const std::bad_alloc&) {
        delete k;
        return hc_fail(ctx, HC_ENOMEM, "host allocation failed");
    }
    std::sort(order.begin(), order.end(), [&](int a, int b) { return heads[a].off < heads[b].off; });
    for (int i = 1; i < n; ++i)
        if (heads[order[i - 1]].off + (int64_t)136 * heads[order[i - 1]].cap > heads[order[i]].off) bad = order[i];
    std::sort(order.begin(), order.end(), [&](int a, int b) { return heads[a].row_off < heads[b].row_off; });
    for (int i = 1; i < n; ++i)
        if (heads[order[i - 1]].row_off + heads[order[i - 1]].cap > heads[order[i]].row_off) bad = order[i];
    if (bad >= 0) {
        delete k;
        return hc_fail(ctx, HC_EINVAL, "hc_kvq_create: head %d: its block or its rows overlap another head's", bad);
    }
    k->magic = HC_KVQ_MAGIC;
    k->ctx = ctx;
    k->n = n;
    k->max_cap = most;
    k->bytes = bytes;
    k->rows = rows;
    k->units = units;
    k->n_chunks = (int)chunks.size();
    k->n_spans = (int)spans.size();
    auto upload = [&](const void* from, size_t size, void** to) {
        hipError_t e = hipMalloc(to, size);
        return e == hipSuccess ? hipMemcpy(*to, from, size, hipMemcpyHostToDevice) : e;
    };
    hipError_t e = upload(heads, (size_t)n * sizeof(hc_kvq_head), (void**)&k->heads);
    if (e == hipSuccess) e = upload(room.data(), (size_t)n * sizeof(int2), (void**)&k->room);
    if (e == hipSuccess) e = upload(chunks.data(), chunks.size() * sizeof(int2), (void**)&k->chunks);
    if (e == hipSuccess) e = upload(spans.data(), spans.size() * sizeof(int2), (void**)&k->spans);
    if (e != hipSuccess) {
        (void)hc_kvq_destroy(k);
        return hc_hip_fail(ctx, e, "hc_kvq_create");
    }
    *out = k;
    return HC_OK;
}

extern "C" hc_status hc_kvq_destroy(hc_kvq* k)
{
    if (!kvq_ok(k)) return HC_ESTATE;
    (void)hipFree(k->heads);
    (void)hipFree(k->room);
    (void)hipFree(k->chunks);
    (void)hipFree(k->spans);
    k->magic = 0;
    delete k;
    return HC_OK;
}

extern "C" size_t hc_kvq_work_bytes(const hc_ctx* ctx, const hc_kvq* kvq)
{
    return hc_ctx_ok(ctx) && kvq_ok(kvq) && kvq->ctx == ctx ? hc_kvq_plan(kvq).bytes : 0;
}

extern "C" hc_status hc_kvq_store(hc_ctx* ctx, const hc_kvq* kvq, const void* kv_prefill, const int64_t* k_off, const int64_t* v_off, const int32_t* first,
                                  const int32_t* count, void* arena, int32_t* state, float* acc, void* stream)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    hc_status s = cache_check(ctx, "hc_kvq_store", kvq, arena, state, acc, false);
    long long tokens = 0;
    if (s == HC_OK) s = hc_check_chunk(ctx, "hc_kvq_store", kv_prefill, k_off, v_off, first, count, &tokens);
    if (s != HC_OK || tokens == 0) return s;
    RowsArgs a{};
    a.arena = (uint8_t*)arena;
    a.kv = (uint16_t*)kv_prefill;
    hipStream_t st = (hipStream_t)stream;
    a.acc = acc;
    return rows_launches(kvq, a, first, count, k_off, v_off, state, [&](dim3 grid) -> hc_status {
        kvq_store_kernel<<<grid, dim3(RW_BLK), 0, st>>>(a);
        HC_HIP(ctx, hipGetLastError());
        if (!a.whole) {
            kvq_count_kernel<<<dim3(1), dim3(RW_BLK), 0, st>>>(a);
            HC_HIP(ctx, hipGetLastError());
        }
        return HC_OK;
    });
}

extern "C" hc_status hc_kvq_load(hc_ctx* ctx, const hc_kvq* kvq, const void* arena, const int32_t* state, const int32_t* first, const int32_t* count,
                                 void* kv_out, const int64_t* k_off, const int64_t* v_off, void* stream)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    hc_status s = cache_check(ctx, "hc_kvq_load", kvq, arena, state, nullptr, false);
    long long tokens = 0;
    if (s == HC_OK) s = hc_check_chunk(ctx, "hc_kvq_load", kv_out, k_off, v_off, first, count, &tokens);
    if (s != HC_OK || tokens == 0) return s;
    RowsArgs a{};
    a.arena = (uint8_t*)const_cast<void*>(arena);
    a.kv = (uint16_t*)kv_out;
    hipStream_t st = (hipStream_t)stream;
    return rows_launches(kvq, a, first, count, k_off, v_off, const_cast<int32_t*>(state), [&](dim3 grid) -> hc_status {
        kvq_load_kernel<<<grid, dim3(RW_BLK), 0, st>>>(a);
        HC_HIP(ctx, hipGetLastError());
        return HC_OK;
    });
}

extern "C" hc_status hc_kvq_append(hc_ctx* ctx, const hc_kvq* kvq, const hc_rope* rope, const void* q, const void* k, const void* v, int64_t q_stride,
                                   int64_t k_stride, int64_t v_stride, int32_t in_type, void* q_out, void* arena, int32_t* state, float* acc, void* stream)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    const hc_rows_in in{q, k, v, q_stride, k_stride, v_stride, in_type == HC_F32};
    hc_status s = cache_check(ctx, "hc_kvq_append", kvq, arena, state, acc, false);
    if (s == HC_OK) s = hc_check_rope(ctx, "hc_kvq_append", rope, in, in_type, q_out);
    if (s != HC_OK) return s;
    TokenArgs a{};
    for (int i = 0; i < rope->rot_dim / 2; ++i) a.turns[i] = rope->freq[i] * (0.5 / M_PI);
    a.q_norm = rope->q_norm;
    a.k_norm = rope->k_norm;
    a.eps = rope->eps;
    a.gain = rope->gain;
    a.rot = rope->rot_dim;
    a.half = rope->layout == HC_ROPE_HALF;
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out = (uint16_t*)q_out;
    a.arena = (uint8_t*)arena;
    a.heads = kvq->heads;
    a.state = (int2*)state;
    a.acc = acc;
    a.Hkv = ctx->cfg.Hkv;
    a.G = ctx->G;
    const dim3 grid((unsigned)kvq->n), block((unsigned)token_threads(ctx->G));
    if (in.f32) kvq_append_kernel<true><<<grid, block, 0, (hipStream_t)stream>>>(a);
    else kvq_append_kernel<false><<<grid, block, 0, (hipStream_t)stream>>>(a);
    HC_HIP(ctx, hipGetLastError());
    return HC_OK;
}

extern "C" hc_status hc_kvq_attn(hc_ctx* ctx, const hc_kvq* kvq, const void* arena, const int32_t* state, const void* q, float* out, float* lse, float* acc,
                                 float decay, void* work, size_t work_bytes, void* stream)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    const hc_status s = cache_check(ctx, "hc_kvq_attn", kvq, arena, state, acc, false);
    if (s != HC_OK) return s;
    if (!q || !out || !lse || !work) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: null pointer");
    if (((uintptr_t)q | (uintptr_t)out) & 15) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: q and out must be 16-byte aligned");
    if ((uintptr_t)lse & 3) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: misaligned float pointer");
    const size_t rows = (size_t)ctx->cfg.B * ctx->cfg.Hq;
    if (overlap(q, rows * HC_D * 2, out, rows * HC_D * 4)) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: out overlaps q");       // (others' queries are read meanwhile)
    if (acc && !(decay >= 0.f && decay <= 1.f)) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: decay must be 0 .. 1");
    if ((uintptr_t)work & 255) return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: work must be 256-byte aligned");
    if (work_bytes < hc_kvq_plan(kvq).bytes)
        return hc_fail(ctx, HC_EINVAL, "hc_kvq_attn: work buffer of %zu bytes, %zu needed", work_bytes, hc_kvq_plan(kvq).bytes);
    return hc_launch_kvq_attn(ctx, kvq, arena, state, q, out, lse, acc, decay, work, (hipStream_t)stream);
}

extern "C" hc_status hc_kvq_evict(hc_ctx* ctx, const hc_kvq* kvq, const void* arena, const int32_t* state, const float* acc, const hc_kvq* to, void* to_arena,
                                  int32_t* to_state, float* to_acc, int32_t* kept, void* work, size_t work_bytes, void* stream)
{
    if (!hc_ctx_ok(ctx)) return HC_ESTATE;
    hc_status s = cache_check(ctx, "hc_kvq_evict", kvq, arena, state, acc, true);
    if (s == HC_OK) s = cache_check(ctx, "hc_kvq_evict", to, to_arena, to_state, to_acc, true);
    if (s != HC_OK) return s;
    if ((uintptr_t)kept & 3) return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: misaligned list");
    const size_t nh = (size_t)kvq->n * 8;
    if (overlap(arena, (size_t)kvq->bytes, to_arena, (size_t)to->bytes) || overlap(state, nh, to_state, nh) ||
        overlap(acc, (size_t)kvq->rows * 4, to_acc, (size_t)to->rows * 4))
        return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: the two caches, their states or their weights overlap");
    if (!work) return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: null pointer");
    if ((uintptr_t)work & 255) return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: work must be 256-byte aligned");
    if (work_bytes < hc_kvq_plan(kvq).bytes)
        return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: work buffer of %zu bytes, %zu needed", work_bytes, hc_kvq_plan(kvq).bytes);
    int32_t most = 1;
    for (int i = 0; i < kvq->n; ++i) {
        const hc_kvq_head& h = to->host[i];
        if (h.budget < std::min((int64_t)kvq->host[i].cap, (int64_t)h.sink + h.recent))
            return hc_fail(ctx, HC_EINVAL, "hc_kvq_evict: head %d: a budget of %d rows has no room for sink %d and recent %d", i, (int)h.budget, (int)h.sink, (int)h.recent);
        most = std::max(most, std::min(h.budget, kvq->host[i].cap));
    }
    hipStream_t st = (hipStream_t)stream;
    const hc_kvq_layout l = hc_kvq_plan(kvq);
    char* const w = (char*)work;
    EvictArgs a{kvq->heads, to->heads, (const int2*)state, (int2*)to_state, acc, to_acc, (const uint8_t*)arena, (uint8_t*)to_arena, kept, 1, kvq->spans,
                (uint32_t*)(w + l.hist), (uint2*)(w + l.found), (uint2*)(w + l.counts)};
    const dim3 heads((unsigned)kvq->n);
    if (kvq->max_cap <= KQ_SHORT) {
        if (!kept) {
            a.list = (int32_t*)(w + l.list);
            a.list_is_to = 0;
        }
        kvq_select_kernel<<<heads, dim3(EV_BLK), 0, st>>>(a);
        HC_HIP(ctx, hipGetLastError());
        for (int h0 = 0; h0 < kvq->n; h0 += 65535) {
            EvictArgs m = a;
            m.heads += h0;
            m.to += h0;
            m.to_state += h0;
            kvq_move_kernel<<<dim3((unsigned)((most + MV_ROWS - 1) / MV_ROWS), (unsigned)std::min(65535, kvq->n - h0)), dim3(MV_BLK), 0, st>>>(m);
            HC_HIP(ctx, hipGetLastError());
        }
        return HC_OK;
    }
    const dim3 spans((unsigned)kvq->n_spans), block(SP_BLK);
    kvq_evict_clear_kernel<<<heads, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_evict_digit_kernel<0><<<spans, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_evict_digit_kernel<1><<<spans, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_evict_digit_kernel<2><<<spans, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_evict_count_kernel<<<spans, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_evict_place_kernel<<<spans, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    return HC_OK;
}
