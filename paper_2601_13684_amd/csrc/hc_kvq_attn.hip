// hc_kvq_attn.hip -- attention of the decode token over the cache held in 4 bits (its format: hc_kvq.h), and every row's share of the weights.
//
//   s_j = q . K[j],   p_j = 2^((s_j - m) log2(e) / sqrt(128)),   out = sum_j p_j V[j] / sum_j p_j,   lse = m / sqrt(128) + ln sum_j p_j
//   acc_j <- decay acc_j + (1/G) sum_g p_gj / sum_i p_gi
//
// References m are logits as they leave the first product, not scaled: a difference of two is off by half a step of its own, whatever their size, and is scaled
// after it.  (A scaled logit's rounding is a step of the logit's: from 2^31 binary orders on more than the exponents hold, so that the row's own weight would be
// infinite, or nothing.)
//
// A workgroup takes an equal share of the tiles of 32 rows of all heads one after the other; lengths are on the device, and each
// wave finds its share by itself.  A wave takes whole tiles, the next one on its way to LDS (asynchronous loads, five to a tile of 4,352 bytes; straight to
// registers they were twenty, and 224K rows took 48 us) under the present one's arithmetic; waves meet at a head's end alone.  S^T = K Q^T and O^T = V^T P^T on the matrix cores (16x16x32), keys along S^T's rows, so that the lane that has a
// weight is the lane that hands it to the second product, and the products' order of the keys is chosen (row 4 x + y of the first is key
// 4 y + x) so that a load of V takes four rows side by side.
//   K   a lane's 16 bytes are 32 values of one scale: what the first product's four steps take; q is laid out alike
//   V   a lane's dword is 8 values of one row; of 8 rows they become, two by two, operands of 8 tiles of 16 values
// Codes become bf16 exactly.  The matrix cores have 16 columns for a group of at most 8 query heads: the others take what the rounding of the weights to
// bf16 leaves, in two steps, so that the weights lose nothing (8 + 8 + 8 bits): columns g, G + g, 2 G + g for the parts of query head g, added at the end.
// Groups of eight take a second product for the last part.
//
// Bound by memory where rows are many: 224K rows of eight heads 39.6 us (250 MB, 6.3 TB/s; a plain read of 1 GiB runs at 5.9) and 4.6 for the partial results, the
// products and the codes' conversion, 222 vector instructions a tile, all but hidden; in groups of eight 43 us.  With weights 45.1 +
// 12.0: logits go through memory, 32 bytes a row in groups of four against 136 for the row.  Two such heads and six of 1,024 to 8,192 rows 14.0 + 5.8, with weights
// 15.5 + 6.4; 16 ragged sequences of 1 to 32K rows, four heads in groups of eight, with weights 21.5 + 9.8: about 5 us of either pass are launch, the search for its
// share and the first loads.  512 heads of 4,096 rows 50.5 + 4.2 us (285 MB).  Few rows: 500 rows of two heads 6.0 us in one launch.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "hc_kvq.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

constexpr int KA_BLK = 256, KA_WAVES = KA_BLK / 64;
constexpr float KA_SCALE = (float)(1.4426950408889634 * 0.08838834764831845);      // log2(e) / sqrt(128)
constexpr float KA_ROOT = 0.08838834764831845f;      // 1 / sqrt(128)
constexpr float KA_LN2 = 0.6931471805599453f;
constexpr float KA_SLACK = 62.0f;            // a logit is at most this far above the reference before that moves: its weight is then below 2^8
constexpr int KA_LEAST = KA_WAVES;           // tiles of a workgroup, where there are so few
// What beginning a head costs a workgroup, in tiles.  us of the split pass with 6, 12 / 16 / 20, 28: 16 ragged sequences in groups of eight 22.5, 19.7 / 19.7 / 19.7, 19.9, with
// weights 23.4, 21.8 / 21.7 / 21.6, 21.9; two heads of 224K rows and six short ones 15.0, 14.2 / 14.2 / 14.0, 14.0.
constexpr int KA_START = 16;

struct AttnArgs {
    const uint8_t* arena;
    const int2* state;
    const hc_kvq_head* heads;
    const int2* room;
    const uint16_t* q;
    float *part_ml, *part_o;                 // [slots][G][2], [slots][G][128]
    int2* plan;                              // [n]: first slot of the head's partial results, and how many; of heads with rows
    float* logits;                           // q . K, [tiles of the caps][8][G][4], or nullptr: place 2 x + y, z of a tile is row 16 y + 4 z + x
    int n;
};

__device__ __forceinline__ int tiles_of(int rows) { return (rows + KQ_TILE - 1) / KQ_TILE; }

// The work is a line on which every head with rows has KA_START places and then one for each of its tiles; workgroup i has the share [i per, (i + 1) per) of it.
__device__ __forceinline__ int places_of(int rows) { return rows > 0 ? KA_START + tiles_of(rows) : 0; }
__device__ __forceinline__ int share(int places, int workgroups) { return max(KA_LEAST, (places + workgroups - 1) / workgroups); }

__device__ __forceinline__ float weight(float s, float ref) { return __builtin_amdgcn_exp2f((s - ref) * KA_SCALE); }
// What sums of reference `ref` come to for reference `top`.
__device__ __forceinline__ float moved(float ref, float top) { return exp2f((ref - top) * KA_SCALE); }
__device__ __forceinline__ float lse_of(float ref, float l) { return l == 0.f ? -INFINITY : fmaf(ref, KA_ROOT, log2f(l) * KA_LN2); }

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
// Sum over the columns of a row of 16 that hold the parts of one query head.
template <int G>
__device__ __forceinline__ float sum_parts(float x)
{
    x = dpp_add<0x128>(x);                   // rotate by 8
    if (G <= 4) x = dpp_add<0x124>(x);       // by 4
    if (G <= 2) x = dpp_add<0x122>(x);
    if (G <= 1) x = dpp_add<0x121>(x);
    return x;
}

// A tile in LDS: K's codes, V's, K's scales, V's.  K's 16-byte chunk c of row r is at place c ^ (r / 4 % 4) of the row's 64 bytes, so that the 16 lanes
// of a phase of the reads (one chunk of 16 rows) go over all banks; the scales of row 4 x + y are at place 8 y + x, so that the eight that a lane takes for V
// lie side by side.
constexpr int T_V = 2048, T_KS = 4096, T_VS = T_KS + 128, T_BYTES = T_VS + 128;
constexpr int KS_BUFS = 4;                   // most buffers of a wave
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

// What a lane reads of a tile.
struct Tile {
    u32x4 k[2];                              // codes and scale of K's rows 16 s + 4 (col % 4) + col / 4
    uint32_t ks[2];
    u32x2 v[4];                              // codes and four scales of V's rows 4 i + grp, i = 0 .. 7
    u32x4 vs[2];
};
// Reads it from buffer BUF once all but `later` of the wave's loads have arrived.  One block with its wait at the end: the compiler does not tell a read of one
// buffer from the loads into the next ones, and would wait for all of them.
template <int BUF, int later>
__device__ __forceinline__ void read_tile(Tile& x, uint32_t k_at, uint32_t s_at, uint32_t v_at, uint32_t f_at)
{
    asm volatile(
        "s_waitcnt vmcnt(%14)\n\t"
        "ds_read_b128 %0, %10 offset:%15\n\t"
        "ds_read_u8 %2, %11 offset:%17\n\t"
        "ds_read_b128 %1, %10 offset:%16\n\t"
        "ds_read_u8 %3, %11 offset:%18\n\t"
        "ds_read2st64_b32 %4, %12 offset0:%19 offset1:%20\n\t"
        "ds_read2st64_b32 %5, %12 offset0:%21 offset1:%22\n\t"
        "ds_read2st64_b32 %6, %12 offset0:%23 offset1:%24\n\t"
        "ds_read2st64_b32 %7, %12 offset0:%25 offset1:%26\n\t"
        "ds_read_b128 %8, %13 offset:%27\n\t"
        "ds_read_b128 %9, %13 offset:%28\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x.k[0]), "=&v"(x.k[1]), "=&v"(x.ks[0]), "=&v"(x.ks[1]), "=&v"(x.v[0]), "=&v"(x.v[1]), "=&v"(x.v[2]), "=&v"(x.v[3]), "=&v"(x.vs[0]), "=&v"(x.vs[1])
        : "v"(k_at), "v"(s_at), "v"(v_at), "v"(f_at), "n"(later), "n"(BUF * T_BYTES), "n"(BUF * T_BYTES + 1024), "n"(BUF * T_BYTES + T_KS),
          "n"(BUF * T_BYTES + T_KS + 16), "n"((BUF * T_BYTES + T_V) / 256), "n"((BUF * T_BYTES + T_V) / 256 + 1), "n"((BUF * T_BYTES + T_V) / 256 + 2),
          "n"((BUF * T_BYTES + T_V) / 256 + 3), "n"((BUF * T_BYTES + T_V) / 256 + 4), "n"((BUF * T_BYTES + T_V) / 256 + 5), "n"((BUF * T_BYTES + T_V) / 256 + 6),
          "n"((BUF * T_BYTES + T_V) / 256 + 7), "n"(BUF * T_BYTES + T_VS), "n"(BUF * T_BYTES + T_VS + 16)
        : "memory");
}
static_assert(T_BYTES % 256 == 0 && T_V % 256 == 0 && KS_BUFS * T_BYTES / 256 < 256, "offsets of the reads");

// One wave's part of a head: what it has of its queries and sums, and where its tiles go.
template <int G>
struct Wave {
    int lane, col, grp;
    int part;                                // of the weights that this column takes
    bool dead;
    uint32_t m1, m2;
    lds_char* lds;
    uint32_t k_read, s_read, v_read, f_read; // what the lane reads of a tile: K's rows 16 s + 4 (col % 4) + col / 4 and V's 4 i + grp
    const uint8_t* block;                    // the head's
    uint32_t cap, k_at, v_at, s_at, k_chunk, v_chunk, s_base;
    int n, c_row, s_row;
    bf16x8 Q[4];
    float ref;                               // of the weights
    f32x4 L;                                 // their sums, of the columns; four times the same
    f32x4 O[8];

    __device__ __forceinline__ explicit Wave(char* tiles)
    {
        lane = threadIdx.x & 63;
        col = lane & 15;
        grp = lane >> 4;
        part = G <= 4 ? col / G : col / 8;
        dead = part > 2;
        m1 = part >= 1 ? 0xffff0000u : 0u;
        m2 = part >= 2 ? 0xffff0000u : 0u;
        lds = (lds_char*)tiles;
        const uint32_t tile0 = (uint32_t)(uintptr_t)lds;
        k_read = tile0 + (4 * (col & 3) + (col >> 2)) * 64 + (grp ^ (col & 3)) * 16;
        s_read = tile0 + (8 * (col >> 2) + (col & 3)) * 4 + grp;
        v_read = tile0 + lane * 4;
        f_read = tile0 + grp * 32;
        asm("" : "+v"(k_read), "+v"(s_read), "+v"(v_read), "+v"(f_read));      // (opaque, so that a buffer goes into an instruction's offset)
        // what it loads: 16 bytes of codes of row lane / 4, and the scales of row 4 (lane % 8) + lane / 8 % 4, K's or V's
        c_row = lane >> 2;
        s_row = 4 * (lane & 7) + (lane >> 3 & 3);
        k_chunk = ((lane & 3) ^ (lane >> 4)) * 16;
        v_chunk = (lane & 3) * 16;
    }
    // The head to load from, and its queries.
    __device__ __forceinline__ void aim(const AttnArgs& a, int bh, int64_t off, uint32_t room, int rows)
    {
        block = a.arena + off;
        cap = room;
        n = rows;
        s_base = (lane < 32 ? 64u : 132u) * cap;
        k_at = c_row * 64 + k_chunk;
        v_at = 68 * cap + c_row * 64 + v_chunk;
        s_at = s_base + s_row * 4;
#pragma unroll
        for (int c = 0; c < 4; ++c) Q[c] = *reinterpret_cast<const bf16x8*>(a.q + ((size_t)bh * G + (col & (G - 1))) * HC_D + 32 * grp + 8 * c);
    }
    __device__ __forceinline__ void reset()
    {
        ref = dead ? FLT_MAX : -FLT_MAX;                     // (beside FLT_MAX a logit weighs nothing, or 1, of which the last part of the weights is nothing)
        L = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) O[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // The queries are there: waits after this count the tiles' loads alone.
    __device__ __forceinline__ void ready()
    {
#pragma unroll
        for (int c = 0; c < 4; ++c) asm volatile("" : "+v"(Q[c]));
    }
    // Tile t to buffer BUF; none from `end` on.
    template <int BUF, int NT>
    __device__ __forceinline__ void load(int t, int end) const
    {
        lds_char* const to = lds + BUF * T_BYTES;
        // (a tile behind the last is loaded from a buffer of no bytes, which costs no memory: the number of loads on their way is then always the same)
        // (the same for all lanes, which the compiler does not see across the parts of a share)
        const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)((uintptr_t)block >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uintptr_t)block);
        const int r0 = __builtin_amdgcn_readfirstlane(t * KQ_TILE);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)at, 0, __builtin_amdgcn_readfirstlane(t < end ? 136u * cap : 0u), 0x00027000);
        uint32_t k0 = k_at, k1 = k_at + 1024, v0 = v_at, v1 = v_at + 1024, s0 = s_at;
        if (r0 + KQ_TILE > n) {                              // rows behind the last repeat it; their weights and values become zeros
            const int last = max(n - 1 - r0, 0);
            k0 = min(c_row, last) * 64 + k_chunk;
            k1 = min(c_row + 16, last) * 64 + k_chunk;
            v0 = 68 * cap + min(c_row, last) * 64 + v_chunk;
            v1 = 68 * cap + min(c_row + 16, last) * 64 + v_chunk;
            s0 = s_base + min(s_row, last) * 4;
        }
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)to, 16, k0, r0 * 64, 0, NT);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + 1024), 16, k1, r0 * 64, 0, NT);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + T_KS), 4, s0, r0 * 4, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + T_V), 16, v0, r0 * 64, 0, NT);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(to + T_V + 1024), 16, v1, r0 * 64, 0, NT);
    }
    // Tile t from buffer BUF, all but LATER of the wave's loads and stores having arrived; S: its logits, q . K.
    template <int BUF, int LATER>
    __device__ __forceinline__ void add(int t, float* logits, f32x4 (&S)[2])
    {
        Tile x;
        read_tile<BUF, LATER>(x, k_read, s_read, v_read, f_read);
        uint32_t xv[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) xv[i] = x.v[i >> 1][i & 1];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            S[s] = f32x4{0.f, 0.f, 0.f, 0.f};
            const float f = kq_scale(x.ks[s]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const u32x4 k{kq_pair<0>(x.k[s][c], f), kq_pair<1>(x.k[s][c], f), kq_pair<2>(x.k[s][c], f), kq_pair<3>(x.k[s][c], f)};
                S[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), Q[c], S[s], 0, 0, 0);
            }
        }
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = kq_scale(__builtin_amdgcn_ubfe(x.vs[i >> 2][i & 3], (col >> 2) * 8, 8));
        const int r0 = t * KQ_TILE;
        if (logits && col < 2 * G)                           // (columns g and G + g have the same: 2 G lanes store half of the eight each)
            *reinterpret_cast<f32x4*>(logits + ((size_t)t * 8 + 2 * grp) * G * 4 + col * 4) = col < G ? S[0] : S[1];
        if (r0 + KQ_TILE > n) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + 4 * i + grp >= n) {
                    S[i >> 2][i & 3] = -INFINITY;
                    xv[i] = 0;
                    f[i] = 1.f;
                }
        }
        float p[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = S[i >> 2][i & 3] - ref;
            top = fmaxf(top, p[i]);
        }
        if (__builtin_amdgcn_ballot_w64(top > KA_SLACK)) {
            float y = S[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) y = fmaxf(y, S[i >> 2][i & 3]);
            y = fmaxf(y, __shfl_xor(y, 16));
            y = fmaxf(y, __shfl_xor(y, 32));
            y = fmaxf(y, ref);
            const float less = moved(ref, y);
            ref = y;
            L *= less;
#pragma unroll
            for (int j = 0; j < 8; ++j) O[j] *= less;
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = S[i >> 2][i & 3] - ref;
        }
        uint32_t P1[8], P2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(p[i] * KA_SCALE);
            const float r1 = e - __uint_as_float(__float_as_uint(e) & (G == 8 ? 0xffff0000u : m1));
            if (G == 8) {
                P1[i] = __float_as_uint(part ? r1 : e);
                P2[i] = part ? 0u : __float_as_uint(r1 - __uint_as_float(__float_as_uint(r1) & 0xffff0000u));
            } else {
                P1[i] = __float_as_uint(r1 - __uint_as_float(__float_as_uint(r1) & m2));
            }
        }
        u32x4 B1, B2;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            B1[i] = __builtin_amdgcn_perm(P1[2 * i + 1], P1[2 * i], 0x07060302u);
            if (G == 8) B2[i] = __builtin_amdgcn_perm(P2[2 * i + 1], P2[2 * i], 0x07060302u);
        }
        // the weights' sum is a product as well: with ones
        const u32x4 ones{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
        L = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, B1), L, 0, 0, 0);
        if (G == 8) L = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), __builtin_bit_cast(bf16x8, B2), L, 0, 0, 0);
        auto values = [&](auto byte) {
            constexpr int B = decltype(byte)::value;
            uint32_t c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = kq_pair<B>(xv[i], f[i]);
            u32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x05040100u);
                hi[i] = __builtin_amdgcn_perm(c[2 * i + 1], c[2 * i], 0x07060302u);
            }
            O[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), __builtin_bit_cast(bf16x8, B1), O[2 * B], 0, 0, 0);
            O[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, B1), O[2 * B + 1], 0, 0, 0);
            if (G == 8) {
                O[2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), __builtin_bit_cast(bf16x8, B2), O[2 * B], 0, 0, 0);
                O[2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), __builtin_bit_cast(bf16x8, B2), O[2 * B + 1], 0, 0, 0);
            }
        };
        values(std::integral_constant<int, 0>{});
        values(std::integral_constant<int, 1>{});
        values(std::integral_constant<int, 2>{});
        values(std::integral_constant<int, 3>{});
    }
    // The parts of a weight, and the groups of lanes, together: to ml [G][2] and o [G][128].
    __device__ __forceinline__ void finish(float (*ml)[2], float* o)
    {
        const float l = sum_parts<G>(L[0]);
        if (lane < G) {
            ml[lane][0] = ref;
            ml[lane][1] = l;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            f32x4 lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = sum_parts<G>(O[j][r]);
                hi[j] = sum_parts<G>(O[4 + j][r]);
            }
            if (col < G) {
                float* const to = o + col * HC_D + 8 * (4 * grp + r);
                *reinterpret_cast<f32x4*>(to) = lo;
                *reinterpret_cast<f32x4*>(to + 4) = hi;
            }
        }
    }
};
static_assert(HC_MAX_G * HC_D * sizeof(float) <= T_BYTES, "a wave's sums go through its first buffer");
constexpr int VMCNT0 = 0x0f70, VMCNT1 = 0x0f71, VMCNT5 = 0x0f75;                  // of s_waitcnt

// The waves' own LDS stores and reads are done, and all waves are here.  (__syncthreads would wait for the tiles on their way to LDS as well.)
__device__ __forceinline__ void meet()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");       // (nothing is moved across by the compiler)
    __builtin_amdgcn_s_waitcnt(0xc07f);                          // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int G, bool LOGITS>
__global__ __launch_bounds__(KA_BLK, KQ_WG_PER_CU) void kvq_attn_kernel(AttnArgs a)
{
    __shared__ float sm_ml[KA_WAVES][G][2];
    __shared__ __attribute__((aligned(16))) float sm_o[KA_WAVES][G][HC_D];
    __shared__ __attribute__((aligned(256))) char sm_tile[KA_WAVES][2][T_BYTES];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;

    // this workgroup's share, and the head that it begins in
    int window = 0, h_rows, h_cap, h_first;                      // a lane's of the 64 heads from `window` on
    int64_t h_off;
    auto look = [&]() {
        const int i = min(window + lane, a.n - 1);
        const int2 room = a.room[i];
        h_rows = min(max(a.state[i].x, 0), room.x);
        h_cap = room.x;
        h_first = room.y;
        h_off = a.heads[i].off;
    };
    look();
    const int each = (a.n + 63) / 64, mine0 = min(a.n, lane * each), mine1 = min(a.n, mine0 + each);
    int sum = 0;
    if (each == 1) sum = lane < a.n ? places_of(h_rows) : 0;
    else
        for (int i = mine0; i < mine0 + each; i += 8) {          // (eight at a time, so that their loads do not follow one another)
            int rows[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) rows[e] = kq_rows(a.state, a.room, min(i + e, a.n - 1));
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += i + e < mine1 ? places_of(rows[e]) : 0;
        }
    int upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    const int total = __builtin_amdgcn_readlane(upto, 63), per = share(total, (int)gridDim.x);
    const int u0 = (int)min((long long)total, (long long)blockIdx.x * per), u1 = min(total, u0 + per);
    if (u0 >= u1) return;
    const int owner = __popcll(__builtin_amdgcn_ballot_w64(upto <= u0));
    int bh = __builtin_amdgcn_readfirstlane(owner * each);
    int before = __builtin_amdgcn_readlane(upto - sum, owner);
    Wave<G> wave(&sm_tile[w][0][0]);
    // Codes are read once: marked so (2), unless the logits on their way to the next kernel share the caches with them.  us of this pass, marked / not:
    // 224K rows of eight heads, no logits 39.4 / 40.6, logits 52.1 / 45.5; two such heads and six short ones 14.0 / 14.9, 18.1 / 15.8.
    static constexpr int NT = LOGITS ? 0 : 2;
    int head = 0, t0 = 0, t1 = 0;                                // of the part at hand: tiles [t0, t1) of a head
    float* logits = nullptr;
    // The next part of the share: where it is, its queries' and its first tiles' loads.
    auto next = [&]() -> bool {
        for (; before < u1 && bh < a.n; ++bh) {
            if (bh >= window + 64) {
                window = bh;
                look();
            }
            const int n = __builtin_amdgcn_readlane(h_rows, bh - window), tiles = tiles_of(n), begin = before + KA_START;
            before += places_of(n);
            t0 = max(u0 - begin, 0);
            t1 = min(tiles, u1 - begin);
            if (t0 >= t1) continue;
            head = bh;
            if (t0 == 0 && tid == 0) a.plan[bh] = make_int2((int)blockIdx.x + bh, (begin + tiles - 1) / per - (int)blockIdx.x + 1);
            const int64_t off = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(h_off >> 32), bh - window) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)h_off, bh - window));
            wave.aim(a, bh, off, (uint32_t)__builtin_amdgcn_readlane(h_cap, bh - window), n);
            if (LOGITS) logits = a.logits + (size_t)__builtin_amdgcn_readlane(h_first, bh - window) * KQ_TILE * G;
            wave.template load<0, NT>(t0 + w, t1);
            wave.template load<1, NT>(t0 + w + KA_WAVES, t1);
            ++bh;
            return true;
        }
        return false;
    };
    for (bool more = next(); more;) {
        wave.reset();
        wave.ready();
        // a wave's tiles, KA_WAVES apart; while one is worked on, the next is on its way.  (More of them in flight, three, two / one, took 224K rows of eight heads
        // 42.5, 41.2 / 39.4 us, ragged batches in groups of eight 20.8, 20.1 / 19.7, with weights 23.8, 22.6 / 21.8; three workgroups to a compute unit 40.5 and 20.9.)
        int t = t0 + w;
        auto step = [&](auto buf) {
            constexpr int BUF = decltype(buf)::value;
            // not waited for: the next tile's loads, and where logits are stored the store before them; behind the last tile there are no loads, and
            // before the first no store
            const bool first = t == t0 + w, last = t + KA_WAVES >= t1;
            if (last && LOGITS && !first) __builtin_amdgcn_s_waitcnt(VMCNT1);
            else if (last) __builtin_amdgcn_s_waitcnt(VMCNT0);
            else if (LOGITS && first) __builtin_amdgcn_s_waitcnt(VMCNT5);
            f32x4 S[2];
            wave.template add<BUF, LOGITS ? 6 : 5>(t, logits, S);
            if (t + 2 * KA_WAVES < t1) wave.template load<BUF, NT>(t + 2 * KA_WAVES, t1);
            t += KA_WAVES;
        };
        while (t < t1) {
            step(std::integral_constant<int, 0>{});
            if (t >= t1) break;
            step(std::integral_constant<int, 1>{});
        }
        if (t == t0 + w) __builtin_amdgcn_s_waitcnt(VMCNT0);     // (no tile: nothing has waited for the loads of none, and others follow into their places)
        const size_t slot = (size_t)blockIdx.x + head;
        more = next();                                           // (its loads are on their way while the waves' sums are put together)
        wave.finish(sm_ml[w], &sm_o[w][0][0]);
        meet();
        for (int i = tid; i < G * HC_D; i += KA_BLK) {
            const int g = i / HC_D, d = i % HC_D;
            float m = sm_ml[0][g][0], o = 0.f, s = 0.f;
#pragma unroll
            for (int k = 1; k < KA_WAVES; ++k) m = fmaxf(m, sm_ml[k][g][0]);
#pragma unroll
            for (int k = 0; k < KA_WAVES; ++k) {
                const float f = moved(sm_ml[k][g][0], m);
                o = fmaf(f, sm_o[k][g][d], o);
                s = fmaf(f, sm_ml[k][g][1], s);
            }
            a.part_o[(slot * G + g) * HC_D + d] = o;
            if (d == 0) {
                a.part_ml[(slot * G + g) * 2] = m;
                a.part_ml[(slot * G + g) * 2 + 1] = s;
            }
        }
        meet();
    }
}

struct CombineArgs {
    const int2* state;
    const int2* room;
    const hc_kvq_head* heads;
    const int2* chunks;
    const int2* plan;
    const float *part_ml, *part_o;
    const float* logits;
    float *out, *lse, *acc;
    float decay;
    int n;
};

// (m, l) and (n, k): sums l and k of weights of references m and n
__device__ __forceinline__ void join(float& m, float& l, float n, float k)
{
    const float top = fmaxf(m, n);
    l = l * moved(m, top) + k * moved(n, top);
    m = top;
}

constexpr int KC_PER_CU = 3;                 // workgroups of 512 threads that a compute unit holds at once: 67 registers, seven waves a SIMD

// The first n G workgroups: output and lse of a query head each, BLK / 32 partial results at a time, 32 lanes of four values to each.  Those behind them:
// KQ_CHUNK rows' weights each.
template <int G, int BLK>
__global__ __launch_bounds__(BLK) void kvq_combine_kernel(CombineArgs a)
{
    constexpr int KC_WAVES = BLK / 64, KC_ROWS = BLK / 32;
    __shared__ float sm_o[KC_ROWS][HC_D];
    __shared__ float sm_w[KQ_MOST_WG];
    __shared__ float sm_m[KC_WAVES > G ? KC_WAVES : G], sm_l[KC_WAVES > G ? KC_WAVES : G];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lead = a.n * G;
    if ((int)blockIdx.x < lead) {
        const int bh = blockIdx.x / G, g = blockIdx.x % G;
        const int2 plan = a.plan[bh];
        const size_t first = (size_t)plan.x;
        const int count = kq_rows(a.state, a.room, bh) ? plan.y : 0;
        const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + first * G + g;
        float m = -FLT_MAX, l = 0.f;
        for (int i = tid; i < count; i += BLK) {
            const float2 x = ml[(size_t)i * G];
            sm_w[i] = x.x;
            join(m, l, x.x, x.y);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) join(m, l, __shfl_xor(m, d), __shfl_xor(l, d));
        if (lane == 0) {
            sm_m[w] = m;
            sm_l[w] = l;
        }
        __syncthreads();
        m = sm_m[0];
        l = sm_l[0];
#pragma unroll
        for (int i = 1; i < KC_WAVES; ++i) join(m, l, sm_m[i], sm_l[i]);
        const int lane32 = tid & 31, row = tid >> 5;
        const float* const po = a.part_o + (first * G + g) * HC_D + 4 * lane32;
        f32x4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = row; i < count; i += KC_ROWS) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(po + (size_t)i * G * HC_D);
            const float f = moved(sm_w[i], m);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[e], o[e]);
        }
        *reinterpret_cast<f32x4*>(&sm_o[row][4 * lane32]) = o;
        __syncthreads();
        if (tid < HC_D) {                                        // (BLK is 128 at least)
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < KC_ROWS; ++i) x += sm_o[i][tid];
            a.out[(size_t)blockIdx.x * HC_D + tid] = count == 0 ? 0.f : x / l;     // (no rows: nothing; nothing but logits of minus infinity: no number)
            if (tid == 0) a.lse[blockIdx.x] = lse_of(m, l);
        }
        return;
    }
    const int2 chunk = a.chunks[blockIdx.x - lead];
    const int bh = chunk.x, n = min(kq_rows(a.state, a.room, bh), chunk.y + KQ_CHUNK);
    if (chunk.y >= n) return;
    constexpr int EACH = KQ_CHUNK / BLK;
    const int64_t row_off = a.heads[bh].row_off;
    const float* const logits = a.logits + (size_t)a.room[bh].y * KQ_TILE * G;
    const int2 plan = a.plan[bh];
    const size_t first = (size_t)plan.x;
    const int count = plan.y;
    float s[EACH][G], old[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = min(chunk.y + k * BLK + tid, n - 1);
        const float* const from = logits + ((size_t)(r / KQ_TILE) * 8 + r % 4 * 2 + r / 16 % 2) * G * 4 + r / 4 % 4;
#pragma unroll
        for (int g = 0; g < G; ++g) s[k][g] = from[g * 4];
        old[k] = a.acc[row_off + r];
    }
    for (int g = w; g < G; g += KC_WAVES) {                      // a wave to a query head
        const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + first * G + g;
        float m = -FLT_MAX, l = 0.f;
#pragma unroll 4
        for (int i = lane; i < count; i += 64) {
            const float2 x = ml[(size_t)i * G];
            join(m, l, x.x, x.y);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) join(m, l, __shfl_xor(m, d), __shfl_xor(l, d));
        if (lane == 0) {
            sm_m[g] = m;
            sm_l[g] = 1.0f / (l * (float)G);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = chunk.y + k * BLK + tid;
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) x = fmaf(weight(s[k][g], sm_m[g]), sm_l[g], x);
        if (r < n) a.acc[row_off + r] = fmaf(old[k], a.decay, x);
    }
}

// ---- heads of few rows: all of one in a workgroup, and no second launch --------------------------------------------------------------------
//
// Where no head of a table has room for more than KS_BUFS KS_ROWS = 1,024 rows; where it is a half or a quarter of that, waves have fewer buffers, and a compute unit holds
// more workgroups: one with four buffers, two with two, with one buffer three (by registers; four without weights in groups of at most four).  4,096 heads of 100 rows, us with four
// buffers / one: groups of one 63 / 25, of four 74 / 30, of eight 85 / 41; with weights 68 / 28, 77 / 36, 89 / 44.  us, this way / split and joined: 500 rows of two heads 6.5 / 5.0 + 3.9 in two launches, 200 rows of eight
// heads 4.8 / 5.1 + 4.8, 1,000 rows of eight heads 7.6 / 5.1 + 5.1, of 512 heads 19.8 / 20.2 + 4.2, with weights 23.9 / 23.1 + 13.4.

constexpr int KS_BLK = 512, KS_WAVES = KS_BLK / 64;
constexpr int KS_ROWS = KS_WAVES * KQ_TILE;  // that a workgroup has at once, to a buffer of its waves: all of its loads are on their way before the first product

struct ShortArgs {
    AttnArgs a;
    float *out, *lse, *acc;
    float decay;
};

template <int G, bool WEIGHTS, int BUFS>
__global__ __launch_bounds__(KS_BLK) void kvq_attn_short_kernel(ShortArgs x)
{
    __shared__ float sm_ml[KS_WAVES][G][2], sm_all[G][2];
    __shared__ __attribute__((aligned(256))) char sm_tile[KS_WAVES][BUFS][T_BYTES];
    const AttnArgs& a = x.a;
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), bh = blockIdx.x;
    const int n = __builtin_amdgcn_readfirstlane(kq_rows(a.state, a.room, bh)), tiles = tiles_of(n);
    const hc_kvq_head hd = a.heads[bh];
    const int64_t off = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(hd.off >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)hd.off));
    Wave<G> wave(&sm_tile[w][0][0]);
    wave.aim(a, bh, off, (uint32_t)__builtin_amdgcn_readfirstlane(hd.cap), n);
    wave.reset();
    const int t = w;                                             // its tiles: KS_WAVES apart
    // a lane's rows of a tile, eight of 4 i + lane / 16: lanes of columns i take row i to the table of weights
    const int col = wave.col, row0 = 4 * (col & 7) + wave.grp;
    float old[BUFS];
    if (WEIGHTS)
#pragma unroll
        for (int b = 0; b < BUFS; ++b) {
            const int r = (t + b * KS_WAVES) * KQ_TILE + row0;
            old[b] = col < 8 && r < n ? x.acc[hd.row_off + r] : 0.f;
        }
    wave.template load<0, 0>(t, tiles);
    if constexpr (BUFS > 1) wave.template load<1, 0>(t + KS_WAVES, tiles);
    if constexpr (BUFS > 2) wave.template load<2, 0>(t + 2 * KS_WAVES, tiles);
    if constexpr (BUFS > 3) wave.template load<3, 0>(t + 3 * KS_WAVES, tiles);
    wave.ready();
    f32x4 S[BUFS][2];
    if (t < tiles) wave.template add<0, 5 * (BUFS - 1)>(t, nullptr, S[0]);
    if constexpr (BUFS > 1)
        if (t + KS_WAVES < tiles) wave.template add<1, 5 * (BUFS - 2)>(t + KS_WAVES, nullptr, S[1]);
    if constexpr (BUFS > 2)
        if (t + 2 * KS_WAVES < tiles) wave.template add<2, 5 * (BUFS - 3)>(t + 2 * KS_WAVES, nullptr, S[2]);
    if constexpr (BUFS > 3)
        if (t + 3 * KS_WAVES < tiles) wave.template add<3, 0>(t + 3 * KS_WAVES, nullptr, S[3]);
    __builtin_amdgcn_s_waitcnt(VMCNT0);                          // sums go through a buffer
    wave.finish(sm_ml[w], reinterpret_cast<float*>(&sm_tile[w][0][0]));
    __syncthreads();
    for (int i = tid; i < G * HC_D; i += KS_BLK) {
        const int g = i / HC_D;
        float m = sm_ml[0][g][0], o = 0.f, l = 0.f;
#pragma unroll
        for (int k = 1; k < KS_WAVES; ++k) m = fmaxf(m, sm_ml[k][g][0]);
#pragma unroll
        for (int k = 0; k < KS_WAVES; ++k) {
            const float f = moved(sm_ml[k][g][0], m);
            o = fmaf(f, reinterpret_cast<const float*>(&sm_tile[k][0][0])[i], o);
            l = fmaf(f, sm_ml[k][g][1], l);
        }
        x.out[(size_t)bh * G * HC_D + i] = n == 0 ? 0.f : o / l;         // (no rows: nothing; nothing but logits of minus infinity: no number)
        if (i % HC_D == 0) {
            x.lse[bh * G + g] = lse_of(m, l);
            sm_all[g][0] = m;
            sm_all[g][1] = 1.0f / (l * (float)G);
        }
    }
    if (!WEIGHTS) return;
    __syncthreads();
    const float ref = sm_all[col & (G - 1)][0], part = sm_all[col & (G - 1)][1];
#pragma unroll
    for (int b = 0; b < BUFS; ++b) {
        if (t + b * KS_WAVES >= tiles) break;
        float mine = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float p = weight(S[b][i >> 2][i & 3], ref) * part;
            if (G > 4) p = dpp_add<0x124>(p);                    // over the queries: columns repeat every G
            if (G > 2) p = dpp_add<0x122>(p);
            if (G > 1) p = dpp_add<0x121>(p);
            mine = (col & 7) == i ? p : mine;
        }
        const int r = (t + b * KS_WAVES) * KQ_TILE + row0;
        if (col < 8 && r < n) x.acc[hd.row_off + r] = fmaf(old[b], x.decay, mine);
    }
}

template <int G, int BUFS>
void launch_short(const ShortArgs& x, hipStream_t st)
{
    if (x.acc) kvq_attn_short_kernel<G, true, BUFS><<<dim3((unsigned)x.a.n), dim3(KS_BLK), 0, st>>>(x);
    else kvq_attn_short_kernel<G, false, BUFS><<<dim3((unsigned)x.a.n), dim3(KS_BLK), 0, st>>>(x);
}

template <int G>
hc_status launch(hc_ctx* ctx, const AttnArgs& a, const CombineArgs& c, int longest, int workgroups, int n_chunks, hipStream_t st)
{
    if (longest <= KS_BUFS * KS_ROWS) {
        const ShortArgs x{a, c.out, c.lse, c.acc, c.decay};
        if (longest <= KS_ROWS) launch_short<G, 1>(x, st);
        else if (longest <= 2 * KS_ROWS) launch_short<G, 2>(x, st);
        else launch_short<G, KS_BUFS>(x, st);
        HC_HIP(ctx, hipGetLastError());
        return HC_OK;
    }
    const dim3 grid((unsigned)workgroups), block(KA_BLK);
    if (a.logits) kvq_attn_kernel<G, true><<<grid, block, 0, st>>>(a);
    else kvq_attn_kernel<G, false><<<grid, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    // Where there are more query heads than the GPU holds workgroups of 512 threads, each has few partial results, and small workgroups take them all at once.
    // KV heads of 1,536 rows in groups of four, us with 512 / 128 threads, and with weights: 64 of them 4.2 / 4.3, 4.2 / 5.0; 128: 4.3 / 4.2, 4.8 / 5.3; 160: 5.1 / 4.1,
    // 6.8 / 6.0; 192, the last that fit: 5.1 / 4.2, 8.0 / 6.2; 224: 6.6 / 4.2, 8.3 / 6.4; 512 of 4,096 rows 10.6 / 4.3, 21.1 / 15.2.
    const dim3 joins((unsigned)(a.n * G + (a.logits ? n_chunks : 0)));
    if (a.n * G > KC_PER_CU * ctx->n_cu) kvq_combine_kernel<G, 128><<<joins, dim3(128), 0, st>>>(c);
    else kvq_combine_kernel<G, 512><<<joins, dim3(512), 0, st>>>(c);
    HC_HIP(ctx, hipGetLastError());
    return HC_OK;
}

}   // namespace

hc_status hc_launch_kvq_attn(hc_ctx* ctx, const hc_kvq* k, const void* arena, const int32_t* state, const void* q, float* out, float* lse, float* acc,
                             float decay, void* work, hipStream_t st)
{
    const hc_kvq_layout l = hc_kvq_plan(k);
    float* const ml = (float*)((char*)work + l.part_ml);
    float* const po = (float*)((char*)work + l.part_o);
    int2* const plan = (int2*)((char*)work + l.plan);
    float* const logits = acc ? (float*)((char*)work + l.logits) : nullptr;
    const int workgroups = (int)std::min((int64_t)hc_kvq_workgroups(ctx), std::max((int64_t)1, (k->units + (int64_t)k->n * KA_START + KA_LEAST - 1) / KA_LEAST));
    const AttnArgs a{(const uint8_t*)arena, (const int2*)state, k->heads, k->room, (const uint16_t*)q, ml, po, plan, logits, k->n};
    const CombineArgs c{(const int2*)state, k->room, k->heads, k->chunks, plan, ml, po, logits, out, lse, acc, decay, k->n};
    switch (ctx->G) {
    case 1: return launch<1>(ctx, a, c, k->max_cap, workgroups, k->n_chunks, st);
    case 2: return launch<2>(ctx, a, c, k->max_cap, workgroups, k->n_chunks, st);
    case 4: return launch<4>(ctx, a, c, k->max_cap, workgroups, k->n_chunks, st);
    default: return launch<8>(ctx, a, c, k->max_cap, workgroups, k->n_chunks, st);
    }
}
