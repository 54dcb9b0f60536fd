// hc_kvq_attn.hip -- attention of the decode token over the cache held in 4 bits (its format: hc_kvq.h), and every row's share of the weights.
//
//   t_j = q . K[j] log2(e) / sqrt(128),   p_j = 2^(t_j - m),   out = sum_j p_j V[j] / sum_j p_j,   lse = (m + log2 sum_j p_j) ln 2
//   acc_j <- decay acc_j + (1/G) sum_g p_gj / sum_i p_gi
//
// A workgroup takes an equal share of the tiles of 32 rows of all heads one after the other; lengths are on the device, and each
// wave finds its share by itself.  A wave takes whole tiles, the next one's loads in flight under the present one's arithmetic, and nothing goes
// through LDS until a head's end.  S^T = K Q^T and O^T = V^T P^T on the matrix cores (16x16x32), keys along S^T's rows, so that the lane that has a
// weight is the lane that hands it to the second product, and the products' order of the keys is chosen (row 4 x + y of the first is key
// 4 y + x) so that a load of V takes four rows side by side.
//   K   a lane's 16 bytes are 32 values of one scale: what the first product's four steps take; q is laid out alike
//   V   a lane's dword is 8 values of one row; of 8 rows they become, two by two, operands of 8 tiles of 16 values
// Codes become bf16 exactly.  The matrix cores have 16 columns for a group of at most 8 query heads: the others take what the rounding of the weights to
// bf16 leaves, in two steps, so that the weights lose nothing (8 + 8 + 8 bits): columns g, G + g, 2 G + g for the parts of query head g, added at the end.
// Groups of eight take a second product for the last part.
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
constexpr float KA_SCALE = 1.4426950408889634f * 0.08838834764831845f;     // log2(e) / sqrt(128)
constexpr float KA_LN2 = 0.6931471805599453f;
constexpr float KA_SLACK = 8.0f;             // a weight is at most 2^8 before the reference moves
constexpr int KA_LEAST = KA_WAVES;           // tiles of a workgroup, where there are so few
constexpr int KA_START = 16;                 // what beginning a head costs a workgroup, in tiles

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
constexpr int KA_BUFS = 4, T_STEP = KA_WAVES * T_BYTES;
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
        : "v"(k_at), "v"(s_at), "v"(v_at), "v"(f_at), "n"(later), "n"(BUF * T_STEP), "n"(BUF * T_STEP + 1024), "n"(BUF * T_STEP + T_KS),
          "n"(BUF * T_STEP + T_KS + 16), "n"((BUF * T_STEP + T_V) / 256), "n"((BUF * T_STEP + T_V) / 256 + 1), "n"((BUF * T_STEP + T_V) / 256 + 2),
          "n"((BUF * T_STEP + T_V) / 256 + 3), "n"((BUF * T_STEP + T_V) / 256 + 4), "n"((BUF * T_STEP + T_V) / 256 + 5), "n"((BUF * T_STEP + T_V) / 256 + 6),
          "n"((BUF * T_STEP + T_V) / 256 + 7), "n"(BUF * T_STEP + T_VS), "n"(BUF * T_STEP + T_VS + 16)
        : "memory");
}
static_assert(T_STEP % 256 == 0 && T_V % 256 == 0 && (KA_BUFS * T_STEP) / 256 <= 272, "offsets of the reads");

template <int G, bool LOGITS>
__global__ __launch_bounds__(KA_BLK, KQ_WG_PER_CU) void kvq_attn_kernel(AttnArgs a)
{
    __shared__ float sm_ml[KA_WAVES][G][2];
    __shared__ __attribute__((aligned(256))) char sm_tile[KA_BUFS][KA_WAVES][T_BYTES];
    static_assert(G * HC_D * sizeof(float) <= T_BYTES, "a wave's sums go through its first buffer");
    auto sm_o = [&](int wave, int g) { return reinterpret_cast<float*>(&sm_tile[0][wave][0]) + g * HC_D; };
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;

    // this workgroup's share, and the head that it begins in
    const int each = (a.n + 63) / 64, mine0 = min(a.n, lane * each), mine1 = min(a.n, mine0 + each);
    int sum = 0;
    for (int i = mine0; i < mine1; ++i) sum += places_of(kq_rows(a.state, a.room, i));
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
    int bh = __builtin_amdgcn_readfirstlane(owner * each), window = bh - 64;
    int before = __builtin_amdgcn_readlane(upto - sum, owner);
    int h_rows = 0, h_cap = 0, h_first = 0;                      // a lane's of the 64 heads from `window` on
    int64_t h_off = 0;

    const int part = G <= 4 ? col / G : col / 8;                 // of the weights that this column takes
    const bool dead = part > 2;
    const uint32_t m1 = part >= 1 ? 0xffff0000u : 0u, m2 = part >= 2 ? 0xffff0000u : 0u;
    const float cs = dead ? 0.f : KA_SCALE;

    // what the lane reads of a tile: K's rows 16 s + 4 (col % 4) + col / 4 and V's 4 i + grp
    const uint32_t tile0 = (uint32_t)(uintptr_t)(lds_char*)&sm_tile[0][w][0];
    uint32_t k_read = tile0 + (4 * (col & 3) + (col >> 2)) * 64 + (grp ^ (col & 3)) * 16, s_read = tile0 + (8 * (col >> 2) + (col & 3)) * 4 + grp;
    uint32_t v_read = tile0 + lane * 4, f_read = tile0 + grp * 32;
    asm("" : "+v"(k_read), "+v"(s_read), "+v"(v_read), "+v"(f_read));      // (opaque, so that a buffer goes into an instruction's offset)
    for (; before < u1 && bh < a.n; ++bh) {
        if (bh >= window + 64) {
            window = bh;
            const int i = min(bh + lane, a.n - 1);
            const int2 room = a.room[i];
            h_rows = min(max(a.state[i].x, 0), room.x);
            h_cap = room.x;
            h_first = room.y;
            h_off = a.heads[i].off;
        }
        const int n = __builtin_amdgcn_readlane(h_rows, bh - window), tiles = tiles_of(n), begin = before + KA_START;
        before += places_of(n);
        const int t0 = max(u0 - begin, 0), t1 = min(tiles, u1 - begin);
        if (t0 >= t1) continue;
        const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(h_off >> 32), bh - window) << 32 |
                             (uint32_t)__builtin_amdgcn_readlane((int)h_off, bh - window);
        const uint32_t cap = __builtin_amdgcn_readlane(h_cap, bh - window);
        const int first_tile = LOGITS ? __builtin_amdgcn_readlane(h_first, bh - window) : 0;
        if (t0 == 0 && tid == 0) a.plan[bh] = make_int2((int)blockIdx.x + bh, (begin + tiles - 1) / per - (int)blockIdx.x + 1);
        bf16x8 Q[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) Q[c] = *reinterpret_cast<const bf16x8*>(a.q + ((size_t)bh * G + (col & (G - 1))) * HC_D + 32 * grp + 8 * c);
        float ref = dead ? FLT_MAX : -FLT_MAX, l = 0.f;
        f32x4 O[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) O[j] = f32x4{0.f, 0.f, 0.f, 0.f};

        // a lane's places: 16 bytes of codes of row lane / 4, and the scales of row 4 (lane % 8) + lane / 8 % 4, K's or V's
        const int c_row = lane >> 2, s_row = 4 * (lane & 7) + (lane >> 3 & 3);
        const uint32_t k_chunk = ((lane & 3) ^ (lane >> 4)) * 16, v_chunk = (lane & 3) * 16, s_base = (lane < 32 ? 64u : 132u) * cap;
        const uint32_t k_at = c_row * 64 + k_chunk, v_at = 68 * cap + c_row * 64 + v_chunk, s_at = s_base + s_row * 4;
        // Codes are read once: marked so (2), unless the logits on their way to the next kernel share the caches with them.  us of this pass, marked / not:
        // 224K rows of eight heads, no logits 42.4 / 43.1, logits 53.3 / 47.6; two such heads and six short ones 16.6 / 18.2, 20.1 / 19.1.
        static constexpr int NT = LOGITS ? 0 : 2;
        auto load = [&](int t, auto buf) {
            lds_char* const to = (lds_char*)&sm_tile[decltype(buf)::value][w][0];
            // (a tile behind the last is loaded from a buffer of no bytes, which costs no memory: the number of loads on their way is then always the same)
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(a.arena + off), 0, t < t1 ? 136u * cap : 0u, 0x00027000);
            const int r0 = t * KQ_TILE;
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
        };
        auto compute = [&](int t, auto buf) {
            Tile x;
            // three tiles' loads, and where logits are stored those of the three tiles before this one: not yet behind the first tiles
            if (LOGITS && t < t0 + 3 * KA_WAVES) __builtin_amdgcn_s_waitcnt(0x0f7f);       // vmcnt(15)
            read_tile<decltype(buf)::value, LOGITS ? 18 : 15>(x, k_read, s_read, v_read, f_read);
            uint32_t xv[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) xv[i] = x.v[i >> 1][i & 1];
            f32x4 S[2];
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
            for (int i = 0; i < 8; ++i) f[i] = kq_scale(x.vs[i >> 2][i & 3] >> (col >> 2) * 8 & 255u);
            const int r0 = t * KQ_TILE;
            if (LOGITS && col < 2 * G)                           // (columns g and G + g have the same: 2 G lanes store half of the eight each)
                *reinterpret_cast<f32x4*>(a.logits + ((size_t)(first_tile + t) * 8 + 2 * grp) * G * 4 + col * 4) = col < G ? S[0] : S[1];
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
                p[i] = fmaf(S[i >> 2][i & 3], cs, -ref);
                top = fmaxf(top, p[i]);
            }
            if (__builtin_amdgcn_ballot_w64(top > KA_SLACK && !dead)) {
                float y = S[0][0] * cs;
#pragma unroll
                for (int i = 1; i < 8; ++i) y = fmaxf(y, S[i >> 2][i & 3] * cs);
                y = fmaxf(y, __shfl_xor(y, 16));
                y = fmaxf(y, __shfl_xor(y, 32));
                y = fmaxf(y, ref);
                const float less = exp2f(ref - y);
                ref = y;
                l *= less;
#pragma unroll
                for (int j = 0; j < 8; ++j) O[j] *= less;
#pragma unroll
                for (int i = 0; i < 8; ++i) p[i] = fmaf(S[i >> 2][i & 3], cs, -ref);
            }
            uint32_t P1[8], P2[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = dead ? 0.f : __builtin_amdgcn_exp2f(p[i]);
                l += e;
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
        };

        // a wave's tiles, KA_WAVES apart; while one is worked on, three are on their way
        using B0 = std::integral_constant<int, 0>;
        using B1 = std::integral_constant<int, 1>;
        using B2 = std::integral_constant<int, 2>;
        using B3 = std::integral_constant<int, 3>;
        int t = t0 + w;
        auto step = [&](auto buf) {
            compute(t, buf);
            load(t + 4 * KA_WAVES, buf);
            t += KA_WAVES;
        };
#pragma unroll
        for (int c = 0; c < 4; ++c) asm volatile("" : "+v"(Q[c]));      // (they are there: the waits below count the tiles' loads alone)
        load(t, B0{});
        load(t + KA_WAVES, B1{});
        load(t + 2 * KA_WAVES, B2{});
        load(t + 3 * KA_WAVES, B3{});
        while (t < t1) {
            step(B0{});
            if (t >= t1) break;
            step(B1{});
            if (t >= t1) break;
            step(B2{});
            if (t >= t1) break;
            step(B3{});
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0): sums go through a buffer

        // the parts of a weight, and the waves, together
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (lane < G) {
            sm_ml[w][lane][0] = ref;
            sm_ml[w][lane][1] = l;
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
                float* const to = sm_o(w, col) + 8 * (4 * grp + r);
                *reinterpret_cast<f32x4*>(to) = lo;
                *reinterpret_cast<f32x4*>(to + 4) = hi;
            }
        }
        __syncthreads();
        const size_t slot = (size_t)blockIdx.x + bh;
        for (int i = tid; i < G * HC_D; i += KA_BLK) {
            const int g = i / HC_D, d = i % HC_D;
            float m = sm_ml[0][g][0], o = 0.f, s = 0.f;
#pragma unroll
            for (int k = 1; k < KA_WAVES; ++k) m = fmaxf(m, sm_ml[k][g][0]);
#pragma unroll
            for (int k = 0; k < KA_WAVES; ++k) {
                const float f = exp2f(sm_ml[k][g][0] - m);
                o = fmaf(f, sm_o(k, g)[d], o);
                s = fmaf(f, sm_ml[k][g][1], s);
            }
            a.part_o[(slot * G + g) * HC_D + d] = o;
            if (d == 0) {
                a.part_ml[(slot * G + g) * 2] = m;
                a.part_ml[(slot * G + g) * 2 + 1] = s;
            }
        }
        __syncthreads();
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

// (m, l) and (n, k): sums l 2^m and k 2^n
__device__ __forceinline__ void join(float& m, float& l, float n, float k)
{
    const float top = fmaxf(m, n);
    l = l * exp2f(m - top) + k * exp2f(n - top);
    m = top;
}

constexpr int KC_BLK = 512, KC_WAVES = KC_BLK / 64, KC_ROWS = KC_BLK / 32;

// The first n G workgroups: output and lse of a query head each, KC_ROWS partial results at a time, 32 lanes of four values to each.  Those behind them:
// KQ_CHUNK rows' weights each.
template <int G>
__global__ __launch_bounds__(KC_BLK) void kvq_combine_kernel(CombineArgs a)
{
    __shared__ float sm_o[KC_ROWS][HC_D];
    __shared__ float sm_w[KQ_MOST_WG];
    __shared__ float sm_m[KC_WAVES], sm_l[KC_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int lead = a.n * G;
    if ((int)blockIdx.x < lead) {
        const int bh = blockIdx.x / G, g = blockIdx.x % G;
        const int2 plan = a.plan[bh];
        const size_t first = (size_t)plan.x;
        const int count = kq_rows(a.state, a.room, bh) ? plan.y : 0;
        const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + first * G + g;
        float m = -FLT_MAX, l = 0.f;
        for (int i = tid; i < count; i += KC_BLK) {
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
            const float f = exp2f(sm_w[i] - m);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[e], o[e]);
        }
        *reinterpret_cast<f32x4*>(&sm_o[row][4 * lane32]) = o;
        __syncthreads();
        if (tid < HC_D) {
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < KC_ROWS; ++i) x += sm_o[i][tid];
            a.out[(size_t)blockIdx.x * HC_D + tid] = l == 0.f ? 0.f : x / l;       // (no rows: nothing)
            if (tid == 0) a.lse[blockIdx.x] = l == 0.f ? -INFINITY : (m + log2f(l)) * KA_LN2;
        }
        return;
    }
    const int2 chunk = a.chunks[blockIdx.x - lead];
    const int bh = chunk.x, n = min(kq_rows(a.state, a.room, bh), chunk.y + KQ_CHUNK);
    if (chunk.y >= n) return;
    constexpr int EACH = KQ_CHUNK / KC_BLK;
    const int64_t row_off = a.heads[bh].row_off;
    const float* const logits = a.logits + (size_t)a.room[bh].y * KQ_TILE * G;
    const int2 plan = a.plan[bh];
    const size_t first = (size_t)plan.x;
    const int count = plan.y;
    float s[EACH][G], old[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = min(chunk.y + k * KC_BLK + tid, n - 1);
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
            sm_l[g] = l == 0.f ? 0.f : 1.0f / (l * (float)G);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = chunk.y + k * KC_BLK + tid;
        float x = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) x = fmaf(__builtin_amdgcn_exp2f(fmaf(s[k][g], KA_SCALE, -sm_m[g])), sm_l[g], x);
        if (r < n) a.acc[row_off + r] = fmaf(old[k], a.decay, x);
    }
}

template <int G>
hc_status launch(hc_ctx* ctx, const AttnArgs& a, const CombineArgs& c, int workgroups, int n_chunks, hipStream_t st)
{
    const dim3 grid((unsigned)workgroups), block(KA_BLK);
    if (a.logits) kvq_attn_kernel<G, true><<<grid, block, 0, st>>>(a);
    else kvq_attn_kernel<G, false><<<grid, block, 0, st>>>(a);
    HC_HIP(ctx, hipGetLastError());
    kvq_combine_kernel<G><<<dim3((unsigned)(a.n * G + (a.logits ? n_chunks : 0))), dim3(KC_BLK), 0, st>>>(c);
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
    case 1: return launch<1>(ctx, a, c, workgroups, k->n_chunks, st);
    case 2: return launch<2>(ctx, a, c, workgroups, k->n_chunks, st);
    case 4: return launch<4>(ctx, a, c, workgroups, k->n_chunks, st);
    default: return launch<8>(ctx, a, c, workgroups, k->n_chunks, st);
    }
}
