// hc_rope.hip -- what happens to a token's query and key heads between the projections and the cache: a norm of each head
// (optional), the rotation by the token's position, and the place of its K and V rows: the prompt's buffer
// (hc_prefill_rope) or the heterogeneous cache (hc_append_rope).
//
//   norm      y = x (mean(x^2) + eps)^(-1/2) w               over the 128 elements of a head
//   rotation  (u, v) -> gain (u cos a - v sin a, v cos a + u sin a),  a = position * freq[i],  for the rot_dim / 2 pairs
//
// The angle is formed in 64 bits, in full turns, and brought to [-1/2, 1/2] turns before it is rounded to 32: at position
// 2^24 a product in 32 bits is off by half a radian, this one by 2^-25 turns.  Everything else is 32-bit, rounded once, to
// the bf16 that caches and attention take.
//
// A row of 128 elements is 16 lanes' work, two chunks of four elements a lane, chosen so that both halves of a pair are the
// same lane's: layout "half" pairs element i with i + rot_dim / 2, so lane l takes chunks [4l, 4l + 4) of either half; where
// pairs lie side by side, and behind the rotating part, a lane takes eight elements in a row.  No exchange between lanes but
// the norm's sum (data-parallel moves inside a row of 16 lanes).
//
// Bound by memory: 32,003 tokens of 32 query and 8 KV heads, bf16, 152 us (786 MB, 5.17 TB/s, where a copy of 2 GiB reaches 4.97); 11,528 tokens of f32
// projections 86.5 us (425 MB, 4.9 TB/s).  Four tokens to a workgroup, a wave's lanes making the table of one token's angles (64-bit products
// are the only arithmetic that could show).  The decode token is bound by the launch: 2.8 us for one sequence of two heads, 3.7 for 64 of eight.
#include <math.h>

#include <algorithm>

#include "hc_internal.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

// hc_rope as the kernels take it: frequencies in full turns a position.
struct RopeArgs {
    double turns[HC_D / 2];
    const float* q_norm;
    const float* k_norm;
    float eps, gain;
    int32_t rot;
    int32_t half;
};

RopeArgs rope_args(const hc_rope* r)
{
    RopeArgs a{};
    for (int i = 0; i < r->rot_dim / 2; ++i) a.turns[i] = r->freq[i] * (0.5 / M_PI);
    a.q_norm = r->q_norm;
    a.k_norm = r->k_norm;
    a.eps = r->eps;
    a.gain = r->gain;
    a.rot = r->rot_dim;
    a.half = r->layout == HC_ROPE_HALF;
    return a;
}

template <int CTRL>
__device__ __forceinline__ float dpp_add(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum16(float x)      // over a row of 16 lanes, in all of them
{
    x = dpp_add<0xB1>(x);        // quad_perm [1,0,3,2]
    x = dpp_add<0x4E>(x);        // quad_perm [2,3,0,1]
    x = dpp_add<0x141>(x);       // half mirror
    return dpp_add<0x128>(x);    // rotate by 8
}

// Where a lane's two chunks begin in a row.
struct Chunks {
    int a, b;
};
__device__ __forceinline__ Chunks chunks(const RopeArgs& r, int lane16)
{
    if (r.half && lane16 < r.rot / 8) return {4 * lane16, r.rot / 2 + 4 * lane16};
    return {8 * lane16, 8 * lane16 + 4};
}

template <bool F32>
__device__ __forceinline__ f32x4 load4(const void* p, size_t at)
{
    if (F32) return *reinterpret_cast<const f32x4*>((const float*)p + at);
    const u32x2 w = *reinterpret_cast<const u32x2*>((const uint16_t*)p + at);
    return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
}

__device__ __forceinline__ u32x2 pack(f32x4 x)
{
    return __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4));
}

// cos and sin of pair i at a position, times the gain.
__device__ __forceinline__ float2 turn(const RopeArgs& r, int i, int pos)
{
    const double t = (double)pos * r.turns[i];
    float s, c;
    sincospif(2.0f * (float)(t - rint(t)), &s, &c);
    return make_float2(c * r.gain, s * r.gain);
}

// Norm and rotation of a lane's two chunks; table: cos and sin of every pair at the row's position.
__device__ __forceinline__ void map_row(const RopeArgs& r, const float* __restrict__ weight, const float2* table, int lane16, Chunks at, f32x4& x, f32x4& y)
{
    if (weight) {
        float q = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) q = fmaf(x[e], x[e], fmaf(y[e], y[e], q));
        const float f = rsqrtf(sum16(q) * (1.0f / HC_D) + r.eps);
        const f32x4 wx = *reinterpret_cast<const f32x4*>(weight + at.a), wy = *reinterpret_cast<const f32x4*>(weight + at.b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] *= f * wx[e];
            y[e] *= f * wy[e];
        }
    }
    if (lane16 >= r.rot / 8) return;
    if (r.half) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 t = table[4 * lane16 + e];
            const float u = x[e], v = y[e];
            x[e] = fmaf(u, t.x, -v * t.y);
            y[e] = fmaf(v, t.x, u * t.y);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float2 s = table[4 * lane16 + e], t = table[4 * lane16 + 2 + e];
            const float u = x[2 * e], v = x[2 * e + 1], m = y[2 * e], n = y[2 * e + 1];
            x[2 * e] = fmaf(u, s.x, -v * s.y);
            x[2 * e + 1] = fmaf(v, s.x, u * s.y);
            y[2 * e] = fmaf(m, t.x, -n * t.y);
            y[2 * e + 1] = fmaf(n, t.x, m * t.y);
        }
    }
}

// ---- a prompt's tokens ----------------------------------------------------------------------------------------------------

constexpr int PR_BLK = 256;
constexpr int PR_TOKENS = PR_BLK / 64;        // of a workgroup: a wave makes the table of one token's angles
constexpr int PR_SEQS = HC_PROMPT_SEQS, PR_HEADS = HC_PROMPT_HEADS;

struct PromptRows {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;   // elements from token to token
    uint16_t *q_out, *kv;
    int Hq, Hkv, n_seq, tokens;
    int end[PR_SEQS];                         // of the launch's packed tokens, sequence by sequence
    int first[PR_SEQS];                       // position of a sequence's first token
    int64_t k_off[PR_HEADS], v_off[PR_HEADS];
};

template <bool F32>
__global__ __launch_bounds__(PR_BLK) void prefill_rope_kernel(RopeArgs r, PromptRows a)
{
    __shared__ float2 sm_turn[PR_TOKENS][HC_D / 2];
    __shared__ int sm_pos[PR_TOKENS], sm_seq[PR_TOKENS];
    const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int t0 = blockIdx.x * PR_TOKENS;
    const int mine = min(t0 + w, a.tokens - 1);
    const int b = __popcll(__builtin_amdgcn_ballot_w64(lane < a.n_seq && a.end[lane] <= mine));      // sequences that end before this token
    const int pos = a.first[b] + mine - (b > 0 ? a.end[b - 1] : 0);
    if (2 * lane < r.rot) sm_turn[w][lane] = turn(r, lane, pos);
    if (lane == 0) {
        sm_pos[w] = pos;
        sm_seq[w] = b;
    }
    __syncthreads();
    const int rows = a.Hq + 2 * a.Hkv, n = min(PR_TOKENS, a.tokens - t0) * rows;
    const int lane16 = tid & 15;
    const Chunks at = chunks(r, lane16);
    for (int i = tid >> 4; i < n; i += PR_BLK / 16) {
        const int t = i / rows, h = i - t * rows, kv = h - a.Hq;
        const size_t token = (size_t)(t0 + t);
        uint16_t* to;
        f32x4 x, y;
        if (kv < 0) {
            const size_t from = token * a.q_stride + (size_t)h * HC_D;
            x = load4<F32>(a.q, from + at.a);
            y = load4<F32>(a.q, from + at.b);
            to = a.q_out + (token * a.Hq + h) * HC_D;
        } else {
            const bool is_v = kv >= a.Hkv;
            const int head = is_v ? kv - a.Hkv : kv, row = sm_seq[t] * a.Hkv + head;
            const size_t from = token * (is_v ? a.v_stride : a.k_stride) + (size_t)head * HC_D;
            const void* src = is_v ? a.v : a.k;
            x = load4<F32>(src, from + at.a);
            y = load4<F32>(src, from + at.b);
            to = a.kv + (is_v ? a.v_off[row] : a.k_off[row]) + (int64_t)sm_pos[t] * HC_D;
        }
        if (kv < a.Hkv) map_row(r, kv < 0 ? r.q_norm : r.k_norm, sm_turn[t], lane16, at, x, y);
        *reinterpret_cast<u32x2*>(to + at.a) = pack(x);
        *reinterpret_cast<u32x2*>(to + at.b) = pack(y);
    }
}

// ---- the decode token ------------------------------------------------------------------------------------------------------

// Threads of a workgroup: 16 for each of the K row, the V row and the G query rows, whole waves.
__host__ __device__ constexpr int append_threads(int G) { return (16 * (G + 2) + 63) / 64 * 64; }

struct AppendRows {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;   // elements from sequence to sequence
    uint16_t *q_out, *arena, *tier;
    HeadDev* heads;
    SegDev* segs;
    BlkDev* blks;
    RepDev* reps;
    int Hkv, G;
};

// One workgroup per KV head and sequence takes the token's K row, V row and the G query rows of the head's group: the position
// is the head's length in the device's table, which the same workgroup moves on once all of it has read it.
template <bool F32>
__global__ __launch_bounds__(append_threads(HC_MAX_G)) void append_rope_kernel(RopeArgs r, AppendRows a)
{
    __shared__ float2 sm_turn[HC_D / 2];
    const int bh = blockIdx.x, b = bh / a.Hkv, h = bh - b * a.Hkv, tid = threadIdx.x;
    const HeadDev hd = a.heads[bh];
    const int pos = hd.ctx;
    const int lane16 = tid & 15, row = tid >> 4;                 // 0: K, 1: V, 2 + g: query head g of the group
    const Chunks at = chunks(r, lane16);
    f32x4 x{}, y{};
    if (row < a.G + 2) {
        const void* src = row == 0 ? a.k : row == 1 ? a.v : a.q;
        const size_t from = row == 0   ? (size_t)b * a.k_stride + (size_t)h * HC_D
                            : row == 1 ? (size_t)b * a.v_stride + (size_t)h * HC_D
                                       : (size_t)b * a.q_stride + (size_t)(h * a.G + row - 2) * HC_D;
        x = load4<F32>(src, from + at.a);
        y = load4<F32>(src, from + at.b);
    }
    if (2 * tid < r.rot) sm_turn[tid] = turn(r, tid, pos);
    __syncthreads();                                             // (and everyone has read the old table entry)
    if (row < a.G + 2) {
        if (row != 1) map_row(r, row == 0 ? r.k_norm : r.q_norm, sm_turn, lane16, at, x, y);
        const u32x2 px = pack(x), py = pack(y);
        auto store = [&](uint16_t* to) {
            *reinterpret_cast<u32x2*>(to + at.a) = px;
            *reinterpret_cast<u32x2*>(to + at.b) = py;
        };
        if (row >= 2) {
            store(a.q_out + ((size_t)bh * a.G + row - 2) * HC_D);
        } else {
            // a full head's row goes behind its last; a compressed head's into the slot of its ring of recent positions that
            // held the position which now leaves the window; a satellite's into its host-tier block as well
            int slot = -1;
            if (hd.role == HC_ROLE_FULL) slot = pos;
            else if (hd.recent > 0) slot = hd.sink + (pos - hd.ctx0) % hd.recent;
            if (slot >= 0) store(a.arena + (row == 0 ? hd.k_off : hd.v_off) + (int64_t)slot * HC_D);
            if (hd.role == HC_ROLE_SATELLITE) store(a.tier + hd.tier_off + ((int64_t)pos * 2 + row) * HC_D);
        }
    }
    if (tid == 0) hc_advance_head(a.heads, a.segs, a.blks, a.reps, bh, hd);
}

}   // namespace

extern "C" hc_status hc_rope_init(hc_rope* out, int32_t layout, int32_t rot_dim, double theta, const hc_rope_scaling* scaling)
{
    if (!out || (layout != HC_ROPE_HALF && layout != HC_ROPE_INTERLEAVED)) return HC_EINVAL;
    if (rot_dim < 0 || rot_dim > HC_D || rot_dim % 8 != 0) return HC_ESHAPE;
    if (!(theta > 0.0) || !isfinite(theta)) return HC_EINVAL;
    hc_rope r{};
    r.layout = layout;
    r.rot_dim = rot_dim;
    r.gain = 1.0f;
    r.eps = 1.0e-6f;
    double base = theta;
    if (scaling) {
        if (!(scaling->factor >= 1.0) || !isfinite(scaling->factor)) return HC_EINVAL;
        if (scaling->kind == HC_ROPE_BASE && rot_dim > 0) base = theta * pow(scaling->factor, rot_dim / (rot_dim - 2.0));
        else if (scaling->kind == HC_ROPE_BANDS) {
            if (!(scaling->low >= 0.0) || !(scaling->high > scaling->low) || !isfinite(scaling->high) || scaling->original < 1) return HC_EINVAL;
        } else if (scaling->kind != HC_ROPE_LINEAR && scaling->kind != HC_ROPE_BASE) return HC_EINVAL;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling && scaling->kind == HC_ROPE_LINEAR) f /= scaling->factor;
        if (scaling && scaling->kind == HC_ROPE_BANDS) {
            const double turns = scaling->original * f / (2.0 * M_PI);
            const double keep = std::min(1.0, std::max(0.0, (turns - scaling->low) / (scaling->high - scaling->low)));
            f = f * keep + f / scaling->factor * (1.0 - keep);
        }
        if (!(f <= HC_ROPE_MAX_FREQ)) return HC_EINVAL;
        r.freq[i] = f;
    }
    *out = r;
    return HC_OK;
}

hc_status hc_launch_prefill_rope(hc_ctx* ctx, const hc_rope* rope, const hc_rows_in& in, const int32_t* first, const int32_t* count, void* q_out,
                                 void* kv, const int64_t* k_off, const int64_t* v_off, hipStream_t st)
{
    const hc_config& c = ctx->cfg;
    const RopeArgs r = rope_args(rope);
    const size_t size = in.f32 ? 4 : 2;
    PromptRows a{};
    a.q_stride = in.q_stride;
    a.k_stride = in.k_stride;
    a.v_stride = in.v_stride;
    a.kv = (uint16_t*)kv;
    a.Hq = c.Hq;
    a.Hkv = c.Hkv;
    // as many sequences at a time as a launch's arguments have room for
    const int most = std::min(PR_SEQS, PR_HEADS / c.Hkv);
    long long done = 0;
    for (int b0 = 0; b0 < c.B; b0 += most) {
        a.n_seq = std::min(most, c.B - b0);
        long long tokens = 0;
        for (int i = 0; i < a.n_seq; ++i) {
            tokens += count[b0 + i];
            a.end[i] = (int)tokens;
            a.first[i] = first[b0 + i];
        }
        if (tokens == 0) continue;
        for (int i = 0; i < a.n_seq * c.Hkv; ++i) {
            a.k_off[i] = k_off[b0 * c.Hkv + i];
            a.v_off[i] = v_off[b0 * c.Hkv + i];
        }
        a.tokens = (int)tokens;
        a.q = (const char*)in.q + (size_t)done * in.q_stride * size;
        a.k = (const char*)in.k + (size_t)done * in.k_stride * size;
        a.v = (const char*)in.v + (size_t)done * in.v_stride * size;
        a.q_out = (uint16_t*)q_out + (size_t)done * c.Hq * HC_D;
        const dim3 grid((unsigned)((tokens + PR_TOKENS - 1) / PR_TOKENS));
        if (in.f32) prefill_rope_kernel<true><<<grid, dim3(PR_BLK), 0, st>>>(r, a);
        else prefill_rope_kernel<false><<<grid, dim3(PR_BLK), 0, st>>>(r, a);
        HC_HIP(ctx, hipGetLastError());
        done += tokens;
    }
    return HC_OK;
}

hc_status hc_launch_append_rope(hc_ctx* ctx, const hc_layer* L, const hc_rope* rope, const hc_rows_in& in, void* q_out, void* arena, void* tier, hipStream_t st)
{
    const RopeArgs r = rope_args(rope);
    const AppendRows a{in.q, in.k, in.v, in.q_stride, in.k_stride, in.v_stride, (uint16_t*)q_out, (uint16_t*)arena, (uint16_t*)tier,
                       L->heads, L->segs, L->blks, L->reps, ctx->cfg.Hkv, ctx->G};
    const dim3 grid((unsigned)L->n_heads), block((unsigned)append_threads(ctx->G));
    if (in.f32) append_rope_kernel<true><<<grid, block, 0, st>>>(r, a);
    else append_rope_kernel<false><<<grid, block, 0, st>>>(r, a);
    HC_HIP(ctx, hipGetLastError());
    return HC_OK;
}
