// RMS norm of every head of q and k and the rotation by the token's position, in one pass over the output of a fused q/k/v projection.
//
// Memory sets the time: 4 bytes a value in 16 bits, and the tables.  head_dim / 8 lanes hold a head, eight consecutive elements each, so a warp
// holds 32 / (head_dim / 8) whole heads side by side in memory; it takes kHeads such sets of one token's q, k or v at once, their loads in
// flight together, with the token's cosines and sines kept in registers for all of them.  The sum of squares is a few shuffles.
//
// Measured (bf16, q, k and v copied): 4608 tokens, 3 x 24 heads of 128, 30.7 us, 5.5 TB/s; 18432 tokens 6.1 TB/s; heads of 64 15.0 us; 64 tokens of 32 + 2 x 8
// heads 3.0 us (latency).  4173 tokens, 3 x 16 heads of 72 in fp16, half of each turned: 15 us, 3.9 TB/s: instructions (27 of 32 lanes hold
// heads, and a sum over nine lanes is four steps of shuffle and test).  Heads of other sizes, 4608 tokens, tensors that are not in L2, all of a head turned:
// 3 x 16 heads of 80 23 us, 3.1 TB/s; 3 x 24 of 96 36, 3.5; 3 x 16 of 160 47, 3.0; 3 x 8 of 256 28, 4.0; 3 x 32 of 32 15, 3.8.
// (One block of threads per token, weights and angles per head from memory: 67 us for the first.)
#include "mxfp4.cuh"
#include "ptx.cuh"
#include "qk_plan.h"
#include "row_ranges.h"

namespace dirotq {
namespace {

constexpr int kThreads = 256;

struct QkParams {
    const void* x;
    void* q_out;
    void* k_out;
    void* v_out;
    long long ldx, ldq, ldk, ldv;
    int hq, hk, D;
    int norm, rope, rot;
    float eps, inv_dim;
    int wdtype;
    const void* qw;
    const void* kw;
    const float* cos_table;
    const float* sin_table;
    long long ld_table;
    int num_positions;
    const int32_t* positions;
    const int32_t* slots;
    int num_slots;
    int copy_v;
    int wide_table;              // rows of both tables are 16-byte aligned
    // how a warp's lanes are used: lanes of a head, heads side by side, the first step of the sum over L lanes, sets of a turn, turns
    // of a token, of all
    int L, per_warp, fold, part_sets, parts_q, parts_k, parts, items;
};

// How the elements of a head lie on its lanes and find their partners.
enum Style {
    PLAIN,    // no rotation: elements 8 sub + i of lane sub
    PAIRS,    // the same; partners are neighbours
    SPLIT,    // halves of the whole head: elements 4 sub + i and D/2 + 4 sub + i, i < 4: partners lie in one lane
    QUARTER,  // halves of half a head: elements 2 sub + i, D/4 + 2 sub + i, i < 2, and, not turned, D/2 + 4 sub + i, i < 4
    HALVES,   // halves of any other part of the head: as PAIRS, partners through shared memory
};

// A lane's eight elements of a head: one piece (16 bytes in 16 bits), or the two or three of its style, in the order of `element`.
template <int STYLE>
__device__ __forceinline__ int element(int i, int sub, int half) {
    if (STYLE == SPLIT) return i < 4 ? 4 * sub + i : half + 4 * sub + i - 4;
    if (STYLE == QUARTER) return i < 2 ? 2 * sub + i : i < 4 ? half + 2 * sub + i - 2 : 2 * half + 4 * sub + i - 4;
    return 8 * sub + i;
}
template <typename T, int STYLE>
__device__ __forceinline__ Raw8<T> load_pieces(const T* head, int sub, int half) {
    Raw8<T> r;
    const int d0 = element<STYLE>(0, sub, half), d2 = element<STYLE>(2, sub, half), d4 = element<STYLE>(4, sub, half);
    uint32_t* w = reinterpret_cast<uint32_t*>(&r);
    if constexpr (STYLE == QUARTER) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(head + d0);
            *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(head + d2);
            *reinterpret_cast<uint4*>(w + 4) = *reinterpret_cast<const uint4*>(head + d4);
        } else {
            w[0] = *reinterpret_cast<const uint32_t*>(head + d0);
            w[1] = *reinterpret_cast<const uint32_t*>(head + d2);
            *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(head + d4);
        }
    } else if constexpr (sizeof(T) == 4) {
        r.u[0] = *reinterpret_cast<const uint4*>(head + d0);
        r.u[1] = *reinterpret_cast<const uint4*>(head + d4);
    } else if constexpr (STYLE == SPLIT) {
        *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(head + d0);
        *reinterpret_cast<uint2*>(w + 2) = *reinterpret_cast<const uint2*>(head + d4);
    } else {
        r.u[0] = *reinterpret_cast<const uint4*>(head + d0);
    }
    return r;
}
template <typename T, int STYLE>
__device__ __forceinline__ void store_pieces(T* head, int sub, int half, const Raw8<T>& r) {
    const int d0 = element<STYLE>(0, sub, half), d2 = element<STYLE>(2, sub, half), d4 = element<STYLE>(4, sub, half);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
    if constexpr (STYLE == QUARTER) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint2*>(head + d0) = *reinterpret_cast<const uint2*>(w);
            *reinterpret_cast<uint2*>(head + d2) = *reinterpret_cast<const uint2*>(w + 2);
            *reinterpret_cast<uint4*>(head + d4) = *reinterpret_cast<const uint4*>(w + 4);
        } else {
            *reinterpret_cast<uint32_t*>(head + d0) = w[0];
            *reinterpret_cast<uint32_t*>(head + d2) = w[1];
            *reinterpret_cast<uint2*>(head + d4) = *reinterpret_cast<const uint2*>(w + 2);
        }
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<uint4*>(head + d0) = r.u[0];
        *reinterpret_cast<uint4*>(head + d4) = r.u[1];
    } else if constexpr (STYLE == SPLIT) {
        *reinterpret_cast<uint2*>(head + d0) = *reinterpret_cast<const uint2*>(w);
        *reinterpret_cast<uint2*>(head + d4) = *reinterpret_cast<const uint2*>(w + 2);
    } else {
        *reinterpret_cast<uint4*>(head + d0) = r.u[0];
    }
}

__device__ __forceinline__ float weight_at(const void* p, int i, int dtype) {
    if (p == nullptr) return 1.f;
    if (dtype == DIROTQ_DTYPE_F32) return __ldg(static_cast<const float*>(p) + i);
    const uint16_t u = __ldg(static_cast<const uint16_t*>(p) + i);
    return dtype == DIROTQ_DTYPE_F16 ? __half2float(__ushort_as_half(u)) : __uint_as_float(static_cast<uint32_t>(u) << 16);
}

template <typename T>
constexpr int kHeads = sizeof(T) == 4 ? 2 : 4;  // sets of heads a warp takes at once

// STYLE; LANES: lanes of a head where head_dim is 64, 72 or 128, 0: p.L, any.  The three are sizes of the models whose layers the library serves; a constant
// unrolls the sum over a head's lanes and, in the QUARTER and HALVES styles, keeps registers from spilling.  4608 tokens, tensors that are not in L2, constant
// against p.L, us: heads of 64 all turned in pairs 31.5 / 35.2, a half turned in halves 32.3 / 42.1, a third 35.2 / 46.5; of 72 20.2 / 22.5, 20.1 / 24.7, 23.7 / 30.6;
// of 128 31.9 / 36.5, 32.9 / 44.2, 36.2 / 49.4; 64 tokens 0.3 to 1.2 us apart.
template <typename T, int STYLE, int LANES>
__global__ void __launch_bounds__(kThreads, STYLE == HALVES && sizeof(T) == 4 ? 2 : 3) qk_norm_rope_kernel(const __grid_constant__ QkParams p) {
    constexpr int HEADS = kHeads<T>;
    constexpr int PITCH = 9;  // words of a lane's eight elements in shared memory: odd, so that a warp's reads of one of them fall into 32 banks
    __shared__ float s_head[STYLE == HALVES ? kThreads / 32 : 1][32 * PITCH];
    __shared__ __align__(16) float s_w[2][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int L = LANES ? LANES : p.L, per_warp = LANES ? 32 / (LANES ? LANES : 1) : p.per_warp;
    const int sub = lane % L, in_warp = lane / L;  // place in the head, head in the set
    const int head0 = lane - sub;                  // the lane that holds the head's first elements
    const bool lives = 32 % (LANES ? LANES : 1) == 0 && LANES ? true : in_warp < per_warp;
    const int half = p.rot >> 1;
    // HALVES: where the partners of this lane's elements will lie; the spare ninth word holds the zero that what is not turned takes instead (an
    // infinity in some partner's place would leave NaN)
    float* const s_mine = &s_head[STYLE == HALVES ? warp : 0][lane * PITCH];
    const float* s_partner[8];
    if constexpr (STYLE == HALVES) {
        s_mine[8] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = 8 * sub + i, from = d < half ? d + half : d - half;
            s_partner[i] = lives && d < p.rot ? &s_head[warp][(head0 + (from >> 3)) * PITCH + (from & 7)] : s_mine + 8;
        }
    }
    const bool weighted = p.qw != nullptr || p.kw != nullptr;
    grid_dependency_wait();  // x is the previous kernel's output
    grid_launch_dependents();
    if (weighted) {
        for (int i = threadIdx.x; i < p.D; i += kThreads) {
            s_w[0][i] = weight_at(p.qw, i, p.wdtype);
            s_w[1][i] = weight_at(p.kw, i, p.wdtype);
        }
        __syncthreads();
    }
    for (int item = blockIdx.x * (kThreads / 32) + warp; item < p.items; item += gridDim.x * (kThreads / 32)) {
        // a turn: one token's q, k or v heads, or a part of them
        const int m = item / p.parts;
        int part = item - m * p.parts;
        const int kind = part < p.parts_q ? 0 : part < p.parts_q + p.parts_k ? 1 : 2;
        part -= kind == 0 ? 0 : kind == 1 ? p.parts_q : p.parts_q + p.parts_k;
        const int set = HEADS * per_warp;
        const int h_end = min(kind == 0 ? p.hq : p.hk, (part + 1) * p.part_sets * set);
        int h0 = part * p.part_sets * set;
        const T* from = static_cast<const T*>(p.x) + static_cast<long long>(m) * p.ldx + (kind == 0 ? 0 : kind == 1 ? p.hq : p.hq + p.hk) * p.D;
        Raw8<T> raw[HEADS];
        auto load_set = [&]() {
#pragma unroll
            for (int j = 0; j < HEADS; ++j) {
                const int h = h0 + j * per_warp + in_warp;
                raw[j] = Raw8<T>();
                if (lives && h < h_end) raw[j] = load_pieces<T, STYLE>(from + h * p.D, sub, half);
            }
        };
        load_set();
        const int pos = STYLE != PLAIN && p.positions != nullptr ? __ldg(p.positions + m) : m;
        const int slot = p.slots != nullptr ? __ldg(p.slots + m) : m;
        // padding (the same for the whole warp)
        if (STYLE != PLAIN && (pos < 0 || pos >= p.num_positions)) continue;
        if (p.slots != nullptr && (slot < 0 || slot >= p.num_slots)) continue;
        T* out = kind == 0   ? static_cast<T*>(p.q_out) + static_cast<long long>(m) * p.ldq
                 : kind == 1 ? static_cast<T*>(p.k_out) + static_cast<long long>(slot) * p.ldk
                             : static_cast<T*>(p.v_out) + static_cast<long long>(slot) * p.ldv;
        if (kind == 2) {
            for (;;) {
#pragma unroll
                for (int j = 0; j < HEADS; ++j) {
                    const int h = h0 + j * per_warp + in_warp;
                    if (lives && h < h_end) store_pieces<T, STYLE>(out + h * p.D, sub, half, raw[j]);
                }
                if ((h0 += set) >= h_end) break;
                load_set();
            }
            continue;
        }
        // With r = 1 / rms, element d becomes r (h[d] w[d] c + h[partner] w[partner] s), s with the sign of d's place in its pair: the weights go
        // into the token's cosines (c) and sines (s) once for all its heads.  (Where nothing is turned c = w and s = 0.)
        float c[8], s[8];
        {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = 1.f;
                s[i] = 0.f;
            }
            if constexpr (STYLE != PLAIN) {
                const float* cs = p.cos_table + static_cast<long long>(pos) * p.ld_table;
                const float* sn = p.sin_table + static_cast<long long>(pos) * p.ld_table;
                auto pair = [&](int first, int second, float cv, float sv) {  // these two of the lane's elements are one pair
                    c[first] = c[second] = cv;
                    s[first] = -sv;
                    s[second] = sv;
                };
                if ((STYLE == SPLIT || (STYLE == PAIRS && 8 * sub + 8 <= p.rot)) && p.wide_table && lives) {
                    const float4 c0 = __ldg(reinterpret_cast<const float4*>(cs + 4 * sub)), s0 = __ldg(reinterpret_cast<const float4*>(sn + 4 * sub));
                    const float cv[4] = {c0.x, c0.y, c0.z, c0.w}, sv[4] = {s0.x, s0.y, s0.z, s0.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) pair(STYLE == PAIRS ? 2 * k : k, STYLE == PAIRS ? 2 * k + 1 : k + 4, cv[k], sv[k]);
                } else if (STYLE == QUARTER && lives) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) pair(k, k + 2, __ldg(cs + 2 * sub + k), __ldg(sn + 2 * sub + k));
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int d = element<STYLE>(i, sub, half);
                        if (lives && d < p.rot) {
                            const int a = STYLE == PAIRS ? d >> 1 : d < half ? d : d - half;
                            const bool second = STYLE == PAIRS ? (d & 1) != 0 : d >= half;
                            c[i] = __ldg(cs + a);
                            s[i] = second ? __ldg(sn + a) : -__ldg(sn + a);
                        }
                    }
                }
            }
            if (weighted && lives) {
                const float* w = s_w[kind];
                float wv[8];
#pragma unroll
                for (int i = 0; i < 8; i += 2) *reinterpret_cast<float2*>(wv + i) = *reinterpret_cast<const float2*>(w + element<STYLE>(i, sub, half));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    c[i] *= wv[i];
                    if constexpr (STYLE == PAIRS) s[i] *= wv[i ^ 1];
                    if constexpr (STYLE == SPLIT) s[i] *= wv[i ^ 4];
                    if constexpr (STYLE == QUARTER) s[i] *= i < 4 ? wv[i ^ 2] : 0.f;
                    if constexpr (STYLE == HALVES) {
                        const int d = 8 * sub + i;
                        s[i] *= w[d >= p.rot ? d : d < half ? d + half : d - half];
                    }
                }
            }
        }
        for (;;) {
#pragma unroll
        for (int j = 0; j < HEADS; ++j) {
            if (h0 + j * per_warp >= h_end) break;  // (the same for the whole warp)
            const int h = h0 + j * per_warp + in_warp;
            float v[8], o[8];
            unpack8<T>(raw[j], v);
            float r = 1.f;
            if (p.norm) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
                if constexpr (LANES == 8 || LANES == 16) {
#pragma unroll
                    for (int f = LANES / 2; f > 0; f >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, f);
                } else {
                    // (the first step is the largest power of two below L)
#pragma unroll
                    for (int f = LANES ? 8 : p.fold; f > 0; f >>= 1) {
                        const float other = __shfl_down_sync(0xffffffffu, ss, f);
                        if (sub + f < L) ss += other;
                    }
                    ss = __shfl_sync(0xffffffffu, ss, head0);
                }
                r = rsqrtf(ss * p.inv_dim + p.eps);
            }
            if constexpr (STYLE == PLAIN) {
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = r * (v[i] * c[i]);
            } else {
                float partner[8];
                if constexpr (STYLE == PAIRS || STYLE == SPLIT || STYLE == QUARTER) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) partner[i] = STYLE == QUARTER && i >= 4 ? 0.f : v[STYLE == PAIRS ? i ^ 1 : STYLE == SPLIT ? i ^ 4 : i ^ 2];
                    if (STYLE == PAIRS && p.rot != p.D) {  // what has no partner takes nothing of one (an infinity there would leave NaN)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (8 * sub + i >= p.rot) partner[i] = 0.f;
                    }
                } else {
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) s_mine[i] = v[i];
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) partner[i] = *s_partner[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = r * fmaf(partner[i], s[i], v[i] * c[i]);
            }
            if (lives && h < h_end) store_pieces<T, STYLE>(out + h * p.D, sub, half, pack8<T>(o));
        }
        if ((h0 += set) >= h_end) break;
        load_set();
        }
    }
}

template <typename T>
cudaError_t launch_t(QkParams& p, int M, cudaStream_t stream) {
    p.L = p.D / 8;
    p.per_warp = 32 / p.L;
    p.fold = 0;
    for (int o = 1; o < p.L; o *= 2) p.fold = o;  // the largest power of two below L
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    // A warp's turn takes all sets of a token's q, k or v where that leaves every SM 32 turns, so that angles and weights are fetched once for
    // all of them; with fewer tokens one set, so that the call is over sooner.  One set against all, us, for 64, 512, 1024, 2048, 2368 (from here
    // on: all), 4608, 9216 tokens: 3 x 24 heads of 128 3.4 / 5.9, 7.0 / 7.5, 10.8 / 9.5, 18.3 / 17.0, 20.4 / 18.5, 34.9 / 32.0, 63.2 / 58.6; 3 x 16 of 72
    // 3.1 / 3.8, 4.6 / 5.6, 7.7 / 6.7, 12.4 / 11.4, 13.1 / 11.7, 21.6 / 20.0, 39.2 / 35.4.  With four q heads to one of k and v turns are of unequal
    // length, and all loses up to between 4608 and 9216 tokens: 32 + 2 x 8 heads of 128 3.2 / 6.7, 5.0 / 8.2, 8.2 / 9.6, 13.0 / 16.6, 14.3 / 17.4,
    // 25.9 / 29.0, 46.7 / 44.0.
    const int per = kHeads<T> * p.per_warp, sets_q = (p.hq + per - 1) / per, sets_k = (p.hk + per - 1) / per;
    const bool whole = static_cast<long long>(M) * 2 >= 32ll * sm_count(device);
    p.part_sets = whole ? (sets_q > sets_k ? sets_q : sets_k) : 1;
    p.parts_q = (sets_q + p.part_sets - 1) / p.part_sets;
    p.parts_k = (sets_k + p.part_sets - 1) / p.part_sets;
    p.parts = p.parts_q + (p.copy_v ? 2 : 1) * p.parts_k;
    const long long items = static_cast<long long>(M) * p.parts;
    if (items > 0x7fffffffll - (1 << 20)) return cudaErrorInvalidValue;  // (the last turn's number stays below 2^31)
    p.items = static_cast<int>(items);
    const long long blocks = (items + kThreads / 32 - 1) / (kThreads / 32), most = 8ll * sm_count(device);
    auto go = [&](auto kern) { return launch_kernel(kern, static_cast<int>(blocks < most ? blocks : most), kThreads, 0, stream, true, p); };
#define DIROTQ_QK_STYLE(STYLE)                                            \
    (p.L == 16  ? go(qk_norm_rope_kernel<T, STYLE, 16>)                   \
     : p.L == 9 ? go(qk_norm_rope_kernel<T, STYLE, 9>)                    \
     : p.L == 8 ? go(qk_norm_rope_kernel<T, STYLE, 8>)                    \
                : go(qk_norm_rope_kernel<T, STYLE, 0>))
    return p.rope == DIROTQ_ROPE_NONE    ? DIROTQ_QK_STYLE(PLAIN)
           : p.rope == DIROTQ_ROPE_PAIRS ? DIROTQ_QK_STYLE(PAIRS)
           : p.rot == p.D                ? DIROTQ_QK_STYLE(SPLIT)
           : 2 * p.rot == p.D            ? DIROTQ_QK_STYLE(QUARTER)
                                         : DIROTQ_QK_STYLE(HALVES);
#undef DIROTQ_QK_STYLE
}

bool bad_float(float v) { return !(v >= 0.f) || v > 3.0e38f; }

}  // namespace

dirotq_status_t qk_check(const dirotq_qk_t* qk, int M) {
    if (!qk || M < 1) return DIROTQ_ERR_INVALID_ARG;
    if (qk->heads_q < 1 || qk->heads_kv < 1 || qk->head_dim < 1) return DIROTQ_ERR_INVALID_ARG;
    if (qk->head_dim % 8 != 0 || qk->head_dim > 256 || qk->heads_q > 65536 || qk->heads_kv > 65536) return DIROTQ_ERR_UNSUPPORTED_SHAPE;
    if (qk->norm != 0 && qk->norm != 1) return DIROTQ_ERR_INVALID_ARG;
    if (qk->norm) {
        if (bad_float(qk->eps) || !dtype_ok(qk->weight_dtype)) return DIROTQ_ERR_INVALID_ARG;
        const size_t es = dtype_size(qk->weight_dtype);
        if (reinterpret_cast<uintptr_t>(qk->q_weight) % es != 0 || reinterpret_cast<uintptr_t>(qk->k_weight) % es != 0) return DIROTQ_ERR_INVALID_ARG;
    }
    if (qk->rope != DIROTQ_ROPE_NONE && qk->rope != DIROTQ_ROPE_PAIRS && qk->rope != DIROTQ_ROPE_HALVES) return DIROTQ_ERR_INVALID_ARG;
    if (qk->rope == DIROTQ_ROPE_NONE) return qk->rot_dim == 0 ? DIROTQ_OK : DIROTQ_ERR_INVALID_ARG;
    if (qk->rot_dim < 2 || qk->rot_dim > qk->head_dim || qk->rot_dim % 2 != 0) return DIROTQ_ERR_INVALID_ARG;
    if (!qk->cos_table || !qk->sin_table || qk->ld_table < qk->rot_dim / 2 || qk->num_positions < 1) return DIROTQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(qk->cos_table) | reinterpret_cast<uintptr_t>(qk->sin_table) | reinterpret_cast<uintptr_t>(qk->positions)) & 3u)
        return DIROTQ_ERR_INVALID_ARG;
    if (!qk->positions && qk->num_positions < M) return DIROTQ_ERR_INVALID_ARG;
    return DIROTQ_OK;
}

cudaError_t launch_qk_norm_rope(const void* x, int dtype, int M, long long ldx, const dirotq_qk_t& qk, void* q_out, long long ldq, void* k_out,
                                long long ldk, void* v_out, long long ldv, const int32_t* slots, int num_slots, cudaStream_t stream) {
    QkParams p = {};
    p.x = x; p.q_out = q_out; p.k_out = k_out; p.v_out = v_out;
    p.ldx = ldx; p.ldq = ldq; p.ldk = ldk; p.ldv = ldv;
    p.hq = qk.heads_q; p.hk = qk.heads_kv; p.D = qk.head_dim;
    p.norm = qk.norm; p.rope = qk.rope; p.rot = qk.rot_dim;
    p.eps = qk.eps;
    p.inv_dim = 1.f / static_cast<float>(qk.head_dim);
    p.wdtype = qk.weight_dtype;
    p.qw = qk.norm ? qk.q_weight : nullptr;
    p.kw = qk.norm ? qk.k_weight : nullptr;
    p.cos_table = qk.cos_table; p.sin_table = qk.sin_table; p.ld_table = qk.ld_table;
    p.num_positions = qk.num_positions;
    p.wide_table = ((reinterpret_cast<uintptr_t>(qk.cos_table) | reinterpret_cast<uintptr_t>(qk.sin_table)) & 15u) == 0 && qk.ld_table % 4 == 0;
    p.positions = qk_positions(qk);
    p.slots = slots; p.num_slots = num_slots;
    // v in its own place needs no copy
    const long long v_off = static_cast<long long>(qk.heads_q + qk.heads_kv) * qk.head_dim * static_cast<long long>(dtype_size(dtype));
    p.copy_v = v_out != nullptr && static_cast<const void*>(v_out) != static_cast<const void*>(static_cast<const char*>(x) + v_off);
    switch (dtype) {
        case DIROTQ_DTYPE_F32: return launch_t<float>(p, M, stream);
        case DIROTQ_DTYPE_BF16: return launch_t<__nv_bfloat16>(p, M, stream);
        default: return launch_t<__half>(p, M, stream);
    }
}

}  // namespace dirotq

using namespace dirotq;

extern "C" {

dirotq_status_t dirotq_qk_norm_rope(const void* x, int dtype, int M, long long ldx, const dirotq_qk_t* qk, void* q_out, long long ldq, void* k_out,
                                    long long ldk, void* v_out, long long ldv, const int32_t* slots, int num_slots, dirotq_stream_t stream) {
    dirotq_status_t st = qk_check(qk, M);
    if (st != DIROTQ_OK) return st;
    if (!x || !q_out || !k_out || !dtype_ok(dtype)) return DIROTQ_ERR_INVALID_ARG;
    const long long es = static_cast<long long>(dtype_size(dtype)), D = qk->head_dim;
    const long long wq = qk->heads_q * D, wk = qk->heads_kv * D, wx = wq + 2 * wk;
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(q_out) | reinterpret_cast<uintptr_t>(k_out) | reinterpret_cast<uintptr_t>(v_out)) & 15u)
        return DIROTQ_ERR_INVALID_ARG;
    // the columns of v are part of a row where v is read; without, a row may end behind k
    if (ldx < (v_out ? wx : wq + wk) || ldq < wq || ldk < wk || (v_out && ldv < wk)) return DIROTQ_ERR_INVALID_ARG;
    if (ldx % 8 != 0 || ldq % 8 != 0 || ldk % 8 != 0 || (v_out && ldv % 8 != 0)) return DIROTQ_ERR_INVALID_ARG;
    if (slots && (num_slots < 1 || (reinterpret_cast<uintptr_t>(slots) & 3u))) return DIROTQ_ERR_INVALID_ARG;
    const char* xb = static_cast<const char*>(x);
    const long long kv_rows = slots ? num_slots : M, xw = (v_out ? wx : wq + wk) * es;
    const bool q_in_place = static_cast<const void*>(q_out) == x && (ldq == ldx || M == 1);
    const bool k_in_place = static_cast<const char*>(k_out) == xb + wq * es && (ldk == ldx || M == 1) && !slots;
    const bool v_in_place = v_out && static_cast<const char*>(v_out) == xb + (wq + wk) * es && (ldv == ldx || M == 1) && !slots;
    if (!q_in_place && rows_overlap(x, M, xw, ldx * es, q_out, M, wq * es, ldq * es)) return DIROTQ_ERR_INVALID_ARG;
    if (!k_in_place && rows_overlap(x, M, xw, ldx * es, k_out, kv_rows, wk * es, ldk * es)) return DIROTQ_ERR_INVALID_ARG;
    if (v_out && !v_in_place && rows_overlap(x, M, xw, ldx * es, v_out, kv_rows, wk * es, ldv * es)) return DIROTQ_ERR_INVALID_ARG;
    if (rows_overlap(q_out, M, wq * es, ldq * es, k_out, kv_rows, wk * es, ldk * es)) return DIROTQ_ERR_INVALID_ARG;
    if (v_out && (rows_overlap(q_out, M, wq * es, ldq * es, v_out, kv_rows, wk * es, ldv * es) ||
                  rows_overlap(k_out, kv_rows, wk * es, ldk * es, v_out, kv_rows, wk * es, ldv * es)))
        return DIROTQ_ERR_INVALID_ARG;
    int dev = 0, major = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
    if (e != cudaSuccess) { set_error("dirotq_qk_norm_rope", e); return DIROTQ_ERR_CUDA; }
    if (major != 10) return DIROTQ_ERR_ARCH;
    e = launch_qk_norm_rope(x, dtype, M, ldx, *qk, q_out, ldq, k_out, ldk, v_out, ldv, slots, num_slots, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { set_error("dirotq_qk_norm_rope", e); return DIROTQ_ERR_CUDA; }
    return DIROTQ_OK;
}

dirotq_status_t dirotq_linear_qkv(const void* x, int M, const dirotq_layer_t* layer, const dirotq_qk_t* qk, void* y, void* workspace,
                                  size_t workspace_bytes, dirotq_stream_t stream) {
    dirotq_status_t st = qk_check(qk, M);
    if (st != DIROTQ_OK) return st;
    st = check_call(layer, M, workspace, workspace_bytes);
    if (st != DIROTQ_OK) return st;
    const int N = layer->geo.N;
    if (static_cast<long long>(qk->heads_q + 2ll * qk->heads_kv) * qk->head_dim != N) return DIROTQ_ERR_INVALID_ARG;
    st = dirotq_linear(x, M, layer, y, workspace, workspace_bytes, stream);
    if (st != DIROTQ_OK) return st;
    const cudaError_t e = launch_qk_norm_rope(y, DIROTQ_DTYPE_BF16, M, N, *qk, y, N, static_cast<uint16_t*>(y) + static_cast<size_t>(qk->heads_q) * qk->head_dim, N,
                                              nullptr, 0, nullptr, 0, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { set_error("dirotq_linear_qkv", e); return DIROTQ_ERR_CUDA; }
    return DIROTQ_OK;
}

}  // extern "C"
