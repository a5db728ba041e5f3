// RMS norm of every head of q and k and the rotation by the token's position, in one pass over the output of a fused q/k/v projection.
//
// A group of LANES lanes (the power of two that covers head_dim at eight elements per lane) holds one head: the sum of squares is a few
// shuffles, pairs (2i, 2i+1) lie in one lane, and the partner half a rotation away is fetched from the lane that holds it, or through shared
// memory where the halves do not fall on whole lanes.  A block of threads serves one token, so that its cosines and sines are read once per
// lane and kept for all of the lane's heads.
#include "mxfp4.cuh"
#include "ptx.cuh"

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
};

__device__ __forceinline__ float weight_at(const void* p, int i, int dtype) {
    if (p == nullptr) return 1.f;
    if (dtype == DIROTQ_DTYPE_F32) return __ldg(static_cast<const float*>(p) + i);
    const uint16_t u = __ldg(static_cast<const uint16_t*>(p) + i);
    return dtype == DIROTQ_DTYPE_F16 ? __half2float(__ushort_as_half(u)) : __uint_as_float(static_cast<uint32_t>(u) << 16);
}

template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const QkParams p) {
    constexpr int GROUPS = kThreads / LANES;
    __shared__ float s_head[GROUPS][LANES * 8];
    const int sub = threadIdx.x & (LANES - 1), group = threadIdx.x / LANES;
    const int d0 = sub * 8;
    const bool has = d0 < p.D;
    grid_dependency_wait();  // x is the previous kernel's output
    grid_launch_dependents();
    const int m = blockIdx.x;
    const int pos = p.positions != nullptr ? __ldg(p.positions + m) : m;
    if (p.rope != DIROTQ_ROPE_NONE && (pos < 0 || pos >= p.num_positions)) return;  // padding
    int slot = m;
    if (p.slots != nullptr) {
        slot = __ldg(p.slots + m);
        if (slot < 0 || slot >= p.num_slots) return;
    }
    // the angles of this lane's elements: element d is turned by c[d], s[d] (s with the sign of its place in the pair)
    float c[8], s[8];
    const int half = p.rot >> 1;
    if (p.rope != DIROTQ_ROPE_NONE) {
        const float* cs = p.cos_table + static_cast<long long>(pos) * p.ld_table;
        const float* sn = p.sin_table + static_cast<long long>(pos) * p.ld_table;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = d0 + i;
            c[i] = 1.f;
            s[i] = 0.f;
            if (d < p.rot) {
                const int a = p.rope == DIROTQ_ROPE_PAIRS ? d >> 1 : d < half ? d : d - half;
                const bool second = p.rope == DIROTQ_ROPE_PAIRS ? (d & 1) != 0 : d >= half;
                c[i] = __ldg(cs + a);
                s[i] = second ? __ldg(sn + a) : -__ldg(sn + a);
            }
        }
    }
    const int heads = p.hq + p.hk + (p.copy_v ? p.hk : 0);
    const T* row = static_cast<const T*>(p.x) + static_cast<long long>(m) * p.ldx;
    // (every lane of a warp makes the same number of turns: shuffles below take whole warps)
    for (int h0 = 0; h0 < heads; h0 += GROUPS) {
        const int h = h0 + group;
        const bool live = h < heads && has;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
        if (live) load8<T>(row + static_cast<long long>(h) * p.D + d0, v);
        const bool is_v = h >= p.hq + p.hk;
        if (p.norm) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float r = rsqrtf(ss * p.inv_dim + p.eps);
            if (live && !is_v) {
                const void* w = h < p.hq ? p.qw : p.kw;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= r * weight_at(w, d0 + i, p.wdtype);
            }
        }
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i];
        if (p.rope == DIROTQ_ROPE_PAIRS) {
            if (!is_v) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    o[i] = v[i] * c[i] + v[i + 1] * s[i];
                    o[i + 1] = v[i + 1] * c[i + 1] + v[i] * s[i + 1];
                }
            }
        } else if (p.rope == DIROTQ_ROPE_HALVES) {
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) s_head[group][d0 + i] = v[i];
            __syncwarp();
            if (!is_v) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int d = d0 + i;
                    if (d < p.rot) o[i] = v[i] * c[i] + s_head[group][d < half ? d + half : d - half] * s[i];
                }
            }
        }
        if (live) {
            T* out = h < p.hq          ? static_cast<T*>(p.q_out) + static_cast<long long>(m) * p.ldq + h * p.D
                     : h < p.hq + p.hk ? static_cast<T*>(p.k_out) + static_cast<long long>(slot) * p.ldk + (h - p.hq) * p.D
                                       : static_cast<T*>(p.v_out) + static_cast<long long>(slot) * p.ldv + (h - p.hq - p.hk) * p.D;
            store8<T>(out + d0, o);
        }
    }
}

template <typename T>
cudaError_t launch_t(const QkParams& p, int M, cudaStream_t stream) {
    auto kern = p.D <= 32 ? qk_norm_rope_kernel<T, 4> : p.D <= 64 ? qk_norm_rope_kernel<T, 8> : p.D <= 128 ? qk_norm_rope_kernel<T, 16> : qk_norm_rope_kernel<T, 32>;
    return launch_kernel(kern, M, kThreads, 0, stream, true, p);
}

bool bad_float(float v) { return !(v >= 0.f) || v > 3.0e38f; }

// Whether the rows [0, rows) of `width` bytes at `stride` bytes from a, and the rows of b, can share a byte: their whole ranges are compared,
// and where both have the same stride, the columns as well.
bool overlap(const void* a, long long rows_a, long long width_a, long long stride_a, const void* b, long long rows_b, long long width_b, long long stride_b) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + static_cast<uintptr_t>((rows_a - 1) * stride_a + width_a), b1 = b0 + static_cast<uintptr_t>((rows_b - 1) * stride_b + width_b);
    if (a1 <= b0 || b1 <= a0) return false;
    if (stride_a == stride_b) {
        const uintptr_t s = static_cast<uintptr_t>(stride_a);
        const uintptr_t off = (b0 >= a0 ? b0 - a0 : s - (a0 - b0) % s) % s;  // b's columns relative to a's
        if (off >= static_cast<uintptr_t>(width_a) && off + static_cast<uintptr_t>(width_b) <= s) return false;
    }
    return true;
}

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
    p.wdtype = qk.weight_dtype; p.qw = qk.q_weight; p.kw = qk.k_weight;
    p.cos_table = qk.cos_table; p.sin_table = qk.sin_table; p.ld_table = qk.ld_table;
    p.num_positions = qk.num_positions;
    p.positions = qk.rope != DIROTQ_ROPE_NONE ? qk.positions : nullptr;
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
    if (!q_in_place && overlap(x, M, xw, ldx * es, q_out, M, wq * es, ldq * es)) return DIROTQ_ERR_INVALID_ARG;
    if (!k_in_place && overlap(x, M, xw, ldx * es, k_out, kv_rows, wk * es, ldk * es)) return DIROTQ_ERR_INVALID_ARG;
    if (v_out && !v_in_place && overlap(x, M, xw, ldx * es, v_out, kv_rows, wk * es, ldv * es)) return DIROTQ_ERR_INVALID_ARG;
    if (overlap(q_out, M, wq * es, ldq * es, k_out, kv_rows, wk * es, ldk * es)) return DIROTQ_ERR_INVALID_ARG;
    if (v_out && (overlap(q_out, M, wq * es, ldq * es, v_out, kv_rows, wk * es, ldv * es) ||
                  overlap(k_out, kv_rows, wk * es, ldk * es, v_out, kv_rows, wk * es, ldv * es)))
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
