// Product of two MXFP4 operands, and the same with the norm and rotation of q and k in its epilogue.
//
//   y[m,n] = round( D[m,n] + bias[n] ),   D = sum over blocks of 32:  2^(sa[m,blk] + sb[n,blk]) * sum_{k in blk} a[m,k] b[n,k]
//
// The scales are applied inside the tensor core (tcgen05.mma kind::mxf4, block32: K = 64 and two E8M0 scales per row and instruction), which
// accumulates in fp32.
//
// Data movement per k-block of 256 elements: packed codes by TMA (rows of 128 bytes, 128-byte swizzle); the scales of 128 rows as two
// 512-byte atoms by cp.async.bulk, copied into tensor memory with tcgen05.cp.32x128b.warpx4 by two copier warps, which hand the stage
// to the MMA warp through an mbarrier.  An atom's 32-bit words hold the scales of two instructions; the instruction descriptor's scale
// ids (0 or 2) pick the half.
//
// Roles (384 threads): warp 0 TMA producer, warp 1 MMA issuer and owner of the tensor memory, warps 2..3 scale copiers, warps 4..11 epilogue,
// a warpgroup per 128 columns.  Plans:
//   PAIR: clusters of two CTAs share every MMA (cta_group::2, M = 256): 256 rows x 256 columns per pair; each CTA holds its own 128 rows of
//         a, half of b's 256 rows, and the scales of both halves.  One 256-column accumulator: the epilogue reads it into registers and
//         hands it back before it converts.
//   single CTAs, 128 x 128: two accumulators, the two epilogue warpgroups take tiles in turn.
// Every plan adds an output element's products in the same order, so that a row's bits do not depend on the plan.
#include "mxfp4.cuh"
#include "ptx.cuh"

namespace dirotq {
namespace {

constexpr int BM = 128;
constexpr int ATOMS = 1024;            // bytes of the scales of 128 rows and one k-block
constexpr int A_BYTES = BM * 128;      // 16 KB
constexpr int NUM_THREADS = 384;
constexpr int NUM_EPI_WARPS = 8;

template <int BN, bool PAIR>
struct MxPlan {
    static constexpr int NB = BN / 128;             // 128-column blocks of a tile
    static constexpr int B_BYTES = 128 * 128;       // this CTA's rows of b: the tile's (single) or half of them (pair)
    static constexpr int STAGE_BYTES = A_BYTES + B_BYTES + (1 + NB) * ATOMS;  // 34 / 35 KB
    static constexpr int STAGES = 5;
    static constexpr int ACC_BUFS = PAIR ? 1 : 2;
    static constexpr int BAR_OFFSET = STAGES * STAGE_BYTES;
    static constexpr int BIAS_OFFSET = BAR_OFFSET + 256;                         // per warpgroup two buffers of 128 values
    static constexpr int HEADW_OFFSET = BIAS_OFFSET + 4 * 128 * 4;               // q and k weights of a head, 128 values each
    static constexpr int STORE_OFFSET = (HEADW_OFFSET + 2 * 128 * 4 + 1023) / 1024 * 1024;  // 32 rows x 128 bytes per epilogue warp
    static constexpr int SMEM_BYTES = STORE_OFFSET + NUM_EPI_WARPS * 4096 + 1024;
    static constexpr int TMEM_SF = ACC_BUFS * BN;   // columns of the scales: per stage 8 for a, 8 per 128 columns
    static constexpr int SF_COLS = 8 * (1 + NB);
    static_assert(PAIR ? BN == 256 : BN == 128, "plans");
    static_assert(TMEM_SF + STAGES * SF_COLS <= 512, "tensor memory plan");
    static_assert(8 * (4 * STAGES + 4) <= 192, "barriers end below the words at +192");
    static_assert(SMEM_BYTES <= 232448, "shared memory plan");
    static_assert(STAGE_BYTES % 1024 == 0, "operand tiles must stay 1024-byte aligned");
};

struct MxKernelParams {
    int M, N, nkb;
    int a_box, b_box;      // rows of the operands' boxes
    const uint8_t* asf;    // scale atoms
    const uint8_t* bsf;
    const void* bias;
    uint8_t* y;
    long long ldy;
    int* status;
    int f16;               // y and bias are fp16 (else bf16)
    int tma_out;           // rows of y may be written by TMA stores
    int early;             // b may be read while the previous kernel runs
    // norm and rotation of q and k
    int q_cols, k_end;     // columns [0, q_cols) are q, [q_cols, k_end) are k
    int head_shift;        // log2 of head_dim: 6 or 7
    int norm, rope;
    float eps, inv_dim;
    int wdtype;
    const void* qw;
    const void* kw;
    const float* cos_table;
    const float* sin_table;
    long long ld_table;
    int num_positions;
    const int32_t* positions;
};

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
                 : "memory");
}

// Shared-memory descriptor of one scale atom for tcgen05.cp: 32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart.
__device__ __forceinline__ uint64_t sf_desc(uint32_t smem_addr) {
    return static_cast<uint64_t>((smem_addr & 0x3FFFF) >> 4) | static_cast<uint64_t>(128 >> 4) << 16 | static_cast<uint64_t>(128 >> 4) << 32 |
           static_cast<uint64_t>(1) << 46;
}

// One atom into 4 columns of tensor memory, replicated to the four lane quadrants (PAIR: each CTA's own atom into its own memory).
template <bool PAIR>
__device__ __forceinline__ void sf_copy(uint32_t taddr, uint64_t desc) {
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// E2M1 x E2M1 -> fp32, E8M0 scales, both operands K-major; `half` (0 or 1): which pair of the four scale bytes of a word applies.
__host__ __device__ constexpr uint32_t mx_idesc(uint32_t M, uint32_t N, uint32_t half) {
    return (2 * half) << 4 | 1u << 7 | 1u << 10 | (N >> 3) << 17 | 1u << 23 | (M >> 4) << 24 | (2 * half) << 29;
}

template <bool PAIR>
__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t tsfa, uint32_t tsfb,
                                          uint32_t accumulate) {
    if constexpr (PAIR)
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t"
            "}\n" ::"r"(d_tmem),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(tsfa), "r"(tsfb)
            : "memory");
    else
        asm volatile(
            "{\n\t"
            ".reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t"
            "}\n" ::"r"(d_tmem),
            "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(tsfa), "r"(tsfb)
            : "memory");
}

__device__ __forceinline__ float load_16(const void* p, int i, int f16) {
    const uint16_t u = __ldg(static_cast<const uint16_t*>(p) + i);
    return f16 ? __half2float(__ushort_as_half(u)) : __uint_as_float(static_cast<uint32_t>(u) << 16);
}
__device__ __forceinline__ float load_weight(const void* p, int i, int dtype) {
    return p == nullptr ? 1.f : dtype == DIROTQ_DTYPE_F32 ? __ldg(static_cast<const float*>(p) + i) : load_16(p, i, dtype == DIROTQ_DTYPE_F16);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, int f16) {
    if (f16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A barrier of the 128 threads of epilogue warpgroup `g` that makes them agree: true if any of them brings true.
__device__ __forceinline__ bool group_any(int g, bool mine) {
    uint32_t any;
    asm volatile(
        "{\n\t"
        ".reg .pred pin, pout;\n\t"
        "setp.ne.u32 pin, %1, 0;\n\t"
        "bar.red.or.pred pout, %2, 128, pin;\n\t"
        "selp.u32 %0, 1, 0, pout;\n\t"
        "}\n"
        : "=r"(any)
        : "r"(static_cast<uint32_t>(mine)), "r"(1 + g)
        : "memory");
    return any != 0;
}

// Norm and rotation of the D elements of one head, in the registers of one thread.
template <int D>
__device__ __forceinline__ void head_norm_rope(float* v, const float* w, const MxKernelParams& p, const float* cs, const float* sn) {
    if (p.norm) {
        float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
        for (int i = 0; i < D; i += 4) {
            s0 = fmaf(v[i], v[i], s0);
            s1 = fmaf(v[i + 1], v[i + 1], s1);
            s2 = fmaf(v[i + 2], v[i + 2], s2);
            s3 = fmaf(v[i + 3], v[i + 3], s3);
        }
        const float r = rsqrtf(((s0 + s1) + (s2 + s3)) * p.inv_dim + p.eps);
#pragma unroll
        for (int i = 0; i < D; i += 4) {
            const float4 wv = *reinterpret_cast<const float4*>(w + i);
            v[i] *= r * wv.x; v[i + 1] *= r * wv.y; v[i + 2] *= r * wv.z; v[i + 3] *= r * wv.w;
        }
    }
    if (p.rope == DIROTQ_ROPE_PAIRS) {
#pragma unroll
        for (int i = 0; i < D / 2; ++i) {
            const float c = __ldg(cs + i), s = __ldg(sn + i), a = v[2 * i], b = v[2 * i + 1];
            v[2 * i] = a * c - b * s;
            v[2 * i + 1] = a * s + b * c;
        }
    } else if (p.rope == DIROTQ_ROPE_HALVES) {
#pragma unroll
        for (int i = 0; i < D / 2; ++i) {
            const float c = __ldg(cs + i), s = __ldg(sn + i), a = v[i], b = v[i + D / 2];
            v[i] = a * c - b * s;
            v[i + D / 2] = a * s + b * c;
        }
    }
}

template <int BN, bool PAIR, bool QKV>
__global__ void __launch_bounds__(NUM_THREADS, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ CUtensorMap tmap_y,
               const __grid_constant__ MxKernelParams p) {
    using P = MxPlan<BN, PAIR>;
    constexpr int NB = P::NB, STAGES = P::STAGES, ACC_BUFS = P::ACC_BUFS, STAGE_BYTES = P::STAGE_BYTES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t bar_base = smem_base + P::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
    auto sfready_bar = [&](int s) { return bar_base + 8u * (2 * STAGES + s); };
    auto peer_bar = [&](int s) { return bar_base + 8u * (3 * STAGES + s); };  // pairs, leader: the other CTA's stage has landed
    auto tfull_bar = [&](int a) { return bar_base + 8u * (4 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (4 * STAGES + 2 + a); };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + P::BAR_OFFSET + 192);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + P::BAR_OFFSET + 196);

    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;
    const uint32_t cta_rank = PAIR ? blockIdx.x & 1u : 0u;
    constexpr int TILE_ROWS = PAIR ? 2 * BM : BM;
    const int tile_first = PAIR ? static_cast<int>(blockIdx.x >> 1) : static_cast<int>(blockIdx.x);
    const int tile_step = PAIR ? static_cast<int>(gridDim.x >> 1) : static_cast<int>(gridDim.x);
    const int num_m_blocks = (p.M + TILE_ROWS - 1) / TILE_ROWS;
    const int num_tiles = num_m_blocks * ((p.N + BN - 1) / BN);

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
            mbar_init(sfready_bar(s), 2);  // one arrival per copier warp
            mbar_init(peer_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), PAIR ? 2 * NUM_EPI_WARPS * 32 : NUM_EPI_WARPS * 32 / 2);
        }
        mbar_init(bar_base + 200u, 1);  // spare: see umma_drain
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tmap_a);
        tma_prefetch_desc(&tmap_b);
        if (p.tma_out) tma_prefetch_desc(&tmap_y);
    }
    if (warp == 1) {
        if constexpr (PAIR) {
            tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
            tmem_relinquish_pair();
        } else {
            tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
            tmem_relinquish();
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();  // the other CTA's barriers are initialised before anything arrives on them
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_wait();  // everything above touched only this CTA's own shared and tensor memory
    grid_launch_dependents();

    if (warp == 0) {
        // ------------------------------------------------------------ producer
        RingPos<STAGES> at;
        bool ok = true;
        for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step) {
            const int m_blk = (tile % num_m_blocks) * (PAIR ? 2 : 1) + static_cast<int>(cta_rank), n_blk = tile / num_m_blocks;
            const int m0 = m_blk * BM, n0 = n_blk * BN + (PAIR ? static_cast<int>(cta_rank) * 128 : 0);
            // (rows past M or N are filled with zeros and still counted; the atoms of 256 rows always exist)
            const uint8_t* asf = p.asf + (static_cast<size_t>(m_blk >> 1) * p.nkb * 2 + (m_blk & 1)) * ATOMS;
            const uint8_t* bsf = PAIR ? p.bsf + static_cast<size_t>(n_blk) * p.nkb * 2 * ATOMS
                                      : p.bsf + (static_cast<size_t>(n_blk >> 1) * p.nkb * 2 + (n_blk & 1)) * ATOMS;
            for (int kb = 0; kb < p.nkb; ++kb, at.next()) {
                const uint32_t s = at.s;
                if (!mbar_wait(empty_bar(s), at.ph ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER)) { ok = false; break; }
                const uint32_t st = smem_base + s * STAGE_BYTES;
                if (!elect_one()) continue;
                mbar_arrive_expect_tx(full_bar(s), (p.a_box + p.b_box) * 128 + (1 + NB) * ATOMS);
                tma_load_2d(st, &tmap_a, full_bar(s), kb * 128, m0);  // byte coordinates
                tma_load_2d(st + A_BYTES, &tmap_b, full_bar(s), kb * 128, n0);
                bulk_load(st + A_BYTES + P::B_BYTES, asf + static_cast<size_t>(kb) * 2 * ATOMS, ATOMS, full_bar(s));
                bulk_load(st + A_BYTES + P::B_BYTES + ATOMS, bsf + static_cast<size_t>(kb) * 2 * ATOMS, NB * ATOMS, full_bar(s));
            }
        }
        if (!ok && lane == 0) {  // a wait gave up: copies in flight land before the CTA leaves
            const uint32_t first = at.it > STAGES ? at.it - STAGES : 0;
            for (uint32_t j = first; j < at.it; ++j) {
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(full_bar(j % STAGES), (j / STAGES) & 1) && globaltimer_ns() - t0 < 100000000ull) {}
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (cta_rank == 0) {
            constexpr uint32_t idesc0 = mx_idesc(TILE_ROWS, BN, 0), idesc1 = mx_idesc(TILE_ROWS, BN, 1);
            const uint64_t desc0 = umma_desc_sw128(smem_base);
            RingPos<STAGES> at;
            uint32_t tcount = 0;
            bool ok = true;
            for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step, ++tcount) {
                const uint32_t acc = tcount % ACC_BUFS;
                if (!mbar_wait(tempty_bar(acc), ((tcount / ACC_BUFS) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_MMA)) { ok = false; break; }
                tc_fence_after_sync();
                const uint32_t d = tmem_base + acc * BN;
                for (int kb = 0; kb < p.nkb; ++kb, at.next()) {
                    const uint32_t s = at.s;
                    // (the copier warps have seen the stage's loads land, in both CTAs of a pair: their barrier covers the operands)
                    if (!mbar_wait(sfready_bar(s), at.ph, abort_flag, p.status, DEV_TIMEOUT_MMA)) { ok = false; break; }
                    tc_fence_after_sync();
                    const uint32_t tsf = tmem_base + P::TMEM_SF + s * P::SF_COLS;
                    const uint64_t adesc = desc0 + s * (STAGE_BYTES >> 4), bdesc = adesc + (A_BYTES >> 4);
                    if (!elect_one()) continue;
#pragma unroll
                    for (int k = 0; k < 4; ++k)  // K = 64 elements = 32 bytes per instruction
                        umma_mxf4<PAIR>(d, adesc + 2 * k, bdesc + 2 * k, (k & 1) ? idesc1 : idesc0, tsf + 4 * (k >> 1), tsf + 8 + 4 * NB * (k >> 1),
                                        (kb | k) != 0);
                    if constexpr (PAIR) umma_commit_pair(empty_bar(s), 3);
                    else umma_commit(empty_bar(s));
                }
                if (ok && elect_one()) {
                    if constexpr (PAIR) umma_commit_pair(tfull_bar(acc), 3);
                    else umma_commit(tfull_bar(acc));
                }
            }
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------ scale copiers
        RingPos<STAGES> at;
        bool ok = true;
        for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step) {
            for (int kb = 0; kb < p.nkb; ++kb, at.next()) {
                const uint32_t s = at.s;
                if (!mbar_wait(full_bar(s), at.ph, abort_flag, p.status, DEV_TIMEOUT_UNPACK)) { ok = false; break; }
                if constexpr (PAIR) {
                    if (cta_rank != 0) {  // this CTA's stage has landed: the leader acts for both
                        if (warp == 2 && elect_one()) mbar_arrive_cluster(map_to_cta(peer_bar(s), 0));
                        continue;
                    }
                    if (!mbar_wait(peer_bar(s), at.ph, abort_flag, p.status, DEV_TIMEOUT_UNPACK)) { ok = false; break; }
                }
                tc_fence_after_sync();
                const uint32_t sf = smem_base + s * STAGE_BYTES + A_BYTES + P::B_BYTES;
                const uint32_t tsf = tmem_base + P::TMEM_SF + s * P::SF_COLS;
                if (!elect_one()) continue;
                // atom i of a at column 4 i; atom i of column block b at 8 + 4 NB i + 4 b (the blocks of a tile side by side)
                if (warp == 2) {
                    sf_copy<PAIR>(tsf, sf_desc(sf));
                    sf_copy<PAIR>(tsf + 4, sf_desc(sf + 512));
                    if constexpr (NB == 2) sf_copy<PAIR>(tsf + 8, sf_desc(sf + ATOMS));
                } else {
                    if constexpr (NB == 1) sf_copy<PAIR>(tsf + 8, sf_desc(sf + ATOMS));
                    if constexpr (NB == 2) sf_copy<PAIR>(tsf + 12, sf_desc(sf + 2 * ATOMS));
#pragma unroll
                    for (int b = 0; b < NB; ++b) sf_copy<PAIR>(tsf + 8 + 4 * NB + 4 * b, sf_desc(sf + (1 + b) * ATOMS + 512));
                }
                if constexpr (PAIR) umma_commit_pair(sfready_bar(s), 1);  // the leader's barrier only
                else umma_commit(sfready_bar(s));
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        // warp % 4 selects the quadrant of tensor-memory lanes (32 rows); a warpgroup has 128 columns: half of a pair's tile, or the whole of
        // every second 128-column tile.  A thread reads its row's 128 columns and hands the accumulator back before it converts them.
        const int q = warp & 3, group = (warp - 4) >> 2, gt = threadIdx.x & 127;
        float* s_hw = reinterpret_cast<float*>(smem_gen + P::HEADW_OFFSET);
        if constexpr (QKV) {  // (both warpgroups write the same values; each reads behind its own barrier below)
            const int i = gt & ((1 << p.head_shift) - 1);
            s_hw[gt] = load_weight(p.qw, i, p.wdtype);
            s_hw[128 + gt] = load_weight(p.kw, i, p.wdtype);
        }
        uint32_t tcount = PAIR ? 0 : group;
        for (int tile = tile_first + (PAIR ? 0 : group * tile_step); tile < num_tiles; tile += PAIR ? tile_step : 2 * tile_step, tcount += PAIR ? 1 : 2) {
            const int m0 = (tile % num_m_blocks) * TILE_ROWS + (PAIR ? static_cast<int>(cta_rank) * BM : 0);
            const int n0 = (tile / num_m_blocks) * BN + (PAIR ? group * 128 : 0);
            const uint32_t acc = tcount % ACC_BUFS, use = tcount / ACC_BUFS;
            // the bias of these columns goes to shared memory while the tile's MMAs run (two buffers: a warp can be a tile ahead); the
            // barrier orders the stores before the reads and makes the warpgroup agree on whether to go on
            float* s_b = reinterpret_cast<float*>(smem_gen + P::BIAS_OFFSET) + (group * 2 + (use & 1)) * 128;
            s_b[gt] = p.bias != nullptr && n0 + gt < p.N ? load_16(p.bias, n0 + gt, p.f16) : 0.f;
            const bool failed = !mbar_wait(tfull_bar(acc), use & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
            if (group_any(group, failed)) break;
            tc_fence_after_sync();
            const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + acc * BN + (PAIR ? group * 128 : 0);
            uint32_t raw[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(taddr + c * 32, raw[c]);
            tmem_ld_wait();
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_fence(raw[c]);
            tc_fence_before_sync();
            if constexpr (PAIR) mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));  // the leader's barrier
            else mbar_arrive(tempty_bar(acc));
            const int row0 = m0 + q * 32;
            float* v = reinterpret_cast<float*>(&raw[0][0]);
#pragma unroll
            for (int i = 0; i < 128; i += 4) {
                const float4 b = *reinterpret_cast<const float4*>(s_b + i);
                v[i] += b.x; v[i + 1] += b.y; v[i + 2] += b.z; v[i + 3] += b.w;
            }
            if constexpr (QKV) {
                // columns are whole heads: 128 is one head of 128 or two of 64
                const int row = row0 + lane;
                int pos = row;
                if (p.positions != nullptr && row < p.M) pos = __ldg(p.positions + row);
                if (n0 < p.k_end && row < p.M && (p.rope == DIROTQ_ROPE_NONE || (pos >= 0 && pos < p.num_positions))) {
                    const float* cs = p.cos_table + static_cast<long long>(pos) * p.ld_table;
                    const float* sn = p.sin_table + static_cast<long long>(pos) * p.ld_table;
                    if (p.head_shift == 7) {
                        head_norm_rope<128>(v, n0 < p.q_cols ? s_hw : s_hw + 128, p, cs, sn);
                    } else {
                        head_norm_rope<64>(v, n0 < p.q_cols ? s_hw : s_hw + 128, p, cs, sn);
                        if (n0 + 64 < p.k_end) head_norm_rope<64>(v + 64, n0 + 64 < p.q_cols ? s_hw : s_hw + 128, p, cs, sn);
                    }
                }
            }
            // outputs leave through a staging tile per warp, 64 columns at a time (128-byte swizzle: a quarter-warp's pieces fall into different
            // banks): a TMA store writes whole lines and clips at M and N; what it cannot address is written by the lanes
            const uint32_t sbuf = smem_base + P::STORE_OFFSET + static_cast<uint32_t>(warp - 4) * 4096u;
#pragma unroll
            for (int cc = 0; cc < 2; ++cc) {
                if (lane == 0) bulk_wait_group_read_all();  // the staging tile's previous contents have been read
                __syncwarp();
#pragma unroll
                for (int p8 = 0; p8 < 8; ++p8) {
                    const float* e = v + cc * 64 + p8 * 8;
                    const uint32_t dst = sbuf + static_cast<uint32_t>(lane) * 128u + (static_cast<uint32_t>(p8 ^ (lane & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(pack2(e[0], e[1], p.f16)), "r"(pack2(e[2], e[3], p.f16)),
                                 "r"(pack2(e[4], e[5], p.f16)), "r"(pack2(e[6], e[7], p.f16))
                                 : "memory");
                }
                const int col0 = n0 + cc * 64;
                // (a TMA store writes 16-byte pieces whole: a ragged last one is left to the lanes)
                if (p.tma_out && (col0 + 64 <= p.N || (p.N & 7) == 0)) {
                    fence_proxy_async_smem();  // these writes -> visible to the copy engine
                    __syncwarp();
                    if (lane == 0 && row0 < p.M && col0 < p.N) {
                        tma_store_2d(&tmap_y, sbuf, col0, row0);
                        bulk_commit_group();
                    }
                } else {
                    __syncwarp();
                    const int rows = min(32, p.M - row0), cols = min(64, p.N - col0);
                    for (int r = 0; r < rows; ++r) {
                        uint16_t* out = reinterpret_cast<uint16_t*>(p.y) + static_cast<long long>(row0 + r) * p.ldy + col0;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int c = lane + 32 * h;
                            uint16_t e;
                            const uint32_t src = sbuf + static_cast<uint32_t>(r) * 128u + (static_cast<uint32_t>((c >> 3) ^ (r & 7)) << 4) + (c & 7) * 2;
                            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(e) : "r"(src) : "memory");
                            if (c < cols) out[c] = e;
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (lane == 0) bulk_wait_group_all();  // this warp's stores are performed before the CTA leaves
    }

    if constexpr (PAIR) {
        if (warp == 1 && lane == 0 && cta_rank == 0 && *abort_flag != 0) umma_drain<true>(bar_base + 200u);  // let issued MMAs finish first
        tc_fence_before_sync();
        cluster_sync_all();  // neither CTA leaves while the other may still read its operands or signal its barriers
        if (warp == 1) {
            tc_fence_after_sync();
            tmem_dealloc_pair(tmem_base, 512);
        }
    } else {
        if (warp == 1 && lane == 0 && *abort_flag != 0) umma_drain(bar_base + 200u);
        tc_fence_before_sync();
        __syncthreads();
        if (warp == 1) {
            tc_fence_after_sync();
            tmem_dealloc(tmem_base, 512);
        }
    }
}

template <int BN, bool PAIR, bool QKV>
dirotq_status_t launch_plan(const MxGemmArgs& a, const CUtensorMap& tmap_y, MxKernelParams& p, cudaStream_t stream) {
    using P = MxPlan<BN, PAIR>;
    auto kern = mx_gemm_kernel<BN, PAIR, QKV>;
    const int device = a.b->device, sms = sm_count(device);
    static SmemOptIn<1> opt_in;
    if (!opt_in.ensure(kern, 0, device, P::SMEM_BYTES)) return DIROTQ_ERR_CUDA;
    const long long rows = PAIR ? 2 * BM : BM;
    const long long tiles = (p.M + rows - 1) / rows * ((p.N + BN - 1) / BN);
    cudaError_t err;
    if constexpr (PAIR) {
        const int pairs = static_cast<int>(tiles < sms / 2 ? tiles : sms / 2);
        err = launch_kernel_pairs(kern, 2 * pairs, NUM_THREADS, P::SMEM_BYTES, stream, true, a.a->tmap, a.b->tmap, tmap_y, p);
    } else {
        err = launch_kernel(kern, static_cast<int>(tiles < sms ? tiles : sms), NUM_THREADS, P::SMEM_BYTES, stream, true, a.a->tmap, a.b->tmap, tmap_y, p);
    }
    if (err != cudaSuccess) set_error("mx_gemm_kernel", err);
    return err == cudaSuccess ? DIROTQ_OK : DIROTQ_ERR_CUDA;
}

}  // namespace

dirotq_status_t launch_mx_gemm(const MxGemmArgs& a, cudaStream_t stream) {
    MxKernelParams p = {};
    p.M = a.a->rows;
    p.N = a.b->rows;
    p.nkb = a.a->lay.nkb;
    p.a_box = a.a->box;
    p.b_box = a.b->box;
    p.asf = reinterpret_cast<const uint8_t*>(a.a->buffer) + a.a->lay.off_scales;
    p.bsf = reinterpret_cast<const uint8_t*>(a.b->buffer) + a.b->lay.off_scales;
    p.bias = a.bias;
    p.y = static_cast<uint8_t*>(a.y);
    p.ldy = a.ldy;
    p.status = a.status;
    p.f16 = a.y_dtype == DIROTQ_DTYPE_F16;
    p.early = a.early_weights;
    p.tma_out = (reinterpret_cast<uintptr_t>(a.y) & 15u) == 0 && a.ldy % 8 == 0;
    CUtensorMap tmap_y = a.a->tmap;  // (not used without TMA stores)
    if (p.tma_out) {
        const dirotq_status_t st =
            encode_tmap_2d(&tmap_y, p.f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, a.y, (uint64_t)p.N, (uint64_t)p.M,
                           (uint64_t)a.ldy * 2, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B);
        if (st != DIROTQ_OK) return st;
    }
    if (a.qk) {
        const dirotq_qk_t& qk = *a.qk;
        p.q_cols = qk.heads_q * qk.head_dim;
        p.k_end = p.q_cols + qk.heads_kv * qk.head_dim;
        p.head_shift = qk.head_dim == 128 ? 7 : 6;
        p.norm = qk.norm;
        p.rope = qk.rope;
        p.eps = qk.eps;
        p.inv_dim = 1.f / static_cast<float>(qk.head_dim);
        p.wdtype = qk.weight_dtype;
        p.qw = qk.norm ? qk.q_weight : nullptr;
        p.kw = qk.norm ? qk.k_weight : nullptr;
        p.cos_table = qk.cos_table;
        p.sin_table = qk.sin_table;
        p.ld_table = qk.ld_table;
        p.num_positions = qk.num_positions;
        p.positions = qk.positions;
    }
    // CTA pairs above 128 rows, where a second row block exists
    if (p.M > BM) return a.qk ? launch_plan<256, true, true>(a, tmap_y, p, stream) : launch_plan<256, true, false>(a, tmap_y, p, stream);
    return a.qk ? launch_plan<128, false, true>(a, tmap_y, p, stream) : launch_plan<128, false, false>(a, tmap_y, p, stream);
}

}  // namespace dirotq
