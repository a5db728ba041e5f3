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
// Roles: warp 0 TMA producer, warp 1 MMA issuer and owner of the tensor memory, warps 2..3 scale copiers, 16 epilogue warps in two
// groups.  Plans:
//   PAIR: clusters of two CTAs share every MMA (cta_group::2, M = 256): 256 rows x 256 columns per pair; each CTA holds its own 128 rows of
//         a, half of b's 256 rows, and the scales of both halves.  One 256-column accumulator, an epilogue group per half of it: the group
//         reads it into registers and hands it back before it converts.
//   single CTAs, 128 rows x 128 or 64 columns: two accumulators, the two epilogue groups take tiles in turn.
//   FUSE (single CTAs, few rows): the activations are quantized by the kernel itself, by every CTA for itself, into shared memory, where
//         their codes and scales stay; the ring carries b alone.
// Every plan adds an output element's products in the same order, so that a row's bits do not depend on the plan.
//
// Measured: 4608 rows, 3072 -> 12288 68 us, 5.1 PFLOP/s; 12288 -> 3072 56 us, 6.2 PFLOP/s (pairs, 1.97 GHz; at the power cap, after
// seconds of it, 1.45 GHz, 84 and 72 us).  With one kind of work left out at a time (12288 -> 12288, us per k-block of 256 rows x 256 columns): everything 0.40; no operand
// loads 0.31, no MMAs 0.25, no scale copies 0.36, no outputs 0.37: loads into shared memory and the tensor core's reads of it share its
// bandwidth, and neither a shorter hand-over (both CTAs' loads counted on the leader's barrier: 0.5 %) nor earlier releases of the accumulator
// (0 %) change that.  4608 tokens of q/k/v (3 x 24 heads of 128): 66 us with norm and rotation, quantizer included, 59 without, 24 for the two as a pass.
#include "mxfp4.cuh"
#include "ptx.cuh"
#include "qk_plan.h"

#include <atomic>
#include <type_traits>

namespace dirotq {
namespace {

constexpr int BM = 128;
constexpr int ATOMS = 1024;            // bytes of the scales of 128 rows and one k-block
constexpr int A_BYTES = BM * 128;      // 16 KB
constexpr int EPI_WARPS = 16;
constexpr int NUM_THREADS = 128 + EPI_WARPS * 32;
constexpr int GROUP_THREADS = EPI_WARPS * 16;  // of one of the two epilogue groups

template <int BN, bool PAIR, bool FUSE>
struct MxPlan {
    static constexpr int NB = BN == 256 ? 2 : 1;                              // 128-column blocks whose scales a stage holds
    // k-blocks per stage: two where a k-block is little work, so that a short call pays for the roles' waits and hand-overs half as often
    // (128 rows, 12288 -> 3072: 9.6 against 10.3 us; 16 rows, 3072 -> 9216: 6.4 against 6.9 with the quantizer).  What is left at 64 columns
    // is 0.15 us a k-block; whether its four MMAs, which add to one accumulator in order, take that or their operands' way into shared memory was not
    // measured apart.
    static constexpr int KBS = BN == 64 || FUSE ? 2 : 1;
    static constexpr int A_STAGE = FUSE ? 0 : A_BYTES;
    static constexpr int B_BYTES = (PAIR ? BN / 2 : BN) * 128;                // this CTA's rows of b: the tile's (single) or half of them (pair)
    static constexpr int B_OFFSET = KBS * A_STAGE;
    static constexpr int SF_OFFSET = B_OFFSET + KBS * B_BYTES;                // scales of a (unless they stay), then of b
    static constexpr int SFB_OFFSET = SF_OFFSET + (FUSE ? 0 : KBS * ATOMS);
    static constexpr int STAGE_BYTES = SFB_OFFSET + KBS * NB * ATOMS;         // pair 35 KB, single 34 / 52 KB, fused 34 / 18 KB
    static constexpr int STAGES = FUSE ? (BN == 64 ? 8 : 4) : (BN == 64 ? 4 : 6);
    static constexpr int RESIDENT = FUSE ? 64 * 1024 : 0;                     // codes and scales of the activations (see kFuseUnits)
    static constexpr int BAR_OFFSET = RESIDENT + STAGES * STAGE_BYTES;
    static constexpr int BIAS_OFFSET = BAR_OFFSET + 512;                      // per epilogue group two buffers of 128 values
    static constexpr int HEADW_OFFSET = BIAS_OFFSET + 4 * 128 * 4;            // q and k weights of a head, 128 values each
    static constexpr int EDGE_OFFSET = HEADW_OFFSET + 2 * 128 * 4;            // 8 rows x 64 bytes per epilogue warp: rows of y of any alignment
    static constexpr int SUM_OFFSET = EDGE_OFFSET + EPI_WARPS * 512;          // sums of squares of 32 rows per epilogue warp
    static constexpr int SMEM_BYTES = SUM_OFFSET + EPI_WARPS * 128 + 1024;
    static constexpr int ACC_BUFS = PAIR ? 1 : 2;
    static constexpr int TMEM_SF = ACC_BUFS * BN;                             // columns of the scales: per k-block 8 for a, 8 per 128 columns
    static constexpr int SF_COLS = 8 * (1 + NB);
    static_assert(PAIR ? BN == 256 && !FUSE : BN == 128 || BN == 64, "plans");
    static_assert(TMEM_SF + STAGES * KBS * SF_COLS <= 512, "tensor memory plan");
    static_assert(8 * ((PAIR ? 4 : 3) * STAGES + 5) <= 480, "barriers end below the words at +480");
    static_assert(SMEM_BYTES <= 232448, "shared memory plan");
    static_assert(STAGE_BYTES % 1024 == 0, "operand tiles must stay 1024-byte aligned");
    // (an MMA reads 128 rows wherever fewer are kept: past the last ones it reads what lies behind, whose results are not stored)
    static_assert(!FUSE || STAGES * STAGE_BYTES >= A_BYTES, "a k-block's 128 rows end inside the ring");
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
    int wide_out;          // rows of y are 16-byte (1) or 32-byte (2) aligned
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
    int wide_table;        // rows of both tables are 32-byte aligned
    int num_positions;
    const int32_t* positions;
    // FUSE: the activations as they are
    const void* x;
    long long ldx;
    int x_dtype, x_wide;   // x_wide: rows are 16-byte aligned
    int K, scale_rule;
    int groups;            // blocks of 8 rows that exist
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
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if constexpr (F16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Named barrier ID of the THREADS of an epilogue group that makes them agree: true if any of them brings true.
template <int ID, int THREADS>
__device__ __forceinline__ bool group_any(bool mine) {
    uint32_t any;
    asm volatile(
        "{\n\t"
        ".reg .pred pin, pout;\n\t"
        "setp.ne.u32 pin, %1, 0;\n\t"
        "bar.red.or.pred pout, %2, %3, pin;\n\t"
        "selp.u32 %0, 1, 0, pout;\n\t"
        "}\n"
        : "=r"(any)
        : "r"(static_cast<uint32_t>(mine)), "n"(ID), "n"(THREADS)
        : "memory");
    return any != 0;
}

// 16 tensor-memory lanes x 256 bits, eight times along the columns (64 columns): register 4 j + 2 h + e of lane l holds row l / 4 + 8 h and
// column 8 j + 2 (l % 4) + e.
__device__ __forceinline__ void tmem_ld_16x256b_x8(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
}

// Within four consecutive lanes: lane t's word k becomes lane k's word t.
__device__ __forceinline__ void transpose4(uint32_t (&w)[4], int t) {
    const bool odd = (t & 1) != 0, upper = (t & 2) != 0;
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, odd ? w[k] : w[k + 1], 1);
        if (odd) w[k] = x;
        else w[k + 1] = x;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, upper ? w[k] : w[k + 2], 2);
        if (upper) w[k] = x;
        else w[k + 2] = x;
    }
}

// Run of 32 columns from n0 of eight rows from row0, lane (l / 4, l % 4) with 8 consecutive columns of its row: straight where rows are wide enough
// apart and whole, else through 512 bytes of shared memory and written by consecutive lanes.
__device__ __forceinline__ void store_run(const MxKernelParams& p, int row0, int rows, int n0, int lane, const uint4& out, uint32_t edge, bool whole) {
    uint16_t* y = reinterpret_cast<uint16_t*>(p.y) + static_cast<long long>(row0) * p.ldy + n0;
    const int t = lane & 3, r4 = lane >> 2;
    if (whole) {
        if (r4 < rows) __stcs(reinterpret_cast<uint4*>(y + r4 * p.ldy + 8 * t), out);
        return;
    }
    __syncwarp();
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(edge + r4 * 64 + t * 16), "r"(out.x), "r"(out.y), "r"(out.z), "r"(out.w) : "memory");
    __syncwarp();
    uint16_t e[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(e[r]) : "r"(edge + r * 64 + 2 * lane) : "memory");
    if (n0 + lane < p.N)
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < rows) y[r * p.ldy + lane] = e[r];
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
    return v;
}
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) { return pair_of(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void split_pair(uint64_t v, uint32_t& lo, uint32_t& hi) { asm("mov.b64 {%0, %1}, %2;" : "=r"(lo), "=r"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// Cosines and sines of eight consecutive angles (`wide`: 32-byte aligned, one load each).
__device__ __forceinline__ void load_angles(const float* cs, const float* sn, int wide, float (&c)[8], float (&s)[8]) {
    if (wide) {
        asm volatile("ld.global.nc.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]), "=f"(c[4]), "=f"(c[5]), "=f"(c[6]), "=f"(c[7])
                     : "l"(cs));
        asm volatile("ld.global.nc.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(s[0]), "=f"(s[1]), "=f"(s[2]), "=f"(s[3]), "=f"(s[4]), "=f"(s[5]), "=f"(s[6]), "=f"(s[7])
                     : "l"(sn));
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            c[k] = __ldg(cs + k);
            s[k] = __ldg(sn + k);
        }
    }
}

// What store_heads needs of its rows besides their values: positions, whether they are turned, and the angles of the rows that it turns next.
template <int SETS, bool HALVES>
struct HeadRows {
    int pos[SETS][2];      // of row 16 set + 8 hi + l / 4
    bool turned[SETS][2];
    bool all;              // every row that exists is turned
    float c[8], s[8];

    __device__ __forceinline__ void start(const MxKernelParams& p, int row0, bool head, int at0, int lane) {
        all = true;
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                const int row = row0 + 16 * set + 8 * hi + (lane >> 2);
                const bool here = head && row < p.M;
                pos[set][hi] = here && p.positions != nullptr ? __ldg(p.positions + row) : row;
                turned[set][hi] = here && (p.rope == DIROTQ_ROPE_NONE || (pos[set][hi] >= 0 && pos[set][hi] < p.num_positions));
                all = all && (turned[set][hi] || !here);
            }
        if (head) fetch(p, 0, 0, at0, lane);
    }
    __device__ __forceinline__ void fetch(const MxKernelParams& p, int set, int hi, int at0, int lane) {
        if (p.rope == DIROTQ_ROPE_NONE) return;
        const long long a = static_cast<long long>(turned[set][hi] ? pos[set][hi] : 0) * p.ld_table + (HALVES ? at0 : at0 >> 1) + 8 * (lane & 3);
        load_angles(p.cos_table + a, p.sin_table + a, p.wide_table, c, s);  // (row 0's where a row is not turned)
    }
};

// The columns of a fused projection's tile that one warp has: two runs of 32 columns, at `run0` and `run1` of the group's, of SETS * 16 rows from
// row0.  raw[set][run][4 k + 2 hi + e] is column 8 k + 2 t + e of the run, row 16 set + 8 hi + l / 4, and is so through bias, sum of squares and
// norm, two fp32 operations at a time; then the row's four lanes exchange it, so that each has whole sectors of the tables and of y.  What counts here is
// latency: with the angles loaded where they are used, 4608 tokens of 3 x 24 heads took 74 us, whether the tables were in L1 or not, with the next rows'
// angles on their way 67, with the first rows' and the positions fetched behind the MMAs 66.  (A row per lane needs no exchange and half the instructions,
// but touches 32 lines a load and store: 79 us, all loads at their use.)
//   HALVES: element i and i + D/2 are in one warp: the runs are the halves of a head of 64 (run1 = run0 + 32), or halves of the halves of one of
//           128 (run1 = run0 + 64); a lane has columns 8 t .. 8 t + 7 of both runs, which are turned with one another by eight angles.
//   else:   64 columns side by side; a lane has columns 16 t .. 16 t + 15, eight pairs.
// The two warps of a head of 128 (`split`) add up their sums of squares through s_sum, `pair_bar` their named barrier.
template <int SETS, bool F16, bool HALVES>
__device__ __forceinline__ void store_heads(uint32_t (&raw)[SETS][2][16], HeadRows<SETS, HALVES>& rows_of, const MxKernelParams& p, int row0, int n0, int run0,
                                            int run1, bool split, int lane, const float* s_b, const float* s_hw, float* s_sum, const float* s_sum_other, int pair_bar,
                                            uint32_t edge, bool whole) {
    const int t = lane & 3, r4 = lane >> 2;
    const bool head = n0 + run0 < p.k_end;  // q or k (the same for the whole warp, and for the two of a head)
    const int at0 = run0 & ((1 << p.head_shift) - 1), at1 = run1 & ((1 << p.head_shift) - 1);  // the runs' places in the head
    uint64_t sum[SETS][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 b = *reinterpret_cast<const float2*>(s_b + (j ? run1 : run0) + 8 * k + 2 * t);
            const uint64_t b2 = pair_of(b.x, b.y);
#pragma unroll
            for (int set = 0; set < SETS; ++set)
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) {
                    uint32_t &x = raw[set][j][4 * k + 2 * hi], &y = raw[set][j][4 * k + 2 * hi + 1];
                    const uint64_t v = add2(pair_of(x, y), b2);
                    sum[set][hi] = j + k ? fma2(v, v, sum[set][hi]) : mul2(v, v);
                    split_pair(v, x, y);
                }
        }
    if (head && p.norm) {
        float ss[SETS][2];
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
                uint32_t x, y;
                split_pair(sum[set][hi], x, y);
                ss[set][hi] = __uint_as_float(x) + __uint_as_float(y);
                ss[set][hi] += __shfl_xor_sync(0xffffffffu, ss[set][hi], 1);
                ss[set][hi] += __shfl_xor_sync(0xffffffffu, ss[set][hi], 2);
                if (split && t == 0) s_sum[16 * set + 8 * hi + r4] = ss[set][hi];
            }
        if (split) {
            asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
#pragma unroll
            for (int set = 0; set < SETS; ++set)
#pragma unroll
                for (int hi = 0; hi < 2; ++hi) ss[set][hi] += s_sum_other[16 * set + 8 * hi + r4];
        }
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) ss[set][hi] = rsqrtf(ss[set][hi] * p.inv_dim + p.eps);
        const float* w = s_hw + (n0 + run0 < p.q_cols ? 0 : 128);
        auto scale = [&](bool every) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 g = *reinterpret_cast<const float2*>(w + (j ? at1 : at0) + 8 * k + 2 * t);
#pragma unroll
                    for (int set = 0; set < SETS; ++set)
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi) {
                            uint32_t &x = raw[set][j][4 * k + 2 * hi], &y = raw[set][j][4 * k + 2 * hi + 1];
                            const uint64_t v = mul2(pair_of(x, y), mul2(pair_of(g.x, g.y), pair_of(ss[set][hi], ss[set][hi])));
                            if (every || rows_of.turned[set][hi]) split_pair(v, x, y);
                        }
                }
        };
        if (__all_sync(0xffffffffu, rows_of.all)) scale(true);
        else scale(false);
    }
#pragma unroll
    for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
            const int row = row0 + 16 * set + 8 * hi + r4;
            // the row's values as this lane has them from here on: HALVES: run0's columns 8 t .., then run1's; else columns 16 t ..
            uint32_t v[16];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t even[4], odd[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int J = HALVES ? 4 * j + k : 2 * k + j;  // columns 8 J + 2 t, + 1 of the 64
                    even[k] = raw[set][J >> 2][4 * (J & 3) + 2 * hi];
                    odd[k] = raw[set][J >> 2][4 * (J & 3) + 2 * hi + 1];
                }
                transpose4(even, t);
                transpose4(odd, t);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v[8 * j + 2 * k] = even[k];
                    v[8 * j + 2 * k + 1] = odd[k];
                }
            }
            if (p.rope != DIROTQ_ROPE_NONE && rows_of.turned[set][hi]) {
                const float(&c)[8] = rows_of.c, (&s)[8] = rows_of.s;
                if constexpr (HALVES) {
#pragma unroll
                    for (int k = 0; k < 8; k += 2) {
                        const uint64_t x = pair_of(v[k], v[k + 1]), y = pair_of(v[8 + k], v[9 + k]), cc = pair_of(c[k], c[k + 1]);
                        split_pair(fma2(x, cc, mul2(y, pair_of(-s[k], -s[k + 1]))), v[k], v[k + 1]);
                        split_pair(fma2(y, cc, mul2(x, pair_of(s[k], s[k + 1]))), v[8 + k], v[9 + k]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float x = __uint_as_float(v[2 * k]), y = __uint_as_float(v[2 * k + 1]);
                        v[2 * k] = __float_as_uint(x * c[k] - y * s[k]);
                        v[2 * k + 1] = __float_as_uint(x * s[k] + y * c[k]);
                    }
                }
            }
            if (head && 2 * set + hi + 1 < 2 * SETS) rows_of.fetch(p, set + hi, hi ^ 1, at0, lane);  // on their way while these rows are packed and stored
            uint32_t o[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = pack2<F16>(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1]));
            const int rows = min(8, p.M - row0 - 16 * set - 8 * hi);  // (none or less where the tile ends before)
            if constexpr (HALVES) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    store_run(p, row - r4, rows, n0 + (j ? run1 : run0), lane, make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]), edge, whole);
            } else if (whole && p.wide_out == 2) {
                if (r4 < rows)
                    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(
                                     reinterpret_cast<uint16_t*>(p.y) + static_cast<long long>(row) * p.ldy + n0 + run0 + 16 * t),
                                 "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7])
                                 : "memory");
            } else {  // (lane t's 16 columns are run t / 2's, from 16 (t % 2): as halves of eight, in the order that store_run has them)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint32_t w4[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int from = (lane & ~3) + 2 * j + (t >> 1);
                        const uint32_t first = __shfl_sync(0xffffffffu, o[i], from), other = __shfl_sync(0xffffffffu, o[4 + i], from);
                        w4[i] = t & 1 ? other : first;
                    }
                    store_run(p, row - r4, rows, n0 + (j ? run1 : run0), lane, make_uint4(w4[0], w4[1], w4[2], w4[3]), edge, whole);
                }
            }
        }
}

// Quantizes all M rows into shared memory (the epilogue's warps): codes at `codes` + (kb groups + row / 8) KB in the layout of a TMA load with the 128-byte
// swizzle, scales at `scales` + kb KB as two atoms.  The arithmetic of mx_quantize_rows_kernel.
template <typename T>
__device__ __forceinline__ void quantize_resident(const MxKernelParams& p, uint32_t codes, uint32_t scales, int warp, int lane) {
    constexpr int AHEAD = 2;  // a warp's units (256 elements of a row), computed side by side
    const T* x = static_cast<const T*>(p.x);
    const int units = p.M * p.nkb;
    int row = warp / p.nkb, kb = warp - row * p.nkb;
    const int rows_on = EPI_WARPS / p.nkb, kb_on = EPI_WARPS - rows_on * p.nkb;
#pragma unroll 1
    for (int u0 = warp; u0 < units; u0 += AHEAD * EPI_WARPS) {
        Raw8<T> raw[AHEAD];
        int rows[AHEAD], kbs[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            rows[j] = row;
            kbs[j] = kb;
            raw[j] = Raw8<T>();
            if (row < p.M) raw[j] = load_raw8<T>(x + row * p.ldx, kb * 256 + lane * 8, p.K, p.x_wide != 0);
            row += rows_on;
            kb += kb_on;
            if (kb >= p.nkb) {
                kb -= p.nkb;
                ++row;
            }
        }
        uint32_t word[AHEAD], sw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            float v[8];
            unpack8<T>(raw[j], v);
            uint32_t am = abs_max_bits<T>(raw[j]);
            am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
            am = max(am, __shfl_xor_sync(0xffffffffu, am, 2));
            const uint32_t byte = p.scale_rule == DIROTQ_MX_SCALE_FLOOR ? mx_scale_byte<DIROTQ_MX_SCALE_FLOOR>(am) : mx_scale_byte<DIROTQ_MX_SCALE_CEIL>(am);
            word[j] = mx_codes8(v, byte);
            sw[j] = byte << (8 * ((lane >> 2) & 3));
            sw[j] |= __shfl_xor_sync(0xffffffffu, sw[j], 4);
            sw[j] |= __shfl_xor_sync(0xffffffffu, sw[j], 8);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (rows[j] >= p.M) break;
            const uint32_t dst = codes + (kbs[j] * p.groups + (rows[j] >> 3)) * 1024 + (rows[j] & 7) * 128 + (((lane >> 2) ^ (rows[j] & 7)) << 4) + (lane & 3) * 4;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst), "r"(word[j]) : "memory");
            if ((lane & 15) == 0)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(scales + kbs[j] * ATOMS + (lane >> 4) * 512 + (rows[j] & 31) * 16 + (rows[j] >> 5) * 4), "r"(sw[j]) : "memory");
        }
    }
}

// HEADS: 0 a product alone, 1 its q and k with norm and rotation of adjacent pairs (or none), 2 of halves (two kernels: one with both branches spills).
template <int BN, bool PAIR, int HEADS, bool F16, bool FUSE>
__global__ void __launch_bounds__(NUM_THREADS, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ MxKernelParams p) {
    using P = MxPlan<BN, PAIR, FUSE>;
    constexpr int NB = P::NB, STAGES = P::STAGES, ACC_BUFS = P::ACC_BUFS, STAGE_BYTES = P::STAGE_BYTES, KBS = P::KBS;
    constexpr int CW = PAIR ? 128 : BN;  // columns of an epilogue group
    constexpr bool QKV = HEADS != 0;
    constexpr bool SPLIT_REGS = QKV || CW == 128;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t ring = smem_base + P::RESIDENT;
    const uint32_t bar_base = smem_base + P::BAR_OFFSET;
    auto full_bar = [&](int s) { return bar_base + 8u * s; };
    auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
    auto sfready_bar = [&](int s) { return bar_base + 8u * (2 * STAGES + s); };
    auto tfull_bar = [&](int a) { return bar_base + 8u * (3 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bar_base + 8u * (3 * STAGES + 2 + a); };
    const uint32_t xready_bar = bar_base + 8u * (3 * STAGES + 4);                  // FUSE: the activations are in shared memory
    auto peer_bar = [&](int s) { return bar_base + 8u * (3 * STAGES + 5 + s); };  // pairs, leader: the other CTA's stage has landed
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + P::BAR_OFFSET + 480);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + P::BAR_OFFSET + 484);
    const uint32_t drain_bar = bar_base + 488u;  // see umma_drain

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
            if constexpr (PAIR) mbar_init(peer_bar(s), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(tfull_bar(a), 1);
            mbar_init(tempty_bar(a), PAIR ? 4 * GROUP_THREADS : GROUP_THREADS);
        }
        mbar_init(xready_bar, EPI_WARPS * 32);
        mbar_init(drain_bar, 1);
        *abort_flag = 0;
        fence_mbar_init();
        if constexpr (!FUSE) tma_prefetch_desc(&tmap_a);
        tma_prefetch_desc(&tmap_b);
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
    // (everything above touched only this CTA's own shared and tensor memory; the warps that touch global memory wait for the previous
    // kernel before they do)

    if (warp < 4) {
        if constexpr (SPLIT_REGS) reg_dealloc<32>();  // 128 * 32 + 512 * 112 registers are the 640 * 96 at launch
        // (before these warps' first waits, all on what comes after the previous kernel: how long that one still runs is no part of a bounded wait.  The
        // producer waits below, behind the loads that need not)
        if (warp != 0) grid_dependency_wait();
        if (warp == 0) {
            // ------------------------------------------------------------ producer
            RingPos<STAGES> at;
            bool ok = true;
            int early = 0;  // stages of the first tile whose rows of b are already on their way
            // k-blocks kb .. of a stage that exist (KBS, but for the last of an odd number)
            auto load_a = [&](int m_blk, int kb, uint32_t st, uint32_t bar) {
#pragma unroll
                for (int j = 0; j < KBS; ++j)
                    if (j == 0 || kb + j < p.nkb) {
                        tma_load_2d(st + j * P::A_STAGE, &tmap_a, bar, (kb + j) * 128, m_blk * BM);  // byte coordinates; rows past M: zeros, counted
                        bulk_load(st + P::SF_OFFSET + j * ATOMS, p.asf + ((static_cast<size_t>(m_blk >> 1) * p.nkb + kb + j) * 2 + (m_blk & 1)) * ATOMS, ATOMS,
                                  bar);
                    }
            };
            auto load_b = [&](int n_blk, int kb, uint32_t st, uint32_t bar) {
                const int rb = n_blk * BN / 128;  // (the atoms of 256 rows always exist)
#pragma unroll
                for (int j = 0; j < KBS; ++j)
                    if (j == 0 || kb + j < p.nkb) {
                        tma_load_2d(st + P::B_OFFSET + j * P::B_BYTES, &tmap_b, bar, (kb + j) * 128, n_blk * BN + (PAIR ? static_cast<int>(cta_rank) * 128 : 0));
                        bulk_load(st + P::SFB_OFFSET + j * NB * ATOMS, p.bsf + ((static_cast<size_t>(rb >> 1) * p.nkb + kb + j) * 2 + (rb & 1)) * ATOMS,
                                  NB * ATOMS, bar);
                    }
            };
            auto stage_tx = [&](int kb) {
                return min(KBS, p.nkb - kb) * (((FUSE ? 0 : p.a_box) + p.b_box) * 128 + (NB + (FUSE ? 0 : 1)) * ATOMS);
            };
            if (!FUSE && p.early && tile_first < num_tiles) {
                // the previous kernel is this call's own quantizer, which does not write b: b's first stages land while it runs
                early = min(STAGES, (p.nkb + KBS - 1) / KBS);
                if (elect_one())
                    for (int i = 0; i < early; ++i) {
                        mbar_arrive_expect_tx(full_bar(i), stage_tx(i * KBS));
                        load_b(tile_first / num_m_blocks, i * KBS, ring + i * STAGE_BYTES, full_bar(i));
                    }
                __syncwarp();
            }
            grid_dependency_wait();
            for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step) {
                const int m_blk = (tile % num_m_blocks) * (PAIR ? 2 : 1) + static_cast<int>(cta_rank), n_blk = tile / num_m_blocks;
                for (int kb = 0; kb < p.nkb; kb += KBS, at.next()) {
                    const uint32_t s = at.s;
                    if (!mbar_wait(empty_bar(s), at.ph ^ 1, abort_flag, p.status, DEV_TIMEOUT_PRODUCER)) { ok = false; break; }
                    const uint32_t st = ring + s * STAGE_BYTES;
                    if (!elect_one()) continue;
                    const bool begun = !FUSE && static_cast<int>(at.it) < early;
                    if (!begun) {
                        mbar_arrive_expect_tx(full_bar(s), stage_tx(kb));
                        load_b(n_blk, kb, st, full_bar(s));
                    }
                    if constexpr (!FUSE) load_a(m_blk, kb, st, full_bar(s));
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
                const uint64_t desc0 = umma_desc_sw128(ring);
                const uint64_t xdesc = umma_desc_sw128(smem_base);  // FUSE: the resident codes
                RingPos<STAGES> at;
                uint32_t tcount = 0;
                bool ok = true;
                if constexpr (FUSE) ok = mbar_wait(xready_bar, 0, abort_flag, p.status, DEV_TIMEOUT_MMA);
                for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step, ++tcount) {
                    const uint32_t acc = tcount % ACC_BUFS;
                    if (!mbar_wait(tempty_bar(acc), ((tcount / ACC_BUFS) & 1) ^ 1, abort_flag, p.status, DEV_TIMEOUT_MMA)) { ok = false; break; }
                    tc_fence_after_sync();
                    const uint32_t d = tmem_base + acc * BN;
                    // a 64-column tile's scales are one half of its 128-column block's: rows 0..63 lie in an atom's first two columns of tensor memory
                    const uint32_t half = BN == 64 ? 2 * ((tile / num_m_blocks) & 1) : 0;
                    for (int kb = 0; kb < p.nkb; kb += KBS, at.next()) {
                        const uint32_t s = at.s;
                        // (the copier warps have seen the stage's loads land, in both CTAs of a pair: their barrier covers the operands)
                        if (!mbar_wait(sfready_bar(s), at.ph, abort_flag, p.status, DEV_TIMEOUT_MMA)) { ok = false; break; }
                        tc_fence_after_sync();
                        const uint64_t sdesc = desc0 + s * (STAGE_BYTES >> 4);
                        if (!elect_one()) continue;
#pragma unroll
                        for (int j = 0; j < KBS; ++j)
                            if (j == 0 || kb + j < p.nkb) {
                                const uint32_t tsf = tmem_base + P::TMEM_SF + (s * KBS + j) * P::SF_COLS;
                                const uint64_t adesc = FUSE ? xdesc + static_cast<uint32_t>((kb + j) * p.groups * (1024 >> 4)) : sdesc + j * (P::A_STAGE >> 4);
                                const uint64_t bdesc = sdesc + (P::B_OFFSET >> 4) + j * (P::B_BYTES >> 4);
#pragma unroll
                                for (int k = 0; k < 4; ++k)  // K = 64 elements = 32 bytes per instruction
                                    umma_mxf4<PAIR>(d, adesc + 2 * k, bdesc + 2 * k, (k & 1) ? idesc1 : idesc0, tsf + 4 * (k >> 1),
                                                    tsf + 8 + 4 * NB * (k >> 1) + half, (kb | j | k) != 0);
                            }
                        if constexpr (PAIR) umma_commit_pair(empty_bar(s), 3);
                        else umma_commit(empty_bar(s));
                    }
                    if (ok && elect_one()) {
                        if constexpr (PAIR) umma_commit_pair(tfull_bar(acc), 3);
                        else umma_commit(tfull_bar(acc));
                    }
                }
            }
        } else {
            // ------------------------------------------------------------ scale copiers
            RingPos<STAGES> at;
            bool ok = true;
            if constexpr (FUSE) ok = mbar_wait(xready_bar, 0, abort_flag, p.status, DEV_TIMEOUT_UNPACK);
            for (int tile = tile_first; ok && tile < num_tiles; tile += tile_step) {
                for (int kb = 0; kb < p.nkb; kb += KBS, at.next()) {
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
                    if (!elect_one()) continue;
#pragma unroll
                    for (int j = 0; j < KBS; ++j)
                        if (j == 0 || kb + j < p.nkb) {
                            const uint32_t sfa = FUSE ? smem_base + p.nkb * p.groups * 1024 + (kb + j) * ATOMS : ring + s * STAGE_BYTES + P::SF_OFFSET + j * ATOMS;
                            const uint32_t sfb = ring + s * STAGE_BYTES + P::SFB_OFFSET + j * NB * ATOMS;
                            const uint32_t tsf = tmem_base + P::TMEM_SF + (s * KBS + j) * P::SF_COLS;
                            // atom i of a at column 4 i; atom i of column block b at 8 + 4 NB i + 4 b (the blocks of a tile side by side)
                            if (warp == 2) {
                                sf_copy<PAIR>(tsf, sf_desc(sfa));
                                sf_copy<PAIR>(tsf + 4, sf_desc(sfa + 512));
                                if constexpr (NB == 2) sf_copy<PAIR>(tsf + 8, sf_desc(sfb));
                            } else {
                                if constexpr (NB == 1) sf_copy<PAIR>(tsf + 8, sf_desc(sfb));
                                if constexpr (NB == 2) sf_copy<PAIR>(tsf + 12, sf_desc(sfb + ATOMS));
#pragma unroll
                                for (int b = 0; b < NB; ++b) sf_copy<PAIR>(tsf + 8 + 4 * NB + 4 * b, sf_desc(sfb + b * ATOMS + 512));
                            }
                        }
                    if constexpr (PAIR) umma_commit_pair(sfready_bar(s), 1);  // the leader's barrier only
                    else umma_commit(sfready_bar(s));
                }
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue
        // Two groups of eight warps; a group has CW columns: half of a pair's tile, or the whole of every second tile.  warp % 4 is the quadrant of
        // tensor-memory lanes (32 rows) that a warp may read; the two warps of a group and quadrant take 16 rows each, or, where 128 columns are
        // heads, 64 columns each (store_heads).  A warp reads its values before it hands the accumulator back and converts.
        //
        // Loads of 16 lanes x 256 bits leave lane l with columns 8 J + 2 t, + 1 (t = l % 4) of rows l / 4 and l / 4 + 8: exchanged within the four lanes
        // of a row (transpose4), each lane has runs of 8 consecutive columns, 32 m + 8 t, of its two rows, 64 bytes of a row side by side in a
        // store.  (Through shared memory and TMA stores instead: the same time at K = 12288, and 32 KB that hold a stage of operands here.)
        if constexpr (SPLIT_REGS) reg_alloc<112>();
        constexpr int RUNS = CW / 32, CH = CW / 64;
        const int q = warp & 3, second = ((warp - 4) >> 2) & 1, group = (warp - 4) >> 3, gt = threadIdx.x - 128 - group * GROUP_THREADS;
        constexpr bool HEADS128 = QKV && CW == 128;  // the second warp of a quadrant takes other columns, not rows
        const int first_row = q * 32 + (HEADS128 ? 0 : second * 16);
        [[maybe_unused]] const int t = lane & 3, r4 = lane >> 2;
        grid_dependency_wait();
        grid_launch_dependents();  // the next kernel may be scheduled as this grid's CTAs leave (it waits for this whole grid)
        if constexpr (FUSE) {
            const uint32_t sfa = smem_base + p.nkb * p.groups * 1024;
            if (p.x_dtype == DIROTQ_DTYPE_BF16) quantize_resident<__nv_bfloat16>(p, smem_base, sfa, warp - 4, lane);
            else if (p.x_dtype == DIROTQ_DTYPE_F16) quantize_resident<__half>(p, smem_base, sfa, warp - 4, lane);
            else quantize_resident<float>(p, smem_base, sfa, warp - 4, lane);
            fence_proxy_async_smem();  // these writes -> visible to the tensor core
            mbar_arrive(xready_bar);
        }
        float* s_hw = reinterpret_cast<float*>(smem_gen + P::HEADW_OFFSET);
        if constexpr (QKV) {  // (both groups write the same values; each reads behind its own barrier below)
            s_hw[gt] = load_weight(gt < 128 ? p.qw : p.kw, gt & ((1 << p.head_shift) - 1), p.wdtype);
        }
        uint32_t tcount = PAIR ? 0 : group;
        for (int tile = tile_first + (PAIR ? 0 : group * tile_step); tile < num_tiles; tile += PAIR ? tile_step : 2 * tile_step, tcount += PAIR ? 1 : 2) {
            const int row0 = (tile % num_m_blocks) * TILE_ROWS + (PAIR ? static_cast<int>(cta_rank) * BM : 0) + first_row;
            const int n0 = (tile / num_m_blocks) * BN + (PAIR ? group * 128 : 0);
            const uint32_t acc = tcount % ACC_BUFS, use = tcount / ACC_BUFS;
            // the bias of these columns goes to shared memory while the tile's MMAs run (two buffers: a warp can be a tile ahead); the
            // barrier orders the stores before the reads and makes the group agree on whether to go on
            float* s_b = reinterpret_cast<float*>(smem_gen + P::BIAS_OFFSET) + (group * 2 + (use & 1)) * 128;
            if (gt < CW) s_b[gt] = p.bias != nullptr && n0 + gt < p.N ? load_16(p.bias, n0 + gt, F16) : 0.f;
            constexpr int SETS = HEADS128 ? 2 : 1;
            const bool split = HEADS128 && p.head_shift == 7, apart = split && HEADS == 2;
            const int run0 = HEADS128 ? (apart ? 32 : 64) * second : 0, run1 = run0 + (apart ? 64 : 32);
            [[maybe_unused]] HeadRows<SETS, HEADS == 2> rows_of;
            if constexpr (QKV)  // positions and the first angles come while the tile's MMAs run
                rows_of.start(p, row0, n0 + run0 < p.k_end, run0 & ((1 << p.head_shift) - 1), lane);
            const bool failed = !mbar_wait(tfull_bar(acc), use & 1, abort_flag, p.status, DEV_TIMEOUT_EPILOGUE);
            if (group == 0 ? group_any<1, GROUP_THREADS>(failed) : group_any<2, GROUP_THREADS>(failed)) break;
            tc_fence_after_sync();
            const uint32_t taddr = tmem_base + (static_cast<uint32_t>(first_row) << 16) + acc * BN + (PAIR ? group * 128 : 0);
            const bool stored = row0 < p.M && n0 < p.N;  // (uniform in the warp, and the same in the two of a quadrant that share heads)
            const bool whole = p.wide_out && n0 + CW <= p.N;
            const uint32_t edge = smem_base + P::EDGE_OFFSET + static_cast<uint32_t>(warp - 4) * 512u;
            auto hand_back = [&]() {
                tc_fence_before_sync();
                if constexpr (PAIR) mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));  // the leader's barrier
                else mbar_arrive(tempty_bar(acc));
            };
            if constexpr (QKV) {
                uint32_t raw[SETS][2][16];
                if (stored) {
#pragma unroll
                    for (int s = 0; s < SETS; ++s) {
                        tmem_ld_16x256b_x4(taddr + (static_cast<uint32_t>(16 * s) << 16) + run0, raw[s][0]);
                        tmem_ld_16x256b_x4(taddr + (static_cast<uint32_t>(16 * s) << 16) + run1, raw[s][1]);
                    }
                    tmem_ld_wait();
#pragma unroll
                    for (int s = 0; s < SETS; ++s) {
                        tmem_ld_fence(raw[s][0]);
                        tmem_ld_fence(raw[s][1]);
                    }
                }
                hand_back();
                if (!stored) continue;
                float* sums = reinterpret_cast<float*>(smem_gen + P::SUM_OFFSET);
                float *mine = sums + (warp - 4) * 32, *other = sums + ((warp - 4) ^ 4) * 32;
                store_heads<SETS, F16, HEADS == 2>(raw, rows_of, p, row0, n0, run0, run1, split, lane, s_b, s_hw, mine, other, 3 + group * 4 + q, edge, whole);
            } else {
                uint32_t raw[CH][32];  // [columns 64 c ..][4 j + 2 (row + 8) + (column + 1)], J = 8 c + j
                if (stored) {
#pragma unroll
                    for (int c = 0; c < CH; ++c) tmem_ld_16x256b_x8(taddr + c * 64, raw[c]);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < CH; ++c) tmem_ld_fence(raw[c]);
                }
                hand_back();
                if (!stored) continue;
                auto convert = [&](int hi, int m) {  // run m of rows l / 4 + 8 hi, rounded and exchanged
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 b = *reinterpret_cast<const float2*>(s_b + 32 * m + 8 * k + 2 * t);
                        w[k] = pack2<F16>(__uint_as_float(raw[m >> 1][16 * (m & 1) + 4 * k + 2 * hi]) + b.x,
                                          __uint_as_float(raw[m >> 1][16 * (m & 1) + 4 * k + 2 * hi + 1]) + b.y);
                    }
                    transpose4(w, t);
                    return make_uint4(w[0], w[1], w[2], w[3]);
                };
                if (whole && row0 + 16 <= p.M) {
                    uint16_t* y = reinterpret_cast<uint16_t*>(p.y) + static_cast<long long>(row0 + r4) * p.ldy + n0 + 8 * t;
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                        for (int m = 0; m < RUNS; ++m) __stcs(reinterpret_cast<uint4*>(y + 8 * hi * p.ldy + 32 * m), convert(hi, m));
                } else {
#pragma unroll
                    for (int hi = 0; hi < 2; ++hi)
#pragma unroll
                        for (int m = 0; m < RUNS; ++m) store_run(p, row0 + 8 * hi, min(8, p.M - row0 - 8 * hi), n0 + 32 * m, lane, convert(hi, m), edge, whole);
                }
            }
        }
    }

    if constexpr (PAIR) {
        if (warp == 1 && lane == 0 && cta_rank == 0 && *abort_flag != 0) umma_drain<true>(drain_bar);  // let issued MMAs finish first
        tc_fence_before_sync();
        cluster_sync_all();  // neither CTA leaves while the other may still read its operands or signal its barriers
        if (warp == 1) {
            tc_fence_after_sync();
            tmem_dealloc_pair(tmem_base, 512);
        }
    } else {
        if (warp == 1 && lane == 0 && *abort_flag != 0) umma_drain(drain_bar);
        tc_fence_before_sync();
        __syncthreads();
        if (warp == 1) {
            tc_fence_after_sync();
            tmem_dealloc(tmem_base, 512);
        }
    }
}

template <int BN, bool PAIR, int HEADS, bool F16, bool FUSE>
dirotq_status_t launch_kernel_of(const MxGemmArgs& a, MxKernelParams& p, cudaStream_t stream) {
    using P = MxPlan<BN, PAIR, FUSE>;
    auto kern = mx_gemm_kernel<BN, PAIR, HEADS, F16, FUSE>;
    const int device = a.b->device, sms = sm_count(device);
    static SmemOptIn<1> opt_in;
    if (!opt_in.ensure(kern, 0, device, P::SMEM_BYTES)) return DIROTQ_ERR_CUDA;
    const long long rows = PAIR ? 2 * BM : BM;
    const long long tiles = (p.M + rows - 1) / rows * ((p.N + BN - 1) / BN);
    const CUtensorMap& tmap_b = BN == 64 ? a.b->tmap64 : a.b->tmap;
    const CUtensorMap& tmap_a = FUSE ? tmap_b : a.a->tmap;  // (not used when the activations are quantized here)
    p.b_box = BN == 64 ? a.b->box64 : a.b->box;
    cudaError_t err;
    if constexpr (PAIR) {
        const int pairs = static_cast<int>(tiles < sms / 2 ? tiles : sms / 2);
        err = launch_kernel_pairs(kern, 2 * pairs, NUM_THREADS, P::SMEM_BYTES, stream, true, tmap_a, tmap_b, p);
    } else {
        err = launch_kernel(kern, static_cast<int>(tiles < sms ? tiles : sms), NUM_THREADS, P::SMEM_BYTES, stream, true, tmap_a, tmap_b, p);
    }
    if (err != cudaSuccess) set_error("mx_gemm_kernel", err);
    return err == cudaSuccess ? DIROTQ_OK : DIROTQ_ERR_CUDA;
}

template <int BN, bool PAIR, bool FUSE>
dirotq_status_t launch_plan(const MxGemmArgs& a, MxKernelParams& p, cudaStream_t stream) {
    const bool f16 = a.y_dtype == DIROTQ_DTYPE_F16;
    if (a.qk && a.qk->rope == DIROTQ_ROPE_HALVES)
        return f16 ? launch_kernel_of<BN, PAIR, 2, true, FUSE>(a, p, stream) : launch_kernel_of<BN, PAIR, 2, false, FUSE>(a, p, stream);
    if (a.qk) return f16 ? launch_kernel_of<BN, PAIR, 1, true, FUSE>(a, p, stream) : launch_kernel_of<BN, PAIR, 1, false, FUSE>(a, p, stream);
    return f16 ? launch_kernel_of<BN, PAIR, 0, true, FUSE>(a, p, stream) : launch_kernel_of<BN, PAIR, 0, false, FUSE>(a, p, stream);
}

std::atomic<int> g_mx_tile{0};  // 0: chosen per call; 64 / 128: single CTAs with that many columns; 512: CTA pairs

// Up to kFuseUnits units (256 elements of a row) the activations are quantized by the product's own CTAs (see FUSE): that takes about 0.3 us per
// unit and warp there, a quantizer of its own about 1.5 us.  (K = 3072 -> 9216: 2 rows, 24 units, 6.1 against 6.6 us, 4 rows 7.1; 1152 -> 1152: 6 rows, 30
// units, 4.7 against 5.5, 8 rows 5.2, 12 rows 6.3; 12288 -> 3072: 1 row, 48 units, 12.6 against 12.1.)
constexpr int kFuseUnits = 32;
bool fuse_fits(int M, int nkb) {
    return static_cast<long long>(M) * nkb <= kFuseUnits && M <= 32 && nkb * ((M + 7) / 8 + 1) * 1024 <= MxPlan<64, false, true>::RESIDENT;
}

// Columns per tile of single CTAs, or 512 for pairs: the shortest schedule, turns of the SMs x the time of a tile.  Microseconds a tile of nkb
// k-blocks takes, from calls of one to nine turns: 64 columns 0.30 + 0.17 nkb, 128 columns 0.55 + 0.235 nkb, pairs 1.0 + 0.36 nkb and 1.3
// once (clusters start later).  (512 rows, K 1152 -> 1152: 3.5, 4.4, 6.2 us; 512 rows, 3072 -> 9216: 11.9, 9.2, 9.6; 4608 rows: pairs 50.)
// Norm and rotation in the epilogue are in none of the three: for 3 x 24 heads of 128 and K = 3072 they move the border between 128 columns and pairs up:
// linear, quantizer included, 512 tokens 12.7 / 12.7 us (128 columns / pairs), 1024 19.3 / 17.4; q/k/v 14.0 / 14.6, 19.9 / 20.2, and 2048 34.6 / 30.8.
int choose_plan(int M, int N, int nkb, const dirotq_qk_t* qk, int sms) {
    const bool heads_of_128 = qk != nullptr && qk->head_dim == 128;  // (a tile's columns are whole heads)
    const int forced = g_mx_tile.load();
    if (forced != 0 && !(forced == 64 && heads_of_128)) return forced;
    auto turns = [](long long tiles, int units) { return static_cast<double>((tiles + units - 1) / units); };
    const long long mb = (M + BM - 1) / BM;
    const double t64 = heads_of_128 ? 1e30 : turns(mb * ((N + 63) / 64), sms) * (0.30 + 0.17 * nkb);
    const double t128 = turns(mb * ((N + 127) / 128), sms) * (0.55 + 0.235 * nkb);
    const double tpair = M <= BM ? 1e30 : 1.3 + turns((M + 2 * BM - 1) / (2 * BM) * ((N + 255ll) / 256), sms / 2) * (1.0 + 0.36 * nkb);
    return tpair < t64 && tpair < t128 ? 512 : t128 < t64 ? 128 : 64;
}

}  // namespace

dirotq_status_t set_mx_tile_columns(int columns) {
    if (columns != 0 && columns != 64 && columns != 128 && columns != 512) return DIROTQ_ERR_INVALID_ARG;
    g_mx_tile.store(columns);
    return DIROTQ_OK;
}

bool mx_fuses(int M, int N, int nkb, const dirotq_qk_t* qk, int device) {
    const int plan = choose_plan(M, N, nkb, qk, sm_count(device));
    return plan != 512 && fuse_fits(M, nkb);
}

dirotq_status_t launch_mx_gemm(const MxGemmArgs& a, cudaStream_t stream) {
    MxKernelParams p = {};
    p.M = a.M;
    p.N = a.b->rows;
    p.nkb = a.b->lay.nkb;
    if (a.a) {
        p.a_box = a.a->box;
        p.asf = reinterpret_cast<const uint8_t*>(a.a->buffer) + a.a->lay.off_scales;
    } else {
        p.x = a.x;
        p.ldx = a.ldx;
        p.x_dtype = a.x_dtype;
        p.x_wide = (reinterpret_cast<uintptr_t>(a.x) & 15u) == 0 && a.ldx * static_cast<long long>(dtype_size(a.x_dtype)) % 16 == 0;
        p.K = a.b->K;
        p.scale_rule = a.scale_rule;
        p.groups = (a.M + 7) / 8;
    }
    p.bsf = reinterpret_cast<const uint8_t*>(a.b->buffer) + a.b->lay.off_scales;
    p.bias = a.bias;
    p.y = static_cast<uint8_t*>(a.y);
    p.ldy = a.ldy;
    p.status = a.status;
    p.early = a.early_weights;
    p.wide_out = (reinterpret_cast<uintptr_t>(a.y) & 15u) != 0 || a.ldy % 8 != 0 ? 0 : (reinterpret_cast<uintptr_t>(a.y) & 31u) != 0 || a.ldy % 16 != 0 ? 1 : 2;
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
        p.wide_table = ((reinterpret_cast<uintptr_t>(qk.cos_table) | reinterpret_cast<uintptr_t>(qk.sin_table)) & 31u) == 0 && qk.ld_table % 8 == 0;
        p.num_positions = qk.num_positions;
        p.positions = qk_positions(qk);
    }
    const int plan = choose_plan(p.M, p.N, p.nkb, a.qk, sm_count(a.b->device));
    if (a.a == nullptr) return plan == 64 ? launch_plan<64, false, true>(a, p, stream) : launch_plan<128, false, true>(a, p, stream);
    return plan == 512   ? launch_plan<256, true, false>(a, p, stream)
           : plan == 128 ? launch_plan<128, false, false>(a, p, stream)
                         : launch_plan<64, false, false>(a, p, stream);
}

}  // namespace dirotq
