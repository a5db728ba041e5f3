// MXFP4 operands: layout of their buffer, host handle, and the element conversions the kernels share.
#pragma once
#include "common.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

namespace dirotq {

// Buffer of an operand [rows, K]:
//   codes   u8 [rows][pitch], pitch = ceil(K / 32) * 16: two E2M1 codes per byte, even k in the low half (the operand layout of
//           tcgen05.mma kind::mxf4); codes behind K are 0
//   scales  512-byte atoms: 128 rows x the 4 scales of 128 elements of K, row r's four bytes at (r % 32) * 16 + (r / 32) * 4 (the order
//           tcgen05.cp.32x128b.warpx4 expects).  Atom `ak` (index along K) of row block `rb` sits at
//           [rb / 2][ak / 2][rb % 2][ak % 2]: the two atoms of a 256-element k-block are contiguous, and so are the four that 256 rows
//           need for it.  Scale bytes behind K are 0 (2^-127: with the zero codes there they add nothing; a NaN byte would).
struct MxLayout {
    int pitch;  // bytes of a row of codes
    int nkb;    // k-blocks of 256 elements
    size_t off_scales, total;
};
inline MxLayout make_mx_layout(int rows, int K) {
    MxLayout l;
    l.pitch = (K + 31) / 32 * 16;
    l.nkb = (K + 255) / 256;
    l.off_scales = align_up(static_cast<size_t>(rows) * l.pitch);
    l.total = l.off_scales + align_up(static_cast<size_t>((rows + 255) / 256) * 256 * l.nkb * 8);
    return l;
}
// Byte offset of the word (4 scale bytes) of `row` for elements [128 ak, 128 ak + 128).
__host__ __device__ inline size_t mx_scale_word(int row, int ak, int nkb) {
    const int rb = row >> 7, r = row & 127;
    return ((((static_cast<size_t>(rb >> 1) * nkb + (ak >> 1)) * 2 + (rb & 1)) * 2) + (ak & 1)) * 512 + (r & 31) * 16 + (r >> 5) * 4;
}

}  // namespace dirotq

struct dirotq_mxfp4 {
    uint32_t magic;
    int device;
    int rows, K;
    dirotq::MxLayout lay;
    char* buffer;      // device
    int box;           // rows of the tensor map's box: 128, or the rows that exist rounded up to 8 (box_rows)
    CUtensorMap tmap;  // u8 [rows][pitch], box 128 x box, 128B swizzle
    int box64;           // the same with boxes of up to 64 rows (tiles of 64 columns)
    CUtensorMap tmap64;
};

namespace dirotq {

constexpr uint32_t kMxMagic = 0x4678694du;  // "Mixf"

// Host side of the operand (mxfp4.cu); `t` need not come from dirotq_mxfp4_create.
dirotq_status_t mx_setup(dirotq_mxfp4* t, int rows, int K, void* buffer, int device, bool both);  // both: the map with boxes of 64 rows too
bool mx_valid(const dirotq_mxfp4* t);
inline size_t dtype_size(int dtype) { return dtype == DIROTQ_DTYPE_F32 ? 4 : 2; }
inline bool dtype_is_16(int dtype) { return dtype == DIROTQ_DTYPE_BF16 || dtype == DIROTQ_DTYPE_F16; }
inline bool dtype_ok(int dtype) { return dtype == DIROTQ_DTYPE_F32 || dtype_is_16(dtype); }

// launchers
cudaError_t launch_mx_quantize(const void* x, int x_dtype, int x_layout, long long ldx, int scale_rule, const dirotq_mxfp4* t,
                               cudaStream_t stream);
struct MxGemmArgs {
    int M;
    const dirotq_mxfp4* a;   // NULL: the kernel quantizes x itself (mx_fuses)
    const void* x;
    int x_dtype;
    long long ldx;
    int scale_rule;
    const dirotq_mxfp4* b;
    const void* bias;
    void* y;
    int y_dtype;
    long long ldy;
    int* status;
    bool early_weights;      // the previous kernel of the stream is this call's own quantizer: b may be read while it runs
    const dirotq_qk_t* qk;   // norm and rotation in the epilogue, or NULL
};
dirotq_status_t launch_mx_gemm(const MxGemmArgs& a, cudaStream_t stream);
bool mx_fuses(int M, int N, int nkb, const dirotq_qk_t* qk, int device);  // whether dirotq_mxfp4_linear / _qkv leaves x to the product's kernel (where y is not in x's memory)

// qk_norm.cu
dirotq_status_t qk_check(const dirotq_qk_t* qk, int M);
cudaError_t launch_qk_norm_rope(const void* x, int dtype, int M, long long ldx, const dirotq_qk_t& qk, void* q_out, long long ldq, void* k_out,
                                long long ldk, void* v_out, long long ldv, const int32_t* slots, int num_slots, cudaStream_t stream);

// ------------------------------------------------------------------ element conversions

// 2^e for e in [-126, 127]
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
// the value of a scale byte (2^-127 is a subnormal number)
__device__ __forceinline__ float e8m0_value(uint32_t s) {
    return s == 255u ? __uint_as_float(0x7fffffffu) : s == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(s << 23);
}
// Scale byte of a block from the bits of its largest magnitude (an unsigned maximum of |x|'s bits: a NaN wins over an infinity, and
// that over every number).  The exponent field of a normal number is floor(log2 a) + 127, so floor(log2 a) - 2 is the field less 2;
// subnormal numbers end at the lower limit either way.  CEIL: a <= 6 2^e = 1.5 2^(e+2) unless the mantissa is above 1.5.
template <int RULE>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t abits) {
    if (abits >= 0x7f800000u) return 255u;
    int b = static_cast<int>(abits >> 23) - 2;
    if (RULE == DIROTQ_MX_SCALE_CEIL) b += (abits & 0x7fffffu) > 0x400000u ? 1 : 0;
    return static_cast<uint32_t>(b < 0 ? 0 : b);
}
// What elements are multiplied by: 2^(127 - byte), exact (byte 0: 2^127; the largest byte of a number is 253).  (A NaN
// block's codes are cleared.)
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == 255u ? 0.f : pow2f(127 - static_cast<int>(byte)); }

__device__ __forceinline__ uint32_t to_e2m1x2(float lo, float hi) {  // nearest, ties to even, saturating; `lo` in bits 0..3
    uint32_t out;
    asm("{\n\t"
        ".reg .b8 t;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\t"
        "cvt.u32.u8 %0, t;\n\t"
        "}\n"
        : "=r"(out)
        : "f"(hi), "f"(lo));
    return out;
}
// The two values of a byte of codes (exact in fp16).
__device__ __forceinline__ float2 from_e2m1x2(uint32_t byte) {
    uint32_t h2;
    asm("{\n\t"
        ".reg .b8 t;\n\t"
        "cvt.u8.u32 t, %1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, t;\n\t"
        "}\n"
        : "=r"(h2)
        : "r"(byte));
    return __half22float2(*reinterpret_cast<const __half2*>(&h2));
}

// The codes of eight elements of a block with this scale byte, the first in bits 0..3.
__device__ __forceinline__ uint32_t mx_codes8(const float (&v)[8], uint32_t byte) {
    const float inv = mx_inverse(byte);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; i += 2) w |= to_e2m1x2(v[i] * inv, v[i + 1] * inv) << (4 * i);
    return byte == 255u ? 0u : w;
}

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <typename T>
struct Raw8 {  // eight elements as they lie in memory
    uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&v)[8]) {
    union { Raw8<T> r; T t[8]; } c;
    c.r = r;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32<T>(c.t[i]);
}
// Bits of the largest magnitude (as fp32) among eight elements as they lie in memory.  In 16 bits the maximum is taken on pairs of patterns without
// their signs, whose order is that of the magnitudes (infinity above every number, NaN above that).
template <typename T>
__device__ __forceinline__ uint32_t abs_max_bits(const Raw8<T>& r) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
        return m;
    } else {
        const uint32_t m = __vmaxu2(__vmaxu2(r.u[0].x & 0x7fff7fffu, r.u[0].y & 0x7fff7fffu), __vmaxu2(r.u[0].z & 0x7fff7fffu, r.u[0].w & 0x7fff7fffu));
        const uint32_t top = max(m & 0xffffu, m >> 16);
        if constexpr (std::is_same_v<T, __nv_bfloat16>) return top << 16;
        else return __float_as_uint(__half2float(__ushort_as_half(static_cast<unsigned short>(top))));
    }
}

// Elements k0 .. k0 + 7 of a row of K as they are, zeros behind K.  (Not converted here: a conversion would wait for the load, and several are to be
// in flight.)
template <typename T>
__device__ __forceinline__ Raw8<T> load_raw8(const T* row, int k0, int K, bool wide) {
    Raw8<T> r;
    if (wide && k0 + 8 <= K) {
#pragma unroll
        for (int u = 0; u < static_cast<int>(sizeof(T) / 2); ++u) r.u[u] = reinterpret_cast<const uint4*>(row + k0)[u];
    } else {
        union { Raw8<T> r; T t[8]; } c;
#pragma unroll
        for (int i = 0; i < 8; ++i) c.t[i] = k0 + i < K ? row[k0 + i] : from_f32<T>(0.f);
        r = c.r;
    }
    return r;
}

template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float (&v)[8]) {
    union { Raw8<T> r; T t[8]; } c;
#pragma unroll
    for (int i = 0; i < 8; ++i) c.t[i] = from_f32<T>(v[i]);
    return c.r;
}

}  // namespace dirotq
