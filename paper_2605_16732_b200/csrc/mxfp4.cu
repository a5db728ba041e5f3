// MXFP4 operands: handles, quantizer, dequantizer, plain import / export, and the entry points of the products.
#include "mxfp4.cuh"
#include "ptx.cuh"
#include "row_ranges.h"

#include <new>
#include <type_traits>

#include <string.h>

namespace dirotq {
namespace {

constexpr int kThreads = 256;

// The quantizers' x and the dequantizer's codes and scales may be what the previous kernel of the stream still writes when these start (dependent launches).  They
// carry no __restrict__: it makes them loads of constant memory, which nothing holds behind the wait for that kernel.  (Where such loads are faster, columns of
// 32-bit weights 24 against 25 us, their addresses are.)

// ------------------------------------------------------------------ quantizer, elements along a row
// A unit is 512 elements of a row (four scale words).  A warp takes UNITS of them, sixteen elements per lane and unit, their loads in flight
// together: two lanes share a block of 32, so its maximum is one shuffle and a scale word three; codes leave as 8 bytes a lane, 256 a warp.  In
// 16 bits the instructions bounded it, not the memory, with eight elements per lane (4608 x 12288: 34 us in bf16, 39 in fp32).  Now 24.6 us in
// bf16, 5.8 TB/s of the 2 + 17/32 bytes an element; 39 us in fp32, 6.6 TB/s; memory bounds both.
template <typename T>
struct Raw16 {
    Raw8<T> h[2];
};
// ALIGN: bytes that rows' pieces of 16 elements are aligned to: 32 (in 16 bits one load), 16, or 0: such rows are read and written an element at a
// time by consecutive lanes, and change places in shared memory (Spread; straight from each lane's own sixteen elements, every access
// would touch 32 sectors)
template <typename T>
struct Spread {  // a unit's 512 elements, lane l with element 32 i + l
    T t[16];
};
template <typename T>
__device__ __forceinline__ Spread<T> load_spread(const T* row, int k0, int K, int lane) {
    Spread<T> e;
#pragma unroll
    for (int i = 0; i < 16; ++i) e.t[i] = k0 + 32 * i + lane < K ? row[k0 + 32 * i + lane] : from_f32<T>(0.f);
    return e;
}
template <typename T>
__device__ __forceinline__ Raw16<T> gather(const Spread<T>& e, T* s, int lane) {  // s: 512 elements of the warp's shared memory
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) s[32 * i + lane] = e.t[i];
    __syncwarp();
    return *reinterpret_cast<const Raw16<T>*>(s + 16 * lane);
}
template <typename T>
__device__ __forceinline__ void store_spread(T* row, int k0, int K, const Raw16<T>& r, T* s, int lane) {
    __syncwarp();
    *reinterpret_cast<Raw16<T>*>(s + 16 * lane) = r;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k0 + 32 * i + lane < K) row[k0 + 32 * i + lane] = s[32 * i + lane];
}

template <typename T, int ALIGN>
__device__ __forceinline__ Raw16<T> load_raw16(const T* row, int k0, int K) {
    Raw16<T> r;
    if (ALIGN == 32 && sizeof(T) == 2 && k0 + 16 <= K) {
        uint4 &a = r.h[0].u[0], &b = r.h[1].u[0];
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
                     : "l"(row + k0));
    } else {
        r.h[0] = load_raw8<T>(row, k0, K, ALIGN != 0);
        r.h[1] = load_raw8<T>(row, k0 + 8, K, ALIGN != 0);
    }
    return r;
}

template <typename T, int RULE, int ALIGN, int UNITS>
__global__ void __launch_bounds__(kThreads) mx_quantize_rows_kernel(const T* x, long long ldx, int rows, int K, int nkb, int pitch,
                                                                    uint8_t* codes, uint8_t* scales) {
    const int lane = threadIdx.x & 31;
    const int per_row = (nkb + 1) >> 1;
    const unsigned units = static_cast<unsigned>(rows) * per_row;  // (at most 2^31 - 1, see check_shape)
    const unsigned first = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * UNITS;
    if (first >= units) return;
    int row = static_cast<int>(first / per_row), u = static_cast<int>(first % per_row);
    // the previous kernel of the stream may still read the workspace this one writes, or write x
    grid_dependency_wait();
    grid_launch_dependents();
    using Loaded = std::conditional_t<ALIGN == 0, Spread<T>, Raw16<T>>;
    __shared__ __align__(16) T s_unit[ALIGN == 0 ? kThreads / 32 : 1][512];
    Loaded loaded[UNITS];
    {
        int r = row, b = u;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            if (r < rows) {
                if constexpr (ALIGN == 0) loaded[j] = load_spread<T>(x + r * ldx, b * 512, K, lane);
                else loaded[j] = load_raw16<T, ALIGN>(x + r * ldx, b * 512 + lane * 16, K);
            }
            if (++b == per_row) { b = 0; ++r; }
        }
    }
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        if (row >= rows) break;  // (the same for the whole warp)
        Raw16<T> raw;
        if constexpr (ALIGN == 0) raw = gather<T>(loaded[j], s_unit[threadIdx.x >> 5], lane);
        else raw = loaded[j];
        uint32_t am = max(abs_max_bits<T>(raw.h[0]), abs_max_bits<T>(raw.h[1]));
        am = max(am, __shfl_xor_sync(0xffffffffu, am, 1));
        const uint32_t byte = mx_scale_byte<RULE>(am);
        float v[8];
        unpack8<T>(raw.h[0], v);
        const uint32_t w0 = mx_codes8(v, byte);
        unpack8<T>(raw.h[1], v);
        const uint32_t w1 = mx_codes8(v, byte);
        const int at = u * 256 + lane * 8;  // of the row's bytes
        if (at < pitch) *reinterpret_cast<uint2*>(codes + static_cast<size_t>(row) * pitch + at) = make_uint2(w0, w1);
        // lane 8 h gathers the bytes of blocks 4 h .. 4 h + 3 of the unit
        uint32_t sw = byte << (8 * ((lane >> 1) & 3));
        sw |= __shfl_xor_sync(0xffffffffu, sw, 2);
        sw |= __shfl_xor_sync(0xffffffffu, sw, 4);
        const int ak = u * 4 + (lane >> 3);
        if ((lane & 7) == 0 && ak < 2 * nkb) *reinterpret_cast<uint32_t*>(scales + mx_scale_word(row, ak, nkb)) = sw;
        if (++u == per_row) { u = 0; ++row; }
    }
}

// ------------------------------------------------------------------ quantizer, elements along a column (weights stored [K, N])
// A block of threads takes COLS * 32 columns x 256 elements along K: a thread has a block of 32 of one column (COLS = 1), or of two adjacent ones
// in 16 bits (COLS = 2: pairs of values are loaded as words, so that a warp reads whole 128-byte lines either way).  Codes leave through
// shared memory so that a column's 128 bytes are written together.  With inputs that are not in L2: 3072 x 12288 in fp32 31.5 us, 5.4 TB/s, near the memory's
// rate; 3072 x 9216 in bf16 19.8 us, 3.6 TB/s, and 23.1 with single 16-bit loads (9217 columns): not the memory there, but which of the 32 small loads a lane
// has, the conversions and the exchange bounds it was not measured.
template <typename T, int RULE, int COLS>
__global__ void __launch_bounds__(kThreads) mx_quantize_cols_kernel(const T* x, long long ldx, int rows, int K, int nkb, int pitch,
                                                                    uint8_t* codes, uint8_t* scales) {
    constexpr int WIDTH = 32 * COLS;
    __shared__ uint4 s_codes[WIDTH][9];  // (a piece of padding: the threads of a warp write different columns' rows)
    __shared__ __align__(16) uint8_t s_scales[WIDTH][8];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int kb = blockIdx.x % nkb;
    const int row0 = blockIdx.x / nkb * WIDTH;
    const int row = row0 + lane * COLS, k0 = kb * 256 + w * 32;
    grid_dependency_wait();
    asm volatile("" : "+l"(x));  // (no address of x is known before this point: none of the loads below can be moved ahead of the wait)
    grid_launch_dependents();
    using Word = std::conditional_t<COLS == 2, uint32_t, T>;
    Word raw[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        raw[i] = Word();
        if (row < rows && k0 + i < K) raw[i] = __ldg(reinterpret_cast<const Word*>(x + (k0 + i) * ldx + row));
    }
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        auto value = [&](int i) {
            if constexpr (COLS == 2) {
                union { uint32_t u; T t[2]; } both;
                both.u = raw[i];
                return to_f32<T>(both.t[c]);
            } else {
                return to_f32<T>(raw[i]);
            }
        };
        uint32_t am = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) am = max(am, __float_as_uint(value(i)) & 0x7fffffffu);
        const uint32_t byte = mx_scale_byte<RULE>(am);
        uint32_t words[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value(8 * g + i);
            words[g] = mx_codes8(v, byte);
        }
        s_codes[lane * COLS + c][w] = make_uint4(words[0], words[1], words[2], words[3]);
        s_scales[lane * COLS + c][w] = static_cast<uint8_t>(byte);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
        const int r = i * 32 + (threadIdx.x >> 3), piece = threadIdx.x & 7;  // columns x 8 pieces of 16 bytes
        if (row0 + r < rows) {
            const int at = kb * 128 + piece * 16;
            if (at < pitch) *reinterpret_cast<uint4*>(codes + static_cast<size_t>(row0 + r) * pitch + at) = s_codes[r][piece];
            if (piece < 2)
                *reinterpret_cast<uint32_t*>(scales + mx_scale_word(row0 + r, kb * 2 + piece, nkb)) =
                    *reinterpret_cast<const uint32_t*>(&s_scales[r][piece * 4]);
        }
    }
}

// ------------------------------------------------------------------ dequantizer: the quantizer's units, backwards
// The values' bytes bound it: 4608 x 12288 to bf16 23.3 us, 6.2 TB/s; to fp32 46 us.
template <typename T, int ALIGN>
__device__ __forceinline__ void store_unit(T* row, int k0, int K, const Raw16<T>& r, T* s, int lane) {
    if constexpr (ALIGN == 0) {
        store_spread<T>(row, k0, K, r, s, lane);
    } else if (ALIGN == 32 && sizeof(T) == 2) {
        const int k = k0 + 16 * lane;
        if (k + 16 <= K) {
            const uint4 &a = r.h[0].u[0], &b = r.h[1].u[0];
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + k), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x),
                         "r"(b.y), "r"(b.z), "r"(b.w)
                         : "memory");
        } else {
            union { Raw16<T> r; T t[16]; } c;
            c.r = r;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (k + i < K) row[k + i] = c.t[i];
        }
    } else {
        // 16-byte pieces change places too, so that a warp writes them side by side (each lane's own pieces straight: 63 instead of 46 us for
        // 4608 x 12288 in fp32)
        constexpr int PIECE = 16 / sizeof(T);
        __syncwarp();
        *reinterpret_cast<Raw16<T>*>(s + 16 * lane) = r;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16 / PIECE; ++i) {
            const int at = (32 * i + lane) * PIECE, k = k0 + at;
            if (k + PIECE <= K) *reinterpret_cast<uint4*>(row + k) = *reinterpret_cast<const uint4*>(s + at);
            else
#pragma unroll
                for (int j = 0; j < PIECE; ++j)
                    if (k + j < K) row[k + j] = s[at + j];
        }
    }
}

template <typename T, int ALIGN, int UNITS>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int rows, int K,
                                                                 int nkb, int pitch, T* y, long long ldy) {
    const int lane = threadIdx.x & 31;
    const int per_row = (nkb + 1) >> 1;
    const unsigned units = static_cast<unsigned>(rows) * per_row;
    const unsigned first = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * UNITS;
    if (first >= units) return;
    int row = static_cast<int>(first / per_row), u = static_cast<int>(first % per_row);
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr bool STAGED = ALIGN != 32 || sizeof(T) != 2;  // (see store_unit)
    __shared__ __align__(16) T s_unit[STAGED ? kThreads / 32 : 1][512];
    uint2 word[UNITS];
    uint32_t sw[UNITS];
    {
        int r = row, b = u;
#pragma unroll
        for (int j = 0; j < UNITS; ++j) {
            word[j] = make_uint2(0, 0);
            sw[j] = 0;
            if (r < rows) {
                const int at = b * 256 + lane * 8, ak = b * 4 + (lane >> 3);
                if (at < pitch) word[j] = *reinterpret_cast<const uint2*>(codes + static_cast<size_t>(r) * pitch + at);
                if (ak < 2 * nkb) sw[j] = *reinterpret_cast<const uint32_t*>(scales + mx_scale_word(r, ak, nkb));
            }
            if (++b == per_row) { b = 0; ++r; }
        }
    }
#pragma unroll
    for (int j = 0; j < UNITS; ++j) {
        if (row >= rows) break;
        const float s = e8m0_value((sw[j] >> (8 * ((lane >> 1) & 3))) & 0xffu);
        Raw16<T> out;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w = h == 0 ? word[j].x : word[j].y;
            float v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 p = from_e2m1x2((w >> (8 * i)) & 0xffu);
                v[2 * i] = p.x * s;
                v[2 * i + 1] = p.y * s;
            }
            out.h[h] = pack8<T>(v);
        }
        store_unit<T, ALIGN>(y + row * ldy, u * 512, K, out, s_unit[STAGED ? threadIdx.x >> 5 : 0], lane);
        if (++u == per_row) { u = 0; ++row; }
    }
}

// ------------------------------------------------------------------ plain form of checkpoints
// One thread per 32-bit word of the operand's codes (and its scale byte where it starts a block); bytes behind K become zeros.  Once per checkpoint, by single
// bytes, whose addresses may be odd: import of 9216 x 3072 23 us, 1.3 TB/s, export 60 us, 0.5 TB/s.
__global__ void __launch_bounds__(kThreads) mx_import_kernel(const uint8_t* __restrict__ in_codes, const uint8_t* __restrict__ in_scales, int rows, int K,
                                                             int nkb, int pitch, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
    const int words = nkb * 32;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= static_cast<long long>(rows) * words) return;
    const int row = static_cast<int>(i / words), w = static_cast<int>(i % words);
    const int k0 = w * 8, kbytes = (K + 1) / 2, nblk = (K + 31) / 32;
    uint32_t word = 0;
    for (int b = 0; b < 4; ++b) {
        const int k = k0 + 2 * b;
        if (k < K) {
            uint32_t c = in_codes[static_cast<size_t>(row) * kbytes + k / 2];
            if (k + 1 == K) c &= 15u;
            word |= c << (8 * b);
        }
    }
    if (k0 < pitch * 2) *reinterpret_cast<uint32_t*>(codes + static_cast<size_t>(row) * pitch + k0 / 2) = word;
    if ((w & 15) == 0) {  // the four scales of 128 elements
        uint32_t sw = 0;
        for (int b = 0; b < 4; ++b) {
            const int blk = k0 / 32 + b;
            if (blk < nblk) sw |= static_cast<uint32_t>(in_scales[static_cast<size_t>(row) * nblk + blk]) << (8 * b);
        }
        *reinterpret_cast<uint32_t*>(scales + mx_scale_word(row, w >> 4, nkb)) = sw;
    }
}

__global__ void __launch_bounds__(kThreads) mx_export_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int rows, int K, int nkb,
                                                             int pitch, uint8_t* __restrict__ out_codes, uint8_t* __restrict__ out_scales) {
    const int kbytes = (K + 1) / 2, nblk = (K + 31) / 32;
    const long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= static_cast<long long>(rows) * kbytes) return;
    const int row = static_cast<int>(i / kbytes), b = static_cast<int>(i % kbytes);
    if (out_codes) out_codes[i] = codes[static_cast<size_t>(row) * pitch + b];
    if (out_scales && (b & 15) == 0)
        out_scales[static_cast<size_t>(row) * nblk + b / 16] = scales[mx_scale_word(row, b >> 6, nkb) + ((b >> 4) & 3)];
}

// What rows at `p`, `ld` elements apart, are aligned to: 32, 16 or 0 (less than 16).
inline int row_alignment(const void* p, long long ld, size_t element) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | static_cast<uintptr_t>(ld * static_cast<long long>(element));
    return (bits & 31u) == 0 ? 32 : (bits & 15u) == 0 ? 16 : 0;
}
// Units of 512 elements per warp: two where that leaves every SM 32 warps, else one, so that a short call is spread out (256 x 1152 1.7
// against 2.3 us).
inline int units_per_warp(const dirotq_mxfp4* t) {
    return static_cast<long long>(t->rows) * ((t->lay.nkb + 1) / 2) >= 64ll * sm_count(t->device) ? 2 : 1;
}
inline int unit_blocks(const dirotq_mxfp4* t, int per_warp) {
    const long long per = (kThreads / 32) * per_warp;
    return static_cast<int>((static_cast<long long>(t->rows) * ((t->lay.nkb + 1) / 2) + per - 1) / per);
}
// go(kernel of that alignment, units per warp)
#define DIROTQ_MX_UNITS(KERNEL, ...)                                                                                             \
    (align == 32   ? (per_warp == 2 ? go(KERNEL<__VA_ARGS__, 32, 2>) : go(KERNEL<__VA_ARGS__, 32, 1>)) \
     : align == 16 ? (per_warp == 2 ? go(KERNEL<__VA_ARGS__, 16, 2>) : go(KERNEL<__VA_ARGS__, 16, 1>)) \
                   : (per_warp == 2 ? go(KERNEL<__VA_ARGS__, 0, 2>) : go(KERNEL<__VA_ARGS__, 0, 1>)))
inline bool fits_grid(long long blocks) { return blocks <= 0x7fffffffll; }

template <typename T>
cudaError_t quantize_t(const void* x, int layout, long long ldx, int rule, const dirotq_mxfp4* t, cudaStream_t stream) {
    const T* in = static_cast<const T*>(x);
    uint8_t* codes = reinterpret_cast<uint8_t*>(t->buffer);
    uint8_t* scales = codes + t->lay.off_scales;
    const bool floor = rule == DIROTQ_MX_SCALE_FLOOR;
    if (layout == DIROTQ_LAYOUT_NK) {
        const int align = row_alignment(x, ldx, sizeof(T)), per_warp = units_per_warp(t);
        auto go = [&](auto kern) {
            return launch_kernel(kern, unit_blocks(t, per_warp), kThreads, 0, stream, true, in, ldx, t->rows, t->K, t->lay.nkb, t->lay.pitch, codes, scales);
        };
        return floor ? DIROTQ_MX_UNITS(mx_quantize_rows_kernel, T, DIROTQ_MX_SCALE_FLOOR) : DIROTQ_MX_UNITS(mx_quantize_rows_kernel, T, DIROTQ_MX_SCALE_CEIL);
    }
    auto kern = floor ? mx_quantize_cols_kernel<T, DIROTQ_MX_SCALE_FLOOR, 1> : mx_quantize_cols_kernel<T, DIROTQ_MX_SCALE_CEIL, 1>;
    int width = 32;
    if constexpr (sizeof(T) == 2) {
        if (t->rows % 2 == 0 && ldx % 2 == 0 && (reinterpret_cast<uintptr_t>(x) & 3u) == 0) {  // pairs of columns are aligned words
            kern = floor ? mx_quantize_cols_kernel<T, DIROTQ_MX_SCALE_FLOOR, 2> : mx_quantize_cols_kernel<T, DIROTQ_MX_SCALE_CEIL, 2>;
            width = 64;
        }
    }
    const unsigned blocks = static_cast<unsigned>((t->rows + width - 1) / width) * t->lay.nkb;
    return launch_kernel(kern, static_cast<int>(blocks), kThreads, 0, stream, true, in, ldx, t->rows, t->K, t->lay.nkb, t->lay.pitch, codes, scales);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

dirotq_status_t current_device(int* device) {
    cudaError_t e = cudaGetDevice(device);
    if (e != cudaSuccess) { set_error("cudaGetDevice", e); return DIROTQ_ERR_CUDA; }
    int major = 0;
    e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *device);
    if (e != cudaSuccess) { set_error("cudaDeviceGetAttribute", e); return DIROTQ_ERR_CUDA; }
    return major == 10 ? DIROTQ_OK : DIROTQ_ERR_ARCH;
}

dirotq_status_t check_shape(int rows, int K) {
    if (rows < 1 || K < 1) return DIROTQ_ERR_INVALID_ARG;
    if (rows > (1 << 24) || K > (1 << 20)) return DIROTQ_ERR_UNSUPPORTED_SHAPE;
    // every kernel's grid: at most one block per 256 bytes of codes
    return fits_grid(static_cast<long long>(rows) * ((K + 255) / 256)) ? DIROTQ_OK : DIROTQ_ERR_UNSUPPORTED_SHAPE;
}

dirotq_status_t check_operand(const dirotq_mxfp4* t) {
    if (!mx_valid(t)) return DIROTQ_ERR_INVALID_ARG;
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) return DIROTQ_ERR_CUDA;
    return dev == t->device ? DIROTQ_OK : DIROTQ_ERR_INVALID_ARG;
}

dirotq_status_t done(const char* what, cudaError_t e) {
    if (e == cudaSuccess) return DIROTQ_OK;
    set_error(what, e);
    return DIROTQ_ERR_CUDA;
}

constexpr size_t kStatusBytes = 256;

dirotq_status_t check_product(const dirotq_mxfp4* a_or_null, const dirotq_mxfp4* b, const void* bias, const void* y, int y_dtype, long long ldy) {
    if (!mx_valid(b) || (a_or_null && !mx_valid(a_or_null)) || !y || !dtype_is_16(y_dtype)) return DIROTQ_ERR_INVALID_ARG;
    if (a_or_null && a_or_null->K != b->K) return DIROTQ_ERR_INVALID_ARG;
    if (ldy < b->rows) return DIROTQ_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(y) & 1u) != 0 || (reinterpret_cast<uintptr_t>(bias) & 1u) != 0) return DIROTQ_ERR_INVALID_ARG;
    return DIROTQ_OK;
}

dirotq_status_t linear(const void* x, int x_dtype, long long ldx, int M, int scale_rule, const dirotq_mxfp4* w, const void* bias,
                       const dirotq_qk_t* qk, void* y, int y_dtype, long long ldy, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
    dirotq_status_t st = check_product(nullptr, w, bias, y, y_dtype, ldy);
    if (st != DIROTQ_OK) return st;
    if (!x || !dtype_ok(x_dtype) || (scale_rule != DIROTQ_MX_SCALE_FLOOR && scale_rule != DIROTQ_MX_SCALE_CEIL)) return DIROTQ_ERR_INVALID_ARG;
    if (ldx < w->K || reinterpret_cast<uintptr_t>(x) % dtype_size(x_dtype) != 0) return DIROTQ_ERR_INVALID_ARG;
    st = check_shape(M, w->K);
    if (st != DIROTQ_OK) return st;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & (kAlign - 1)) != 0) return DIROTQ_ERR_INVALID_ARG;
    if (workspace_bytes < kAlign + make_mx_layout(M, w->K).total) return DIROTQ_ERR_BUFFER_TOO_SMALL;
    if (qk) {
        st = qk_check(qk, M);
        if (st != DIROTQ_OK) return st;
        if (static_cast<long long>(qk->heads_q + 2ll * qk->heads_kv) * qk->head_dim != w->rows) return DIROTQ_ERR_INVALID_ARG;
        if ((qk->head_dim != 64 && qk->head_dim != 128) || (qk->rot_dim != 0 && qk->rot_dim != qk->head_dim)) return DIROTQ_ERR_UNSUPPORTED_SHAPE;
    }
    st = check_operand(w);
    if (st != DIROTQ_OK) return st;
    // A product that quantizes x itself has blocks that write y while others still read x: with y in x's memory the quantizer runs alone, before
    // anything of y is written, as it does for more rows.
    const long long es = static_cast<long long>(dtype_size(x_dtype));
    const bool apart = !rows_overlap(x, M, w->K * es, ldx * es, y, M, w->rows * 2ll, ldy * 2);
    if (apart && mx_fuses(M, w->rows, w->lay.nkb, qk, w->device)) {
        const MxGemmArgs ga = {M, nullptr, x, x_dtype, ldx, scale_rule, w, bias, y, y_dtype, ldy, static_cast<int*>(workspace), false, qk};
        return launch_mx_gemm(ga, stream);
    }
    dirotq_mxfp4 a;
    st = mx_setup(&a, M, w->K, static_cast<char*>(workspace) + kAlign, w->device, false);
    if (st != DIROTQ_OK) return st;
    st = done("dirotq_mxfp4_linear", launch_mx_quantize(x, x_dtype, DIROTQ_LAYOUT_NK, ldx, scale_rule, &a, stream));
    if (st != DIROTQ_OK) return st;
    const MxGemmArgs ga = {M, &a, nullptr, 0, 0, 0, w, bias, y, y_dtype, ldy, static_cast<int*>(workspace), true, qk};
    return launch_mx_gemm(ga, stream);
}

}  // namespace

bool mx_valid(const dirotq_mxfp4* t) { return t != nullptr && t->magic == kMxMagic; }

dirotq_status_t mx_setup(dirotq_mxfp4* t, int rows, int K, void* buffer, int device, bool both) {
    memset(t, 0, sizeof *t);
    t->magic = kMxMagic;
    t->device = device;
    t->rows = rows;
    t->K = K;
    t->lay = make_mx_layout(rows, K);
    t->buffer = static_cast<char*>(buffer);
    t->box = box_rows(rows);
    t->box64 = rows < 64 ? t->box : 64;
    if (both) {
        const dirotq_status_t st = encode_tmap_2d(&t->tmap64, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, buffer, (uint64_t)t->lay.pitch, (uint64_t)rows,
                                                  (uint64_t)t->lay.pitch, 128, t->box64, CU_TENSOR_MAP_SWIZZLE_128B);
        if (st != DIROTQ_OK) return st;
    }
    return encode_tmap_2d(&t->tmap, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, buffer, (uint64_t)t->lay.pitch, (uint64_t)rows, (uint64_t)t->lay.pitch, 128,
                          t->box, CU_TENSOR_MAP_SWIZZLE_128B);
}

cudaError_t launch_mx_quantize(const void* x, int x_dtype, int x_layout, long long ldx, int scale_rule, const dirotq_mxfp4* t, cudaStream_t stream) {
    switch (x_dtype) {
        case DIROTQ_DTYPE_F32: return quantize_t<float>(x, x_layout, ldx, scale_rule, t, stream);
        case DIROTQ_DTYPE_BF16: return quantize_t<__nv_bfloat16>(x, x_layout, ldx, scale_rule, t, stream);
        default: return quantize_t<__half>(x, x_layout, ldx, scale_rule, t, stream);
    }
}

}  // namespace dirotq

using namespace dirotq;

extern "C" {

dirotq_status_t dirotq_mxfp4_bytes(int rows, int K, size_t* bytes) {
    if (!bytes) return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_shape(rows, K);
    if (st != DIROTQ_OK) return st;
    *bytes = make_mx_layout(rows, K).total;
    return DIROTQ_OK;
}

dirotq_status_t dirotq_mxfp4_create(int rows, int K, void* buffer, size_t buffer_bytes, dirotq_mxfp4_t** out) {
    if (!buffer || !out || (reinterpret_cast<uintptr_t>(buffer) & (kAlign - 1)) != 0) return DIROTQ_ERR_INVALID_ARG;
    dirotq_status_t st = check_shape(rows, K);
    if (st != DIROTQ_OK) return st;
    if (buffer_bytes < make_mx_layout(rows, K).total) return DIROTQ_ERR_BUFFER_TOO_SMALL;
    int dev = 0;
    st = current_device(&dev);
    if (st != DIROTQ_OK) return st;
    dirotq_mxfp4* t = new (std::nothrow) dirotq_mxfp4;
    if (!t) return DIROTQ_ERR_INVALID_ARG;
    st = mx_setup(t, rows, K, buffer, dev, true);
    if (st != DIROTQ_OK) {
        delete t;
        return st;
    }
    *out = t;
    return DIROTQ_OK;
}

dirotq_status_t dirotq_mxfp4_destroy(dirotq_mxfp4_t* t) {
    if (!mx_valid(t)) return DIROTQ_ERR_INVALID_ARG;
    t->magic = 0;
    delete t;
    return DIROTQ_OK;
}

dirotq_status_t dirotq_mxfp4_info(const dirotq_mxfp4_t* t, int* rows, int* K) {
    if (!mx_valid(t)) return DIROTQ_ERR_INVALID_ARG;
    if (rows) *rows = t->rows;
    if (K) *K = t->K;
    return DIROTQ_OK;
}

dirotq_status_t dirotq_mxfp4_quantize(const void* x, int x_dtype, int x_layout, long long ldx, int scale_rule, const dirotq_mxfp4_t* out,
                                      dirotq_stream_t stream) {
    if (!mx_valid(out) || !x || !dtype_ok(x_dtype) || (x_layout != DIROTQ_LAYOUT_NK && x_layout != DIROTQ_LAYOUT_KN))
        return DIROTQ_ERR_INVALID_ARG;
    if (scale_rule != DIROTQ_MX_SCALE_FLOOR && scale_rule != DIROTQ_MX_SCALE_CEIL) return DIROTQ_ERR_INVALID_ARG;
    if (ldx < (x_layout == DIROTQ_LAYOUT_NK ? out->K : out->rows) || reinterpret_cast<uintptr_t>(x) % dtype_size(x_dtype) != 0)
        return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_operand(out);
    if (st != DIROTQ_OK) return st;
    return done("dirotq_mxfp4_quantize", launch_mx_quantize(x, x_dtype, x_layout, ldx, scale_rule, out, static_cast<cudaStream_t>(stream)));
}

dirotq_status_t dirotq_mxfp4_dequantize(const dirotq_mxfp4_t* t, void* y, int y_dtype, long long ldy, dirotq_stream_t stream) {
    if (!mx_valid(t) || !y || !dtype_ok(y_dtype) || ldy < t->K || reinterpret_cast<uintptr_t>(y) % dtype_size(y_dtype) != 0)
        return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_operand(t);
    if (st != DIROTQ_OK) return st;
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(t->buffer);
    const uint8_t* scales = codes + t->lay.off_scales;
    const int align = row_alignment(y, ldy, dtype_size(y_dtype)), per_warp = units_per_warp(t);
    auto of_type = [&](auto* out) {
        using T = std::remove_pointer_t<decltype(out)>;
        auto go = [&](auto kern) {
            return launch_kernel(kern, unit_blocks(t, per_warp), kThreads, 0, static_cast<cudaStream_t>(stream), true, codes, scales, t->rows, t->K, t->lay.nkb,
                                 t->lay.pitch, out, ldy);
        };
        return DIROTQ_MX_UNITS(mx_dequantize_kernel, T);
    };
    return done("dirotq_mxfp4_dequantize", y_dtype == DIROTQ_DTYPE_F32    ? of_type(static_cast<float*>(y))
                                           : y_dtype == DIROTQ_DTYPE_BF16 ? of_type(static_cast<__nv_bfloat16*>(y))
                                                                          : of_type(static_cast<__half*>(y)));
}

dirotq_status_t dirotq_mxfp4_import(const uint8_t* codes, const uint8_t* scales, const dirotq_mxfp4_t* out, dirotq_stream_t stream) {
    if (!mx_valid(out) || !codes || !scales) return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_operand(out);
    if (st != DIROTQ_OK) return st;
    uint8_t* to = reinterpret_cast<uint8_t*>(out->buffer);
    const long long words = static_cast<long long>(out->rows) * out->lay.nkb * 32;
    return done("dirotq_mxfp4_import",
                launch_kernel(mx_import_kernel, static_cast<int>((words + kThreads - 1) / kThreads), kThreads, 0, static_cast<cudaStream_t>(stream), false,
                              codes, scales, out->rows, out->K, out->lay.nkb, out->lay.pitch, to, to + out->lay.off_scales));
}

dirotq_status_t dirotq_mxfp4_export(const dirotq_mxfp4_t* t, uint8_t* codes, uint8_t* scales, dirotq_stream_t stream) {
    if (!mx_valid(t)) return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_operand(t);
    if (st != DIROTQ_OK) return st;
    const uint8_t* from = reinterpret_cast<const uint8_t*>(t->buffer);
    const long long n = static_cast<long long>(t->rows) * ((t->K + 1) / 2);
    return done("dirotq_mxfp4_export",
                launch_kernel(mx_export_kernel, static_cast<int>((n + kThreads - 1) / kThreads), kThreads, 0, static_cast<cudaStream_t>(stream), false, from,
                              from + t->lay.off_scales, t->rows, t->K, t->lay.nkb, t->lay.pitch, codes, scales));
}

dirotq_status_t dirotq_mxfp4_workspace_bytes(int M, int K, size_t* bytes) {
    if (!bytes) return DIROTQ_ERR_INVALID_ARG;
    const dirotq_status_t st = check_shape(M, K);
    if (st != DIROTQ_OK) return st;
    *bytes = kAlign + make_mx_layout(M, K).total;
    return DIROTQ_OK;
}

dirotq_status_t dirotq_mxfp4_gemm(const dirotq_mxfp4_t* a, const dirotq_mxfp4_t* b, const void* bias, void* y, int y_dtype, long long ldy,
                                  void* workspace, size_t workspace_bytes, dirotq_stream_t stream) {
    if (!a) return DIROTQ_ERR_INVALID_ARG;
    dirotq_status_t st = check_product(a, b, bias, y, y_dtype, ldy);
    if (st != DIROTQ_OK) return st;
    if (!workspace || !aligned16(workspace)) return DIROTQ_ERR_INVALID_ARG;
    if (workspace_bytes < kStatusBytes) return DIROTQ_ERR_BUFFER_TOO_SMALL;
    st = check_operand(a);
    if (st == DIROTQ_OK) st = check_operand(b);
    if (st != DIROTQ_OK) return st;
    const MxGemmArgs ga = {a->rows, a, nullptr, 0, 0, 0, b, bias, y, y_dtype, ldy, static_cast<int*>(workspace), false, nullptr};
    return launch_mx_gemm(ga, static_cast<cudaStream_t>(stream));
}

dirotq_status_t dirotq_mxfp4_linear(const void* x, int x_dtype, long long ldx, int M, int scale_rule, const dirotq_mxfp4_t* w, const void* bias,
                                    void* y, int y_dtype, long long ldy, void* workspace, size_t workspace_bytes, dirotq_stream_t stream) {
    return linear(x, x_dtype, ldx, M, scale_rule, w, bias, nullptr, y, y_dtype, ldy, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

dirotq_status_t dirotq_mxfp4_qkv(const void* x, int x_dtype, long long ldx, int M, int scale_rule, const dirotq_mxfp4_t* w, const void* bias,
                                 const dirotq_qk_t* qk, void* y, int y_dtype, long long ldy, void* workspace, size_t workspace_bytes,
                                 dirotq_stream_t stream) {
    if (!qk) return DIROTQ_ERR_INVALID_ARG;
    return linear(x, x_dtype, ldx, M, scale_rule, w, bias, qk, y, y_dtype, ldy, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
