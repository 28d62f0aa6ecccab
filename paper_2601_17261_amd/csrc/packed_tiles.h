// Tiles of attention in LDS and registers, as its kernels share them: 64 positions of keys or values, read as rows and with transposition, fragments of the
// 32 x 32 x 16 matrix instruction, and what goes over a wave's lanes.
#pragma once
#include "agzo_internal.h"

namespace agzo {

namespace {

typedef __bf16 pk_bf16x8 __attribute__((ext_vector_type(8)));
typedef float pk_floatx16 __attribute__((ext_vector_type(16)));
typedef uint32_t pk_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) void* pk_lptr;
typedef __attribute__((address_space(3))) char* pk_lchar;
typedef const __attribute__((address_space(1))) void* pk_gptr;
union PkFrag { uint4 u; uint32_t w[4]; pk_bf16x8 v; };

constexpr int PK_T = 64;                    // positions of a tile in LDS
constexpr float PK_LOG2E = 1.44269504088896341f, PK_LN2 = 0.693147180559945309f;

__device__ __forceinline__ pk_floatx16 pk_mfma(const PkFrag& a, const PkFrag& b, const pk_floatx16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ float pk_max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pk_sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint4 pk_load16(__amdgpu_buffer_rsrc_t rsrc, int off, int uniform) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, uniform, 0);
    return make_uint4(v[0], v[1], v[2], v[3]);
}

// A tile of 64 positions of HD values, 16-byte chunk c of row r at place c ^ swz(r).  Reads of 16 rows' same chunk, and reads with
// transposition of 4 rows' four neighbouring chunks, then meet each bank once
template <int HD>
__device__ __forceinline__ int pk_swz(int r) { return HD == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : ((r & 2) << 1) | ((r >> 2) & 3); }

// Byte offsets, in a tile, of what a lane reads.  rows: chunk (lane / 32) of row lane % 32 (chunk 2 ks + lane / 32: ^ ks << 5; rows 32 further on: + 32
// rows' bytes).  trans: for 16 positions, those 4 (lane / 32) .. + 4 of the first eight and of the second eight, dims 0 .. 32 (32 db ..: ^ db << 6;
// 16 positions further on: + 16 rows' bytes)
template <int HD>
struct PkOffsets {
    int rows, trans[2];
    __device__ __forceinline__ PkOffsets() {
        const int lane = threadIdx.x & 63, r = lane & 31, hi = lane >> 5, n16 = lane & 15, dg = (lane >> 4) & 1;
        rows = r * (HD * 2) + ((hi ^ pk_swz<HD>(r)) << 4);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int tr = 8 * s + 4 * hi + (n16 >> 2);
            trans[s] = tr * (HD * 2) + (((2 * dg + ((n16 & 3) >> 1)) ^ pk_swz<HD>(tr)) << 4) + (n16 & 1) * 8;
        }
    }
    // addresses in LDS of a tile that starts at `at`, a multiple of 256.  (Values that the compiler does not know: it would work out every read's address ahead of
    // the loop over tiles and spill them, and a wait for a reload is one for the next tile's loads too)
    __device__ __forceinline__ PkOffsets(const PkOffsets& of, int at) : rows(of.rows + at), trans{of.trans[0] + at, of.trans[1] + at} {
        asm volatile("" : "+v"(rows), "+v"(trans[0]), "+v"(trans[1]));
    }
    // ... from two offsets kept: the second eight positions are 8 rows on, and their chunks ^ 2
    __device__ __forceinline__ PkOffsets(int rows_, int trans_, int at) : rows(rows_ + at), trans{trans_ + at, ((trans_ + at) ^ 32) + 8 * HD * 2} {
        asm volatile("" : "+v"(rows), "+v"(trans[0]), "+v"(trans[1]));
    }
    // chunk 2 ks + lane / 32 of row 32 h + lane % 32
    __device__ __forceinline__ pk_bf16x8 row(int h, int ks, int more = 0) const {
        typedef const __attribute__((address_space(3))) pk_bf16x8* ptr;
        return *(ptr)(uintptr_t)(uint32_t)((rows ^ (ks << 5)) + h * 32 * HD * 2 + more);
    }
};

// a fragment with transposition: 16 positions (from place `at` of a tile on) x 32 dims
typedef __bf16 pk_bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) pk_bf16x4* pk_trptr;
template <int HD>
__device__ __forceinline__ void pk_read_trans(const PkOffsets<HD>& o, int at, int db, PkFrag& f) {
    union { pk_bf16x4 v; uint2 u; } lo, hi;
    lo.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((pk_trptr)(uintptr_t)(uint32_t)((o.trans[0] ^ (db << 6)) + at));
    hi.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((pk_trptr)(uintptr_t)(uint32_t)((o.trans[1] ^ (db << 6)) + at));
    f.u = make_uint4(lo.u.x, lo.u.y, hi.u.x, hi.u.y);
}

// acc[db] += (positions x dims of a tile)^T times fragments FROM .. TO of 16 positions each
template <int HD, int FROM, int TO>
__device__ __forceinline__ void pk_second(const PkOffsets<HD>& o, int at, const PkFrag (&p)[4], pk_floatx16 (&acc)[HD / 32]) {
#pragma unroll
    for (int s = FROM; s < TO; ++s)
#pragma unroll
        for (int db = 0; db < HD / 32; ++db) {
            PkFrag f;
            pk_read_trans<HD>(o, at + s * 16 * HD * 2, db, f);
            acc[db] = pk_mfma(f, p[s], acc[db]);
        }
}

// The same with care: values that are not finite are taken out, and with INF, where `seen` (fragments of ones and zeros) has a one for them, the
// sum becomes what they make of it: a product of seen with 1 for inf, 2^12 for -inf and 2^23 for NaN has at most 64 of each.  LOW: p has a
// second part
template <int HD, bool INF, bool LOW>
__device__ __forceinline__ void pk_second_careful(const char* tile, const PkFrag (&p)[4], const PkFrag (&low)[4], const PkFrag (&seen)[4], pk_floatx16 (&acc)[HD / 32]) {
    const int lane = threadIdx.x & 63, hi = lane >> 5;
#pragma unroll
    for (int db = 0; db < HD / 32; ++db) {
        const int dim = 32 * db + (lane & 31);
        pk_floatx16 c = {};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            PkFrag f, k;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t fw = 0, kw = 0;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int i = 2 * w + b, r = 16 * s + (i >> 2) * 8 + 4 * hi + (i & 3);
                    const uint32_t x = *reinterpret_cast<const bf16_t*>(tile + r * (HD * 2) + (((dim >> 3) ^ pk_swz<HD>(r)) << 4) + (dim & 7) * 2);
                    const bool bad = (x & 0x7F80u) == 0x7F80u;
                    fw |= (bad ? 0u : x) << (16 * b);
                    // 2^23, 2^12 and 1 in bf16
                    kw |= (!bad ? 0u : (x & 0x7Fu) ? 0x4B00u : (x & 0x8000u) ? 0x4580u : 0x3F80u) << (16 * b);
                }
                f.w[w] = fw;
                k.w[w] = kw;
            }
            acc[db] = pk_mfma(f, p[s], acc[db]);       // (in the order of pk_second: the same bits)
            if (LOW) acc[db] = pk_mfma(f, low[s], acc[db]);
            if (INF) c = pk_mfma(k, seen[s], c);
        }
        if (INF) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool nan = c[e] >= 8388608.f, neg = c[e] >= 4096.f, pos = c[e] - 4096.f * floorf(c[e] * (1.f / 4096.f)) > 0.f;
                acc[db][e] += c[e] == 0.f ? 0.f : nan || (neg && pos) ? NAN : neg ? -INFINITY : INFINITY;
            }
        }
    }
}

// whether any of a lane's sums is not finite
template <int N>
__device__ __forceinline__ bool pk_not_finite(const pk_floatx16 (&acc)[N], float z = 0.f) {
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) z = fmaf(acc[d][e], 0.f, z);
    return !(z == 0.f);
}

// a lane's sums of its column (rows of the instruction: dims) times f, as bf16, to `row` (its row's first value): the halves of a wave
// exchange what makes 16 bytes
template <int HD>
__device__ __forceinline__ void pk_store(const pk_floatx16 (&acc)[HD / 32], float f, bf16_t* row, bool store) {
    const int hi = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int db = 0; db < HD / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            const uint32_t a0 = pack_bf16x2(acc[db][4 * g] * f, acc[db][4 * g + 1] * f), a1 = pack_bf16x2(acc[db][4 * g + 2] * f, acc[db][4 * g + 3] * f);
            const uint32_t b0 = pack_bf16x2(acc[db][4 * g + 4] * f, acc[db][4 * g + 5] * f), b1 = pack_bf16x2(acc[db][4 * g + 6] * f, acc[db][4 * g + 7] * f);
            const auto r0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), r1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            if (store) *reinterpret_cast<uint4*>(row + 32 * db + 8 * (g + hi)) = make_uint4(r0[0], r1[0], r0[1], r1[1]);
        }
}

// x / d for 0 <= x < 2^31, 1 <= d: the quotient by a multiplication is at most one short.  (A division is some 30 instructions, of 64 bits 100: three of them
// and the scan below were half of what a workgroup did before its first load)
struct PkDiv {
    uint32_t d, m;
    __device__ __forceinline__ explicit PkDiv(int by) : d((uint32_t)by), m((uint32_t)(0x100000000ull / (uint32_t)by - (by == 1))) {}
    __device__ __forceinline__ int operator()(int x) const {
        uint32_t q = __umulhi((uint32_t)x, m);
        q += (uint32_t)x - q * d >= d;
        return (int)q;
    }
};

// sums over the lanes up to each, and the sum of all
__device__ __forceinline__ int pk_scan(int x) {
#pragma unroll
    for (int shift = 1; shift < 16; shift <<= 1) {
        // row_shr: within 16 lanes
        const int o = shift == 1 ? __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true) : shift == 2 ? __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true)
                    : shift == 4 ? __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true) : __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
        x += o;
    }
    const int a = __builtin_amdgcn_readlane(x, 15), b = a + __builtin_amdgcn_readlane(x, 31), c = b + __builtin_amdgcn_readlane(x, 47);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row == 0 ? 0 : row == 1 ? a : row == 2 ? b : c);
}

// sum over the lanes
__device__ __forceinline__ int pk_total(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    return __builtin_amdgcn_readlane(x, 15) + __builtin_amdgcn_readlane(x, 31) + __builtin_amdgcn_readlane(x, 47) + __builtin_amdgcn_readlane(x, 63);
}

__device__ __forceinline__ void pk_zero(pk_floatx16& x) {
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = 0.f;
}

// e's position in a block of 32
__device__ __forceinline__ int pk_pos(int e) { return 8 * (e >> 2) + (e & 3); }      // + 4 (lane / 32)

}  // namespace

}  // namespace agzo
