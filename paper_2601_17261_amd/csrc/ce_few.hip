// Token cross-entropy of a layer's outputs, and its gradient, for few tokens (answers that are scored, a short sentence; see ce_few_fits): what counts is that W is read, and dW
// written, at the rate of memory.  Products are v_mfma_f32_32x32x16_bf16 with W's rows or dims as the instruction's rows and the tokens as its columns.
//
// Logits, 32 tokens at a time: a workgroup has 32 outputs, its four waves every fourth 256 bytes of their rows, requested a round ahead straight into registers in the
// layout of the instruction: whole lines, 8 KB a wave, and nothing that a wave waits for another with until the four sums meet in LDS.
// 7 tokens, 2048 -> 32000 (131 MB): 30 us, and the 256 x 256 tiles of gemm_bf16_aligned.hip 54.  (Two blocks of tokens to a wave
// leave room for one wave a SIMD: 40 tokens, 1024 -> 50000: 52 us, the tiles 38.)
#include "gemm_bf16_common.h"

namespace agzo {

namespace {

union FewFrag { uint4 u; uint2 h[2]; bf16x8 v; };
constexpr int FEW_OUT = 32, FEW_K = 128;                 // outputs of a workgroup, values of a row that a wave reads at a time
constexpr float FEW_LOG2E = 1.44269504088896341f;

__device__ __forceinline__ uint4 few_load(__amdgpu_buffer_rsrc_t r, int off) {
    const auto v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
    return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t few_rsrc(const bf16_t* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(base), 0, (int)(uint32_t)kPastEnd, 0x00020000);
}

struct FewArgs {
    const bf16_t* X; int64_t ldx;
    const bf16_t* W; int64_t ldw;
    int M; int64_t V, d;
    const int32_t* ids;
    // statistics of 32 outputs each, [token][outputs / 32], and the targets' logits
    float2* ms; float* tl; int64_t nch;
    // gradient: D [M][ldd], D^T [V][32]
    const float* lse; const double* g; bf16_t* D; int64_t ldd; bf16_t* Dt; int64_t ldt; float* scale;
    int blocks;                     // of 32 tokens
};

template <bool GRAD>
__global__ __launch_bounds__(256) void ce_few_kernel(const FewArgs a) {
    __shared__ float red[4][FEW_OUT][33];
    __shared__ float2 part[8][32];
    __shared__ __align__(16) bf16_t tile[GRAD ? FEW_OUT : 1][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, hi = lane >> 5;
    // workgroups of the same outputs follow each other on one XCD (ids are dealt round-robin over the eight), so that W comes out of its L2 for all but the first
    const int at = blockIdx.x >> 3, m0 = at % a.blocks * 32, M = min(32, a.M - m0);
    const int64_t chunk = (int64_t)(at / a.blocks) * 8 + (blockIdx.x & 7), out0 = chunk * FEW_OUT;
    if (out0 >= a.V) return;
    const int left = (int)min((int64_t)FEW_OUT, a.V - out0);
    const auto rw = few_rsrc(a.W + out0 * a.ldw), rx = few_rsrc(a.X + (M > 0 ? (int64_t)m0 * a.ldx : 0));        // (M <= 0: only zeros of D^T are wanted)
    // (outputs and tokens past the end repeat the last ones, uncounted)
    const int woff = min(r, left - 1) * (int)(2 * a.ldw) + 16 * hi, xoff = min(r, max(M, 1) - 1) * (int)(2 * a.ldx) + 16 * hi;
    const int nchunk = (int)((a.d + FEW_K - 1) / FEW_K);
    FewFrag w0[8], x0[8], w1[8], x1[8];
    auto load = [&](int c, FewFrag (&w)[8], FewFrag (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const int at = c * (2 * FEW_K) + 32 * s;
            const bool in = c * FEW_K + 16 * s + 8 * hi < (int)a.d;            // (past the row: zeros)
            w[s].u = few_load(rw, in ? woff + at : kPastEnd);
            x[s].u = few_load(rx, in ? xoff + at : kPastEnd);
        }
    };
    floatx16 acc = {};
    auto multiply = [&](const FewFrag (&w)[8], const FewFrag (&x)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < 8; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[s].v, x[s].v, acc, 0, 0, 0);
    };
    if (wave < nchunk) load(wave, w0, x0);
    for (int c = wave; c < nchunk; c += 8) {
        if (c + 4 < nchunk) load(c + 4, w1, x1);
        multiply(w0, x0);
        if (c + 4 >= nchunk) break;
        if (c + 8 < nchunk) load(c + 8, w0, x0);
        multiply(w1, x1);
    }
    // a lane's sums: token r, outputs 8 (e / 4) + 4 hi + e % 4
#pragma unroll
    for (int e = 0; e < 16; ++e) red[wave][8 * (e >> 2) + 4 * hi + (e & 3)][r] = acc[e];
    if (GRAD) {
        if (tid < FEW_OUT * 4) reinterpret_cast<uint4*>(&tile[0][0])[tid] = make_uint4(0, 0, 0, 0);
        if (blockIdx.x == 0 && wave == 0) {
            int count = 0;
            for (int t = 0; t < a.M; t += 64) {
                const int id = t + lane < a.M ? a.ids[t + lane] : -1;
                count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(id >= 0 && id < a.V));
            }
            if (lane == 0) *a.scale = (float)((a.g ? *a.g : 1.0) / (double)max(count, 1));
        }
    }
    __syncthreads();
    // four outputs of a token a thread
    const int grp = tid >> 5, tok = tid & 31;
    float y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) y[u] = (red[0][4 * grp + u][tok] + red[1][4 * grp + u][tok]) + (red[2][4 * grp + u][tok] + red[3][4 * grp + u][tok]);
    const int64_t id = tok < M ? a.ids[m0 + tok] : -1;
    if (!GRAD) {
        float mx = -INFINITY, s = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (4 * grp + u < left) {
                mx = fmaxf(mx, y[u]);
                if (out0 + 4 * grp + u == id) a.tl[m0 + tok] = y[u];
            }
        // (a NaN among them stays in the sum)
        const float m0 = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (4 * grp + u < left) s += __builtin_amdgcn_exp2f((y[u] - m0) * FEW_LOG2E);
        part[grp][tok] = make_float2(mx, s);
    } else {
        const bool counted = id >= 0 && id < a.V;
        const float l = tok < M ? a.lse[m0 + tok] : 0.f;
        float v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float p = __builtin_amdgcn_exp2f((y[u] - l) * FEW_LOG2E);
            v[u] = counted && 4 * grp + u < left ? (out0 + 4 * grp + u == id ? p - 1.f : p) : 0.f;
        }
        const uint2 two = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        if (tok < M) {
            *reinterpret_cast<uint2*>(a.D + (int64_t)(m0 + tok) * a.ldd + out0 + 4 * grp) = two;
            tile[4 * grp][tok] = (bf16_t)two.x; tile[4 * grp + 1][tok] = (bf16_t)(two.x >> 16);
            tile[4 * grp + 2][tok] = (bf16_t)two.y; tile[4 * grp + 3][tok] = (bf16_t)(two.y >> 16);
        }
    }
    __syncthreads();
    if (GRAD) {
        if (a.Dt && tid < 4 * left) *reinterpret_cast<uint4*>(a.Dt + (out0 + (tid >> 2)) * a.ldt + m0 + (tid & 3) * 8) = reinterpret_cast<const uint4*>(&tile[0][0])[tid];
        return;
    }
    if (tid >= M) return;
    float mx = -INFINITY, s = 0.f;
#pragma unroll
    for (int g8 = 0; g8 < 8; ++g8) mx = fmaxf(mx, part[g8][tid].x);
#pragma unroll
    for (int g8 = 0; g8 < 8; ++g8) {
        const float2 p = part[g8][tid];
        s += p.y == 0.f ? 0.f : p.y * __builtin_amdgcn_exp2f((p.x - (mx == -INFINITY ? 0.f : mx)) * FEW_LOG2E);
    }
    a.ms[(m0 + tid) * a.nch + chunk] = make_float2(mx, s);
}

// Loss and lse from the statistics: a workgroup has up to 32 tokens, 1, 2, 4, 8 or 16 waves to each, so that up to 16 are looked at at once; sums in fp64.  One
// workgroup: the loss; several: {sum, count} of each, which loss.hip's last launch adds
__global__ __launch_bounds__(1024) void ce_few_finish_kernel(const float2* __restrict__ ms, const float* __restrict__ tl, const int32_t* __restrict__ ids, int M, int64_t V, int64_t nch,
                                                             float* __restrict__ lse, double* __restrict__ scratch, double* __restrict__ out) {
    const int m0 = blockIdx.x * 32;
    ms += m0 * nch;
    tl += m0;
    ids += m0;
    M = min(32, M - m0);
    __shared__ float tops[16];
    __shared__ double sums[16], logs[32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // (the first wave's lanes: a token each)
    const int id = threadIdx.x < M ? ids[threadIdx.x] : -1;
    const bool counted = id >= 0 && id < V;
    const float target = counted ? tl[threadIdx.x] : 0.f;
    const int each = M > 8 ? 1 : M > 4 ? 2 : M > 2 ? 4 : M > 1 ? 8 : 16, stride = 64 * each, first = (wave % each) * 64 + lane;
    for (int t0 = 0; t0 < M; t0 += 16 / each) {
        const int t = t0 + wave / each;
        float top = -INFINITY;
        double s = 0.0;
        if (t < M) {
            const float2* m = ms + t * nch;
            for (int64_t c0 = first; c0 < nch; c0 += stride * 8) {
                float2 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = m[min(c0 + stride * u, nch - 1)];
                float now = top;
#pragma unroll
                for (int u = 0; u < 8; ++u) now = fmaxf(now, v[u].x);              // (one that is there twice changes nothing)
                const float base = now == -INFINITY ? 0.f : now;
                s *= (double)__builtin_amdgcn_exp2f((top - base) * FEW_LOG2E);      // (0 to begin with)
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (c0 + stride * u < nch && v[u].y != 0.f) s += (double)(v[u].y * __builtin_amdgcn_exp2f((v[u].x - base) * FEW_LOG2E));
                top = now;
            }
            float all = top;
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) all = fmaxf(all, __shfl_xor(all, off));
            s = s == 0.0 ? 0.0 : s * (double)__builtin_amdgcn_exp2f((top - all) * FEW_LOG2E);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off);
            top = all;
        }
        if (lane == 0) { tops[wave] = top; sums[wave] = s; }
        __syncthreads();
        if (lane == 0 && wave % each == 0 && t < M) {
            float all = top;
            for (int w = 1; w < each; ++w) all = fmaxf(all, tops[wave + w]);
            double sum = 0.0;
            for (int w = 0; w < each; ++w) sum += sums[wave + w] == 0.0 ? 0.0 : sums[wave + w] * exp((double)tops[wave + w] - (double)all);
            logs[t] = log(sum) + (double)all;
        }
        __syncthreads();
    }
    if (wave != 0) return;
    const double l = lane < M ? logs[lane] : 0.0;
    if (lse && lane < M) lse[m0 + lane] = (float)l;
    double loss = counted ? l - (double)target : 0.0;
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(counted));
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) loss += __shfl_xor(loss, off);
    if (lane != 0) return;
    if (gridDim.x == 1) { *out = n > 0 ? loss / n : 0.0; return; }
    scratch[2 * blockIdx.x] = loss;
    scratch[2 * blockIdx.x + 1] = n;
}

// A tile of 32 rows of 128 values, for a wave or a workgroup, which is read transposed: a lane gets four rows' values of a column with each read
typedef __bf16 few_bf16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) few_bf16x4* few_trptr;
// 16 bytes c of row i lie at place c ^ few_swz(i): no two rows that a write or a read touches at once share banks
__device__ __forceinline__ int few_swz(int i) { return ((i & 3) << 2) | ((i >> 2) & 3); }
struct FewTrans {
    int at[2];
    __device__ __forceinline__ explicit FewTrans(int lane) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int n16 = lane & 15, tr = 8 * s + 4 * (lane >> 5) + (n16 >> 2), c = 2 * ((lane >> 4) & 1) + ((n16 & 3) >> 1);
            at[s] = tr * 256 + ((c ^ few_swz(tr)) << 4) + (n16 & 1) * 8;
        }
    }
    // columns 32 b .. 32 b + 31 as the instruction's rows; contracted rows 16 s + 4 hi .. + 3 and 16 s + 8 + 4 hi .. + 3
    __device__ __forceinline__ FewFrag read(const char* tile, int s, int b) const {
        union { few_bf16x4 v; uint2 u; } lo, up;
        lo.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((few_trptr)(tile + s * 4096 + (at[0] ^ (b << 6))));
        up.v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((few_trptr)(tile + s * 4096 + (at[1] ^ (b << 6))));
        FewFrag f;
        f.h[0] = lo.u;
        f.h[1] = up.u;
        return f;
    }
};
// the other operand, its columns' rows in that order
__device__ __forceinline__ FewFrag few_order(const bf16_t* row, int s) {
    FewFrag f;
    f.h[0] = *reinterpret_cast<const uint2*>(row + 16 * s);
    f.h[1] = *reinterpret_cast<const uint2*>(row + 16 * s + 8);
    return f;
}

// dX = D W for up to 255 tokens, or for rows too short for a tile's 256: a workgroup has 128 dims, 32 TB tokens and a share of the outputs, its waves 32 outputs in
// turn.  Rows of W go through LDS, a wave's own 8 KB, so that no wave waits for another and no transposed copy of W is made; D's values straight from memory.
// sums [shares][M][d], added to if this is not the first piece of the outputs.  7 tokens, 2048 <- 32000: 22 us (5.9 TB/s: W lies in the last cache by then);
// a transposed copy and a product of it 51 and 340.  200 tokens, four blocks that read W each: 102, and 51 and 347
struct FewDx { const bf16_t* D; int64_t ldd; const bf16_t* W; int64_t ldw; int64_t M, n, d; bool add; float* sums; int slices, shares; };
constexpr int FEW_LDS = 4 * 32 * 256 + 4 * 32 * 33 * 4;
template <int TB>
__device__ __forceinline__ void ce_few_dx(const FewDx& a, char* lds, int64_t block) {
    char (*stage)[32 * 256] = reinterpret_cast<char (*)[32 * 256]>(lds);
    float (*red)[32][33] = reinterpret_cast<float (*)[32][33]>(lds + 4 * 32 * 256);
    const bf16_t *const D = a.D, *const W = a.W;
    const int64_t ldd = a.ldd, ldw = a.ldw, M = a.M, n = a.n, d = a.d;
    // (a slice of dims, a share of the outputs, some tokens)
    const int64_t slice = block % a.slices, share = block / a.slices % a.shares;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, hi = lane >> 5;
    const int64_t d0 = slice * 128, m0 = block / a.slices / a.shares * (32 * TB);
    const int64_t blocks = (n + 31) / 32;
    char* own = stage[wave];
    const FewTrans trans(lane);
    uint4 data[8];
    auto load = [&](int64_t b) __attribute__((always_inline)) {
        const auto rs = few_rsrc(W + b * 32 * ldw + d0);
        const int left = (int)min((int64_t)32, n - b * 32);
        // (rows past the end repeat the last one: their D is 0)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int row = 4 * q + (lane >> 4), chunk = (lane & 15) ^ few_swz(row);
            data[q] = few_load(rs, d0 + 8 * chunk < d ? min(row, left - 1) * (int)(2 * ldw) + 16 * chunk : kPastEnd);
        }
    };
    const bf16_t* drow[TB];
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) drow[tb] = D + min(m0 + 32 * tb + r, M - 1) * ldd + 4 * hi;
    floatx16 acc[TB][4] = {};
    const int64_t first = share * 4 + wave, step = (int64_t)a.shares * 4;
    if (first < blocks) load(first);
    for (int64_t b = first; b < blocks; b += step) {
#pragma unroll
        for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(own + q * 1024 + lane * 16) = data[q];
        FewFrag x[TB][2];
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
#pragma unroll
            for (int s = 0; s < 2; ++s) x[tb][s] = few_order(drow[tb] + b * 32, s);
        if (b + step < blocks) load(b + step);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const FewFrag w = trans.read(own, s, db);
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) acc[tb][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w.v, x[tb][s].v, acc[tb][db], 0, 0, 0);
            }
    }
    // the waves' sums, 32 dims of 32 tokens at a time
#pragma unroll
    for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int db = 0; db < 4; ++db) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 16; ++e) red[wave][8 * (e >> 2) + 4 * hi + (e & 3)][r] = acc[tb][db][e];
            __syncthreads();
            const int dim = tid & 31;
            if (d0 + 32 * db + dim < d)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int c = (tid >> 5) + 8 * u;
                    const int64_t tok = m0 + 32 * tb + c;
                    if (tok >= M) continue;
                    float* to = a.sums + (share * M + tok) * d + d0 + 32 * db + dim;
                    const float s = (red[0][dim][c] + red[1][dim][c]) + (red[2][dim][c] + red[3][dim][c]);
                    *to = a.add ? *to + s : s;
                }
        }
}

// dW = *scale D^T X for up to 32 KB tokens, as many as D^T [n][32 KB] has columns: a workgroup has 128 dims, whose X lies in LDS (rows that are not counted as
// zeros: D is 0 there, and a value that is not finite would make NaNs of it) and in registers from there, and its waves take 32 outputs in turn.
// Bound by what it writes.  7 tokens, 2048 x 32000: 27 us (4.8 TB/s), a product of X transposed 72
struct FewDw { const bf16_t* Dt; const bf16_t* X; int64_t ldx; int M; int64_t n, d; const int32_t* ids; int64_t V; const float* scale; bf16_t* dW; int64_t lddw; int slices, groups; };
template <int KB>
__device__ __forceinline__ void ce_few_dw(const FewDw& a, char* lds, int64_t block) {
    char (*xs)[32 * 256] = reinterpret_cast<char (*)[32 * 256]>(lds);
    const bf16_t *const Dt = a.Dt, *const X = a.X;
    const int32_t* const ids = a.ids;
    bf16_t* const dW = a.dW;
    const int64_t ldx = a.ldx, n = a.n, d = a.d, V = a.V, lddw = a.lddw, group = block / a.slices;
    const int M = a.M;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, hi = lane >> 5;
    const int64_t d0 = block % a.slices * 128, blocks = (n + 31) / 32;
    const float f = *a.scale;
    for (int i = tid; i < 32 * KB * 16; i += 256) {
        const int row = i >> 4, c = i & 15, id = row < M ? ids[row] : -1;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (id >= 0 && id < V && d0 + 8 * c < d) v = *reinterpret_cast<const uint4*>(X + row * ldx + d0 + 8 * c);
        *reinterpret_cast<uint4*>(xs[row >> 5] + (row & 31) * 256 + ((c ^ few_swz(row & 31)) << 4)) = v;
    }
    __syncthreads();
    const FewTrans trans(lane);
    FewFrag x[2 * KB][4];
#pragma unroll
    for (int s = 0; s < 2 * KB; ++s)
#pragma unroll
        for (int db = 0; db < 4; ++db) x[s][db] = trans.read(xs[s >> 1], s & 1, db);
    for (int64_t b = group * 4 + wave; b < blocks; b += (int64_t)a.groups * 4) {
        const int64_t out = b * 32 + r;
        const bf16_t* row = Dt + min(out, n - 1) * (32 * KB) + 4 * hi;
        FewFrag t[2 * KB];
#pragma unroll
        for (int s = 0; s < 2 * KB; ++s) t[s] = few_order(row, s);
        bf16_t* to = dW + out * lddw + d0 + 8 * hi;
#pragma unroll
        for (int db = 0; db < 4; ++db) {
            floatx16 acc = {};
#pragma unroll
            for (int s = 0; s < 2 * KB; ++s) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[s][db].v, t[s].v, acc, 0, 0, 0);
            // dims 16 h + 8 hi .. + 7 after the halves have changed places
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t a0 = pack_bf16x2(acc[8 * h] * f, acc[8 * h + 1] * f), a1 = pack_bf16x2(acc[8 * h + 2] * f, acc[8 * h + 3] * f);
                const uint32_t b0 = pack_bf16x2(acc[8 * h + 4] * f, acc[8 * h + 5] * f), b1 = pack_bf16x2(acc[8 * h + 6] * f, acc[8 * h + 7] * f);
                const auto p = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), q = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
                if (out < n && d0 + 32 * db + 16 * h + 8 * hi < d) *reinterpret_cast<uint4*>(to + 32 * db + 16 * h) = make_uint4(p[0], q[0], p[1], q[1]);
            }
        }
    }
}

// Both beside each other, dX's workgroups first: what reads W out of the last cache leaves what writes dW the memory.  7 tokens, 2048 x 32000: 46 us for 22 and 27.  (With
// four blocks of tokens the registers leave one wave a SIMD: 100 tokens, 1024 -> 50000: a gradient of 182 us, two launches 162)
template <int TB, int KB>
__global__ __launch_bounds__(256) void ce_few_grad_kernel(const FewDx x, const FewDw w, int64_t x_blocks) {
    __shared__ __align__(1024) char lds[FEW_LDS];
    if (blockIdx.x < x_blocks) ce_few_dx<TB>(x, lds, blockIdx.x);
    else ce_few_dw<KB>(w, lds, blockIdx.x - x_blocks);
}
template <int TB>
__global__ __launch_bounds__(256) void ce_few_dx_kernel(const FewDx x) {
    __shared__ __align__(1024) char lds[FEW_LDS];
    ce_few_dx<TB>(x, lds, blockIdx.x);
}
template <int KB>
__global__ __launch_bounds__(256) void ce_few_dw_kernel(const FewDw w) {
    __shared__ __align__(1024) char lds[KB * 32 * 256];
    ce_few_dw<KB>(w, lds, blockIdx.x);
}

FewArgs few_args(const bf16_t* X, int64_t ldx, const bf16_t* W, int64_t ldw, int64_t M, int64_t V, int64_t d, const int32_t* ids) {
    FewArgs a{};
    a.X = X; a.ldx = ldx; a.W = W; a.ldw = ldw; a.M = (int)M; a.V = V; a.d = d; a.ids = ids; a.blocks = (int)((M + 31) / 32);
    return a;
}
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Up to 32 tokens, and more (in blocks of 32, W out of the XCD's L2 for all but the first) while that is at most seven workgroups to a compute unit: beyond, the tiles
// of the layers' forward, bound by how deep d is, are faster.  60 tokens, 1000 -> 10000: loss in 27 us, tiles 44; 146, 2488 -> 4588: 41 and 91; 120, 2000 -> 10000:
// 48 and 70; 240, 1000 -> 10000 (ten workgroups): 51 and 48; 40, 1024 -> 50000 (twelve): 73 and 51
bool ce_few_fits(int64_t M, int64_t V) { return M <= 32 || (M <= kCeFewTokens && (M + 31) / 32 * ((V + FEW_OUT - 1) / FEW_OUT) <= 7 * 256); }

size_t ce_few_workspace_bytes(int64_t M, int64_t V) { return up256((size_t)((V + FEW_OUT - 1) / FEW_OUT) * M * sizeof(float2)) + up256((size_t)M * 4) + up256(8 * 2 * 8); }

hipError_t launch_ce_few(const bf16_t* X, int64_t ldx, const bf16_t* W, int64_t ldw, int64_t M, int64_t V, int64_t d, const int32_t* ids, float* lse, double* out, void* workspace, hipStream_t st) {
    if (M < 1 || M > kCeFewTokens) return hipErrorInvalidValue;
    FewArgs a = few_args(X, ldx, W, ldw, M, V, d, ids);
    a.nch = (V + FEW_OUT - 1) / FEW_OUT;
    char* ws = static_cast<char*>(workspace);
    a.ms = reinterpret_cast<float2*>(ws);
    a.tl = reinterpret_cast<float*>(ws + up256((size_t)a.nch * M * sizeof(float2)));
    double* scratch = reinterpret_cast<double*>(reinterpret_cast<char*>(a.tl) + up256((size_t)M * 4));
    hipLaunchKernelGGL(ce_few_kernel<false>, dim3((unsigned)((a.nch + 7) / 8 * 8 * a.blocks)), dim3(256), 0, st, a);
    hipLaunchKernelGGL(ce_few_finish_kernel, dim3(a.blocks), dim3(1024), 0, st, a.ms, a.tl, ids, (int)M, V, a.nch, lse, scratch, out);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || a.blocks == 1 ? e : launch_ce_finish(scratch, a.blocks, out, st);
}

hipError_t launch_ce_few_d(const bf16_t* X, int64_t ldx, const bf16_t* W, int64_t ldw, int64_t M, int64_t V, int64_t d, const int32_t* ids, const float* lse, const double* g,
                           float* scale, bf16_t* D, int64_t ldd, bf16_t* Dt, int64_t ldt, hipStream_t st) {
    if (M < 1 || M > kCeFewTokens || ldd < (V + 31) / 32 * 32 || ldd % 4 || (Dt && (ldt % 32 || ldt < M))) return hipErrorInvalidValue;
    FewArgs a = few_args(X, ldx, W, ldw, M, V, d, ids);
    a.lse = lse; a.g = g; a.scale = scale; a.D = D; a.ldd = ldd; a.Dt = Dt; a.ldt = ldt;
    // (the columns of D^T behind the tokens too)
    if (Dt) a.blocks = (int)(ldt / 32);
    hipLaunchKernelGGL(ce_few_kernel<true>, dim3((unsigned)(((V + FEW_OUT - 1) / FEW_OUT + 7) / 8 * 8 * a.blocks)), dim3(256), 0, st, a);
    return hipGetLastError();
}

// for two workgroups to a compute unit, of four blocks of 32 outputs to a wave at least
int ce_few_dx_shares(int64_t M, int64_t n, int64_t d) {
    const int64_t tiles = (d + 127) / 128 * ((M + 63) / 64), blocks = (n + 31) / 32;
    return (int)std::max<int64_t>(1, std::min<int64_t>({512 / tiles, blocks / 16, 64}));
}

hipError_t launch_ce_few_grad(const CeFewGrad& a, hipStream_t st) {
    const int64_t M = a.M, n = a.n, d = a.d, slices = (d + 127) / 128;
    const bool dx = a.sums != nullptr, dw = a.dW != nullptr;
    if (M < 1 || (dx && (a.shares < 1 || a.ldd < (n + 31) / 32 * 32 || a.ldd % 4)) || (dw && (M > a.ldt || (a.ldt != 32 && a.ldt != 64 && a.ldt != 128)))) return hipErrorInvalidValue;
    const FewDx x{a.D, a.ldd, a.W, a.ldw, M, n, d, a.add, a.sums, (int)slices, a.shares};
    // dW: eight workgroups to a compute unit, no more: each has to read X first
    const FewDw w{a.Dt, a.X, a.ldx, (int)M, n, d, a.ids, a.V, a.scale, a.dW, a.lddw, (int)slices, (int)std::max<int64_t>(1, std::min((n + 127) / 128, 2048 / slices))};
    const bool one = M <= 32;
    const int64_t xb = dx ? slices * a.shares * ((M + (one ? 31 : 63)) / (one ? 32 : 64)) : 0, wb = dw ? slices * w.groups : 0;
    if (xb + wb == 0) return hipSuccess;
    if (xb + wb > 0x7FFFFFFFLL) return hipErrorInvalidValue;
    const dim3 wg(256);
    if (dx && dw && a.ldt != 128) {
        if (one) hipLaunchKernelGGL((ce_few_grad_kernel<1, 1>), dim3((unsigned)(xb + wb)), wg, 0, st, x, w, xb);
        else hipLaunchKernelGGL((ce_few_grad_kernel<2, 2>), dim3((unsigned)(xb + wb)), wg, 0, st, x, w, xb);
        return hipGetLastError();
    }
    if (dx) {
        if (one) hipLaunchKernelGGL(ce_few_dx_kernel<1>, dim3((unsigned)xb), wg, 0, st, x);
        else hipLaunchKernelGGL(ce_few_dx_kernel<2>, dim3((unsigned)xb), wg, 0, st, x);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || !dw) return e;
    }
    if (a.ldt == 32) hipLaunchKernelGGL(ce_few_dw_kernel<1>, dim3((unsigned)wb), wg, 0, st, w);
    else if (a.ldt == 64) hipLaunchKernelGGL(ce_few_dw_kernel<2>, dim3((unsigned)wb), wg, 0, st, w);
    else hipLaunchKernelGGL(ce_few_dw_kernel<4>, dim3((unsigned)wb), wg, 0, st, w);
    return hipGetLastError();
}

}  // namespace agzo
