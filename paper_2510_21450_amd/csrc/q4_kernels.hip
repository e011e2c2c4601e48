// The input projection with 4-bit weights, and one token of a gated layer.
//
//   u[r][g][c] = sum_j q[g][c][j] s[g][c][j / group] x[r][head(c) dh + j] + bias[g][c],   q = -8 .. 7
//
// Few rows: the time is that of reading the weights, so they go from memory straight into the matrix cores' operand
// registers.  A unit is 16 output channels x 64 inputs (512 bytes, 8 a lane); rows of x are the other operand, 16 at a time.
// A code becomes a bf16 number by one masked OR: the bits of q + 8 are put into the mantissa of 16, which gives
// 24 + q, exactly.  The 24 is taken out by a product of the same x with -24, which the products of all gates start from:
//   sum (24 + q) x - sum 24 x, each term exact in fp32, one more matrix instruction for each group of inputs.
// Groups are scaled in fp32 as their sums are added up.  fp32 inputs are split into three bf16 terms (24 bits), and codes are
// operands without the 24, whose sums would lose three of those bits.
#include <algorithm>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pararnn.h"
#include "pararnn/common.h"
#include "pararnn/launch.h"
#include "proj.h"
#include "q4.h"

namespace pararnn {
namespace {

typedef float f4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef unsigned int u2v __attribute__((ext_vector_type(2)));
typedef unsigned int u4v __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ layout
// Unit (row tile rt of 16 outputs, k unit ku of 64 inputs) at ((rt nu + ku) 64 + lane) 8 bytes; lane = 16 kq + n holds output n,
// word s the inputs 64 ku + 32 s + 8 kq + 0 .. 7: inputs 2p and 2p + 1 in bits 4p and 16 + 4p, as q + 8.
__device__ __forceinline__ unsigned int pack8(const int (&q)[8])
{
    unsigned int w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (unsigned int)(q[e] + 8) << (4 * (e >> 1) + 16 * (e & 1));
    return w;
}
__device__ __forceinline__ int code_at(unsigned int w, int e) { return (int)(w >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8; }

// the eight numbers 24 + q of a word, as the matrix cores take them
__device__ __forceinline__ bf8v operand(unsigned int w)
{
    constexpr unsigned int mask = 0x00780078u, one = 0x41804180u;        // the mantissa bits above 1/8, and 16.0 twice
    const u4v r = {((w << 3) & mask) | one, ((w >> 1) & mask) | one, ((w >> 5) & mask) | one, ((w >> 9) & mask) | one};
    return __builtin_bit_cast(bf8v, r);
}

// the same less 24, exact too: for fp32, where the 24 and its product would cost the sums three bits
__device__ __forceinline__ bf8v operand_signed(unsigned int w)
{
    const u4v r = __builtin_bit_cast(u4v, operand(w));
    u4v q;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const unsigned int lo = __float_as_uint(__uint_as_float(r[p] << 16) - 24.0f);
        const unsigned int hi = __float_as_uint(__uint_as_float(r[p] & 0xffff0000u) - 24.0f);
        q[p] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);       // the upper halves of both
    }
    return __builtin_bit_cast(bf8v, q);
}

struct PrepArgs {
    const float *W;
    const signed char *codes;
    const unsigned short *code_scales;
    const u2v *packed;
    const unsigned short *scales;
    u2v *packed_out;
    unsigned short *scales_out;
    float *W_out;
    unsigned short *Wb_out;
    int *tickets;
    int nu, group, dh;
    long long units;              // of `per` k units each
};

// A wave takes PER k units of 16 outputs: one, or the two that share a scale.  Memory-bound: 4.5 bytes a weight.
template <int PER> __global__ __launch_bounds__(256) void q4_quantize_kernel(const PrepArgs a)
{
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= a.units) return;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
    const int per_row = a.nu / PER;
    const long long rt = id / per_row;
    const int ku = (int)(id - rt * per_row) * PER;
    const float *src = a.W + (rt * 16 + n) * a.dh + ku * 64 + 8 * kq;
    float v[PER * 2][8], big[PER * 2];
#pragma unroll
    for (int s = 0; s < PER * 2; ++s) {
        // 4-byte alignment is all the caller owes
        __builtin_memcpy(v[s], src + 32 * s, 32);
        float m = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = nanmax(m, fabsf(v[s][e]));
        m = nanmax(m, __shfl_xor(m, 16, 64));
        big[s] = nanmax(m, __shfl_xor(m, 32, 64));
    }
    const int steps = a.group / 32, ng = a.dh / a.group;
#pragma unroll
    for (int s = 0; s < PER * 2; ++s) {
        float m = big[s];
        for (int q = 1; q < steps; q *= 2) {
#pragma unroll
            for (int o = 0; o < PER * 2; ++o)
                if (o / steps == s / steps) m = nanmax(m, big[o]);
        }
        const unsigned short sc = m < __builtin_inff() ? f32_to_bf16(m / 7.0f) : (unsigned short)0x7fc0u;
        const float scale = bf16_to_f32(sc);
        int q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // the quotient of an fp32 and a bf16 number is rounded to the middle between two codes only where it is that exactly
            const float r = scale > 0.0f ? rintf(v[s][e] / scale) : 0.0f;
            q[e] = (int)fminf(fmaxf(r, -7.0f), 7.0f);
        }
        const unsigned int w = pack8(q);
        reinterpret_cast<unsigned int *>(a.packed_out + (rt * a.nu + ku + s / 2) * 64 + lane)[s & 1] = w;
        if (s % steps == 0 && kq == 0) a.scales_out[(rt * ng + (ku * 2 + s) / steps) * 16 + n] = sc;
    }
}

__global__ __launch_bounds__(256) void q4_pack_kernel(const PrepArgs a)
{
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= a.units) return;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
    const long long rt = id / a.nu;
    const int ku = (int)(id - rt * a.nu);
    const signed char *src = a.codes + (rt * 16 + n) * a.dh + ku * 64 + 8 * kq;
    unsigned int w[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        signed char c[8];
        __builtin_memcpy(c, src + 32 * s, 8);
        int q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = c[e] < -8 ? -8 : c[e] > 7 ? 7 : c[e];
        w[s] = pack8(q);
    }
    a.packed_out[id * 64 + lane] = u2v{w[0], w[1]};
    const int ng = a.dh / a.group;
    if (kq == 0)
        for (int k = ku * 64; k < ku * 64 + 64; k += 32)
            if (k % a.group == 0) a.scales_out[(rt * ng + k / a.group) * 16 + n] = a.code_scales[(rt * 16 + n) * ng + k / a.group];
}

// Wx fp32, or rounded to bf16 for the matrix products of many rows
template <bool BF16> __global__ __launch_bounds__(256) void q4_dequantize_kernel(const PrepArgs a)
{
    if (BF16 && blockIdx.x == 0 && threadIdx.x < 8) a.tickets[threadIdx.x] = 0;      // for the product that follows
    const long long id = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (id >= a.units) return;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
    const long long rt = id / a.nu;
    const int ku = (int)(id - rt * a.nu), ng = a.dh / a.group;
    const u2v w = a.packed[id * 64 + lane];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int k = ku * 64 + 32 * s;
        const float scale = bf16_to_f32(a.scales[(rt * ng + k / a.group) * 16 + n]);
        const long long at = (rt * 16 + n) * a.dh + k + 8 * kq;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = scale * (float)code_at(w[s], e);
        if constexpr (BF16) {
            u4v r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = f32_to_bf16(v[2 * e]) | (unsigned int)f32_to_bf16(v[2 * e + 1]) << 16;
            *reinterpret_cast<u4v *>(a.Wb_out + at) = r;
        } else {
            __builtin_memcpy(a.W_out + at, v, 32);
        }
    }
}

// ------------------------------------------------------------------ products of few rows
struct RowsQ4Args {
    const void *x;
    const u2v *packed;
    const unsigned short *scales;
    const float *bias, *h;
    void *out;                    // u, or y of a step
    float *h_next;
    int rows, H, G, dh, nu, group;
};

// Eight inputs of a row as they lie in memory, and as operands
template <typename T> struct Eight;
template <> struct Eight<unsigned short> {
    static constexpr int TERMS = 1;
    u4v v;
    __device__ __forceinline__ void load(const unsigned short *p) { v = *reinterpret_cast<const u4v *>(p); }
    __device__ __forceinline__ void zero() { v = u4v{0, 0, 0, 0}; }
    __device__ __forceinline__ void terms(bf8v (&t)[1]) const { t[0] = __builtin_bit_cast(bf8v, v); }
};
template <> struct Eight<float> {
    static constexpr int TERMS = 3;
    f4v lo, hi;
    __device__ __forceinline__ void load(const float *p)
    {
        lo = *reinterpret_cast<const f4v *>(p);
        hi = *reinterpret_cast<const f4v *>(p + 4);
    }
    __device__ __forceinline__ void zero() { lo = hi = f4v{0, 0, 0, 0}; }
    // x = t0 + t1 + t2: what a term leaves is exact in fp32, and eight bits of mantissa three times are all 24
    __device__ __forceinline__ void terms(bf8v (&t)[3]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = e < 4 ? lo[e & 3] : hi[e & 3];
            t[0][e] = (__bf16)x;
            const float r = x - (float)t[0][e];
            t[1][e] = (__bf16)r;
            t[2][e] = (__bf16)(r - (float)t[1][e]);
        }
    }
};

// A workgroup: 16 channels (STEP: of all NG gates; else of one gate's rows of the weights) x 16 MT rows; its waves share the inputs of
// a head among them and add up in LDS.  G32: groups of 32 inputs, else of 64 and more.
template <typename T, int MT, int NG, bool STEP, bool G32>
__global__ __launch_bounds__(512) void q4_rows_kernel(const RowsQ4Args a)
{
    constexpr int U = MT * NG * (sizeof(T) / 2) <= 3 ? 4 : 2;      // units in flight
    constexpr int TERMS = Eight<T>::TERMS;
    extern __shared__ float s_red[];
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4, w = threadIdx.x >> 6, W = blockDim.x >> 6;
    const int tiles = a.H / 16;                              // row tiles of a gate
    const int g0 = STEP ? 0 : (int)blockIdx.x / tiles, ct = (int)blockIdx.x - g0 * tiles;
    const int m0 = (int)blockIdx.y * 16 * MT;
    const int head = ct * 16 / a.dh, ng = a.dh / a.group;
    const T *x = static_cast<const T *>(a.x) + (size_t)head * a.dh + 8 * kq;

    const u4v minus24 = {0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u};
    const bf8v offset = __builtin_bit_cast(bf8v, minus24);
    f4v total[NG][MT];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m) total[g][m] = f4v{0, 0, 0, 0};

    for (int base = w; base < a.nu; base += W * U) {
        u2v q[U][NG];
        float sc[U][NG][2];
        Eight<T> xr[U][MT][2];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int unit = base + i * W;
            const bool live = unit < a.nu;
            const int ku = live ? unit : base;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const size_t rt = (size_t)(g0 + g) * tiles + ct;
                q[i][g] = a.packed[(rt * a.nu + ku) * 64 + lane];
                const unsigned short *s = a.scales + (rt * ng) * 16 + n;
                if constexpr (G32) {
                    sc[i][g][0] = bf16_to_f32(s[(2 * ku) * 16]);
                    sc[i][g][1] = bf16_to_f32(s[(2 * ku + 1) * 16]);
                } else {
                    sc[i][g][0] = bf16_to_f32(s[(ku * 64 / a.group) * 16]);
                }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int row = m0 + 16 * m + n;
                const bool ok = live && row < a.rows;
                const T *p = x + (size_t)(row < a.rows ? row : a.rows - 1) * a.H + ku * 64;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    xr[i][m][s].load(p + 32 * s);
                    if (!ok) xr[i][m][s].zero();
                }
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                bf8v t[2][TERMS];
                xr[i][m][0].terms(t[0]);
                xr[i][m][1].terms(t[1]);
                f4v start[2] = {f4v{0, 0, 0, 0}, f4v{0, 0, 0, 0}};
                if constexpr (TERMS == 1)
#pragma unroll
                    for (int s = 0; s < 2; ++s)
                        start[G32 ? s : 0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[s][0], offset, start[G32 ? s : 0], 0, 0, 0);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    f4v acc = start[0];
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const bf8v b = TERMS == 1 ? operand(q[i][g][s]) : operand_signed(q[i][g][s]);
                        if (G32 && s == 1) {
                            total[g][m] += sc[i][g][0] * acc;
                            acc = start[1];
                        }
#pragma unroll
                        for (int e = TERMS - 1; e >= 0; --e) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[s][e], b, acc, 0, 0, 0);
                    }
                    // a lane's four sums are rows 4 kq .. 4 kq + 3 of channel n
                    total[g][m] += sc[i][g][G32 ? 1 : 0] * acc;
                }
            }
    }
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) s_red[((w * NG + g) * MT + m) * 256 + j * 64 + lane] = total[g][m][j];
    __syncthreads();
    for (int id = threadIdx.x; id < MT * 256; id += blockDim.x) {
        const int m = id >> 8, j = id >> 6 & 3, l = id & 63;
        const int row = m0 + 16 * m + 4 * (l >> 4) + j, ch = ct * 16 + (l & 15);
        if (row >= a.rows) continue;
        float u[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            u[g] = a.bias ? a.bias[(size_t)(g0 + g) * a.H + ch] : 0.0f;
            for (int p = 0; p < W; ++p) u[g] += s_red[((p * NG + g) * MT) * 256 + id];
        }
        if constexpr (STEP) {
            const size_t at = (size_t)row * a.H + ch;
            const float f = fast_sigmoid(u[0]), i = fast_sigmoid(NG == 2 ? -u[0] : u[NG - 2]);
            const float next = fmaf(f, a.h ? a.h[at] : 0.0f, i * u[NG - 1]);
            a.h_next[at] = next;
            if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = next;
            else static_cast<unsigned short *>(a.out)[at] = f32_to_bf16(next);
        } else {
            const size_t at = ((size_t)row * a.G + g0) * a.H + ch;
            if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = u[0];
            else static_cast<unsigned short *>(a.out)[at] = f32_to_bf16(u[0]);
        }
    }
}

// ------------------------------------------------------------------ host
constexpr int kExactRows = 64;

bool weights_ok(int H, int G, int n_heads) { return H >= 1 && G >= 1 && G <= 8 && n_heads >= 1 && H % n_heads == 0; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
// what the kernels have no form for
bool unsupported(int H, int n_heads, int group)
{
    const int dh = H / n_heads;
    return H > (1 << 20) || dh % 64 || dh % group;
}
bool misaligned(const void *p, size_t n) { return (uintptr_t)p % n != 0; }

PrepArgs prep_args(int H, int G, int n_heads, int group, int per)
{
    PrepArgs a = {};
    a.dh = H / n_heads;
    a.nu = a.dh / 64;
    a.group = group;
    a.units = (long long)G * H / 16 * (a.nu / per);
    return a;
}
unsigned prep_blocks(const PrepArgs &a) { return (unsigned)((a.units + 3) / 4); }

template <typename T, int MT, int NG, bool STEP, bool G32> hipError_t launch_rows(const RowsQ4Args &a, hipStream_t st)
{
    int W = a.nu < 8 ? a.nu : 8;
    const int most = 48 / (NG * MT);                          // sums of a wave: NG MT KB of LDS
    if (W > most) W = most;
    const unsigned tiles = (unsigned)(a.H / 16) * (STEP ? 1 : a.G), mb = (unsigned)((a.rows + 16 * MT - 1) / (16 * MT));
    hipLaunchKernelGGL((q4_rows_kernel<T, MT, NG, STEP, G32>), dim3(tiles, mb), dim3(64 * W), (size_t)W * NG * MT * 1024, st, a);
    return hipGetLastError();
}
template <typename T, int NG, bool STEP> hipError_t launch_rows_of(const RowsQ4Args &a, hipStream_t st)
{
#define PARARNN_Q4(MT) (a.group == 32 ? launch_rows<T, MT, NG, STEP, true>(a, st) : launch_rows<T, MT, NG, STEP, false>(a, st))
    if (a.rows <= 16) return PARARNN_Q4(1);
    if (a.rows <= 32) return PARARNN_Q4(2);
    return PARARNN_Q4(4);
#undef PARARNN_Q4
}

}  // namespace

size_t q4_packed_bytes(int H, int G, int n_heads)
{
    if (!weights_ok(H, G, n_heads) || unsupported(H, n_heads, 32)) return 0;
    return (size_t)G * H * (H / n_heads) / 2;
}

size_t q4_scale_bytes(int H, int G, int n_heads, int group)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || unsupported(H, n_heads, group)) return 0;
    return (size_t)G * H * (H / n_heads / group) * 2;
}

int q4_quantize(const float *Wx, int H, int G, int n_heads, int group, void *packed, void *scales, hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !Wx || !packed || !scales || misaligned(Wx, 4) || misaligned(packed, 16) ||
        misaligned(scales, 2))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, group == 128 ? 2 : 1);
    a.W = Wx; a.packed_out = static_cast<u2v *>(packed); a.scales_out = static_cast<unsigned short *>(scales);
    if (group == 128) hipLaunchKernelGGL(q4_quantize_kernel<2>, dim3(prep_blocks(a)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(q4_quantize_kernel<1>, dim3(prep_blocks(a)), dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_pack(const signed char *codes, const void *code_scales, int H, int G, int n_heads, int group, void *packed, void *scales,
            hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !codes || !code_scales || !packed || !scales || misaligned(code_scales, 2) ||
        misaligned(packed, 16) || misaligned(scales, 2))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, 1);
    a.codes = codes; a.code_scales = static_cast<const unsigned short *>(code_scales);
    a.packed_out = static_cast<u2v *>(packed); a.scales_out = static_cast<unsigned short *>(scales);
    hipLaunchKernelGGL(q4_pack_kernel, dim3(prep_blocks(a)), dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_dequantize(const void *packed, const void *scales, int H, int G, int n_heads, int group, float *Wx, hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !packed || !scales || !Wx || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(Wx, 4))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, 1);
    a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.W_out = Wx;
    hipLaunchKernelGGL(q4_dequantize_kernel<false>, dim3(prep_blocks(a)), dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_exact_rows(int H, int G, int n_heads)
{
    return weights_ok(H, G, n_heads) && !unsupported(H, n_heads, 32) ? kExactRows : -1;
}

size_t q4_workspace_bytes(int dtype, int B, int L, int H, int G, int n_heads, int group)
{
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || L < 1 || (double)B * L > 1e9 || q4_scale_bytes(H, G, n_heads, group) == 0) return 0;
    if (dtype == PARARNN_F32 || (long long)B * L <= kExactRows) return 256;
    return proj_workspace_bytes(dtype, B, L, H, G, n_heads, 0);
}

int q4_project(int dtype, const void *x, const void *packed, const void *scales, const float *bias, int B, int L, int H, int G,
               int n_heads, int group, void *u, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || L < 1 || !weights_ok(H, G, n_heads) || !group_ok(group) || !x ||
        !packed || !scales || !u || !workspace || misaligned(x, 16) || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(bias, 4) || misaligned(u, es) || misaligned(workspace, 256))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, n_heads, group)) return PARARNN_UNSUPPORTED;
    const size_t need = q4_workspace_bytes(dtype, B, L, H, G, n_heads, group);
    if (need == 0) return PARARNN_INVALID_ARG;
    if (workspace_bytes < need) return PARARNN_WORKSPACE_TOO_SMALL;
    const int rows = B * L;
    if (dtype == PARARNN_BF16 && rows > kExactRows) {
        if (misaligned(u, 16)) return PARARNN_UNSUPPORTED;
        int *tickets = nullptr;
        unsigned short *Wb = proj_weights_at(workspace, &tickets);
        PrepArgs p = prep_args(H, G, n_heads, group, 1);
        p.packed = static_cast<const u2v *>(packed); p.scales = static_cast<const unsigned short *>(scales);
        p.Wb_out = Wb; p.tickets = tickets;
        hipLaunchKernelGGL(q4_dequantize_kernel<true>, dim3(prep_blocks(p)), dim3(256), 0, st, p);
        if (hipGetLastError() != hipSuccess) return PARARNN_HIP_ERROR;
        return proj_product(dtype, x, Wb, bias, B, L, H, G, n_heads, u, tickets, st);
    }
    RowsQ4Args a = {};
    a.x = x; a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.bias = bias; a.out = u;
    a.rows = rows; a.H = H; a.G = G; a.dh = H / n_heads; a.nu = a.dh / 64; a.group = group;
    const hipError_t e = dtype == PARARNN_BF16 ? launch_rows_of<unsigned short, 1, false>(a, st) : launch_rows_of<float, 1, false>(a, st);
    return e == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_step(int dtype, const void *x, const void *packed, const void *scales, const float *bias, const float *h, int B, int H, int G,
            int n_heads, int group, void *y, float *h_next, hipStream_t st)
{
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || (G != 2 && G != 3) || !weights_ok(H, G, n_heads) || !group_ok(group) ||
        !x || !packed || !scales || !y || !h_next || misaligned(x, 16) || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(bias, 4) || misaligned(h, 4) || misaligned(h_next, 4) || misaligned(y, es))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, n_heads, group) || B > (1 << 20)) return PARARNN_UNSUPPORTED;
    RowsQ4Args a = {};
    a.x = x; a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.bias = bias; a.h = h;
    a.out = y; a.h_next = h_next;
    a.rows = B; a.H = H; a.G = G; a.dh = H / n_heads; a.nu = a.dh / 64; a.group = group;
    const hipError_t e = dtype == PARARNN_BF16
                             ? (G == 2 ? launch_rows_of<unsigned short, 2, true>(a, st) : launch_rows_of<unsigned short, 3, true>(a, st))
                             : (G == 2 ? launch_rows_of<float, 2, true>(a, st) : launch_rows_of<float, 3, true>(a, st));
    return e == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

}  // namespace pararnn
