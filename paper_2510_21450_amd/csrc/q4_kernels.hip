// The input projection with 4-bit weights, and one token of a gated layer.
//
//   u[r][g][c] = sum_j q[g][c][j] s[g][c][j / group] x[r][head(c) dh + j] + bias[g][c],   q = -8 .. 7
//
// Few rows: the time is that of reading the weights, so they go from memory straight into the matrix cores' operand
// registers.  A unit is 16 output channels x 64 inputs (512 bytes, 8 a lane); rows of x are the other operand, 16 at a time.
// A code becomes a bf16 number by one masked OR: the bits of q + 8 are put into the mantissa of 16, which gives
// 24 + q, exactly.  The 24 is taken out by a product of the same x with -24, which the products of all gates start from:
//   sum (24 + q) x - sum 24 x, each term exact in fp32, one more matrix instruction for each group of inputs.
// (What a sum carries is up to eight times larger for it, and its roundings with it.)  Groups are scaled in fp32 as their sums are added up.  fp32 inputs are split into three bf16 terms (24 bits), and codes are
// operands without the 24, whose sums would lose three of those bits.
#include <algorithm>
#include <atomic>
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

// 16.0 twice, in a vector register: an instruction takes one scalar, and the mask is one
__device__ __forceinline__ unsigned int sixteens()
{
    unsigned int x = 0x41804180u;
    asm("" : "+v"(x));
    return x;
}
// the eight numbers 24 + q of a word, as the matrix cores take them
__device__ __forceinline__ bf8v operand(unsigned int w, unsigned int one)
{
    constexpr unsigned int mask = 0x00780078u;                           // the mantissa bits above 1/8
    const u4v r = {((w << 3) & mask) | one, ((w >> 1) & mask) | one, ((w >> 5) & mask) | one, ((w >> 9) & mask) | one};
    return __builtin_bit_cast(bf8v, r);
}

// q / 16 by table, exact: for fp32, where the 24 and its product would cost the sums three bits
__device__ __forceinline__ bf8v operand_signed(unsigned int w)
{
    const unsigned int even = w ^ 0x88888888u, odd = even >> 4;      // two's complement
    u4v r;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        float lo, hi;
        const unsigned int from = p & 1 ? odd : even;
        if (p < 2) {
            asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD src0_sel:BYTE_0" : "=v"(lo) : "v"(from));
            asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD src0_sel:BYTE_2" : "=v"(hi) : "v"(from));
        } else {
            asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD src0_sel:BYTE_1" : "=v"(lo) : "v"(from));
            asm("v_cvt_off_f32_i4_sdwa %0, %1 dst_sel:DWORD src0_sel:BYTE_3" : "=v"(hi) : "v"(from));
        }
        r[p] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);      // the upper halves of both
    }
    return __builtin_bit_cast(bf8v, r);
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
    int per_row;                  // k units of a row tile, PER taken as one
    unsigned int blocks;          // workgroups that share a row tile, four units each
};

// Row tile and k unit of a wave.  Neighbouring workgroups take neighbouring units of the same rows (the other order: 55 -> 68 us for 2 x 4096
// x 4096 weights to 4 bits and back).
__device__ __forceinline__ bool unit_of(const PrepArgs &a, long long *rt, int *ku)
{
    const unsigned int r = blockIdx.x / a.blocks;
    *rt = r;
    *ku = (int)((blockIdx.x - r * a.blocks) * 4 + (threadIdx.x >> 6));
    return *ku < a.per_row;
}

// A wave takes PER k units of 16 outputs: one, or the two that share a scale.  Memory-bound, 4.53 bytes a weight: 30 us for 2 x 4096 x 4096
// weights, 5.1 TB/s (vector issue 0.9 of the time, most of it the quotients, which are exact so that halves go to the even code).
template <int PER> __global__ __launch_bounds__(256) void q4_quantize_kernel(const PrepArgs a)
{
    long long rt;
    int ku;
    if (!unit_of(a, &rt, &ku)) return;
    ku *= PER;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
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
    long long rt;
    int ku;
    if (!unit_of(a, &rt, &ku)) return;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4;
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
    a.packed_out[(rt * a.nu + ku) * 64 + lane] = u2v{w[0], w[1]};
    const int ng = a.dh / a.group;
    if (kq == 0)
        for (int k = ku * 64; k < ku * 64 + 64; k += 32)
            if (k % a.group == 0) a.scales_out[(rt * ng + k / a.group) * 16 + n] = a.code_scales[(rt * 16 + n) * ng + k / a.group];
}

// Wx fp32, or rounded to bf16 for the matrix products of many rows where the caller asks for those.  Memory-bound: 25 us for 2 x 4096 x 4096 weights to fp32, 6.0 TB/s.
template <bool BF16> __global__ __launch_bounds__(256) void q4_dequantize_kernel(const PrepArgs a)
{
    if (BF16 && blockIdx.x == 0 && threadIdx.x < 8) a.tickets[threadIdx.x] = 0;      // for the product that follows
    long long rt;
    int ku;
    if (!unit_of(a, &rt, &ku)) return;
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4, ng = a.dh / a.group;
    const u2v w = a.packed[(rt * a.nu + ku) * 64 + lane];
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
    int rows, H, G, dh;
    int nu, ng, tiles;            // units and groups of a head's inputs; 16-channel tiles of a gate
    int unit_shift;               // a unit's group is unit >> this (groups of 64 and 128)
};

// Waves whose sums of `tiles` KB each are in LDS at once: 64 KB
constexpr __host__ __device__ int sums_in_lds(int tiles) { return 64 / tiles < 8 ? 64 / tiles : 8; }

// Eight inputs of a row as they lie in memory, and as operands
template <typename T> struct Eight;
template <> struct Eight<unsigned short> {
    static constexpr int TERMS = 1;
    static constexpr int CHUNKS = 1;       // of 16 bytes
    u4v c[1];
    __device__ __forceinline__ void load(const unsigned short *p) { c[0] = *reinterpret_cast<const u4v *>(p); }
    __device__ __forceinline__ void terms(bf8v (&t)[1]) const { t[0] = __builtin_bit_cast(bf8v, c[0]); }
};
template <> struct Eight<float> {
    static constexpr int TERMS = 3;
    static constexpr int CHUNKS = 2;
    u4v c[2];
    __device__ __forceinline__ void load(const float *p)
    {
        c[0] = *reinterpret_cast<const u4v *>(p);
        c[1] = *reinterpret_cast<const u4v *>(p + 4);
    }
    // x = t0 + t1 + t2, cut off and not rounded: eight bits of mantissa three times are all 24, and what a term leaves is exact.  (An infinity
    // leaves a NaN.)
    __device__ __forceinline__ void terms(bf8v (&t)[3]) const
    {
        u4v r[3];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            float x[2] = {__uint_as_float(c[p >> 1][2 * p & 3]), __uint_as_float(c[p >> 1][(2 * p & 3) + 1])};
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                r[k][p] = __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u);
#pragma unroll
                for (int e = 0; e < 2; ++e) x[e] -= __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
            }
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) t[k] = __builtin_bit_cast(bf8v, r[k]);
    }
};

// A workgroup: 16 CT channels (STEP: of all NG gates; else of one gate) x 16 MT rows; its waves share the inputs of a head among
// them and add up in LDS.  A row's inputs are read once for the NG CT tiles of weights and a weight once for the 16 MT rows.
// Few rows are bound by the way to memory and back, so a wave asks for its units at once (its whole share of up to 4096 inputs for
// one row), and for what it adds to the sums before the first of them comes.  G32: groups of 32 inputs, else of 64 and more.
// One row in a graph, weights read from memory: 3 x 4096 x 4096 (27 MB) 11 us, 2.4 TB/s; a step with 2 x 4096 x 4096 7.7, 2.3 TB/s; with the
// weights in the memory-side cache 7.9 and 5.6.  Launch, loads and sums of a small one 3.0 to 4.3.
template <typename T, int MT, int NG, int CT, bool STEP, bool G32>
__global__ __launch_bounds__(512, MT * NG * CT == 1 ? 4 : 2) void q4_rows_kernel(const RowsQ4Args a)
{
    constexpr int NT = NG * CT;
    constexpr int TERMS = Eight<T>::TERMS;
    extern __shared__ __align__(16) float s_red[];
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int W = blockDim.x >> 6;
    const unsigned int per_gate = a.tiles / CT, all = STEP ? per_gate : per_gate * a.G;
    const unsigned int mb = blockIdx.x / all, tile = blockIdx.x - mb * all;
    const int g0 = STEP ? 0 : (int)(tile / per_gate), ct = (int)(tile - g0 * per_gate) * CT;
    const int m0 = (int)mb * 16 * MT;
    const int head = ct * 16 / a.dh;                         // (a multiple of 64 channels: the CT tiles are of one head)
    // bases that all lanes share and scalar registers hold, and 32-bit offsets from them: no address arithmetic for a load.  Rows behind the last are read as the block's first: a row of x
    // reaches that row's sums alone, and those are not written.
    const T *x = static_cast<const T *>(a.x) + (size_t)m0 * a.H + (size_t)head * a.dh;
    auto weights = [&](int g) { return a.packed + ((size_t)(g0 + g / CT) * a.tiles + ct + g % CT) * a.nu * 64; };
    auto scales = [&](int g) { return a.scales + ((size_t)(g0 + g / CT) * a.tiles + ct + g % CT) * a.ng * 16; };
    auto row_at = [&](int r) { return (unsigned int)(m0 + r < a.rows ? r : 0) * a.H; };

    const u4v minus24 = {0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u};
    const bf8v offset = __builtin_bit_cast(bf8v, minus24);
    const unsigned int one = sixteens();
    f4v total[NT][MT];
#pragma unroll
    for (int g = 0; g < NT; ++g)
#pragma unroll
        for (int m = 0; m < MT; ++m) total[g][m] = f4v{0, 0, 0, 0};

    // A lane's four sums of a tile, rows 4 kq .. 4 kq + 3 of channel n, lie together.  A thread finishes PER of them at a time: all four
    // where there are tiles for every thread, else one (a step of 48 rows: 3.9 us to 4.4).
    constexpr int PER = CT * MT >= 4 ? 4 : 1;
    auto place = [&](int id, int *c, int *m, int *j) {       // tile of channels, of rows, first of the sums; returns the channel
        *j = PER == 4 ? 0 : id / 64 % 4;
        const int quad = id / (64 * (4 / PER));
        *c = quad / MT;
        *m = quad % MT;
        return (ct + *c) * 16 + n;
    };
    constexpr int PLACES = CT * MT * 64 * (4 / PER);
    float bias[NT], first_h[PER];
#pragma unroll
    for (int g = 0; g < NT; ++g) bias[g] = a.bias ? a.bias[(size_t)(g0 + g / CT) * a.H + (ct + g % CT) * 16 + n] : 0.0f;
    if constexpr (STEP) {
        int c, m, j;
        const int ch = place(threadIdx.x, &c, &m, &j), row = m0 + 16 * m + 4 * kq + j;
#pragma unroll
        for (int e = 0; e < PER; ++e) first_h[e] = a.h && (int)threadIdx.x < PLACES && row + e < a.rows ? a.h[(size_t)(row + e) * a.H + ch] : 0.0f;
    }

    // one unit's products; x(m, s): the eight inputs of 16 rows m at step s that this lane multiplies
    auto multiply = [&](const u2v (&q)[NT], const unsigned int (&sc)[NT][2], auto &&x_at) {
        // parts of a unit: its groups; three terms of both steps at once would not fit the registers
        constexpr int PARTS = G32 || TERMS == 3 ? 2 : 1, STEPS = 2 / PARTS;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            bf8v t[MT][STEPS][TERMS];
            f4v start[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                start[m] = f4v{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    x_at(m, p * STEPS + s).terms(t[m][s]);
                    if constexpr (TERMS == 1) start[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[m][s][0], offset, start[m], 0, 0, 0);
                }
            }
#pragma unroll
            for (int g = 0; g < NT; ++g) {
                bf8v b[STEPS];
#pragma unroll
                for (int s = 0; s < STEPS; ++s) b[s] = TERMS == 1 ? operand(q[g][p * STEPS + s], one) : operand_signed(q[g][p * STEPS + s]);
                const float scale = (TERMS == 1 ? 1.0f : 16.0f) * __uint_as_float(sc[g][G32 ? p : 0] << 16);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    f4v acc = start[m];
#pragma unroll
                    for (int s = 0; s < STEPS; ++s)
#pragma unroll
                        for (int e = TERMS - 1; e >= 0; --e) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[m][s][e], b[s], acc, 0, 0, 0);
                    // a lane's four sums are rows 4 kq .. 4 kq + 3 of channel n
                    total[g][m] += scale * acc;
                }
            }
        }
    };
    auto load_weights = [&](int ku, u2v (&q)[NT], unsigned int (&sc)[NT][2]) {
#pragma unroll
        for (int g = 0; g < NT; ++g) {
            q[g] = (weights(g) + (size_t)ku * 64)[(unsigned)lane];
            const unsigned short *s = scales(g) + (size_t)(G32 ? 2 * ku : ku >> a.unit_shift) * 16;
            sc[g][0] = s[(unsigned)n];
            if constexpr (G32) sc[g][1] = s[16u + (unsigned)n];
        }
    };
    if constexpr (MT == 1) {
        constexpr int U = sizeof(T) == 2 ? (G32 ? 6 : 8) : 4;             // units asked for at once
        const unsigned int at = row_at(n) + 8 * kq;
        for (int base = w; base < a.nu; base += W * U) {
            u2v q[U][NT];
            unsigned int sc[U][NT][2];            // (whole registers: halves would be put together, one load waiting for the other)
            Eight<T> xr[U][2];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int ku = base + i * W;
                if (ku >= a.nu) break;
                load_weights(ku, q[i], sc[i]);
#pragma unroll
                for (int s = 0; s < 2; ++s) xr[i][s].load((x + (size_t)ku * 64 + 32 * s) + at);
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (base + i * W >= a.nu) break;
                multiply(q[i], sc[i], [&](int, int s) -> const Eight<T> & { return xr[i][s]; });
            }
        }
    } else {
        // Rows are read along themselves and turned in LDS, where a wave has a place for its unit of x to itself: lanes that each read a row of
        // their own (the operand's order) touch 64 lines in one load.  A row's 16-byte chunks are turned round by its number, so that the
        // eight lanes of a read's quarter find them in eight different places.  The next unit is on its way from memory while this one is multiplied.
        constexpr int CH = 4 * sizeof(T), LOADS = MT * 16 * CH / 64;      // chunks of a row's 64 inputs; chunks a lane brings
        u4v *const mine = reinterpret_cast<u4v *>(s_red) + w * (MT * 16 * CH);
        unsigned int from[LOADS], to[LOADS];
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int id = j * 64 + lane, r = id / CH, c = id % CH;
            from[j] = row_at(r) + c * (16 / sizeof(T));
            to[j] = r * CH + (c ^ (r & (CH - 1)));
        }
        u4v raw[LOADS];
        u2v q[NT], q_next[NT];
        unsigned int sc[NT][2], sc_next[NT][2];
        auto load = [&](int ku) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) raw[j] = *reinterpret_cast<const u4v *>((x + (size_t)ku * 64) + from[j]);
            load_weights(ku, q_next, sc_next);
        };
        if (w < a.nu) load(w);
        for (int ku = w; ku < a.nu; ku += W) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) mine[to[j]] = raw[j];
#pragma unroll
            for (int g = 0; g < NT; ++g) {
                q[g] = q_next[g];
                sc[g][0] = sc_next[g][0];
                sc[g][1] = sc_next[g][1];
            }
            __builtin_amdgcn_wave_barrier();
            if (ku + W < a.nu) load(ku + W);
            multiply(q, sc, [&](int m, int s) {
                Eight<T> e;
#pragma unroll
                for (int k = 0; k < Eight<T>::CHUNKS; ++k) {
                    const int c = (4 * s + kq) * Eight<T>::CHUNKS + k;
                    e.c[k] = mine[(16 * m + n) * CH + (c ^ (n & (CH - 1)))];
                }
                return e;
            });
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();                                                  // the places are where the sums go
    }
    // the waves' sums, in a fixed order; upper halves are added to the lower ones while LDS does not hold those of all
    f4v *const red = reinterpret_cast<f4v *>(s_red) + lane;
    auto put = [&](int at) {
#pragma unroll
        for (int g = 0; g < NT; ++g)
#pragma unroll
            for (int m = 0; m < MT; ++m) red[((at * NT + g) * MT + m) * 64] = total[g][m];
    };
    while (W > sums_in_lds(NT * MT)) {
        const int half = (W + 1) / 2;
        if (w >= half && w < W) put(w - half);
        __syncthreads();
        if (w < W - half)
#pragma unroll
            for (int g = 0; g < NT; ++g)
#pragma unroll
                for (int m = 0; m < MT; ++m) total[g][m] += red[((w * NT + g) * MT + m) * 64];
        __syncthreads();
        W = half;
    }
    if (w < W) put(w);
    __syncthreads();
    for (int id = threadIdx.x; id < PLACES; id += blockDim.x) {
        int c, m, j;
        const int ch = place(id, &c, &m, &j), row = m0 + 16 * m + 4 * kq + j;
        if (row >= a.rows) continue;
        float u[NG][PER];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float b = bias[g * CT];
#pragma unroll
            for (int k = 1; k < CT; ++k) b = c == k ? bias[g * CT + k] : b;
#pragma unroll
            for (int e = 0; e < PER; ++e) u[g][e] = b;
            for (int p = 0; p < W; ++p) {
                const f4v *at = red + ((p * NT + g * CT + c) * MT + m) * 64;
                if constexpr (PER == 4) {
                    const f4v v = *at;
#pragma unroll
                    for (int e = 0; e < PER; ++e) u[g][e] += v[e];
                } else {
                    u[g][0] += reinterpret_cast<const float *>(at)[j];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            if (row + e >= a.rows) break;
            float out = u[0][e];
            size_t at;
            if constexpr (STEP) {
                at = (size_t)(row + e) * a.H + ch;
                const float h = id == (int)threadIdx.x ? first_h[e] : a.h ? a.h[at] : 0.0f;
                const float f = fast_sigmoid(u[0][e]), i = fast_sigmoid(NG == 2 ? -u[0][e] : u[NG - 2][e]);
                out = fmaf(f, h, i * u[NG - 1][e]);
                a.h_next[at] = out;
            } else {
                at = ((size_t)(row + e) * a.G + g0) * a.H + ch;
            }
            if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at] = out;
            else static_cast<unsigned short *>(a.out)[at] = f32_to_bf16(out);
        }
    }
}

// ------------------------------------------------------------------ products of many rows
// A workgroup: 128 rows x 64 NW channels of a head, waves of 16 MT rows x 64 channels that go through the inputs together, a unit at a time (KS = 2:
// a unit each for two halves of the waves, whose sums are added in LDS).  Rows come into LDS once for all waves (fp32: as their three
// terms), two places in turn with one barrier a unit; weights go from memory into the operand registers as above, the next unit's
// on their way meanwhile.  Bound by instruction issue: for 64 x 64 x 64 a wave issues 40 matrix and 160 vector instructions, 64 of which
// scale the sums of a group (MT = 8 halves those that unpack; groups of 128 are scaled by units too), and fp32 96 and 340.  0.80 PFLOP/s
// with heads of 1024 inputs and 4096 rows, fp32 0.35; 0.57 at 1024 rows of 2816 x 4 x 704.  Without effect: loads two units ahead,
// reads of LDS a step ahead, three waves a SIMD.
template <typename T, int MT, int NW, int KS, bool G32>
__global__ __launch_bounds__(64 * 8 / MT * NW * KS, 2) void q4_tiles_kernel(const RowsQ4Args a)
{
    constexpr int TERMS = Eight<T>::TERMS, M = 128, NT = 4, WM = 8 / MT, THREADS = 64 * WM * NW;
    constexpr int LOADS = M * 8 / THREADS;                    // eights of x that a thread brings
    __shared__ u4v s_x[KS][2][TERMS][M * 8];
    const int lane = threadIdx.x & 63, n = lane & 15, kq = lane >> 4, all_w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = KS == 1 ? 0 : all_w / (WM * NW), w = KS == 1 ? all_w : all_w % (WM * NW);
    // the tiles of 64 channels of all gates that have a head's inputs, NW at a time
    const unsigned int in_head = (unsigned)a.dh / 64, all = in_head * a.G, across = (all + NW - 1) / NW, per_rows = across * (a.tiles / 4 / in_head);
    const unsigned int mb = blockIdx.x / per_rows, rest = blockIdx.x - mb * per_rows, head = rest / across;
    unsigned int tile = (rest - head * across) * NW + w / WM;
    const bool mine = tile < all;                             // (a wave behind the last tile multiplies that one again and writes nothing)
    tile = mine ? tile : all - 1;
    const int gate = (int)(tile / in_head), ct = (int)(head * in_head + tile - gate * in_head) * 4, wm = w % WM * 16 * MT;
    const int m0 = (int)mb * M;
    const T *x = static_cast<const T *>(a.x) + (size_t)m0 * a.H + (size_t)head * a.dh;
    // loads by resources: what all lanes share is in scalar registers, and nothing is added up for a load
    auto resource = [](const void *p, size_t bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (unsigned int)bytes, 0x27000); };
    const unsigned int esH = a.H * (unsigned int)sizeof(T);
    const buf_rsrc rx = resource(x, (size_t)(a.rows - m0 < M ? a.rows - m0 : M) * esH - (size_t)head * a.dh * sizeof(T));
    const size_t tile0 = (size_t)gate * a.tiles + ct;
    const buf_rsrc rw = resource(a.packed + tile0 * a.nu * 64, (size_t)NT * a.nu * 512);
    const buf_rsrc rs = resource(a.scales + tile0 * a.ng * 16, (size_t)NT * a.ng * 32);

    unsigned int from[LOADS], to[LOADS];                      // bytes, places
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
        const int id = j * THREADS + threadIdx.x % THREADS, r = id / 8, c = id % 8;
        from[j] = ((unsigned int)(m0 + r < a.rows ? r : 0) * a.H + c * 8) * sizeof(T);
        to[j] = r * 8 + (c ^ (r & 7));
    }
    Eight<T> raw[LOADS];
    u2v q[NT];
    unsigned int sc[NT][2];
    const int last = a.nu - 1;                                // (behind it, it is read again: a load without a branch has no wait of its own)
    auto load_x = [&](int ku) {
        const unsigned int k = (unsigned)(ku < last ? ku : last) * 64 * (unsigned)sizeof(T);
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
#pragma unroll
            for (int h = 0; h < Eight<T>::CHUNKS; ++h) raw[j].c[h] = __builtin_amdgcn_raw_buffer_load_b128(rx, from[j] + 16 * h, k, 0);
    };
    auto store_x = [&](int buf) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            bf8v t[TERMS];
            raw[j].terms(t);
#pragma unroll
            for (int e = 0; e < TERMS; ++e) s_x[part][buf][e][to[j]] = __builtin_bit_cast(u4v, t[e]);
        }
    };
    auto load_weights = [&](int ku) {
        ku = ku < last ? ku : last;
#pragma unroll
        for (int c = 0; c < NT; ++c) {
            q[c] = __builtin_amdgcn_raw_buffer_load_b64(rw, lane * 8, (unsigned)(c * a.nu + ku) * 512, 0);
            const unsigned int group = c * a.ng + (G32 ? 2 * ku : ku >> a.unit_shift);
            sc[c][0] = __builtin_amdgcn_raw_buffer_load_b16(rs, n * 2, group * 32, 0);
            if constexpr (G32) sc[c][1] = __builtin_amdgcn_raw_buffer_load_b16(rs, n * 2, group * 32 + 32, 0);
        }
    };
    float bias[NT];
#pragma unroll
    for (int c = 0; c < NT; ++c) bias[c] = a.bias ? a.bias[(size_t)gate * a.H + (ct + c) * 16 + n] : 0.0f;
    const u4v minus24 = {0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u, 0xc1c0c1c0u};
    const bf8v offset = __builtin_bit_cast(bf8v, minus24);
    const unsigned int one = sixteens();
    f4v total[NT][MT];
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int m = 0; m < MT; ++m) total[c][m] = f4v{0, 0, 0, 0};

    load_x(part);
    load_weights(part);
    store_x(0);
    load_x(part + KS);
    for (int i = 0, ku = part; i * KS < a.nu; ++i, ku += KS) {
        __syncthreads();               // this unit's x is there, and nobody reads the other place any more
        store_x(~i & 1);
        load_x(ku + 2 * KS);
        bf8v b[NT][2];
        float scale[NT][2];
#pragma unroll
        for (int c = 0; c < NT; ++c) {
#pragma unroll
            for (int s = 0; s < 2; ++s) b[c][s] = TERMS == 1 ? operand(q[c][s], one) : operand_signed(q[c][s]);
            scale[c][0] = (TERMS == 1 ? 1.0f : 16.0f) * __uint_as_float(sc[c][0] << 16);
            if constexpr (G32) scale[c][1] = (TERMS == 1 ? 1.0f : 16.0f) * __uint_as_float(sc[c][1] << 16);
        }
        load_weights(ku + KS);
        if (KS > 1 && ku >= a.nu) break;      // (the last round, and the barriers are behind)
        const u4v(*const xs)[M * 8] = s_x[part][i & 1];
        constexpr int PARTS = G32 || TERMS == 3 ? 2 : 1, STEPS = 2 / PARTS;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                bf8v t[STEPS][TERMS];
                f4v start = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
#pragma unroll
                    for (int e = 0; e < TERMS; ++e)
                        t[s][e] = __builtin_bit_cast(bf8v, xs[e][(wm + 16 * m + n) * 8 + ((4 * (p * STEPS + s) + kq) ^ (n & 7))]);
                    if constexpr (TERMS == 1) start = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[s][0], offset, start, 0, 0, 0);
                }
                f4v acc[NT];
#pragma unroll
                for (int c = 0; c < NT; ++c) acc[c] = start;
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int e = TERMS - 1; e >= 0; --e)
#pragma unroll
                        for (int c = 0; c < NT; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(t[s][e], b[c][p * STEPS + s], acc[c], 0, 0, 0);
#pragma unroll
                for (int c = 0; c < NT; ++c) total[c][m] += scale[c][G32 ? p : 0] * acc[c];
                if constexpr (G32 && TERMS == 1 && KS == 1) __builtin_amdgcn_sched_barrier(0);
            }
    }
    if constexpr (KS == 2) {
        // one sum of both halves, where x was
        f4v *const sums = reinterpret_cast<f4v *>(s_x) + w * (NT * MT * 64) + lane;
        static_assert(sizeof(s_x) >= WM * NW * NT * MT * 64 * sizeof(f4v), "");
        __syncthreads();
        if (part == 1)
#pragma unroll
            for (int c = 0; c < NT; ++c)
#pragma unroll
                for (int m = 0; m < MT; ++m) sums[(c * MT + m) * 64] = total[c][m];
        __syncthreads();
        if (part == 1) return;
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
            for (int m = 0; m < MT; ++m) total[c][m] += sums[(c * MT + m) * 64];
    }
    if (!mine) return;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = m0 + wm + 16 * m + 4 * kq + e;
            if (row >= a.rows) continue;
            const size_t at = ((size_t)row * a.G + gate) * a.H + ct * 16 + n;
#pragma unroll
            for (int c = 0; c < NT; ++c) {
                const float u = total[c][m][e] + bias[c];
                if constexpr (sizeof(T) == 4) static_cast<float *>(a.out)[at + c * 16] = u;
                else static_cast<unsigned short *>(a.out)[at + c * 16] = f32_to_bf16(u);
            }
        }
}

// ------------------------------------------------------------------ host
// pararnn_set_q4_products: 0: products with the codes whatever the rows, 1: beyond exact_rows with the weights rounded to bf16
std::atomic<int> g_products{0};

// Rows from which the weights rounded to bf16 and written out for the tiles of the projection, whose rate is higher but which start with
// that, are ahead of the codes themselves.  A weight has up to 11 significant bits and loses up to three of them, so a caller has to
// ask for it: products of one layer would else see other weights in a long prompt than in the tokens after it.  In units of what 256 of the projection's tiles (256 x 256) take: those
// take 8 us and, for every 256 tiles begun, 10 us and 1.4 for each 64 inputs of a head (2048 x 2 x 2048: 56 us for 65 rows, 61 for 2048,
// 72 for 4096, 116 for 6000; 4096 x 3 x 1024: 41 to 45 up to 1024 rows, 73 for 2048, 106 for 4096); q4_tiles_kernel takes 2 us and 5 + 2.15 for
// each 64 inputs, in proportion to the rows (46 us for 2048, 76 for 4096, 113 for 6000; 38, 64 and 120), with groups of 32 a fifth
// more.  The projection may take over where it is ahead for a seventh of such a round at least, and never for heads of few inputs.
int exact_rows(int H, int G, int n_heads)
{
    const double nu = H / n_heads / 64, round = 10.0 + 1.41 * nu, own = 5.0 + 2.15 * nu;
    for (int r = 1; r < 64; ++r) {
        const double rounds = (6.0 + r * round) / own;
        if (rounds < r - 0.15) return std::max(64, (int)std::min(1e9, rounds * (1 << 24) / ((double)G * H)));
    }
    return 1000000000;
}
bool weights_ok(int H, int G, int n_heads) { return H >= 1 && G >= 1 && G <= 8 && n_heads >= 1 && H % n_heads == 0; }
bool group_ok(int group) { return group == 32 || group == 64 || group == 128; }
// what the kernels have no form for (6e10 weights: the threads of a launch are numbered in 32 bits, 16 weights each)
bool unsupported(int H, int G, int n_heads, int group)
{
    const int dh = H / n_heads;
    return H > (1 << 20) || dh % 64 || dh % group || (double)G * H * dh > 6e10;
}
int status_of(hipError_t e) { return e == hipSuccess ? PARARNN_OK : e == hipErrorInvalidConfiguration ? PARARNN_UNSUPPORTED : PARARNN_HIP_ERROR; }
bool misaligned(const void *p, size_t n) { return (uintptr_t)p % n != 0; }

PrepArgs prep_args(int H, int G, int n_heads, int group, int per)
{
    PrepArgs a = {};
    a.dh = H / n_heads;
    a.nu = a.dh / 64;
    a.group = group;
    a.per_row = a.nu / per;
    a.blocks = (unsigned)(a.per_row + 3) / 4;
    return a;
}
dim3 prep_grid(const PrepArgs &a, int H, int G) { return dim3((unsigned)((long long)G * H / 16) * a.blocks); }
dim3 prep_block(const PrepArgs &a) { return dim3(64 * (a.per_row < 4 ? a.per_row : 4)); }

template <typename T, int MT, int NG, int CT, bool STEP> hipError_t launch_rows(const RowsQ4Args &a, int group, hipStream_t st)
{
    const int W = a.nu < 8 ? a.nu : 8;
    const int held = sums_in_lds(NG * CT * MT);
    const long long blocks = (long long)(a.tiles / CT) * (STEP ? 1 : a.G) * ((a.rows + 16 * MT - 1) / (16 * MT));
    if (blocks * 512 >= (1ll << 32)) return hipErrorInvalidConfiguration;      // threads of a launch are numbered in 32 bits
    const dim3 grid((unsigned)blocks), block(64 * W);
    const size_t sums = (size_t)std::min(W, held) * NG * CT * MT * 1024;
    const size_t lds = MT == 1 ? sums : std::max(sums, (size_t)W * MT * 16 * 64 * sizeof(T));
    if (group == 32) hipLaunchKernelGGL((q4_rows_kernel<T, MT, NG, CT, STEP, true>), grid, block, lds, st, a);
    else hipLaunchKernelGGL((q4_rows_kernel<T, MT, NG, CT, STEP, false>), grid, block, lds, st, a);
    return hipGetLastError();
}
// Whether tiles of 128 rows beat the kernel of few rows.  They use a weight for twice the rows or more and need no sums of eight waves, but have
// fewer workgroups, which take a unit in 0.7 us (fp32 2.9): it pays from a number of the latter's workgroups (64 rows x 64 channels,
// fp32 32 x 64) on.  Both level, bf16, units of a head: that number: 1: 90, 4: 340, 8: 300, 11: 340, 16: 390, 32: 580; 4096 rows: 9.9 to
// 5.6 us, 32 to 18, 45 to 18, 245 to 83, 155 to 64, 146 to 75.  fp32: 6: 1000, 16: 1800 (512 rows 29 to 21.5, 80 to 48; 4096 rows 215 to 72, 622 to
// 298), and not with too few of either (512 x 2 x 256: 2048 rows 11.0 to 15, 4096 20.4 to 16.6).
bool tiles_better(const RowsQ4Args &a, bool bf16)
{
    if (a.rows <= 64) return false;
    const double groups = (double)(a.H / 64) * a.G * ((a.rows + (bf16 ? 63 : 31)) / (bf16 ? 64 : 32));
    if (bf16) return groups > std::min(90.0 * a.nu, 300.0 + 8.0 * a.nu);
    return groups > std::max(1100.0, 256.0 * (1.0 + 3.1 * a.nu) / (2.3 + 0.33 * a.nu));
}
template <typename T, int MT, int NW, int KS> hipError_t launch_tiles(const RowsQ4Args &a, long long blocks, int group, hipStream_t st)
{
    if (blocks * 512 >= (1ll << 32)) return hipErrorInvalidConfiguration;      // threads of a launch are numbered in 32 bits
    const dim3 grid((unsigned)blocks), block(64 * 8 / MT * NW * KS);
    if (group == 32) hipLaunchKernelGGL((q4_tiles_kernel<T, MT, NW, KS, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((q4_tiles_kernel<T, MT, NW, KS, false>), grid, block, 0, st, a);
    return hipGetLastError();
}
// bf16: 128 channels in four waves, 64 rows x 64 channels each.  Where there is not one such workgroup for each compute unit, twice the waves share
// the inputs (2048 x 2 x 2048, 686 rows: 30.2 to 24.6 us; with two for each 46 to 51).  Where there is one of 256 channels for each, and a head's
// channels fill them, waves of 128 rows x 64 channels, which unpack a weight once for all of them (4096 rows: 4096 x 3 x 1024 142 to 120, 2816
// x 4 x 704 97 to 83; 264 and 288 workgroups 28.0 to 26.2, 37.1 to 35.1, 192 23.6 to 25.5; groups of 32 with 256 18.6 to 23.8).
// fp32: 256 channels in eight waves, for the terms of x are formed once for all of them (4096 x 3 x 1024, 4096 rows: 498 to 310).
template <typename T> hipError_t launch_tiles(const RowsQ4Args &a, int group, hipStream_t st)
{
    const int all = a.G * (a.dh / 64);                        // of a head
    auto blocks_of = [&](int NW) { return (long long)(a.H / a.dh) * ((all + NW - 1) / NW) * ((a.rows + 127) / 128); };
    const long long narrow = blocks_of(2), wide = blocks_of(4);
    if constexpr (sizeof(T) == 4) {
        return launch_tiles<T, 4, 4, 1>(a, wide, group, st);
    } else {
        if (narrow <= 256 && a.nu >= 8) return launch_tiles<T, 4, 2, 2>(a, narrow, group, st);
        if (wide >= (group == 32 ? 512 : 256) && 10 * wide <= 6 * narrow) return launch_tiles<T, 8, 4, 1>(a, wide, group, st);
        return launch_tiles<T, 4, 2, 1>(a, narrow, group, st);
    }
}
constexpr int kWorkgroups = 192;        // fewer leave too much of the device idle
// Rows and channels of a workgroup: the more, the fewer times weights and inputs are read, as long as there are workgroups for the
// device.  In a graph, weights read from memory, one row and 16 of bf16, 16 x 16 against 32 x 64 (a step: 32 x 16 of each gate): 3 x 4096 x 4096
// 11.4 us and 15.9 against 10.8 and 10.9 (weights in the memory-side cache 8.4 and 15.0 against 9.6 and 9.7), a step with 2 x 8192 x 1024 6.3 and 7.4
// against 6.3 and 6.5, with 2 x 4096 x 4096 7.9 and 9.2 against 8.7 and 8.9; with too few workgroups, 3 x 2048 x 1024, 3.9 and 5.1
// against 5.5 twice.  fp32, whose terms cost more than the weights, 4, 8 and 16 rows: 18.2, 19.5 and 27.5 against 20.0, 19.9 and
// 20.1, a step with 2 x 4096 x 4096 11.0, 10.9 and 12.8 against 15.0.
template <typename T, int NG, bool STEP> hipError_t launch_rows_of(RowsQ4Args a, int n_heads, int group, hipStream_t st)
{
    a.dh = a.H / n_heads; a.nu = a.dh / 64; a.ng = a.dh / group; a.tiles = (unsigned)a.H / 16;
    a.unit_shift = group == 128 ? 1 : 0;
    const long long tiles = (long long)a.tiles * (STEP ? 1 : a.G);
    auto enough = [&](int mt, int ct) { return tiles / ct * ((a.rows + 16 * mt - 1) / (16 * mt)) >= kWorkgroups; };
    constexpr int C4 = STEP ? 1 : 4;
    constexpr bool bf16 = sizeof(T) == 2;
    if constexpr (!STEP)
        if (tiles_better(a, bf16)) return launch_tiles<T>(a, group, st);
    // (three terms of fp32 leave no registers for 64 rows: 46 -> 88 us for 64 of 3 x 4096 x 4096)
    if constexpr (bf16)
        if (a.rows > 32 && enough(4, C4)) return launch_rows<T, 4, NG, C4, STEP>(a, group, st);
    if (a.rows > (bf16 || !STEP ? 8 : 16) && enough(2, C4)) return launch_rows<T, 2, NG, C4, STEP>(a, group, st);
    if (a.rows > 16 && enough(2, 1)) return launch_rows<T, 2, NG, 1, STEP>(a, group, st);
    return launch_rows<T, 1, NG, 1, STEP>(a, group, st);
}

}  // namespace

size_t q4_packed_bytes(int H, int G, int n_heads)
{
    if (!weights_ok(H, G, n_heads) || unsupported(H, G, n_heads, 32)) return 0;
    return (size_t)G * H * (H / n_heads) / 2;
}

size_t q4_scale_bytes(int H, int G, int n_heads, int group)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || unsupported(H, G, n_heads, group)) return 0;
    return (size_t)G * H * (H / n_heads / group) * 2;
}

int q4_quantize(const float *Wx, int H, int G, int n_heads, int group, void *packed, void *scales, hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !Wx || !packed || !scales || misaligned(Wx, 4) || misaligned(packed, 16) ||
        misaligned(scales, 2))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, G, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, group == 128 ? 2 : 1);
    a.W = Wx; a.packed_out = static_cast<u2v *>(packed); a.scales_out = static_cast<unsigned short *>(scales);
    if (group == 128) hipLaunchKernelGGL(q4_quantize_kernel<2>, prep_grid(a, H, G), prep_block(a), 0, st, a);
    else hipLaunchKernelGGL(q4_quantize_kernel<1>, prep_grid(a, H, G), prep_block(a), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_pack(const signed char *codes, const void *code_scales, int H, int G, int n_heads, int group, void *packed, void *scales,
            hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !codes || !code_scales || !packed || !scales || misaligned(code_scales, 2) ||
        misaligned(packed, 16) || misaligned(scales, 2))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, G, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, 1);
    a.codes = codes; a.code_scales = static_cast<const unsigned short *>(code_scales);
    a.packed_out = static_cast<u2v *>(packed); a.scales_out = static_cast<unsigned short *>(scales);
    hipLaunchKernelGGL(q4_pack_kernel, prep_grid(a, H, G), prep_block(a), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_dequantize(const void *packed, const void *scales, int H, int G, int n_heads, int group, float *Wx, hipStream_t st)
{
    if (!weights_ok(H, G, n_heads) || !group_ok(group) || !packed || !scales || !Wx || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(Wx, 4))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, G, n_heads, group)) return PARARNN_UNSUPPORTED;
    PrepArgs a = prep_args(H, G, n_heads, group, 1);
    a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.W_out = Wx;
    hipLaunchKernelGGL(q4_dequantize_kernel<false>, prep_grid(a, H, G), prep_block(a), 0, st, a);
    return hipGetLastError() == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

int q4_set_products(int mode)
{
    if (mode < 0 || mode > 1) return PARARNN_INVALID_ARG;
    g_products.store(mode, std::memory_order_relaxed);
    return PARARNN_OK;
}

int q4_products() { return g_products.load(std::memory_order_relaxed); }

int q4_exact_rows(int H, int G, int n_heads)
{
    return weights_ok(H, G, n_heads) && !unsupported(H, G, n_heads, 32) ? exact_rows(H, G, n_heads) : -1;
}

size_t q4_workspace_bytes(int dtype, int B, int L, int H, int G, int n_heads, int group)
{
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || L < 1 || (double)B * L > 1e9 || q4_scale_bytes(H, G, n_heads, group) == 0) return 0;
    if (dtype == PARARNN_F32 || (long long)B * L <= exact_rows(H, G, n_heads)) return 256;
    return proj_workspace_bytes(dtype, B, L, H, G, n_heads, 0);
}

int q4_project(int dtype, const void *x, const void *packed, const void *scales, const float *bias, int B, int L, int H, int G,
               int n_heads, int group, void *u, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || L < 1 || !weights_ok(H, G, n_heads) || !group_ok(group) || !x ||
        !packed || !scales || !u || misaligned(x, 16) || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(bias, 4) || misaligned(u, es) || misaligned(workspace, 256))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, G, n_heads, group)) return PARARNN_UNSUPPORTED;
    const size_t need = q4_workspace_bytes(dtype, B, L, H, G, n_heads, group);
    if (need == 0) return PARARNN_INVALID_ARG;
    const int rows = B * L;
    const bool many = dtype == PARARNN_BF16 && rows > exact_rows(H, G, n_heads), rounded = many && q4_products() == 1;
    if (rounded && !workspace) return PARARNN_INVALID_ARG;
    if (workspace && workspace_bytes < need) return PARARNN_WORKSPACE_TOO_SMALL;
    if (many && misaligned(u, 16)) return PARARNN_UNSUPPORTED;      // (with either products, as the workspace: the choice may change between calls)
    if (rounded) {
        int *tickets = nullptr;
        unsigned short *Wb = proj_weights_at(workspace, &tickets);
        PrepArgs p = prep_args(H, G, n_heads, group, 1);
        p.packed = static_cast<const u2v *>(packed); p.scales = static_cast<const unsigned short *>(scales);
        p.Wb_out = Wb; p.tickets = tickets;
        hipLaunchKernelGGL(q4_dequantize_kernel<true>, prep_grid(p, H, G), prep_block(p), 0, st, p);
        if (hipGetLastError() != hipSuccess) return PARARNN_HIP_ERROR;
        return proj_product(dtype, x, Wb, bias, B, L, H, G, n_heads, u, tickets, st);
    }
    RowsQ4Args a = {};
    a.x = x; a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.bias = bias; a.out = u;
    a.rows = rows; a.H = H; a.G = G;
    const hipError_t e = dtype == PARARNN_BF16 ? launch_rows_of<unsigned short, 1, false>(a, n_heads, group, st) : launch_rows_of<float, 1, false>(a, n_heads, group, st);
    return status_of(e);
}

int q4_step(int dtype, const void *x, const void *packed, const void *scales, const float *bias, const float *h, int B, int H, int G,
            int n_heads, int group, void *y, float *h_next, hipStream_t st)
{
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || (G != 2 && G != 3) || !weights_ok(H, G, n_heads) || !group_ok(group) ||
        !x || !packed || !scales || !y || !h_next || misaligned(x, 16) || misaligned(packed, 16) || misaligned(scales, 2) ||
        misaligned(bias, 4) || misaligned(h, 4) || misaligned(h_next, 4) || misaligned(y, es))
        return PARARNN_INVALID_ARG;
    if (unsupported(H, G, n_heads, group) || B > (1 << 20)) return PARARNN_UNSUPPORTED;
    RowsQ4Args a = {};
    a.x = x; a.packed = static_cast<const u2v *>(packed); a.scales = static_cast<const unsigned short *>(scales); a.bias = bias; a.h = h;
    a.out = y; a.h_next = h_next;
    a.rows = B; a.H = H; a.G = G;
    const hipError_t e = dtype == PARARNN_BF16
                             ? (G == 2 ? launch_rows_of<unsigned short, 2, true>(a, n_heads, group, st) : launch_rows_of<unsigned short, 3, true>(a, n_heads, group, st))
                             : (G == 2 ? launch_rows_of<float, 2, true>(a, n_heads, group, st) : launch_rows_of<float, 3, true>(a, n_heads, group, st));
    return status_of(e);
}

}  // namespace pararnn
