// The gated linear recurrence h_t = f_t h_{t-1} + i_t v_t and its adjoint over whole sequences.
//
//   gates    G = 2: (f, v) with f = sig(u_f), i = 1 - f = sig(-u_f), v = u_v;  G = 3: (f, i, v) with i = sig(u_i)
//   forward  the map of a stretch of steps is h -> A h + S; maps compose as (A2 A1, A2 S1 + S2)
//   adjoint  mu_t = f_t (g_t + mu_{t+1}) is the gradient of h_{t-1}, lam_t = g_t + mu_{t+1} that of h_t:
//            du_v = lam i,  du_i = lam v i (1 - i),  du_f = lam h_{t-1} f (1 - f)  (G = 2: lam (h_{t-1} - v) f (1 - f))
//
// A tile is CW channels x TT steps of one sequence (64 x 128, 16 x 512 or, alone, shorter).  It is read from memory once: a thread takes VEC channels of C
// consecutive steps, 64 / LPR segments of a wave are joined by shuffles, the waves through LDS, the tiles along L by carry
// records (look-back).  The forward pass leaves the fp32 state in front of every tile behind (checkpoints, 4 bytes a channel
// for TT steps); the adjoint recomputes the states inside a tile from there, which reads 2 bytes a step and channel less than
// the stored states would take and keeps their rounding out of the gradients.
//
// States, maps and adjoints are fp32; h and dL_du are rounded once when they are written.
//
// Long sequences are bound by memory: (G + 1) elements a step and channel forward, 2 G + 1 backward.  4 x 65536 x 4096 bf16, G = 2: 1.28 ms
// and 2.08, 5.0 and 5.2 TB/s of those bytes (a copy: 4.7); 16 x 4096 x 1024 fp32 0.16 and 0.25, 5.0 and 5.4.  Short ones are bound by
// the launch and the way to memory and back: 2.5 to 4.5 us for one tile along time, 6 to 13 where a few wait for each other.
// Two channels a thread for either type: eight hold so many values that few waves fit (the same backward pass 5.0 ms).
#include <algorithm>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gated.h"
#include "pararnn.h"
#include "pararnn/common.h"
#include "pararnn/launch.h"

namespace pararnn {
namespace {

// Tiles: 64 channels x 128 steps, or 16 x 512 (narrow rows, and problems of few tiles); a single tile along L may be shorter
constexpr int kWide = 64, kNarrow = 16;
constexpr __host__ __device__ int tile_steps(int channels) { return 8192 / channels; }
constexpr int kQueues = 16;              // counters that hand out tiles, kQueuePitch words apart (a line each)
constexpr int kQueuePitch = 32;
constexpr int kWaves = 8;                // of a tile's workgroup
constexpr int kBatch = 4;                // steps that a thread which walks a sequence reads at once

// ------------------------------------------------------------------ accesses
typedef unsigned int u2v __attribute__((ext_vector_type(2)));
typedef unsigned int u4v __attribute__((ext_vector_type(4)));

// VEC storage elements as they lie in memory
template <typename T, int VEC> struct Raw {
    unsigned int w[(sizeof(T) * VEC + 3) / 4];
    __device__ __forceinline__ float at(int k) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
};

// The bounds of the resource are the bounds of the tile's valid rows: a load behind them gives zeros, a store nothing.
// The row is part of the vector offset, which the bounds check covers (the scalar offset is outside it).
template <typename T, int VEC> __device__ __forceinline__ Raw<T, VEC> load_raw_at(buf_rsrc r, unsigned int off)
{
    Raw<T, VEC> x;
    constexpr int BYTES = sizeof(T) * VEC;
    if constexpr (BYTES == 2) x.w[0] = __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0);
    else if constexpr (BYTES == 4) x.w[0] = __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0);
    else if constexpr (BYTES == 8) {
        const u2v v = __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0);
        x.w[0] = v.x; x.w[1] = v.y;
    } else {
        static_assert(BYTES == 16, "");
        const u4v v = __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0);
        x.w[0] = v.x; x.w[1] = v.y; x.w[2] = v.z; x.w[3] = v.w;
    }
    return x;
}
template <typename T, int VEC> __device__ __forceinline__ void store_at(buf_rsrc r, unsigned int off, const float (&in)[VEC])
{
    constexpr int BYTES = sizeof(T) * VEC;
    unsigned int w[(BYTES + 3) / 4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) w[k] = __float_as_uint(in[k]);
    } else if constexpr (VEC == 1) {
        w[0] = f32_to_bf16(in[0]);
    } else {
#pragma unroll
        for (int k = 0; k < VEC / 2; ++k) w[k] = f32_to_bf16(in[2 * k]) | (unsigned int)f32_to_bf16(in[2 * k + 1]) << 16;
    }
    if constexpr (BYTES == 2) __builtin_amdgcn_raw_buffer_store_b16((unsigned short)w[0], r, off, 0, 0);
    else if constexpr (BYTES == 4) __builtin_amdgcn_raw_buffer_store_b32(w[0], r, off, 0, 0);
    else if constexpr (BYTES == 8) __builtin_amdgcn_raw_buffer_store_b64(u2v{w[0], w[1]}, r, off, 0, 0);
    else {
        const u4v v = {w[0], w[1], w[2], w[3]};
        __builtin_amdgcn_raw_buffer_store_b128(v, r, off, 0, 0);
    }
}
__device__ __forceinline__ buf_rsrc rsrc_of(const void *base, unsigned int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x27000);
}
constexpr unsigned int kOutside = 0x80000000u;        // an offset behind every bound, with any row's added (a tile's rows stay below 2^31 bytes)
// Registers are what the number of waves hangs on, so values are held to where they are formed:
// unknown(): a value the compiler knows nothing about.  Offsets of stores are formed where the stores are, not kept (one for each row
// and gate) from the loads of the same rows on, and packed elements are unpacked again at their second use.
// formed(): what is computed before this point is not put off behind it, with all its operands alive until then.
__device__ __forceinline__ unsigned int unknown(unsigned int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ void formed(float &x) { asm volatile("" : "+v"(x)); }

// ------------------------------------------------------------------ gates
// f = sig(x) and 1 - f, the latter as e^-x f: exact where f rounds to 1.  e^-x is held below 2^126, so that its product with f is
// 1 and not inf times 0 for very negative x (f is then 2^-126 instead of less).  NaN stays NaN.
__device__ __forceinline__ void sigmoid2(float x, float *f, float *one_minus)
{
    float p = -1.4426950408889634f * x;
    p = p > 126.0f ? 126.0f : p;
    const float e = __builtin_amdgcn_exp2f(p);
    *f = __builtin_amdgcn_rcpf(1.0f + e);
    *one_minus = e * *f;
}

// The factor of a stretch's map.  Every gate is above 0, so a product of them that underflows is held at the least fp32 number in place of 0:
// an infinite state or gradient stays one behind the stretch, as it does step by step, where 0 times it would be NaN.  What that adds is below
// 2^-149 of the state.  (As whole numbers, where a NaN is larger than all that is compared here; one instruction.)
__device__ __forceinline__ float factor(float a)
{
    const unsigned int w = __float_as_uint(a);
    return __uint_as_float(w > 1u ? w : 1u);
}

// ------------------------------------------------------------------ carry records
// Three 64-bit words {value, tag} for a tile and channel: A and S of the tile's map, and the state behind it.  A word is written
// and read whole and validates itself (tag = number of the call and state), so no fence is needed.
typedef unsigned long long word_t;
__device__ __forceinline__ void put(word_t *p, float v, unsigned int tag)
{
    __hip_atomic_store(p, (word_t)tag << 32 | __float_as_uint(v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ word_t get(const word_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool has_tag(word_t w, unsigned int tag) { return (unsigned int)(w >> 32) == tag; }
__device__ __forceinline__ float value(word_t w) { return __uint_as_float((unsigned int)w); }

// The values that enter tile lt from its neighbours in direction dir: the state behind the nearest tile that has one, carried through
// the maps of those in between in the order and with the roundings those tiles themselves use, so that the result has the same
// bits whichever tile that is.  The whole workgroup looks: wave w at the tile w + 1 steps away, a lane for each channel (or at the
// next LK x 64 / CW tiles), so that W and more tiles are asked in one trip to memory and no wave keeps many of them in registers.  Returns the number of maps
// between (the tiles found are in LDS then, carry_of() puts them together), or -1 when the wait ran out.
// Tiles are numbered by a ticket in the order of their chain: every tile in front has been started by a workgroup that never
// waits for this one, and the first of a chain publishes its state without waiting, so the wait ends.  A bound on the polls
// ends it whatever happens; the result is then NaN.
template <int W, int LK, int CW> struct Seen {
    static constexpr int SUB = 64 / CW, N = W * LK * SUB;    // tiles that a wave looks at in one load; in one trip
    static_assert(N <= 64, "");
    float a[2][N][CW], s[2][N][CW];                          // s: of a map, or the state behind the tile
    int what[2][N];                                          // 2: a state, 1: a map, 0: neither yet
};
// active: whether this lane's channel, lane % CW, is one of the tile's
template <int W, int LK, int CW>
__device__ __forceinline__ int look_back(Seen<W, LK, CW> &seen, const word_t *rec, int dir, int lt, int n_lt, bool active,
                                         unsigned int tag, unsigned int spin_limit, int *parity)
{
    constexpr int SUB = Seen<W, LK, CW>::SUB, N = Seen<W, LK, CW>::N;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane / CW, col = lane % CW;
    for (unsigned int spins = 0; spins < spin_limit; ++spins) {
        const int b = spins & 1;
        word_t x[LK], a[LK], s[LK];
        bool exists[LK];
#pragma unroll
        for (int k = 0; k < LK; ++k) {
            const int j = lt + ((w * LK + k) * SUB + sub + 1) * dir;
            exists[k] = j >= 0 && j < n_lt;
            const word_t *p = rec + (long long)(exists[k] ? j - lt : dir) * 3 * CW + col;      // lt + dir exists
            x[k] = get(p + 2 * CW);
            a[k] = get(p);
            s[k] = get(p + CW);
        }
#pragma unroll
        for (int k = 0; k < LK; ++k) {
            // votes of the lanes that look at the same tile
            auto all_of = [&](bool ok) { return (__ballot(!active || ok) >> (sub * CW) & (~0ull >> (64 - CW))) == ~0ull >> (64 - CW); };
            const bool state = all_of(has_tag(x[k], tag + 2)), map = all_of(has_tag(a[k], tag + 1) && has_tag(s[k], tag + 1));
            const int at = (w * LK + k) * SUB + sub;
            seen.a[b][at][col] = value(a[k]);
            seen.s[b][at][col] = state ? value(x[k]) : value(s[k]);
            if (col == 0) seen.what[b][at] = !exists[k] ? 0 : state ? 2 : map ? 1 : 0;
        }
        __syncthreads();
        // (two buffers: a wave that goes on writes the other one, and is held by the next barrier until all have read this one)
        const int what = seen.what[b][lane % N];
        const unsigned long long states = __ballot(what == 2), gaps = __ballot(what == 0);
        if (states && (!gaps || __builtin_ctzll(states) < __builtin_ctzll(gaps))) {
            *parity = b;
            return __builtin_ctzll(states);
        }
        __builtin_amdgcn_s_sleep(1);
    }
    return -1;
}
// K channels from c on: what the look found
template <int K, int W, int LK, int CW>
__device__ __forceinline__ void carry_of(const Seen<W, LK, CW> &seen, int found, int parity, int c, float (&v)[K])
{
    if (found < 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = __uint_as_float(0x7fc00000u);
        return;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = seen.s[parity][found][c + k];
    for (int q = found - 1; q >= 0; --q)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = fmaf(seen.a[parity][q][c + k], v[k], seen.s[parity][q][c + k]);
}

struct GatedArgs {
    const void *u;
    const float *h0;              // forward, or NULL
    const int *lengths;           // or NULL
    void *h;                      // forward: out
    float *last;                  // forward: state behind the last step, or NULL
    float *ckpt;                  // forward: out or NULL; backward: in
    const void *g;                // backward, or NULL
    const float *dlast;           // backward, or NULL
    void *du;                     // backward: out
    float *dh0;                   // backward: out or NULL
    unsigned int *ticket;
    word_t *rec;                  // [chain][tile][3][CW]
    unsigned int tag;             // of this call: aggregates carry tag + 1, states tag + 2
    unsigned int spin_limit;
    int B, L, H, n_lt, groups, chains, queues;
};

// Where a workgroup's tile lies.
struct Place {
    int b, grp, lt, chain;
    int rows, rows_all;           // valid steps, and all steps, of the tile
};

// Chains are shared out among up to kQueues queues, neighbours to the same one: a queue hands out the tiles of its chains with a
// ticket, along time first for none of them (all chains' first tiles, then all second ones).  One counter for all tiles
// bounds a launch: its atomics take 12.5 ns each, 1.7 ms for 131072 tiles that move 6.4 GB.  Of 8 or 16 queues, queue q's workgroups
// are launched q, q + queues, ..., which are on one XCD, so that a line shared by two groups of channels is in its L2; not the last
// tiles of unequal queues (fewer than 16 chains' worth), nor those of another number of queues, which fewer than 16 chains make.
// The last workgroup of a queue leaves the counter at zero for the next call.
template <bool LOOK, bool REVERSE, int TT> __device__ __forceinline__ Place place_of(const GatedArgs &a, int *s_id)
{
    Place p;
    if constexpr (LOOK) {
        const int each = a.chains / a.queues, more = a.chains - each * a.queues;      // the first `more` queues have one chain more
        const int even = a.queues * each * a.n_lt, block = (int)blockIdx.x;
        const int q = block < even ? block % a.queues : (block - even) % more;
        const int n = each + (q < more), first = q * each + (q < more ? q : more);
        if (threadIdx.x == 0) {
            unsigned int *ticket = a.ticket + q * kQueuePitch;
            const unsigned int t = atomicAdd(ticket, 1u);
            if (t + 1 == (unsigned int)n * (unsigned int)a.n_lt) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            *s_id = (int)t;
        }
        __syncthreads();
        const int id = __builtin_amdgcn_readfirstlane(*s_id);
        p.lt = id / n;
        p.chain = first + id - p.lt * n;
    } else {
        p.lt = 0;
        p.chain = (int)blockIdx.x;
    }
    if (REVERSE) p.lt = a.n_lt - 1 - p.lt;
    p.b = p.chain / a.groups;
    p.grp = p.chain - p.b * a.groups;
    int len = a.L;
    if (a.lengths) {
        len = __builtin_amdgcn_readfirstlane(a.lengths[p.b]);
        len = len < 0 ? 0 : len > a.L ? a.L : len;
    }
    p.rows = len - p.lt * TT;
    p.rows = p.rows < 0 ? 0 : p.rows > TT ? TT : p.rows;
    p.rows_all = a.L - p.lt * TT;
    p.rows_all = p.rows_all > TT ? TT : p.rows_all;
    // the same in all lanes, which the compiler does not see through the divisions: resources built from them would be used lane by lane
    p.b = __builtin_amdgcn_readfirstlane(p.b);
    p.grp = __builtin_amdgcn_readfirstlane(p.grp);
    p.lt = __builtin_amdgcn_readfirstlane(p.lt);
    p.chain = __builtin_amdgcn_readfirstlane(p.chain);
    p.rows = __builtin_amdgcn_readfirstlane(p.rows);
    p.rows_all = __builtin_amdgcn_readfirstlane(p.rows_all);
    return p;
}

// Bytes from the tile's first channel to the end of its n rows of `width` elements.
__device__ __forceinline__ unsigned int extent(int n, unsigned int row_bytes, unsigned int first)
{
    return n > 0 ? (unsigned int)n * row_bytes - first : 0u;
}

template <typename T, int G, int VEC, int CW, int W, int C, int LK>
__global__ __launch_bounds__(64 * W) void gated_forward_kernel(const GatedArgs a)
{
    constexpr int LPR = CW / VEC, SEG = 64 / LPR;
    constexpr int TT = W * SEG * C;
    static_assert(LK == 0 || TT == tile_steps(CW), "");
    __shared__ float s_a[W][CW], s_s[W][CW], s_in[CW];
    constexpr bool LOOK = LK > 0;
    __shared__ Seen<LOOK ? W : 1, LOOK ? LK : 1, CW> s_seen;
    __shared__ int s_id;
    const Place p = place_of<LOOK, false, TT>(a, &s_id);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sg = lane / LPR, c0 = (lane % LPR) * VEC;
    const int t0 = (w * SEG + sg) * C;
    const unsigned int es = sizeof(T), H = (unsigned int)a.H, first = (unsigned int)p.grp * CW;
    const bool active = first + c0 < H;
    const unsigned int row_bytes = H * es, at_h = (active ? c0 * es : kOutside) + (unsigned int)t0 * row_bytes;
    const unsigned int at_u = at_h + (unsigned int)t0 * (G - 1) * row_bytes;

    const size_t row = (size_t)p.b * a.L + (size_t)p.lt * TT;
    const buf_rsrc ru = rsrc_of(static_cast<const T *>(a.u) + row * G * H + first, extent(p.rows, G * H * es, first * es));
    Raw<T, VEC> raw[C][G];
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int g = 0; g < G; ++g)
            raw[j][g] = load_raw_at<T, VEC>(ru, at_u + (unsigned int)(j * G + g) * row_bytes);

    const unsigned int ch = first + lane % CW;               // wave 0: a lane for each channel of the tile
    const bool act = ch < H, one = lane < CW && act;
    const float in0 = w == 0 && p.lt == 0 && one && a.h0 ? a.h0[(size_t)p.b * H + ch] : 0.0f;

    float f[C][VEC], b[C][VEC], A[VEC], S[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { A[k] = 1.0f; S[k] = 0.0f; }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const bool valid = t0 < p.rows - j;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            float ff, om, i;
            sigmoid2(raw[j][0].at(k), &ff, &om);
            i = om;
            if constexpr (G == 3) i = fast_sigmoid(raw[j][1].at(k));
            f[j][k] = valid ? ff : 1.0f;
            b[j][k] = valid ? i * raw[j][G - 1].at(k) : 0.0f;
            A[k] *= f[j][k];
            S[k] = fmaf(f[j][k], S[k], b[j][k]);
        }
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) A[k] = factor(A[k]);
    // maps of the wave's segments up to and including this one, then without it
#pragma unroll
    for (int d = LPR; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float a1 = __shfl_up(A[k], d, 64), s1 = __shfl_up(S[k], d, 64);
            S[k] = fmaf(A[k], lane >= d ? s1 : 0.0f, S[k]);
            A[k] = factor(A[k] * (lane >= d ? a1 : 1.0f));
        }
    if (sg == SEG - 1)
#pragma unroll
        for (int k = 0; k < VEC; ++k) { s_a[w][c0 + k] = A[k]; s_s[w][c0 + k] = S[k]; }
    if constexpr (SEG > 1) {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float a1 = __shfl_up(A[k], LPR, 64), s1 = __shfl_up(S[k], LPR, 64);
            A[k] = sg ? a1 : 1.0f;
            S[k] = sg ? s1 : 0.0f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) { A[k] = 1.0f; S[k] = 0.0f; }
    }
    if (w == 0 && lane < CW) s_in[lane] = in0;
    __syncthreads();
    // this wave's place among the waves
    float x[VEC], pa[VEC], ps[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { pa[k] = 1.0f; ps[k] = 0.0f; }
    for (int q = 0; q < w; ++q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) { ps[k] = fmaf(s_a[q][c0 + k], ps[k], s_s[q][c0 + k]); pa[k] *= s_a[q][c0 + k]; }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {                          // of all steps of the tile in front of this thread's
        S[k] = fmaf(A[k], ps[k], S[k]);
        A[k] = factor(A[k] * pa[k]);
    }
    const bool more = LOOK && p.lt + 1 < a.n_lt;
    word_t *rec = a.rec + ((size_t)p.chain * a.n_lt + p.lt) * (3 * CW);
    float ta = 1.0f, ts = 0.0f;
    if (w == 0 && lane < CW) {
#pragma unroll
        for (int q = 0; q < W; ++q) { ts = fmaf(s_a[q][lane], ts, s_s[q][lane]); ta *= s_a[q][lane]; }
        ta = factor(ta);
        if (more && act && p.lt > 0) { put(rec + lane, ta, a.tag + 1); put(rec + CW + lane, ts, a.tag + 1); }
    }
    int found = -1, parity = 0;
    if constexpr (LOOK)
        if (p.lt > 0) found = look_back(s_seen, rec, -1, p.lt, a.n_lt, act, a.tag, a.spin_limit, &parity);
    auto entering = [&](int c, auto &v) {                    // the state in front of the tile
        if constexpr (LOOK)
            if (p.lt > 0) return carry_of(s_seen, found, parity, c, v);
#pragma unroll
        for (int k = 0; k < (int)(sizeof(v) / sizeof(v[0])); ++k) v[k] = s_in[c + k];
    };
    if (w == 0 && one) {
        float in1[1];
        entering(lane, in1);
        const float in = in1[0], out = fmaf(ta, in, ts);
        if (more) put(rec + 2 * CW + lane, out, a.tag + 2);
        if (a.ckpt) a.ckpt[((size_t)p.b * a.n_lt + p.lt) * H + ch] = in;
        if (a.last && p.lt + 1 == a.n_lt) a.last[(size_t)p.b * H + ch] = out;      // (may be h0: read before the first state was published)
    }
    entering(c0, x);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = fmaf(A[k], x[k], S[k]);

    const unsigned int at_out = unknown(at_h);
    const buf_rsrc rh = rsrc_of(static_cast<T *>(a.h) + row * H + first, extent(p.rows_all, H * es, first * es));
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const bool valid = t0 < p.rows - j;
        float o[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            x[k] = fmaf(f[j][k], x[k], b[j][k]);
            o[k] = valid ? x[k] : 0.0f;
        }
        store_at<T, VEC>(rh, at_out + (unsigned int)j * row_bytes, o);
    }
}

template <typename T, int G, int VEC, int CW, int W, int C, int LK>
__global__ __launch_bounds__(64 * W, 4) void gated_backward_kernel(const GatedArgs a)
{
    constexpr int LPR = CW / VEC, SEG = 64 / LPR;
    constexpr int TT = W * SEG * C;
    static_assert(LK == 0 || TT == tile_steps(CW), "");
    __shared__ float s_a[W][CW], s_s[W][CW], s_m[W][CW], s_in[CW];
    constexpr bool LOOK = LK > 0;
    __shared__ Seen<LOOK ? W : 1, LOOK ? LK : 1, CW> s_seen;
    __shared__ int s_id;
    const Place p = place_of<LOOK, true, TT>(a, &s_id);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sg = lane / LPR, c0 = (lane % LPR) * VEC;
    const int t0 = (w * SEG + sg) * C;
    const unsigned int es = sizeof(T), H = (unsigned int)a.H, first = (unsigned int)p.grp * CW;
    const bool active = first + c0 < H;
    const unsigned int row_bytes = H * es, at_h = (active ? c0 * es : kOutside) + (unsigned int)t0 * row_bytes;
    const unsigned int at_u = at_h + (unsigned int)t0 * (G - 1) * row_bytes;

    const size_t row = (size_t)p.b * a.L + (size_t)p.lt * TT;
    const buf_rsrc ru = rsrc_of(static_cast<const T *>(a.u) + row * G * H + first, extent(p.rows, G * H * es, first * es));
    const buf_rsrc rg = rsrc_of(static_cast<const T *>(a.g) + row * H + first, extent(a.g ? p.rows : 0, H * es, first * es));
    Raw<T, VEC> raw[C][G], rawg[C];
#pragma unroll
    for (int j = 0; j < C; ++j) {
#pragma unroll
        for (int g = 0; g < G; ++g)
            raw[j][g] = load_raw_at<T, VEC>(ru, at_u + (unsigned int)(j * G + g) * row_bytes);
        rawg[j] = load_raw_at<T, VEC>(rg, at_h + (unsigned int)j * row_bytes);
    }
    const unsigned int ch = first + lane % CW;               // wave 0: a lane for each channel of the tile
    const bool act = ch < H, one = lane < CW && act;
    const float in0 = w == 0 && p.lt + 1 == a.n_lt && one && a.dlast ? a.dlast[(size_t)p.b * H + ch] : 0.0f;
    float before[VEC];                                       // the state in front of the tile
#pragma unroll
    for (int k = 0; k < VEC; ++k) before[k] = active ? a.ckpt[((size_t)p.b * a.n_lt + p.lt) * H + first + c0 + k] : 0.0f;

    // cf, ci and i: what lam is multiplied by for the gradients of the gates and of v (cf first without the state)
    float f[C][VEC], i[C][VEC], cf[C][VEC], ci[G == 3 ? C : 1][VEC], A[VEC], S[VEC], M[VEC], RA[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { A[k] = 1.0f; S[k] = M[k] = 0.0f; }
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const bool valid = t0 < p.rows - j;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float v = raw[j][G - 1].at(k);             // (zero behind the valid steps)
            float ff, om;
            sigmoid2(raw[j][0].at(k), &ff, &om);
            if constexpr (G == 3) {
                float ii, oi;
                sigmoid2(raw[j][1].at(k), &ii, &oi);
                ci[j][k] = v * (ii * oi);
                formed(ci[j][k]);
                i[j][k] = ii;
            } else {
                i[j][k] = om;
            }
            cf[j][k] = ff * om;
            formed(cf[j][k]);
            f[j][k] = valid ? ff : 1.0f;
            A[k] *= f[j][k];
            S[k] = fmaf(f[j][k], S[k], i[j][k] * v);
        }
    }
#pragma unroll
    for (int j = C - 1; j >= 0; --j)
#pragma unroll
        for (int k = 0; k < VEC; ++k) M[k] = f[j][k] * (rawg[j].at(k) + M[k]);
    if constexpr (sizeof(T) == 2)
#pragma unroll
        for (int j = 0; j < C; ++j) {
#pragma unroll
            for (unsigned k = 0; k < sizeof(rawg[j].w) / 4; ++k) {
                rawg[j].w[k] = unknown(rawg[j].w[k]);
                raw[j][G - 1].w[k] = unknown(raw[j][G - 1].w[k]);
            }
        }
#pragma unroll
    for (int k = 0; k < VEC; ++k) RA[k] = A[k] = factor(A[k]);
    // along time for the states, against it for the adjoint
#pragma unroll
    for (int d = LPR; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float a1 = __shfl_up(A[k], d, 64), s1 = __shfl_up(S[k], d, 64);
            const float a2 = __shfl_down(RA[k], d, 64), m2 = __shfl_down(M[k], d, 64);
            S[k] = fmaf(A[k], lane >= d ? s1 : 0.0f, S[k]);
            A[k] = factor(A[k] * (lane >= d ? a1 : 1.0f));
            M[k] = fmaf(RA[k], lane + d < 64 ? m2 : 0.0f, M[k]);
            RA[k] = factor(RA[k] * (lane + d < 64 ? a2 : 1.0f));
        }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        if (sg == SEG - 1) { s_a[w][c0 + k] = A[k]; s_s[w][c0 + k] = S[k]; }
        if (sg == 0) s_m[w][c0 + k] = M[k];
    }
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        if constexpr (SEG > 1) {
            const float a1 = __shfl_up(A[k], LPR, 64), s1 = __shfl_up(S[k], LPR, 64);
            const float a2 = __shfl_down(RA[k], LPR, 64), m2 = __shfl_down(M[k], LPR, 64);
            A[k] = sg ? a1 : 1.0f;
            S[k] = sg ? s1 : 0.0f;
            RA[k] = sg + 1 < SEG ? a2 : 1.0f;
            M[k] = sg + 1 < SEG ? m2 : 0.0f;
        } else {
            A[k] = RA[k] = 1.0f;
            S[k] = M[k] = 0.0f;
        }
    }
    if (w == 0 && lane < CW) s_in[lane] = in0;
    __syncthreads();
    const bool more = LOOK && p.lt > 0;
    word_t *rec = a.rec + ((size_t)p.chain * a.n_lt + p.lt) * (3 * CW);
    float ta = 1.0f, tm = 0.0f;
    if (w == 0 && lane < CW) {
#pragma unroll
        for (int q = W - 1; q >= 0; --q) { tm = fmaf(s_a[q][lane], tm, s_m[q][lane]); ta *= s_a[q][lane]; }
        ta = factor(ta);
        if (more && act && p.lt + 1 < a.n_lt) { put(rec + lane, ta, a.tag + 1); put(rec + CW + lane, tm, a.tag + 1); }
    }
    // the state in front of each of this thread's steps
    for (int q = 0; q < w; ++q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) before[k] = fmaf(s_a[q][c0 + k], before[k], s_s[q][c0 + k]);
#pragma unroll
    for (int k = 0; k < VEC; ++k) before[k] = fmaf(A[k], before[k], S[k]);
#pragma unroll
    for (int j = 0; j < C; ++j)
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float v = raw[j][G - 1].at(k);
            cf[j][k] *= G == 2 ? before[k] - v : before[k];
            formed(cf[j][k]);
            before[k] = fmaf(f[j][k], before[k], i[j][k] * v);
        }
    float pa[VEC], pm[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) { pa[k] = 1.0f; pm[k] = 0.0f; }
    for (int q = W - 1; q > w; --q)
#pragma unroll
        for (int k = 0; k < VEC; ++k) { pm[k] = fmaf(s_a[q][c0 + k], pm[k], s_m[q][c0 + k]); pa[k] *= s_a[q][c0 + k]; }
#pragma unroll
    for (int k = 0; k < VEC; ++k) pa[k] = factor(pa[k]);
    int found = -1, parity = 0;
    if constexpr (LOOK)
        if (p.lt + 1 < a.n_lt) found = look_back(s_seen, rec, 1, p.lt, a.n_lt, act, a.tag, a.spin_limit, &parity);
    auto entering = [&](int c, auto &v) {                    // the adjoint behind the tile
        if constexpr (LOOK)
            if (p.lt + 1 < a.n_lt) return carry_of(s_seen, found, parity, c, v);
#pragma unroll
        for (int k = 0; k < (int)(sizeof(v) / sizeof(v[0])); ++k) v[k] = s_in[c + k];
    };
    if (w == 0 && one) {
        float in1[1];
        entering(lane, in1);
        const float out = fmaf(ta, in1[0], tm);
        if (more) put(rec + 2 * CW + lane, out, a.tag + 2);
        if (a.dh0 && p.lt == 0) a.dh0[(size_t)p.b * H + ch] = out;
    }
    float m[VEC];
    entering(c0, m);
#pragma unroll
    for (int k = 0; k < VEC; ++k) m[k] = fmaf(RA[k], fmaf(pa[k], m[k], pm[k]), M[k]);

    const unsigned int at_out = unknown(at_u);
    const buf_rsrc rd = rsrc_of(static_cast<T *>(a.du) + row * G * H + first, extent(p.rows_all, G * H * es, first * es));
#pragma unroll
    for (int j = C - 1; j >= 0; --j) {
        const bool valid = t0 < p.rows - j;
        float o[G][VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float lam = rawg[j].at(k) + m[k];
            o[0][k] = valid ? lam * cf[j][k] : 0.0f;
            if constexpr (G == 3) o[1][k] = valid ? lam * ci[j][k] : 0.0f;
            o[G - 1][k] = valid ? lam * i[j][k] : 0.0f;
            m[k] = f[j][k] * lam;
        }
#pragma unroll
        for (int g = 0; g < G; ++g)
            store_at<T, VEC>(rd, at_out + (unsigned int)(j * G + g) * row_bytes, o[g]);
    }
}

// A few steps: a thread walks them for VEC channels, kBatch steps read at once.  One launch, no workspace; bound by latency: 32 x 1 x 1024 bf16
// 3.2 us in a graph (an empty kernel 1.75), 5.1 as a call.
template <typename T, int G, int VEC> __global__ __launch_bounds__(256) void gated_walk_kernel(const GatedArgs a)
{
    const int per_row = a.H / VEC;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    if (id >= (long long)a.B * per_row) return;
    const int b = (int)(id / per_row), c0 = (int)(id - (long long)b * per_row) * VEC;
    int len = a.L;
    if (a.lengths) {
        len = a.lengths[b];
        len = len < 0 ? 0 : len > a.L ? a.L : len;
    }
    const T *u = static_cast<const T *>(a.u) + (size_t)b * a.L * G * a.H + c0;
    T *h = static_cast<T *>(a.h) + (size_t)b * a.L * a.H + c0;
    using E = typename RawVec<T, VEC>::type;
    float x[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
        x[k] = a.h0 ? a.h0[(size_t)b * a.H + c0 + k] : 0.0f;
        if (a.ckpt) a.ckpt[(size_t)b * a.H + c0 + k] = x[k];
    }
    for (int t = 0; t < a.L; t += kBatch) {
        E r[kBatch][G];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (t + j < len)
#pragma unroll
                for (int g = 0; g < G; ++g) r[j][g] = *reinterpret_cast<const E *>(u + ((size_t)(t + j) * G + g) * a.H);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (t + j >= a.L) break;
            float o[VEC] = {};
            if (t + j < len) {
                float in[G][VEC];
#pragma unroll
                for (int g = 0; g < G; ++g) raw_to_float<T, VEC>(r[j][g], in[g]);
#pragma unroll
                for (int k = 0; k < VEC; ++k) {
                    float f, i;
                    sigmoid2(in[0][k], &f, &i);
                    if constexpr (G == 3) i = fast_sigmoid(in[1][k]);
                    x[k] = fmaf(f, x[k], i * in[G - 1][k]);
                    o[k] = x[k];
                }
            }
            store_vec<VEC>(h + (size_t)(t + j) * a.H, o);
        }
    }
    if (a.last)
#pragma unroll
        for (int k = 0; k < VEC; ++k) a.last[(size_t)b * a.H + c0 + k] = x[k];
}

__global__ __launch_bounds__(256) void gated_clear_kernel(ulonglong2 *p, size_t n)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = make_ulonglong2(0, 0);
}

// ------------------------------------------------------------------ host
constexpr size_t kCtrl = (size_t)kQueues * kQueuePitch * sizeof(unsigned int);
struct Shape {
    int cw, n_lt, groups;
    long long chains, tiles;
    size_t bytes;                 // control block, and carry records where there is more than one tile along L
};

// 16 channels x 512 steps in place of 64 x 128.  Rows that leave most of a wide tile idle: forward 8 x 21715 x 16 bf16 26 -> 9 us, 64 x
// 20000 x 16 fp32, three gates 134 -> 67, 64 x 2000 x 32 13 -> 9; with 38 channels 59 -> 76.  And sequences that one such tile
// holds, which nobody then waits for, as long as the device holds them all at once: 4 x 469 x 464 5.9 -> 4.4, 64 x 300 x 64 6.5 ->
// 4.6; with twice as many 8.5 -> 12.5 (8 x 400 x 1000: a row's 32 bytes come with lines of 128).  Backward alike.
bool narrow_tiles(int B, int L, int H)
{
    const long long chains = (long long)B * ((H + kNarrow - 1) / kNarrow);
    return L > tile_steps(kWide) && (H <= 32 || (L <= tile_steps(kNarrow) && chains <= 256));
}
bool shape_of(int dtype, int B, int L, int H, int G, Shape *s)
{
    if ((dtype != PARARNN_F32 && dtype != PARARNN_BF16) || B < 1 || L < 1 || H < 1 || (G != 2 && G != 3)) return false;
    auto cut = [&](int cw) {
        s->cw = cw;
        s->n_lt = (int)(((long long)L + tile_steps(cw) - 1) / tile_steps(cw));
        s->groups = (H + cw - 1) / cw;
        s->chains = (long long)B * s->groups;
        s->tiles = s->chains * s->n_lt;
    };
    cut(narrow_tiles(B, L, H) ? kNarrow : kWide);
    s->bytes = s->n_lt > 1 ? kCtrl + (size_t)s->tiles * 3 * s->cw * sizeof(word_t) : 256;
    return true;
}

// Row offsets of a tile are 32-bit (128 steps x 3 gates x 4 bytes x 2^20 channels; 512 steps of up to 4096), and so are the numbers of a launch's threads (512 of
// a tile; one for each channel of a walk).
bool size_ok(const Shape &s, int B, int H)
{
    return H <= (1 << 20) && s.tiles < (1ll << 23) && (long long)B * H < (1ll << 32) - 256;
}

// Whether rows can be taken n elements at a time
bool rows_of(int n, int H, int dtype, std::initializer_list<const void *> ptrs)
{
    uintptr_t m = 0;
    for (const void *p : ptrs) m |= (uintptr_t)p;
    return m % ((dtype == PARARNN_BF16 ? 2 : 4) * n) == 0 && H % n == 0;
}

// A look at 32 tiles in place of 8: few and long chains, whose tiles are on the device all at once and wait for the chain.  4 chains of 512
// tiles: 92 -> 48 us (forward, 1 x 65536 x 256 bf16), 86 -> 51 (backward); 16 chains of 32 are level, of 64 lose 23 -> 26 and
// 29 -> 32 (2 x 8192 x 512), 64 of 128 107 -> 120 (2 x 16384 x 2048).
bool wide_look(const GatedArgs &a) { return a.chains <= 8 && a.n_lt > kWaves; }

hipError_t launch_clear(void *ws, size_t bytes, hipStream_t st)
{
    const size_t n = bytes / 16;
    const size_t blocks = std::min<size_t>((n + 255) / 256, (size_t)std::max(1, device_cu_count()) * 8);
    hipLaunchKernelGGL(gated_clear_kernel, dim3((unsigned)blocks), dim3(256), 0, st, static_cast<ulonglong2 *>(ws), n);
    return hipGetLastError();
}

// LK: 0 for a single tile along L, of TT steps
template <typename T, int G, int VEC, int CW, int LK, int TT = tile_steps(CW)> void launch_tiles(const GatedArgs &a, bool backward, hipStream_t st)
{
    constexpr int C = TT / (kWaves * (64 * VEC / CW));
    const dim3 grid((unsigned)a.chains * a.n_lt), block(64 * kWaves);
    if (backward) hipLaunchKernelGGL((gated_backward_kernel<T, G, VEC, CW, kWaves, C, LK>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((gated_forward_kernel<T, G, VEC, CW, kWaves, C, LK>), grid, block, 0, st, a);
}
template <typename T, int G> hipError_t launch_tiles_of(const GatedArgs &a, int cw, bool backward, bool pairs, hipStream_t st)
{
    const int look = a.n_lt == 1 ? 0 : wide_look(a) ? 4 : 1;
#define PARARNN_GATED(VEC)                                                    \
    do {                                                                      \
        if (cw == kNarrow && look == 0) launch_tiles<T, G, VEC, kNarrow, 0>(a, backward, st);        \
        else if (cw == kNarrow) launch_tiles<T, G, VEC, kNarrow, 1>(a, backward, st);                 \
        else if (look == 0 && a.L <= 32) launch_tiles<T, G, VEC, kWide, 0, 32>(a, backward, st);      \
        else if (look == 0 && a.L <= 64) launch_tiles<T, G, VEC, kWide, 0, 64>(a, backward, st);      \
        else if (look == 0) launch_tiles<T, G, VEC, kWide, 0>(a, backward, st);                       \
        else if (look == 1) launch_tiles<T, G, VEC, kWide, 1>(a, backward, st);                       \
        else launch_tiles<T, G, VEC, kWide, 4>(a, backward, st);                                      \
    } while (0)
    if (pairs) PARARNN_GATED(2);
    else PARARNN_GATED(1);
#undef PARARNN_GATED
    return hipGetLastError();
}

int launch_of(int dtype, int G, const GatedArgs &a, int cw, bool backward, bool pairs, hipStream_t st)
{
    const hipError_t e = dtype == PARARNN_BF16
                             ? (G == 2 ? launch_tiles_of<unsigned short, 2>(a, cw, backward, pairs, st) : launch_tiles_of<unsigned short, 3>(a, cw, backward, pairs, st))
                             : (G == 2 ? launch_tiles_of<float, 2>(a, cw, backward, pairs, st) : launch_tiles_of<float, 3>(a, cw, backward, pairs, st));
    return e == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
}

template <typename T, int G> hipError_t launch_walk(const GatedArgs &a, bool pairs, hipStream_t st)
{
    const long long n = (long long)a.B * (a.H / (pairs ? 2 : 1));
    const unsigned blocks = (unsigned)((n + 255) / 256);
    if (pairs) hipLaunchKernelGGL((gated_walk_kernel<T, G, 2>), dim3(blocks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((gated_walk_kernel<T, G, 1>), dim3(blocks), dim3(256), 0, st, a);
    return hipGetLastError();
}

// Control block and carry records for the call: cleared, unless the library knows what an earlier call left in this workspace.
// False: a launch failed.
bool take_workspace(void *workspace, const Shape &s, unsigned int spin_limit, GatedArgs *a, hipStream_t st)
{
    char *ws = static_cast<char *>(workspace);
    a->ticket = reinterpret_cast<unsigned int *>(ws);
    a->rec = reinterpret_cast<word_t *>(ws + kCtrl);
    a->queues = (int)std::min<long long>(kQueues, s.chains);
    a->spin_limit = spin_limit;
    // FNV-1a; what the words are used for depends on the tiles alone
    unsigned long long sig = 1469598103934665603ull;
    for (unsigned long long v : {0x6761746564ull, (unsigned long long)s.n_lt, (unsigned long long)s.chains, (unsigned long long)s.cw})
        for (int i = 0; i < 8; ++i) sig = (sig ^ (v >> (8 * i) & 0xff)) * 1099511628211ull;
    bool fill = true;
    a->tag = workspace_epoch(workspace, sig ? sig : 1, st, &fill);
    return !fill || launch_clear(ws, s.bytes, st) == hipSuccess;
}

// A walk takes 2 us and 0.1 to 0.2 for a step; a tile of 32 steps 2.5 to 2.8 us, from 30000 channels on more: 65536 (B x H) 4.5 to 5.6, 262144
// 15 to 20, whatever there is of its steps.  Channels, steps at which both took the same (bf16 two gates / fp32 three): 512 6 / 4, 8192
// 6 / 5, 65536 16 / 14, 262144 beyond 48 (a tile of 64 there) / 36.
bool walked(int B, int L, int H) { return L <= 48 && L <= 5 + (long long)B * H / 6500; }

bool misaligned(const void *p, size_t n) { return (uintptr_t)p % n != 0; }

}  // namespace

size_t gated_workspace_bytes(int dtype, int B, int L, int H, int G)
{
    Shape s;
    return shape_of(dtype, B, L, H, G, &s) && size_ok(s, B, H) ? s.bytes : 0;
}

size_t gated_checkpoint_bytes(int dtype, int B, int L, int H, int G)
{
    Shape s;
    return shape_of(dtype, B, L, H, G, &s) && size_ok(s, B, H) ? (size_t)B * s.n_lt * H * sizeof(float) : 0;
}

int gated_forward(int dtype, const void *u, const float *h0, const int *lengths, int B, int L, int H, int G, void *h,
                  float *h_last, float *checkpoints, void *workspace, size_t workspace_bytes, unsigned int spin_limit, hipStream_t st)
{
    Shape s;
    if (!shape_of(dtype, B, L, H, G, &s) || !u || !h || (!workspace && s.n_lt > 1) || misaligned(workspace, 256)) return PARARNN_INVALID_ARG;
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if (misaligned(u, es) || misaligned(h, es) || misaligned(h0, 4) || misaligned(lengths, 4) || misaligned(h_last, 4) ||
        misaligned(checkpoints, 4))
        return PARARNN_INVALID_ARG;
    if (!size_ok(s, B, H)) return PARARNN_UNSUPPORTED;
    if (s.n_lt > 1 && workspace_bytes < s.bytes) return PARARNN_WORKSPACE_TOO_SMALL;
    GatedArgs a = {};
    a.u = u; a.h0 = h0; a.lengths = lengths; a.h = h; a.last = h_last; a.ckpt = checkpoints;
    a.B = B; a.L = L; a.H = H; a.n_lt = s.n_lt; a.groups = s.groups; a.chains = (int)s.chains;
    if (walked(B, L, H)) {
        const bool pairs = rows_of(2, H, dtype, {u, h});
        const hipError_t e = dtype == PARARNN_BF16 ? (G == 2 ? launch_walk<unsigned short, 2>(a, pairs, st) : launch_walk<unsigned short, 3>(a, pairs, st))
                                                   : (G == 2 ? launch_walk<float, 2>(a, pairs, st) : launch_walk<float, 3>(a, pairs, st));
        return e == hipSuccess ? PARARNN_OK : PARARNN_HIP_ERROR;
    }
    if (s.n_lt > 1 && !take_workspace(workspace, s, spin_limit, &a, st)) {
        workspace_forget(workspace);
        return PARARNN_HIP_ERROR;
    }
    const int rc = launch_of(dtype, G, a, s.cw, false, rows_of(2, H, dtype, {u, h}), st);
    if (rc != PARARNN_OK && s.n_lt > 1) workspace_forget(workspace);
    return rc;
}

int gated_backward(int dtype, const void *u, const float *checkpoints, const int *lengths, const void *dL_dh,
                   const float *dL_dlast, int B, int L, int H, int G, void *dL_du, float *dL_dh0, void *workspace,
                   size_t workspace_bytes, unsigned int spin_limit, hipStream_t st)
{
    Shape s;
    if (!shape_of(dtype, B, L, H, G, &s) || !u || !checkpoints || !dL_du || (!workspace && s.n_lt > 1) || misaligned(workspace, 256))
        return PARARNN_INVALID_ARG;
    const size_t es = dtype == PARARNN_BF16 ? 2 : 4;
    if (misaligned(u, es) || misaligned(dL_dh, es) || misaligned(dL_du, es) || misaligned(checkpoints, 4) || misaligned(lengths, 4) ||
        misaligned(dL_dlast, 4) || misaligned(dL_dh0, 4))
        return PARARNN_INVALID_ARG;
    if (!size_ok(s, B, H)) return PARARNN_UNSUPPORTED;
    if (s.n_lt > 1 && workspace_bytes < s.bytes) return PARARNN_WORKSPACE_TOO_SMALL;
    GatedArgs a = {};
    a.u = u; a.lengths = lengths; a.ckpt = const_cast<float *>(checkpoints); a.g = dL_dh; a.dlast = dL_dlast; a.du = dL_du; a.dh0 = dL_dh0;
    a.B = B; a.L = L; a.H = H; a.n_lt = s.n_lt; a.groups = s.groups; a.chains = (int)s.chains;
    if (s.n_lt > 1 && !take_workspace(workspace, s, spin_limit, &a, st)) {
        workspace_forget(workspace);
        return PARARNN_HIP_ERROR;
    }
    const int rc = launch_of(dtype, G, a, s.cw, true, rows_of(2, H, dtype, {u, dL_dh, dL_du}), st);
    if (rc != PARARNN_OK && s.n_lt > 1) workspace_forget(workspace);
    return rc;
}

}  // namespace pararnn
