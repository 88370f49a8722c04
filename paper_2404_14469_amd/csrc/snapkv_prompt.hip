// Causal attention over whole prompts packed one behind the other, with grouped heads and the rows' log-sum-exp:
//
//   out[i, h] = sum_{j <= i} softmax_j(q[i, h] . k[j, h / g] / sqrt(D)) v[j, h / g],
//   lse[h, i] = log sum_{j <= i} exp(q[i, h] . k[j, h / g] / sqrt(D)),      i, j within one prompt.
//
// One pass over the keys with the running maximum and sum of a softmax, in base two; 4 D operations per visible pair make
// the matrix units the bound of all but the shortest prompts.
//
// Work split.  A workgroup takes a tile of query rows of one head, each wave 32 of them, and walks the keys in tiles of 64
// that all its waves share through LDS.
//
// MFMA layout (32x32x16, 64 lanes): lane l supplies row (left operand) or column (right operand) l%32 and contraction
// elements 8*(l/32) .. +7; accumulator register r of lane l is row 8*(r/4) + 4*(l/32) + r%4, column l%32.
//
//   logits^T = K Q^T: a lane gets 16 logits of ONE query per 32 keys, so the softmax is arithmetic within the lane and one
//     exchange with the lane that has the other half of the keys; the maximum, the sum and the factor that rescales the
//     output are one register each.
//   out^T = V^T P^T: contraction element e of lane l stands for key 8*(e/4) + 4*(l/32) + e%4 of 16, which is where the
//     logits left that key's probability: P never moves between lanes.  V^T comes from LDS by the transposing read (a lane
//     gets four keys of one column).
//
// The probabilities enter the last product rounded to the storage type, as its operand must be: each is off by at most half
// a step (bf16 2^-8, fp16 2^-11, relative; the fp16 ones are taken 2^8 times as large, so those down to 2^-22 of the
// largest are normal numbers), which adds to an output about what its own rounding does.  Their sum is taken in fp32 from
// the unrounded values.
#include "snapkv_internal.h"

#include <cmath>

namespace snapkv {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 pbf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 pf16x8;
typedef __attribute__((ext_vector_type(16))) float pfx16;
typedef __attribute__((ext_vector_type(4))) short ps16x4;

struct p_bf16 {
    typedef __bf16 elem;
    typedef pbf16x8 frag;
    static constexpr float kShift = 0.f;
};
struct p_f16 {
    typedef _Float16 elem;
    typedef pf16x8 frag;
    static constexpr float kShift = 7.f;
};
__device__ __forceinline__ pfx16 mma32(pbf16x8 a, pbf16x8 b, pfx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ pfx16 mma32(pf16x8 a, pf16x8 b, pfx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kKeys = 64;      // keys of a tile

typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) ps16x4* lds_s16x4;

// Which 16-byte piece of its row an LDS slot of a tile holds: the pieces of a row are permuted so that the lanes of a read,
// which go down the rows, meet all banks.
template <int D> __device__ __forceinline__ int k_slot(int row, int piece) { return piece ^ (row & (D / 8 - 1)); }
template <int D> __device__ __forceinline__ int v_slot(int row, int piece) { return piece ^ ((row & (D / 32 - 1)) << 2); }

// The tile of rank `rank` in descending order of its number of visible keys: sequence and row tile, or false.  A sequence
// of n row tiles has one of each cost 1 .. n; F(c) counts the tiles of cost c and more.
template <int ROWS>
__device__ bool locate(const PromptArgs& A, int rank, int lane, int& seq, int& tile, int& begin, int& len) {
    auto span = [&](int b, int& s0, int& n) {
        s0 = 0;
        n = 0;
        if (b < A.B) {
            const int a = A.cu[b], e = A.cu[b + 1];
            s0 = a < 0 ? 0 : a;
            const int e1 = e > A.T ? (int)A.T : e;
            n = e1 > s0 ? e1 - s0 : 0;
        }
    };
    int most = 0, total = 0;
    for (int b0 = 0; b0 < A.B; b0 += 64) {
        int s0, n;
        span(b0 + lane, s0, n);
        const int nt = (n + ROWS - 1) / ROWS;
        int x = nt, t = nt;
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            x = max(x, __shfl_xor(x, d));
            t += __shfl_xor(t, d);
        }
        most = max(most, x);
        total += t;
    }
    if (rank >= total) return false;
    auto count = [&](int c) {                              // F(c)
        int t = 0;
        for (int b0 = 0; b0 < A.B; b0 += 64) {
            int s0, n;
            span(b0 + lane, s0, n);
            const int nt = (n + ROWS - 1) / ROWS;
            t += max(0, nt - c + 1);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) t += __shfl_xor(t, d);
        return t;
    };
    int lo = 1, hi = most + 1;                             // F(lo) > rank >= F(hi)
    while (hi - lo > 1) {
        const int c = (lo + hi) / 2;
        if (count(c) > rank) lo = c; else hi = c;
    }
    int within = rank - count(lo + 1);
    for (int b0 = 0; b0 < A.B; b0 += 64) {
        int s0, n;
        span(b0 + lane, s0, n);
        const unsigned long long has = __ballot((n + ROWS - 1) / ROWS >= lo);
        const int here = __popcll(has);
        if (within < here) {
            unsigned long long rest = has;
            for (int i = 0; i < within; ++i) rest &= rest - 1;
            const int l = __ffsll((long long)rest) - 1;
            seq = b0 + l;
            begin = __builtin_amdgcn_readlane(s0, l);
            len = __builtin_amdgcn_readlane(n, l);
            tile = lo - 1;
            return true;
        }
        within -= here;
    }
    return false;
}

// The other half of the wave: lane l gets lane l ^ 32's value.
__device__ __forceinline__ float other_half(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? y[0] : y[1]);
}

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void prompt_attn(const PromptArgs A) {
    typedef typename T::elem elem;
    typedef typename T::frag frag;
    constexpr int ROWS = WAVES * 32;            // query rows of a workgroup
    constexpr int ROW = D * 2, PIECES = D / 8;  // bytes and 16-byte pieces of a row
    constexpr int NC = D / 16, ND = D / 32;     // contraction steps of a logit; 32-column blocks of the output
    __shared__ __align__(16) char s_k0[kKeys * ROW], s_v0[kKeys * ROW], s_k1[kKeys * ROW], s_v1[kKeys * ROW];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, h2 = lane >> 5;

    // KV heads are dealt to the XCDs (workgroup i runs on XCD i % 8), so the workgroups that read a head share an L2
    const int m8 = (A.Hkv & 7) == 0 ? 8 : ((A.Hkv & 3) == 0 ? 4 : ((A.Hkv & 1) == 0 ? 2 : 1));
    const int rest = blockIdx.x / m8;
    const int per = A.ranks * A.g;
    const int kvh = blockIdx.x % m8 + m8 * (rest / per);
    const int rank = rest % per / A.g, hq = kvh * A.g + rest % A.g;

    int seq, tile, begin, len;
    if (!locate<ROWS>(A, rank, lane, seq, tile, begin, len)) return;

    const int row0 = tile * ROWS + wave * 32;               // the wave's first query row within the prompt
    const int row = row0 + n32, row_in = row < len ? row : len - 1;
    frag qf[NC];
    {
        const char* qr = A.q + (int64_t)(begin + row_in) * A.q_rs + (int64_t)hq * A.q_hs + h2 * 16;
#pragma unroll
        for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const frag*>(qr + 32 * c);
    }
    float m = -INFINITY, lsum = 0.f;
    pfx16 acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    const char* kh = A.k + (int64_t)kvh * A.k_hs + (int64_t)begin * A.k_rs;
    const char* vh = A.v + (int64_t)kvh * A.v_hs + (int64_t)begin * A.v_rs;
    const int last = min(len, (tile + 1) * ROWS) - 1;        // the last key any of the tile's rows sees
    const int ntiles = last / kKeys + 1;
    constexpr int PER = kKeys * PIECES / 64;                 // 1 KB loads of a tile
    auto load = [&](int kt, char* dk, char* dv) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < PER / WAVES; ++i) {
            const int at = (i * WAVES + wave) * 64;
            const int r = (at + lane) / PIECES, s = (at + lane) % PIECES;
            const int key = min(kt * kKeys + r, len - 1);
            __builtin_amdgcn_global_load_lds((global_ptr)(kh + (int64_t)key * A.k_rs + k_slot<D>(r, s) * 16), (lds_ptr)(dk + at * 16), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((global_ptr)(vh + (int64_t)key * A.v_rs + v_slot<D>(r, s) * 16), (lds_ptr)(dv + at * 16), 16, 0, 0);
        }
    };
    auto step = [&](int kt, const char* s_k, const char* s_v) __attribute__((always_inline)) {
        if (kt * kKeys > row0 + 31) return;                  // all of it lies behind the wave's rows
        pfx16 x[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[kb][r] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int kr = 32 * kb + n32;
                const frag kf = *reinterpret_cast<const frag*>(s_k + kr * ROW + k_slot<D>(kr, 2 * c + h2) * 16);
                x[kb] = mma32(kf, qf[c], x[kb]);
            }
        }
        if (kt * kKeys + kKeys - 1 > row0) {                 // keys behind a row are hidden from it (and those behind the prompt)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (kt * kKeys + 32 * kb + 8 * (r / 4) + 4 * h2 + r % 4 > row) x[kb][r] = -INFINITY;
        }
        float top = x[0][0];
#pragma unroll
        for (int r = 1; r < 32; ++r) top = fmaxf(top, x[r / 16][r % 16]);
        top = fmaxf(top, other_half(top)) * A.scale2;        // finite in the first tile: it holds the prompt's key 0
        // The shift of the exponentials need not be the maximum itself: it is moved, and sums and outputs rescaled, only
        // when some row of the wave has outgrown it by 2^8
        if (__any(top > m + 8.f)) {
            const float mn = fmaxf(m, top);
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            lsum *= alpha;
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
        }
        float sum = 0.f;
        frag pf[4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[kb][r], A.scale2, T::kShift - m));
                sum += p;
                pf[2 * kb + r / 8][r % 8] = (elem)p;
            }
        lsum += sum;
#pragma unroll
        for (int j = 0; j < 4; ++j) {                        // 16 keys
            const int kr = 16 * j + 4 * h2 + (lane & 15) / 4;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const int piece = 4 * i + 2 * ((lane >> 4) & 1) + (lane & 3) / 2;
                const char* a0 = s_v + kr * ROW + v_slot<D>(kr, piece) * 16 + (lane & 1) * 8;
                const char* a1 = s_v + (kr + 8) * ROW + v_slot<D>(kr + 8, piece) * 16 + (lane & 1) * 8;
                const ps16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)a0);
                const ps16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)a1);
                const frag vf = __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                acc[i] = mma32(vf, pf[j], acc[i]);
            }
        }
    };
    load(0, s_k0, s_v0);
    for (int kt = 0;;) {
        __syncthreads();                                     // this tile has arrived, the other buffer has been read
        if (kt + 1 < ntiles) load(kt + 1, s_k1, s_v1);
        step(kt, s_k0, s_v0);
        if (++kt >= ntiles) break;
        __syncthreads();
        if (kt + 1 < ntiles) load(kt + 1, s_k0, s_v0);
        step(kt, s_k1, s_v1);
        if (++kt >= ntiles) break;
    }
    lsum += other_half(lsum);
    if (row < len) {
        const float inv = 1.f / lsum;
        elem* o = reinterpret_cast<elem*>(A.out) + ((int64_t)(begin + row) * A.Hq + hq) * D + 4 * h2;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                typedef __attribute__((ext_vector_type(4))) elem elem4;
                elem4 y;
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = (elem)(acc[i][4 * r4 + r] * inv);
                *reinterpret_cast<elem4*>(o + 32 * i + 8 * r4) = y;
            }
        if (A.lse && h2 == 0)
            A.lse[(int64_t)hq * A.T + begin + row] = (m - T::kShift + __builtin_amdgcn_logf(lsum)) * 0.6931471805599453f;
    }
}

}  // namespace

hipError_t launch_prompt(int dtype, int D, PromptArgs A, hipStream_t st) {
    A.scale2 = (float)(1.4426950408889634 / std::sqrt((double)D));
    constexpr int WAVES = 4, ROWS = WAVES * 32;
    A.ranks = (int)(A.T / ROWS) + A.B;                       // every prompt has at most one tile that is not full
    const int64_t groups = (int64_t)A.ranks * A.Hq;
    if (groups >= (int64_t)1 << 31) return hipErrorInvalidValue;
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(WAVES * 64), 0, st, A); };
    if (dtype == 0 && D == 128) launch(prompt_attn<p_bf16, 128, WAVES>);
    else if (dtype == 0 && D == 64) launch(prompt_attn<p_bf16, 64, WAVES>);
    else if (dtype == 2 && D == 128) launch(prompt_attn<p_f16, 128, WAVES>);
    else if (dtype == 2 && D == 64) launch(prompt_attn<p_f16, 64, WAVES>);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace snapkv
