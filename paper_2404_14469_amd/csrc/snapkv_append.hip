// Appending new tokens' keys and values to a paged cache, keys and queries rotated by their positions on the way.
//
// Rotation of a row x by position t, over its first R elements: pairs (x_i, x_{i + R/2}) (or, interleaved, (x_2i, x_2i+1)),
// i < R/2, become (a cos - b sin, b cos + a sin) with the cosine and sine of row t of the caller's fp32 tables.  Products
// and sums are fp32, rounded to the storage type once.
//
// Bound by HBM: every row is read once and written once or twice.  A wave owns a token, so the search for its
// sequence, its row, page and position are done once for all heads, and the token's cosines and sines stay in registers:
// a lane keeps the same 32 bytes of a head (its unit) in every head that it meets, 8 heads of 128 two-byte elements at a
// time.  The two 16-byte pieces of a unit are the two partners of eight pairs (halves) or four pairs each (interleaved).
// Fewer than 1024 tokens are shared out by head groups instead, so that a step's few tokens meet more waves.  65319 tokens
// of 32/32 heads, rotated, queries too, keys twice: 3.8 GB in 735 us, 5.1 TB/s; 8 tokens of 32/8 heads 3.7 us.
#include "snapkv_sequence.h"
#include "snapkv_serve.h"

namespace snapkv {
namespace {

struct a_bf16 {
    typedef __attribute__((ext_vector_type(8))) __bf16 piece;
    static constexpr int N = 8;
};
struct a_f16 {
    typedef __attribute__((ext_vector_type(8))) _Float16 piece;
    static constexpr int N = 8;
};
struct a_f32 {
    typedef __attribute__((ext_vector_type(4))) float piece;
    static constexpr int N = 4;
};

template <typename T, int D, bool INTERLEAVED>
__global__ __launch_bounds__(256) void append_paged(const AppendArgs A) {
    typedef typename T::piece piece;
    constexpr int N = T::N, U = D / (2 * N);          // elements of a piece; units of a head
    constexpr int HW = 64 / U;                        // heads that a wave meets at a time
    constexpr int E = sizeof(piece) / N;
    const int lane = threadIdx.x & 63;
    const unsigned item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(item / (unsigned)A.parts), part = (int)(item % (unsigned)A.parts);
    if (t >= A.T) return;
    int b = t, first = t;
    if (A.cu) {
        b = sequence_of(A.cu, A.B, t, lane);
        if (b >= A.B) return;                         // behind the last sequence
        first = A.cu[b];
        if (first > t) return;                        // before the first
    }
    int64_t row = (int64_t)A.starts[b] + (t - first);
    int64_t slot = -1;
    if (row >= 0 && row < A.table_rows) {
        const int64_t pg = (unsigned)row / (unsigned)A.page;   // (a start and a token's place are below 2^31 each)
        const int64_t at = A.table[(int64_t)b * A.table_stride + pg];
        if (at >= 0 && at < A.pages) slot = at * A.page + (row - pg * A.page);
    }
    // the unit's two pieces: partners of the rotation, or neighbours in what is not rotated
    const int u = lane % U, hl = lane / U;
    const int nr = A.rot / (2 * N);
    const bool turn = u < nr;
    const int c0 = (INTERLEAVED || !turn) ? 2 * u : u, c1 = (INTERLEAVED || !turn) ? 2 * u + 1 : u + nr;
    float cs[N] = {}, sn[N] = {};
    if (turn) {
        int64_t pos = A.positions ? (int64_t)A.positions[t] : row;
        pos = pos < 0 ? 0 : (pos >= A.npos ? A.npos - 1 : pos);
        const float4* cr = reinterpret_cast<const float4*>(A.cos + pos * (A.rot / 2) + N * u);
        const float4* sr = reinterpret_cast<const float4*>(A.sin + pos * (A.rot / 2) + N * u);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            *reinterpret_cast<float4*>(cs + 4 * i) = cr[i];
            *reinterpret_cast<float4*>(sn + 4 * i) = sr[i];
        }
    }
    const int heads = A.Hq + 2 * A.Hkv;               // query heads, key heads, value heads
    for (int h = part * HW + hl; h < heads; h += A.parts * HW) {
        const bool is_q = h < A.Hq, is_k = !is_q && h < A.Hq + A.Hkv;
        const int hh = is_q ? h : (is_k ? h - A.Hq : h - A.Hq - A.Hkv);
        const char* src = is_q ? A.q + t * A.q_rs + hh * A.q_hs : (is_k ? A.k + t * A.k_rs + hh * A.k_hs : A.v + t * A.v_rs + hh * A.v_hs);
        piece x0 = reinterpret_cast<const piece*>(src)[c0], x1 = reinterpret_cast<const piece*>(src)[c1];
        if (turn && (is_q || is_k)) {
            piece y0, y1;
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < N; i += 2) {
                    const float a0 = (float)x0[i], b0 = (float)x0[i + 1], a1 = (float)x1[i], b1 = (float)x1[i + 1];
                    const float p0 = cs[i / 2], q0 = sn[i / 2], p1 = cs[N / 2 + i / 2], q1 = sn[N / 2 + i / 2];
                    y0[i] = a0 * p0 - b0 * q0;
                    y0[i + 1] = b0 * p0 + a0 * q0;
                    y1[i] = a1 * p1 - b1 * q1;
                    y1[i + 1] = b1 * p1 + a1 * q1;
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float a = (float)x0[i], c = (float)x1[i];
                    y0[i] = a * cs[i] - c * sn[i];
                    y1[i] = c * cs[i] + a * sn[i];
                }
            }
            x0 = y0;
            x1 = y1;
        }
        if (is_q || (is_k && A.k_out)) {
            char* o = is_q ? A.q_out + t * A.qo_rs + hh * A.qo_hs : A.k_out + t * A.ko_rs + hh * A.ko_hs;
            reinterpret_cast<piece*>(o)[c0] = x0;
            reinterpret_cast<piece*>(o)[c1] = x1;
        }
        if (!is_q && slot >= 0) {
            char* o = (is_k ? A.k_pages : A.v_pages) + (slot * A.Hkv + hh) * (int64_t)(D * E);
            reinterpret_cast<piece*>(o)[c0] = x0;
            reinterpret_cast<piece*>(o)[c1] = x1;
        }
    }
}

}  // namespace

hipError_t launch_append(int dtype, int D, bool interleaved, AppendArgs A, hipStream_t st) {
    const int units = D * (dtype == 1 ? 4 : 2) / 32, per = 64 / units;
    const int heads = A.Hq + 2 * A.Hkv, groups = (heads + per - 1) / per;
    A.parts = A.T < 1024 ? groups : 1;
    const int64_t items = A.T * A.parts;
    const dim3 grid((unsigned)((items + 3) / 4)), block(256);
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, st, A); };
    auto form = [&](auto t, auto d) {
        typedef decltype(t) T;
        constexpr int DD = decltype(d)::value;
        interleaved ? launch(append_paged<T, DD, true>) : launch(append_paged<T, DD, false>);
    };
    typedef std::integral_constant<int, 64> d64;
    typedef std::integral_constant<int, 128> d128;
    if (dtype == 0) D == 128 ? form(a_bf16{}, d128{}) : form(a_bf16{}, d64{});
    else if (dtype == 1) D == 128 ? form(a_f32{}, d128{}) : form(a_f32{}, d64{});
    else if (dtype == 2) D == 128 ? form(a_f16{}, d128{}) : form(a_f16{}, d64{});
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace snapkv
