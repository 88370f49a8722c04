// Microscaled paged caches: rows quantised as they are written, keys rotated by their positions on the way, and read back.
//
// A row of D values lies in blocks of 32.  With A a block's largest magnitude and M the largest value of the element type (e4m3
// 448, e2m1 6), e is the smallest integer with A <= M 2^e, at least -117; the block's byte is e + 127 and an element's code the
// nearest value to x 2^-e, ties to the even code.  A code times 2^e is a bfloat16 number then, subnormal ones of e4m3 among
// them (2^-9 2^-117 is the smallest normal one).  A block with an infinity or NaN has byte 255 and codes of zero and reads as NaN.
//
// A code jumps at the border between two values, so a key is rotated in 64 bits, where products of its 24 bits at most are
// exact, and brought to float32 with its last bit set where anything was lost: what is rounded once more from there, to
// 4 bits or 2, is rounded as the 64-bit value would be; so is the keys' second copy in bfloat16 and fp16, and in float32 it is the 64-bit value
// rounded to nearest.  Queries are rotated in float32 and rounded once.
//
// Both ways are bound by memory.  65319 tokens of 32 heads in 4 bits: written, with queries rotated, in 471 us (2.46 GB, 5.2 TB/s; a copy
// reaches 5.1), read back in 258 (1.35 GB, 5.3 TB/s).  32749 rows of 8 heads in 8 bits read back in 31.8 us of a call (203 MB).  Eight rows: 5.0 and 4.0 us,
// a launch's latency.
#include "snapkv_sequence.h"
#include "snapkv_serve.h"

#include <type_traits>

namespace snapkv {
namespace {

typedef __attribute__((ext_vector_type(2))) float fx2;

struct m_bf16 {
    typedef __bf16 elem;
    static constexpr int N = 8;
};
struct m_f16 {
    typedef _Float16 elem;
    static constexpr int N = 8;
};
struct m_f32 {
    typedef float elem;
    static constexpr int N = 4;
};
template <typename T> using piece_of = __attribute__((ext_vector_type(T::N))) typename T::elem;

// CACHE 1: e4m3 codes of 8 bits; 2: e2m1 codes of 4, two to a byte.
template <int CACHE> struct mx;
template <> struct mx<1> {
    static constexpr int kTop = 8;                    // exponent of the largest value, and its fraction's bits
    static constexpr unsigned kFraction = 0x600000u;
};
template <> struct mx<2> {
    static constexpr int kTop = 2;
    static constexpr unsigned kFraction = 0x400000u;
};

// N codes of one piece; y is within the element type's range.
template <int N> __device__ __forceinline__ void store_codes(mx<1>, char* row, int at, const float* y) {
    unsigned w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], lo, true);
    }
    if constexpr (N == 8) *reinterpret_cast<uint2*>(row + at) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<unsigned*>(row + at) = w[0];
}
template <int N> __device__ __forceinline__ void store_codes(mx<2>, char* row, int at, const float* y) {
    unsigned w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[2], y[3], 1.f, 1);
    if constexpr (N == 8) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[4], y[5], 1.f, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, y[6], y[7], 1.f, 3);
        *reinterpret_cast<unsigned*>(row + at / 2) = w;
    } else {
        *reinterpret_cast<unsigned short*>(row + at / 2) = (unsigned short)w;
    }
}

// x in float32 with the last bit set where x has more bits (a value beyond the largest finite one becomes that).
__device__ __forceinline__ float to_odd(double x) {
    const float f = (float)x;
    unsigned u = __float_as_uint(f);
    if ((double)f != x) {
        u -= fabs((double)f) > fabs(x);
        u |= 1;
    }
    return __uint_as_float(u);
}

// Output rows may go past the caches (launch_append_mx and launch_read_mx say when).
template <bool PAST, typename P> __device__ __forceinline__ void store_row(P* to, P x) {
    if constexpr (PAST) __builtin_nontemporal_store(x, to);
    else *to = x;
}

template <int CTRL> __device__ __forceinline__ unsigned across(unsigned x) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
// Largest x of the U neighbouring lanes, U = 4, 8 or 16.
template <int U> __device__ __forceinline__ unsigned most_of(unsigned x) {
    x = max(x, across<0xB1>(x));                      // lane ^ 1
    x = max(x, across<0x4E>(x));                      // lane ^ 2
    if constexpr (U >= 8) x = max(x, across<0x141>(x));   // 7 - lane of 8
    if constexpr (U >= 16) x = max(x, across<0x140>(x));  // 15 - lane of 16
    return x;
}

template <typename T, int CACHE, int D, bool INTERLEAVED, bool PAST>
__global__ __launch_bounds__(256) void append_mx(const AppendArgs A) {
    typedef piece_of<T> piece;
    constexpr int N = T::N, U = D / (2 * N);          // elements of a piece; units of a head: a lane has one, its two pieces
    constexpr int HW = 64 / U;                        // heads that a wave meets at a time
    constexpr int NB = D / 32;                        // blocks of a row
    constexpr int ROW = CACHE == 1 ? D : D / 2;
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
    // a pair's cosine and sine: halves, pair i is (x0[i], x1[i]); interleaved, (x0[2i], x0[2i + 1]), then those of x1
    const int heads = A.Hq + 2 * A.Hkv;               // query heads, key heads, value heads
    for (int h = part * HW + hl; h < heads; h += A.parts * HW) {
        const bool is_q = h < A.Hq, is_k = !is_q && h < A.Hq + A.Hkv;
        const int hh = is_q ? h : (is_k ? h - A.Hq : h - A.Hq - A.Hkv);
        const char* src = is_q ? A.q + t * A.q_rs + hh * A.q_hs : (is_k ? A.k + t * A.k_rs + hh * A.k_hs : A.v + t * A.v_rs + hh * A.v_hs);
        const piece x0 = reinterpret_cast<const piece*>(src)[c0], x1 = reinterpret_cast<const piece*>(src)[c1];
        constexpr bool kSingle = std::is_same<typename T::elem, float>::value;
        float y[2 * N], copy[kSingle ? 2 * N : 1];    // copy: float32 rows as the keys' second copy has them
#pragma unroll
        for (int i = 0; i < N; ++i) {
            y[i] = (float)x0[i];
            y[N + i] = (float)x1[i];
        }
        if (is_q) {
            if (turn) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int a = INTERLEAVED ? 2 * i : i, c = INTERLEAVED ? 2 * i + 1 : N + i;
                    const float ya = y[a], yc = y[c];
                    y[a] = ya * cs[i] - yc * sn[i];
                    y[c] = yc * cs[i] + ya * sn[i];
                }
            }
        } else if (is_k && turn) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int a = INTERLEAVED ? 2 * i : i, c = INTERLEAVED ? 2 * i + 1 : N + i;
                const double ya = y[a], yc = y[c], dc = cs[i], ds = sn[i], da = ya * dc - yc * ds, db = yc * dc + ya * ds;
                y[a] = to_odd(da);
                y[c] = to_odd(db);
                if constexpr (kSingle) {
                    copy[a] = (float)da;
                    copy[c] = (float)db;
                }
            }
        }
        if (is_q || (is_k && A.k_out)) {
            piece y0, y1;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                y0[i] = (typename T::elem)y[i];
                y1[i] = (typename T::elem)y[N + i];
            }
            if constexpr (kSingle) {
                if (is_k && turn) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        y0[i] = copy[i];
                        y1[i] = copy[N + i];
                    }
                }
            }
            char* o = is_q ? A.q_out + t * A.qo_rs + hh * A.qo_hs : A.k_out + t * A.ko_rs + hh * A.ko_hs;
            store_row<PAST>(reinterpret_cast<piece*>(o) + c0, y0);
            store_row<PAST>(reinterpret_cast<piece*>(o) + c1, y1);
        }
        if (is_q || slot < 0) continue;               // (a head's lanes go on together: the exchanges below stay within them)
        // magnitudes compare as whole numbers, infinities and NaN behind all others
        unsigned m0 = 0, m1 = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m0 = max(m0, __float_as_uint(y[i]) & 0x7FFFFFFFu);
            m1 = max(m1, __float_as_uint(y[N + i]) & 0x7FFFFFFFu);
        }
        const int b0 = c0 * N / 32, b1 = c1 * N / 32;
        unsigned bytes = 0, e0 = 0, e1 = 0;
#pragma unroll
        for (int k = 0; k < NB; ++k) {
            const unsigned m = most_of<U>(max(b0 == k ? m0 : 0u, b1 == k ? m1 : 0u));
            int e = (int)(m >> 23) - mx<CACHE>::kTop + ((m & 0x7FFFFFu) > mx<CACHE>::kFraction);
            e = m >= 0x7F800000u ? 255 : max(e, 10);
            bytes |= (unsigned)e << (8 * k);
            if (b0 == k) e0 = e;
            if (b1 == k) e1 = e;
        }
        const float f0 = __uint_as_float((254 - e0) << 23), f1 = __uint_as_float((254 - e1) << 23);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            y[i] = e0 == 255 ? 0.f : y[i] * f0;
            y[N + i] = e1 == 255 ? 0.f : y[N + i] * f1;
        }
        const int64_t at = slot * A.Hkv + hh;
        char* o = (is_k ? A.k_pages : A.v_pages) + at * ROW;
        store_codes<N>(mx<CACHE>{}, o, c0 * N, y);
        store_codes<N>(mx<CACHE>{}, o, c1 * N, y + N);
        if (u == 0) {
            unsigned char* s = (is_k ? A.k_scales : A.v_scales) + at * NB;
            if constexpr (NB == 4) *reinterpret_cast<unsigned*>(s) = bytes;
            else *reinterpret_cast<unsigned short*>(s) = (unsigned short)bytes;
        }
    }
}

// One piece's codes as they lie in a row, and the N values that they stand for, times 2^(byte - 127).
template <int CACHE, int N> struct codes_of;
template <> struct codes_of<1, 8> { typedef uint2 type; };
template <> struct codes_of<1, 4> { typedef unsigned type; };
template <> struct codes_of<2, 8> { typedef unsigned type; };
template <> struct codes_of<2, 4> { typedef unsigned short type; };
__device__ __forceinline__ void four_values(unsigned w, float unit, float* y) {
    const fx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, unit, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, unit, true);
    y[0] = a.x;
    y[1] = a.y;
    y[2] = b.x;
    y[3] = b.y;
}
__device__ __forceinline__ void values(mx<1>, uint2 w, float unit, float* y) {
    four_values(w.x, unit, y);
    four_values(w.y, unit, y + 4);
}
__device__ __forceinline__ void values(mx<1>, unsigned w, float unit, float* y) { four_values(w, unit, y); }
__device__ __forceinline__ void values(mx<2>, unsigned short w, float unit, float* y) {
    const fx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
    y[0] = a.x;
    y[1] = a.y;
    y[2] = b.x;
    y[3] = b.y;
}
__device__ __forceinline__ void values(mx<2>, unsigned w, float unit, float* y) {
    values(mx<2>{}, (unsigned short)w, unit, y);
    const fx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3);
    y[4] = a.x;
    y[5] = a.y;
    y[6] = b.x;
    y[7] = b.y;
}

// A wave takes a token, a lane one piece of a head at a time, and of four heads before the first is stored.
template <typename T, int CACHE, int D, bool PAST>
__global__ __launch_bounds__(256) void read_mx(const AppendArgs A) {
    typedef piece_of<T> piece;
    constexpr int N = T::N, P = D / N, HW = 64 / P;   // pieces of a row; heads that a wave meets at a time
    constexpr int ROW = CACHE == 1 ? D : D / 2;
    const int lane = threadIdx.x & 63;
    const unsigned item = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(item / (unsigned)A.parts), part = (int)(item % (unsigned)A.parts);
    if (t >= A.T) return;
    int b = t, first = t;
    if (A.cu) {
        b = sequence_of(A.cu, A.B, t, lane);
        if (b >= A.B) return;
        first = A.cu[b];
        if (first > t) return;
    }
    const int64_t row = (int64_t)A.starts[b] + (t - first);
    if (row < 0 || row >= A.table_rows) return;
    const int64_t pg = (unsigned)row / (unsigned)A.page;
    const int64_t page = A.table[(int64_t)b * A.table_stride + pg];
    if (page < 0 || page >= A.pages) return;
    const int64_t slot = page * A.page + (row - pg * A.page);
    const int c = lane % P;
    constexpr int BATCH = 4;
    for (int h0 = part * HW + lane / P; h0 < 2 * A.Hkv; h0 += A.parts * HW * BATCH) {
        typename codes_of<CACHE, N>::type w[BATCH];
        unsigned s[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = min(h0 + i * A.parts * HW, 2 * A.Hkv - 1);           // (behind the last: it again, and nothing is stored)
            const bool is_k = h < A.Hkv;
            const int64_t at = slot * A.Hkv + (is_k ? h : h - A.Hkv);
            s[i] = (is_k ? A.k_scales : A.v_scales)[at * (D / 32) + c * N / 32];
            w[i] = *reinterpret_cast<const typename codes_of<CACHE, N>::type*>((is_k ? A.k_pages : A.v_pages) + at * ROW + c * N * ROW / D);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int h = h0 + i * A.parts * HW;
            if (h >= 2 * A.Hkv) break;
            float y[N];
            values(mx<CACHE>{}, w[i], __uint_as_float(s[i] << 23), y);
            piece x;
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = (typename T::elem)y[e];
            char* o = h < A.Hkv ? A.k_out + t * A.ko_rs + h * A.ko_hs : A.v_out + t * A.vo_rs + (h - A.Hkv) * A.vo_hs;
            store_row<PAST>(reinterpret_cast<piece*>(o) + c, x);
        }
    }
}

template <typename F> hipError_t by_form(int dtype, int cache, int D, F form) {
    typedef std::integral_constant<int, 64> d64;
    typedef std::integral_constant<int, 128> d128;
    typedef std::integral_constant<int, 1> fp8;
    typedef std::integral_constant<int, 2> fp4;
    auto of = [&](auto t) {
        if (cache == 1) D == 128 ? form(t, fp8{}, d128{}) : form(t, fp8{}, d64{});
        else D == 128 ? form(t, fp4{}, d128{}) : form(t, fp4{}, d64{});
    };
    if (dtype == 0) of(m_bf16{});
    else if (dtype == 1) of(m_f32{});
    else if (dtype == 2) of(m_f16{});
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace

// Output bytes from which a call's rows go past the caches.  What counts is the call and the one behind it, which reads these rows.  Microseconds past / through
// the caches.  Append with the attention over the prompts behind it: 1070 MB 4245 / 4265, 819 MB 2983 / 2995, 512 MB 1775 / 1782; 246 MB 869 / 866, 213 MB 534 / 531,
// 154 MB 458 / 449, 4 MB (8192 tokens of 2/2 heads of 64) 64 / 55: past from about twice the last-level cache's 256 MB on.
// Read with the compression behind it, into the same rows as before or others in turn: 1070 MB 404 / 420, 537 MB 232 / 237; 459 MB 220 / 211 and 221 / 212, 328 MB
// 159 / 154 and 161 / 158, 213 MB 94 / 106 and 112 / 104, 154 MB 77 / 76 and 79 / 82, 134 MB (32749 tokens of 8 heads) 84 / 83 and 91 / 87, 32 heads 73 / 71 and 75 / 81;
// 57 MB 47 / 45 and 46 / 44, 46 MB 45 / 43 and 41 / 40, 25 MB 51.5 / 51.1 and 47.0 / 46.4, 8 MB 31.6 / 31.2.  The read alone: 213 MB 44 / 60, 134 MB 32 / 43, 25 MB
// 6.9 / 8.9.  So from 64 MB on the pair takes the same within a few percent either way and the read alone less; below, what the read takes less comes back in the
// compression, which finds no rows in the caches, and more.
constexpr int64_t kPastAppend = 500000000, kPastRead = 64000000;

hipError_t launch_append_mx(int dtype, int cache, int D, bool interleaved, AppendArgs A, hipStream_t st) {
    const int units = D * (dtype == 1 ? 4 : 2) / 32, per = 64 / units;
    const int heads = A.Hq + 2 * A.Hkv, groups = (heads + per - 1) / per;
    A.parts = A.T < 1024 ? groups : 1;
    const bool past = A.T * (A.Hq + (A.k_out ? A.Hkv : 0)) * D * (dtype == 1 ? 4 : 2) > kPastAppend;
    const dim3 grid((unsigned)((A.T * A.parts + 3) / 4)), block(256);
    return by_form(dtype, cache, D, [&](auto t, auto c, auto d) {
        typedef decltype(t) T;
        constexpr int C = decltype(c)::value, DD = decltype(d)::value;
        auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, st, A); };
        if (past) launch(interleaved ? append_mx<T, C, DD, true, true> : append_mx<T, C, DD, false, true>);
        else launch(interleaved ? append_mx<T, C, DD, true, false> : append_mx<T, C, DD, false, false>);
    });
}

hipError_t launch_read_mx(int dtype, int cache, int D, AppendArgs A, hipStream_t st) {
    const int per = 64 * 16 / (D * (dtype == 1 ? 4 : 2));
    const int groups = (2 * A.Hkv + per - 1) / per;
    A.parts = A.T < 1024 ? groups : 1;
    const bool past = 2 * A.T * A.Hkv * D * (dtype == 1 ? 4 : 2) > kPastRead;
    const dim3 grid((unsigned)((A.T * A.parts + 3) / 4)), block(256);
    return by_form(dtype, cache, D, [&](auto t, auto c, auto d) {
        typedef decltype(t) T;
        constexpr int C = decltype(c)::value, DD = decltype(d)::value;
        auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, st, A); };
        launch(past ? read_mx<T, C, DD, true> : read_mx<T, C, DD, false>);
    });
}

}  // namespace snapkv
