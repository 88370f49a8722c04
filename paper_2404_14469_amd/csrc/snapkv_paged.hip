// Attention of one new token per sequence over a paged cache of [pages, page, Hkv, D] rows.
//
//   out[b, h] = sum_j softmax_j(q[b, h] . k_j / sqrt(D)) v_j,   lse[b, h] = log sum_j exp(q[b, h] . k_j / sqrt(D)),
//
// j over the lens[b] rows of sequence b: one pass with the running maximum and sum.  Every row is read once, so HBM bounds
// the step, and one short sequence the latency of its few loads.  The arithmetic is that of the step over compacted
// caches (snapkv_decode.hip): 16x16x32 products with the g query heads of a KV head as the 16 columns, probabilities in two
// parts of the storage type, value tiles transposed by a 0/1 product.
//
// Work split: a workgroup of four waves takes a share of the keys of one (sequence, KV head).  The host fixes how many shares a
// sequence can have, the device how long they are, by the sequence's own length (share_of): a cache may be far longer than what
// it holds.  Workgroups beyond a sequence's end return at once.  Sequences of one share are finished by their workgroup; the
// partial (max, sum, output) of longer ones are joined by a second kernel.  Rows behind a sequence's end are never read: their lanes read the last row again.
// The rows of a step (a table entry, then K and V) are looked up one step ahead.  Eight sequences of about 16000 rows, 32 KV
// heads: 2.07 GB in 365 us with the join, 5.7 TB/s; one of 131072 rows, 8 KV heads 103 us and 6 for the join; one of 2113 rows 6.0 and 3.8.
#include "snapkv_attn.h"
#include "snapkv_serve.h"

#include <algorithm>
#include <cmath>

namespace snapkv {
namespace {

constexpr int kWaves = 4;
constexpr int64_t kMostGroups = 16384;   // workgroups of a step whose sequences' shares are bounded by it

// Keys of a share of a sequence of S: whole steps of all waves, so many that nchunk shares hold it, and at least `least`.
__device__ __forceinline__ int share_of(int S, int nchunk, int least) {
    const int c = (S + nchunk - 1) / nchunk;
    return max(least, (c + 127) / 128 * 128);
}

template <typename T> struct store_type;
template <> struct store_type<dec_bf16> {
    typedef __bf16 type;
    static constexpr float kShift = 0.f;
};
// fp16 probabilities are taken 2^15 times as large (the largest, 2^15, is below fp16's largest number).  Two parts of one then lose
// less than 2^-20 of it, or a step of fp16's smallest numbers, 2^-39 of the row's largest; taken as they are, those of about
// 2^-17, of which a long cache can have as many as weigh all, would lose up to 2^-7 of themselves.
template <> struct store_type<dec_f16> {
    typedef _Float16 type;
    static constexpr float kShift = 15.f;
};

template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void paged_attn(const PagedArgs A) {
    typedef typename store_type<T>::type elem;
    constexpr int NP = D / 32;        // 16-byte pieces per lane and row
    constexpr int NB = D / 16;        // 16-column blocks of the output
    constexpr int ROW = D * 2;
    constexpr float kShift = store_type<T>::kShift;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n16 = lane & 15, kg = lane >> 4;
    // A share's heads run together.  With several sequences they run on one XCD too (workgroup i runs on XCD i % 8), which then
    // reads whole rows; a sequence has an odd number of places (`places`, at most one of them empty), so that the first shares, which
    // are all that short sequences have, do not meet on a few XCDs.
    int kvh = blockIdx.x % A.Hkv, chunk = blockIdx.x / A.Hkv;
    if (A.by_xcd) {
        kvh = blockIdx.x / 8 % A.Hkv;
        chunk = blockIdx.x / (8 * A.Hkv) * 8 + blockIdx.x % 8;
    }
    const int b = chunk / A.places;
    chunk %= A.places;
    if (chunk >= A.nchunk || b >= A.B) return;
    int64_t len = A.lens[b];
    const int S = (int)(len < 0 ? 0 : (len > A.max_len ? A.max_len : len));
    if (chunk > 0 && chunk * A.least >= S) return;                 // (most of what returns, before the division)
    const int share = share_of(S, A.nchunk, A.least), begin = chunk * share;
    if (chunk > 0 && begin >= S) return;
    const int end = begin + share < S ? begin + share : S;         // keys begin .. end - 1
    const int32_t* table = A.table + (int64_t)b * A.table_stride;
    const int64_t token = (int64_t)A.Hkv * ROW;                    // bytes between the rows of a page
    const char* kbase = A.k + (int64_t)kvh * ROW;
    const char* vbase = A.v + (int64_t)kvh * ROW;

    uint4 qf[NP];
#pragma unroll
    for (int c = 0; c < NP; ++c) qf[c] = make_uint4(0, 0, 0, 0);
    if (n16 < A.g) {
        const char* qrow = A.q + ((int64_t)b * A.Hq + (int64_t)kvh * A.g + n16) * ROW;
#pragma unroll
        for (int c = 0; c < NP; ++c) qf[c] = *reinterpret_cast<const uint4*>(qrow + (4 * c + kg) * 16);
    }
    const uint4 sel0 = selector<T>(lane, 0), sel1 = selector<T>(lane, 1);

    float m = -3.4028235e38f, lsum = 0.f;              // (finite: logits of -infinity have probability 0 and not NaN)
    dfx4 acc[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[i] = dfx4{0.f, 0.f, 0.f, 0.f};

    auto offset_of = [&](int key) {                    // byte offset of the row of a key, 64 bits
        const int r = key < end ? key : end - 1;
        const int pg = (int)(((uint64_t)(unsigned)r * A.page_magic) >> A.page_shift);
        int64_t at = table[pg];
        at = at < 0 ? 0 : (at >= A.pages ? A.pages - 1 : at);
        return (at * A.page + (r - pg * A.page)) * token;
    };
    struct Rows {                                      // the rows of a lane's two keys
        int64_t x, y;
    };
    auto find = [&](int key0) { return Rows{offset_of(key0 + n16), offset_of(key0 + 16 + n16)}; };
    auto process = [&](const Rows& at, int key0) {
        uint4 kx[NP], ky[NP], vx[NP], vy[NP];
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            kx[c] = *reinterpret_cast<const uint4*>(kbase + at.x + (4 * c + kg) * 16);
            ky[c] = *reinterpret_cast<const uint4*>(kbase + at.y + (4 * c + kg) * 16);
        }
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            vx[c] = *reinterpret_cast<const uint4*>(vbase + at.x + (4 * c + kg) * 16);
            vy[c] = *reinterpret_cast<const uint4*>(vbase + at.y + (4 * c + kg) * 16);
        }
        __builtin_amdgcn_sched_barrier(0);
        dfx4 sx = {0.f, 0.f, 0.f, 0.f}, sy = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            sx = mma(T{}, kx[c], qf[c], sx);
            sy = mma(T{}, ky[c], qf[c], sy);
        }
        const int k0 = key0 + 4 * kg;
        float e[8];
        float tmax = -INFINITY;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            e[r] = k0 + r < end ? sx[r] * A.scale2 : -INFINITY;
            e[4 + r] = k0 + 16 + r < end ? sy[r] * A.scale2 : -INFINITY;
            tmax = fmaxf(tmax, fmaxf(e[r], e[4 + r]));
        }
        tmax = fmaxf(tmax, __shfl_xor(tmax, 16));
        tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
        const float mn = fmaxf(m, tmax);
        const float alpha = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        const float least = mn - kShift;
        float psum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = __builtin_amdgcn_exp2f(e[j] - least);
            psum += e[j];
        }
        lsum = lsum * alpha + psum;
        uint4 ph, pl;
        split2(T{}, e[0], e[1], ph.x, pl.x);
        split2(T{}, e[2], e[3], ph.y, pl.y);
        split2(T{}, e[4], e[5], ph.z, pl.z);
        split2(T{}, e[6], e[7], ph.w, pl.w);
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[i] *= alpha;
#pragma unroll
        for (int c = 0; c < NP; ++c) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const dfx4 z = {0.f, 0.f, 0.f, 0.f};
                const dfx4 tx = mma(T{}, vx[c], half ? sel1 : sel0, z);
                const dfx4 ty = mma(T{}, vy[c], half ? sel1 : sel0, z);
                uint4 vt;
                vt.x = pack_exact(T{}, tx[0], tx[1]);
                vt.y = pack_exact(T{}, tx[2], tx[3]);
                vt.z = pack_exact(T{}, ty[0], ty[1]);
                vt.w = pack_exact(T{}, ty[2], ty[3]);
                dfx4 o = acc[2 * c + half];
                o = mma(T{}, vt, ph, o);
                o = mma(T{}, vt, pl, o);
                acc[2 * c + half] = o;
            }
        }
    };
    constexpr int STEP = 32 * kWaves;
    int key = begin + 32 * wave;
    if (key < end) {
        Rows at = find(key);
        for (;;) {
            const Rows next = find(key + STEP);        // (behind the end: the last row)
            process(at, key);
            key += STEP;
            if (key >= end) break;
            at = next;
        }
    }
    lsum += __shfl_xor(lsum, 16);
    lsum += __shfl_xor(lsum, 32);

    __shared__ float s_acc[kWaves][16][D + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
#pragma unroll
    for (int i = 0; i < NB; ++i)
        *reinterpret_cast<float4*>(&s_acc[wave][n16][16 * i + 4 * kg]) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    if (kg == 0) {
        s_m[wave][n16] = m;
        s_l[wave][n16] = lsum;
    }
    __syncthreads();
    constexpr int DT = D / 16;
    const int qi = tid >> 4, d0 = (tid & 15) * DT;
    if (qi < A.g) {
        float M = s_m[0][qi];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][qi]);
        float Lq = 0.f, o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][qi] - M);
            Lq += s_l[w][qi] * f;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] += s_acc[w][qi][d0 + d] * f;
        }
        const int64_t hq = (int64_t)b * A.Hq + (int64_t)kvh * A.g + qi;
        if (S <= share) {
            const float inv = Lq == 0.f ? 0.f : 1.f / Lq;      // (no rows; a sum that is NaN makes the row's answer NaN)
            elem* out = reinterpret_cast<elem*>(A.out) + hq * D + d0;
#pragma unroll
            for (int d = 0; d < DT; ++d) out[d] = (elem)(o[d] * inv);
            if (A.lse && (tid & 15) == 0)
                A.lse[hq] = Lq == 0.f ? -INFINITY : (M - kShift + __builtin_amdgcn_logf(Lq)) * 0.6931471805599453f;
        } else {
            float* pa = A.part_acc + (hq * A.nchunk + chunk) * D;
#pragma unroll
            for (int d = 0; d < DT; ++d) pa[d0 + d] = o[d];
            if ((tid & 15) == 0) A.part_ml[hq * A.nchunk + chunk] = make_float2(M, Lq);
        }
    }
}

// Joins the partials of the sequences of more than one chunk: a workgroup per query head, its waves a quarter of the chunks each,
// eight partial outputs in flight at a time.
template <typename T, int D>
__global__ __launch_bounds__(kWaves * 64) void paged_join(const PagedArgs A) {
    typedef typename store_type<T>::type elem;
    constexpr int E = D / 64, BATCH = 8;
    constexpr float kShift = store_type<T>::kShift;
    const int64_t hq = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = (int)(hq / A.Hq);
    int64_t len = A.lens[b];
    const int S = (int)(len < 0 ? 0 : (len > A.max_len ? A.max_len : len));
    const int share = share_of(S, A.nchunk, A.least);
    if (S <= share) return;
    const int n = (S + share - 1) / share;
    const float2* ml = A.part_ml + hq * A.nchunk;
    const float* pa = A.part_acc + hq * A.nchunk * D + lane * E;
    float M = -INFINITY;
    for (int i = lane; i < n; i += 64) M = fmaxf(M, ml[i].x);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    float Lq = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int i0 = wave * BATCH; i0 < n; i0 += kWaves * BATCH) {
        float2 p[BATCH];
        float x[BATCH][E];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int c = i0 + i < n ? i0 + i : n - 1;
            p[i] = ml[c];
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = pa[(int64_t)c * D + e];
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float f = i0 + i < n ? __builtin_amdgcn_exp2f(p[i].x - M) : 0.f;
            Lq += p[i].y * f;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += x[i][e] * f;
        }
    }
    __shared__ float s_o[kWaves][D], s_l[kWaves];
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[wave][lane * E + e] = o[e];
    if (lane == 0) s_l[wave] = Lq;
    __syncthreads();
    Lq = s_l[0] + s_l[1] + s_l[2] + s_l[3];
    if (threadIdx.x < D) {
        const int d = threadIdx.x;
        const float y = s_o[0][d] + s_o[1][d] + s_o[2][d] + s_o[3][d];
        reinterpret_cast<elem*>(A.out)[hq * D + d] = (elem)(Lq == 0.f ? 0.f : y / Lq);
    }
    if (A.lse && threadIdx.x == 0) A.lse[hq] = Lq == 0.f ? -INFINITY : (M - kShift + __builtin_amdgcn_logf(Lq)) * 0.6931471805599453f;
}

}  // namespace

// Shares of a sequence: as many as give 1024 workgroups, four per compute unit, if all sequences are as long as they may be, of 128
// keys, one step of each wave, at least; but a sequence of up to 512 is not cut, so that short steps are one launch.  At most 1024
// keys, and 512 where even those give 2048 workgroups: sequences are of different lengths, which only the device knows, and
// small shares even that out.  Microseconds with at most 512 / 1024 / 2048 / 4096 keys: 32 sequences of 1 to 16384
// keys, 8 KV heads 120 / 125 / 149 / 224; eight of about 16000, 32 KV heads 374 / 373 / 378 / 385; one of 131072 keys, 8 KV heads
// 114 / 107 / 108 / -.  Shares of sequences that are shorter than they may be are as much shorter, down to 128 keys where there
// are few (sequence, KV head) pairs.
// Workgroups and workspace go by how long sequences may be, so no more shares than give 16384 workgroups, or seven, whatever that
// is; sequences that are long then have longer ones.  With this bound / without it, 8 KV heads, tables for 131072 rows: 32 sequences
// of 2000 rows 61 / 100, 128 of 1000 122 / 303, 32 of 1 to 131072 278 / 314; 32 KV heads, 256 sequences of 1 to 8192 656 / 700.
PagedPlan paged_plan(int B, int Hq, int Hkv, int D, int64_t max_len) {
    const int64_t pairs = (int64_t)B * Hkv, keys = pairs * max_len;
    int64_t chunk = std::max<int64_t>(128, (keys / 1024 + 127) / 128 * 128);
    chunk = std::min<int64_t>(chunk, keys >= 2048 * 1024 ? 512 : 1024);
    if (max_len <= 512) chunk = 512;
    PagedPlan P;
    P.nchunk = (int)std::min((max_len + chunk - 1) / chunk, std::max<int64_t>(7, kMostGroups / pairs));
    P.least = P.nchunk == 1 || pairs > 128 ? 512 : (pairs > 64 ? 256 : 128);
    const size_t heads = (size_t)B * Hq;
    P.bytes = P.nchunk <= 1 ? 0 : ((heads * P.nchunk * D * sizeof(float) + 255) & ~(size_t)255) + heads * P.nchunk * sizeof(float2);
    return P;
}

hipError_t launch_paged(int dtype, int D, PagedArgs A, void* workspace, hipStream_t st) {
    const PagedPlan P = paged_plan(A.B, A.Hq, A.Hkv, D, A.max_len);
    A.nchunk = P.nchunk;
    A.least = P.least;
    // r / page for 0 <= r < 2^31: with 2^(l-1) < page <= 2^l, ceil(2^(31+l) / page) fits 32 bits and its product's error stays
    // below one part in r (page 1: 2^31 and a shift by 31)
    int l = 0;
    while (l < 31 && (1ll << l) < A.page) ++l;
    A.page_magic = (unsigned)(((1ull << (31 + l)) + A.page - 1) / A.page);
    A.page_shift = 31 + l;
    A.scale2 = (float)(1.4426950408889634 / std::sqrt((double)D));
    A.part_acc = nullptr;
    A.part_ml = nullptr;
    const size_t heads = (size_t)A.B * A.Hq;
    if (P.nchunk > 1) {
        A.part_acc = static_cast<float*>(workspace);
        A.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + ((heads * P.nchunk * D * sizeof(float) + 255) & ~(size_t)255));
    }
    // (8 x 16000 rows, 32 KV heads 366 us so, 378 with heads dealt to XCDs; 32 sequences of 1 to 16384 rows 119 / 121; one of 131072
    // rows 112 / 109)
    A.by_xcd = A.B > 1 && (int64_t)P.nchunk * A.B >= 64;
    // (256 sequences of 300 rows, one share each, 63; 71 with places in eights)
    A.places = A.by_xcd ? P.nchunk | 1 : P.nchunk;
    int64_t units = (int64_t)A.places * A.B;
    if (A.by_xcd) units = (units + 7) / 8 * 8;
    auto launch = [&](auto step, auto join) {
        hipLaunchKernelGGL(step, dim3((unsigned)(units * A.Hkv)), dim3(kWaves * 64), 0, st, A);
        if (P.nchunk > 1) hipLaunchKernelGGL(join, dim3((unsigned)heads), dim3(kWaves * 64), 0, st, A);
    };
    if (dtype == 0 && D == 128) launch(paged_attn<dec_bf16, 128>, paged_join<dec_bf16, 128>);
    else if (dtype == 0 && D == 64) launch(paged_attn<dec_bf16, 64>, paged_join<dec_bf16, 64>);
    else if (dtype == 2 && D == 128) launch(paged_attn<dec_f16, 128>, paged_join<dec_f16, 128>);
    else if (dtype == 2 && D == 64) launch(paged_attn<dec_f16, 64>, paged_join<dec_f16, 64>);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace snapkv
