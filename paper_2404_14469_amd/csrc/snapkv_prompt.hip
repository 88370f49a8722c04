// Causal attention over whole prompts packed one behind the other, with grouped heads and the rows' log-sum-exp:
//
//   out[i, h] = sum_{j <= i} softmax_j(q[i, h] . k[j, h / g] / sqrt(D)) v[j, h / g],
//   lse[h, i] = log sum_{j <= i} exp(q[i, h] . k[j, h / g] / sqrt(D)),      i, j within one prompt.
//
// One pass over the keys with the running maximum and sum of a softmax, in base two; 4 D operations per visible pair make
// the matrix units the bound of all but the shortest prompts.
//
// Work split.  A workgroup of four waves takes 128 query rows of one head, each wave 32 of them, and walks the keys in tiles of 64 that
// its waves share through LDS; two workgroups share a compute unit (187 registers and 64 KB each), so one's waits are the
// other's time.  Calls of few rows give a workgroup 32 rows, and each wave every fourth block of 32 keys (split_keys says which).
// 32749 tokens of 32/8 heads of 128 take 7.1 to 7.6 ms by card, 1.15 to 1.24 PFLOP/s, with the card at its power limit; 88 to 91 % of
// a 16384^3 bf16 product's rate where both were timed.  A batch of 7499 tokens in eight prompts takes 0.13 ms, 4 heads of 2048 tokens 17 us, 78 tokens 7 us, where finding
// the tile, fetching and storing are most of the time.
//
// MFMA layout (32x32x16, 64 lanes): lane l supplies row (left operand) or column (right operand) l%32 and contraction
// elements 8*(l/32) .. +7; accumulator register r of lane l is row 8*(r/4) + 4*(l/32) + r%4, column l%32.
//
//   logits^T = K Q^T: a lane gets 16 logits of ONE query per 32 keys, so the softmax is arithmetic within the lane (and, when
//     the shift moves, one exchange with the lane that has the other half of the keys); the shift, the sum and the factor that
//     rescales the output are one register each.
//   out^T = V^T P^T: contraction element e of lane l stands for key 8*(e/4) + 4*(l/32) + e%4 of 16, which is where the
//     logits left that key's probability: P never moves between lanes.  V^T comes from LDS by the transposing read (a lane
//     gets four keys of one column).
//
// The probabilities enter the last product rounded to the storage type, as its operand must be: each is off by at most half
// a step (bf16 2^-8, fp16 2^-11, relative; the fp16 ones are taken 2^7 times as large, so those down to 2^-21 of the
// largest are normal numbers), which adds to an output about what its own rounding does.  Their sum is taken in fp32 from
// the unrounded values.
#include "snapkv_serve.h"

#include <cmath>

namespace snapkv {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 pbf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 pf16x8;
typedef __attribute__((ext_vector_type(16))) float pfx16;
typedef __attribute__((ext_vector_type(4))) short ps16x4;
typedef __attribute__((ext_vector_type(4))) unsigned pu32x4;

struct p_bf16 {
    typedef __bf16 elem;
    typedef pbf16x8 frag;
    // exponent that the probabilities are raised by; most that 16 may sum up to (2^20 times what the maximum alone gives: bf16 has the
    // range; 16384 tokens with queries three times as long 1.98 ms, with 2^8 2.05)
    static constexpr float kShift = 0.f, kMost = 1048576.f;
    static constexpr unsigned kExp = 0x7F80;                 // all ones: an infinity or NaN
    static constexpr float kLargest = INFINITY;              // that a mean can round beyond
};
struct p_f16 {
    typedef _Float16 elem;
    typedef pf16x8 frag;
    static constexpr float kShift = 7.f, kMost = 32768.f;    // (2^8 times; below fp16's largest number)
    static constexpr unsigned kExp = 0x7C00;
    static constexpr float kLargest = 65504.f;
};
__device__ __forceinline__ pfx16 mma32(pbf16x8 a, pbf16x8 b, pfx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ pfx16 mma32(pf16x8 a, pf16x8 b, pfx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

constexpr int kKeys = 64;      // keys of a tile
constexpr int kWaves = 4;

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) char* lds_char;
typedef __attribute__((address_space(3))) ps16x4* lds_s16x4;

// Which 16-byte piece of its row an LDS slot of a tile holds: the pieces of a row are permuted so that the lanes of a read,
// which go down the rows, meet all banks.
template <int D> __device__ __forceinline__ int k_slot(int row, int piece) { return piece ^ (row & (D / 8 - 1)); }
template <int D> __device__ __forceinline__ int v_slot(int row, int piece) { return piece ^ ((row & (D / 32 - 1)) << 2); }

// The row tile of rank `rank`: its sequence's first token and length, and which tile of it; false where there is none.
//
// Up to 64 sequences are taken in descending order of the tiles' visible keys, so that the long ones start first.  A sequence of n
// tiles has one of each cost 1 .. n, so F(c) = sum over sequences of max(0, n - c + 1) tiles cost c or more, and the tile's cost is
// the largest c with F(c) > rank.  Every lane counts another c, 63 of them and one beyond the range at a time, over the
// sequences one by one.
//
// More sequences are short ones or many: there sequence b has the ranks from floor(cu[b] / ROWS) + b on, which leaves it enough
// of them, and is found by search, 64 places at a time.  Within it the longest tile comes first.
template <int ROWS>
__device__ __forceinline__ bool locate(const PromptArgs& A, int rank, int lane, int& begin, int& len, int& tile) {
    auto token = [&](int b) __attribute__((always_inline)) { return (int)min(max((int64_t)A.cu[b], (int64_t)0), A.T); };
    if (A.B > 64) {
        int lo = 0;
        for (int width = A.B; width > 1;) {                          // b is in lo .. lo + width - 1
            const int w = (width + 63) / 64, b = lo + lane * w;
            const int k = __popcll(__ballot(lane * w < width && token(min(b, A.B)) / ROWS + b <= rank));
            if (k == 0) return false;                                // (tokens before the first sequence)
            lo += (k - 1) * w;
            width = min(w, width - (k - 1) * w);
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        begin = __builtin_amdgcn_readfirstlane(token(lo));
        len = __builtin_amdgcn_readfirstlane(token(lo + 1)) - begin;
        tile = (len + ROWS - 1) / ROWS - 1 - (rank - begin / ROWS - lo);
        return len > 0 && tile >= 0 && rank >= begin / ROWS + lo;
    }
    int from = 0, n = 0;                                             // of the lane's sequence: first token, tokens
    if (lane < A.B) {
        from = token(lane);
        n = max(token(lane + 1) - from, 0);
    }
    const int nt = (n + ROWS - 1) / ROWS;
    int most = 0, total = 0;
    for (int i = 0; i < A.B; ++i) {
        const int x = __builtin_amdgcn_readlane(nt, i);
        most = max(most, x);
        total += x;
    }
    if (rank >= total) return false;
    int lo = 1, width = most, after = 0;                             // F(lo) > rank >= F(lo + width); after = F(lo + 1) at the end
    for (bool more = true; more;) {
        const int w = (width + 62) / 63, c = lo + lane * w;
        int f = 0;
        for (int i = 0; i < A.B; ++i) f += max(__builtin_amdgcn_readlane(nt, i) - c + 1, 0);
        const int k = __popcll(__ballot(f > rank));                  // (at least 1, at most 63)
        after = __builtin_amdgcn_readlane(f, k);
        lo += (k - 1) * w;
        width = w;
        more = w > 1;
    }
    unsigned long long has = __ballot(nt >= lo);                     // the tile is that of the (rank - after)-th sequence of lo tiles or more
    for (int within = rank - after; within > 0; --within) has &= has - 1;
    const int l = __ffsll((long long)has) - 1;
    begin = __builtin_amdgcn_readlane(from, l);
    len = __builtin_amdgcn_readlane(n, l);
    tile = lo - 1;
    return true;
}

// What the wave fetched straight into LDS has arrived.  The wait is explicit: those loads write no register that the compiler
// would wait for, and a barrier alone does not.
// All of it, or all but the last N loads.
template <int N = 0>
__device__ __forceinline__ void fetched() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// The other half of the wave: lane l gets lane l ^ 32's value.
__device__ __forceinline__ float other_half(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? y[0] : y[1]);
}

// An output that rounds to no infinity.  Probabilities that were rounded up can carry a mean of numbers near fp16's largest one,
// 65504, past the 65520 from which on numbers round to infinity; a mean of finite values is at most the largest of them.
// Infinities stay.  (bf16 has fp32's range, where the sum itself would be infinite.)
template <typename T> __device__ __forceinline__ float in_range(float y) {
    if constexpr (T::kLargest == INFINITY) return y;
    else return __builtin_fabsf(y) < INFINITY ? __builtin_amdgcn_fmed3f(y, -T::kLargest, T::kLargest) : y;
}

template <typename T, int D, bool SPLIT>
__global__ __launch_bounds__(kWaves * 64, D == 64 && !SPLIT ? 3 : 2) void prompt_attn(const PromptArgs A) {
    typedef typename T::elem elem;
    typedef typename T::frag frag;
    constexpr int WAVES = kWaves, STEP = SPLIT ? WAVES : 1;   // blocks of 32 keys from one of a wave to its next
    constexpr int ROWS = SPLIT ? 32 : WAVES * 32;            // query rows of a workgroup
    constexpr int ROW = D * 2, PIECES = D / 8;  // bytes and 16-byte pieces of a row
    constexpr int NC = D / 16, ND = D / 32;     // contraction steps of a logit; 32-column blocks of the output
    constexpr int TILE = (SPLIT ? WAVES * 32 : kKeys) * ROW; // (split: a block of each wave's own)
    __shared__ __align__(16) char m_k0[TILE], m_v0[TILE], m_k1[SPLIT ? 16 : TILE], m_v1[SPLIT ? 16 : TILE];
    const lds_char s_k0 = (lds_char)m_k0, s_v0 = (lds_char)m_v0, s_k1 = (lds_char)m_k1, s_v1 = (lds_char)m_v1;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, h2 = lane >> 5;

    // KV heads are dealt to the XCDs (workgroup i runs on XCD i % 8), so the workgroups that read a head share an L2; the
    // longest row tiles of all heads come first.
    const int m8 = (A.Hkv & 7) == 0 ? 8 : ((A.Hkv & 3) == 0 ? 4 : ((A.Hkv & 1) == 0 ? 2 : 1));
    const int rank = blockIdx.x / A.Hq, rest = blockIdx.x % A.Hq / m8;
    const int kvh = blockIdx.x % m8 + m8 * (rest / A.g), hq = kvh * A.g + rest % A.g;

    int tile, begin, len;
    if (!locate<ROWS>(A, rank, lane, begin, len, tile)) return;

    const int row0 = tile * ROWS + (SPLIT ? 0 : wave * 32);  // the wave's first query row within the prompt
    const int row = row0 + n32;
    frag qf[NC];
    const char* qr = A.q + (int64_t)(begin + min(row, len - 1)) * A.q_rs + (int64_t)hq * A.q_hs + h2 * 16;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[c] = *reinterpret_cast<const frag*>(qr + 32 * c);
    // The shift of the exponentials (finite from the start: logits of -infinity, if a row sees nothing else yet, then have
    // probability 0 and not NaN) and their sum.
    float m = -3.4028235e38f, lsum = 0.f;
    pfx16 acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    const char* kh = A.k + (int64_t)kvh * A.k_hs + (int64_t)begin * A.k_rs;
    const char* vh = A.v + (int64_t)kvh * A.v_hs + (int64_t)begin * A.v_rs;
    const int mine = row0 < len ? row0 / 32 + 1 : 0;         // blocks of 32 keys that the wave's rows see; the last one in part

    // Loads of 64 keys by all waves, or (split) of 32 by each: SHARE KB at a time, a KB (RPL rows) per wave, straight into LDS.
    // Addresses are a uniform 64-bit one of the first row and 32-bit offsets of at most 63 rows, never negative.
    constexpr int SHARE = SPLIT ? 1 : WAVES, RPL = 1024 / ROW, PER = (SPLIT ? 32 : kKeys) / (RPL * SHARE);
    const int part = SPLIT ? 0 : wave, lr = part * RPL + lane / PIECES, own = SPLIT ? wave * 32 * ROW : 0;
    // (what a lane's rows differ by changes its place in the permutation by the same number, mostly 0, whatever the lane)
    constexpr int K_TURN = RPL * SHARE % PIECES * 16;
    static_assert(RPL * SHARE % (D / 32) == 0 && (K_TURN == 0 || RPL * SHARE * 16 == K_TURN), "rows of a lane and the permutations");
    int k_piece = k_slot<D>(lr, lane % PIECES) * 16, v_piece = v_slot<D>(lr, lane % PIECES) * 16;
    auto load = [&](const char* base, int rs, int piece, int turn, int first, lds_char to) __attribute__((always_inline)) {
        const int at = min(first, len - 1);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base) + (int64_t)at * rs, 0, -1, 0x00020000);
        if (first + (SPLIT ? 32 : kKeys) <= len) {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(to + own + (i * SHARE + part) * 1024), 16, lr * rs + (piece ^ (i * turn & (ROW - 1))), i * RPL * SHARE * rs, 0, 0);
        } else {                                             // rows behind the prompt: its last row again
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int down = min(first + i * RPL * SHARE + lr, len - 1) - at;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(to + own + (i * SHARE + part) * 1024), 16, down * rs + (piece ^ (i * turn & (ROW - 1))), 0, 0, 0);
            }
        }
    };
    auto load_k = [&](int first, lds_char to) __attribute__((always_inline)) { load(kh, (int)A.k_rs, k_piece, K_TURN, first, to); };
    auto load_v = [&](int first, lds_char to) __attribute__((always_inline)) { load(vh, (int)A.v_rs, v_piece, 0, first, to); };

    // A lane's places in a tile: its pieces of key row n32 (the 32 rows below have the same permutation), and of the first value
    // row that it transposes (so have those 8 and 16 below).
    int k_at[NC], v_at[ND];
#pragma unroll
    for (int c = 0; c < NC; ++c) k_at[c] = own + n32 * ROW + k_slot<D>(n32, 2 * c + h2) * 16;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
        const int vr = 4 * h2 + (lane & 15) / 4;
        v_at[i] = own + vr * ROW + v_slot<D>(vr, 4 * i + 2 * ((lane >> 4) & 1) + (lane & 3) / 2) * 16 + (lane & 1) * 8;
    }
    // Operands of product i of a block of 32 keys: of its logits, of its part of the output (16 keys of 32 columns, transposed).
    constexpr int NQ = NC, NV = 2 * ND;
    auto k_frag = [&](lds_char s_k, int i) __attribute__((always_inline)) {
        return *reinterpret_cast<const __attribute__((address_space(3))) frag*>(s_k + k_at[i]);
    };
    auto v_frag = [&](lds_char s_v, int i) __attribute__((always_inline)) {
        lds_char at = s_v + v_at[i % ND] + 16 * ROW * (i / ND);
        const ps16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)at);
        const ps16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(at + 8 * ROW));
        return __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto product = [&](frag kf, int i, pfx16& x) __attribute__((always_inline)) {          // product i of a block's logits
        pfx16 z;
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = 0.f;
        x = mma32(kf, qf[i], i == 0 ? z : x);
    };
    // Logits of block b that lie behind their row, and so those behind the prompt, are hidden.
    auto hide = [&](int b, pfx16& x) __attribute__((always_inline)) {
        if (b < mine - 1) return;
        const int seen = row - b * 32 - 4 * h2;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (8 * (r / 4) + r % 4 > seen) x[r] = -INFINITY;
    };
    // The probabilities of a lane's 16 logits, rounded to pf, and their sums (two: shorter chains), in three stages, so that no
    // instruction waits for the one before.
    auto probabilities = [&](const pfx16& x, frag* pf, float* sum) __attribute__((always_inline)) {
        const float shift = T::kShift - m;
        float e[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r] = __builtin_fmaf(x[r], A.scale2, shift);
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r] = __builtin_amdgcn_exp2f(e[r]);
        sum[0] = e[0];
        sum[1] = e[1];
#pragma unroll
        for (int r = 2; r < 16; ++r) sum[r & 1] += e[r];
#pragma unroll
        for (int r = 0; r < 16; ++r) pf[r / 8][r % 8] = (elem)e[r];
    };
    // The shift need not be the maximum: a row's is moved to it, its sum and output rescaled and the block's probabilities taken
    // anew, only when those of one of its two lanes sum up to more than kMost.  So no probability is larger than that, and no maximum
    // is looked for as long as none is.  The wave's other rows keep their shift, their factor is 1 and their probabilities come out
    // as before: what a row gives depends on what it sees alone.
    auto settle = [&](const pfx16& x, frag* pf, float* sum) __attribute__((always_inline)) {
        const float both = sum[0] + sum[1];
        if (__any(both > T::kMost)) {
            float big = x[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) big = fmaxf(big, x[r]);
            const float others = other_half(both), top = fmaxf(big, other_half(big)) * A.scale2;   // (all lanes exchange)
            const float mn = both > T::kMost || others > T::kMost ? fmaxf(m, top) : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            lsum *= alpha;
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
            probabilities(x, pf, sum);
        }
        lsum += sum[0] + sum[1];
    };
    // A block's softmax, which only vector instructions do, then the products of the wave's next block's logits (which take the
    // place of this one's) and of this block's part of the output, which only matrix instructions do: the other wave of the SIMD
    // is in the other half meanwhile, and a wave with products goes first (32749 tokens 7.27 -> 7.08 ms; with the softmax's
    // instructions between the logits' products instead 7.1 to 7.4, and two prompts with 20 heads of 64 103 us instead of 98).
    // Operands are read from LDS AHEAD products before their own.
    constexpr int AHEAD = SPLIT ? 2 : 3;
    pfx16 x;
    auto pass = [&](int b, lds_char k_next, lds_char v_now) __attribute__((always_inline)) {
        if (b + STEP >= mine) return;
        frag pf[2], kf[NQ], vf[NV];
        float sum[2];
        if constexpr (SPLIT) fetched<PER>();                 // its keys; its values (PER loads) may still be on their way
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) kf[i] = k_frag(k_next, i);
        __builtin_amdgcn_sched_barrier(0);
        probabilities(x, pf, sum);
        settle(x, pf, sum);
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (SPLIT && i + AHEAD == NQ) fetched();
            if (i + AHEAD < NQ) kf[i + AHEAD] = k_frag(k_next, i + AHEAD);
            else vf[i + AHEAD - NQ] = v_frag(v_now, i + AHEAD - NQ);
            product(kf[i], i, x);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (SPLIT)                                 // (all products with the keys there have been issued, so they have been read)
            if (b + 2 * STEP < mine) load_k((b + 2 * STEP) * 32, k_next);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i + AHEAD < NV) vf[i + AHEAD] = v_frag(v_now, i + AHEAD);
            acc[i % ND] = mma32(vf[i], pf[i / ND], acc[i % ND]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        hide(b + STEP, x);
        if constexpr (SPLIT) load_v((b + STEP) * 32, v_now);
    };
    // (a lane's places are kept as they are, and a buffer's address is the constant offset of a read: sums of the two, made once
    // in front of the loop, would take 24 registers)
    auto keep_places = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NC; ++c) asm volatile("" : "+v"(k_at[c]));
#pragma unroll
        for (int i = 0; i < ND; ++i) asm volatile("" : "+v"(v_at[i]));
        asm volatile("" : "+v"(k_piece), "+v"(v_piece));
    };
    auto begin_with = [&](int b, lds_char s_k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) product(k_frag(s_k, i), i, x);
        __builtin_amdgcn_sched_barrier(0);                   // (the products stand in front of the loads that reuse the buffer)
        hide(b, x);
    };
    lds_char v_last = s_v0;                                  // values of the wave's last block
    if constexpr (SPLIT) {
        // A wave's blocks are its own from their loads on: nothing to wait for but its own fetches.  One buffer for keys, which the
        // next block's replace as soon as their logits are taken, and one for values: 64 KB, so two workgroups share a compute
        // unit, and one's arithmetic covers the other's fetches.
        int b = wave;
        if (b < mine) {
            load_k(b * 32, s_k0);
            load_v(b * 32, s_v0);
            fetched<PER>();
            begin_with(b, s_k0);
            if (b + STEP < mine) load_k((b + STEP) * 32, s_k0);
            fetched();
        }
        for (; b + STEP < mine; b += STEP) {
            keep_places();
            pass(b, s_k0, s_v0);
        }
        fetched();
    } else {
        // Keys are half a tile ahead of values: tile t of V is blocks 2 t and 2 t + 1, that of K blocks 2 t + 1 and 2 t + 2, whose
        // logits are taken meanwhile.  The next tiles arrive in the other two buffers.
        const int ntiles = (min(len, (tile + 1) * ROWS) - 1) / kKeys + 1;      // of keys that any of the rows sees
        auto two_blocks = [&](int t, lds_char k_now, lds_char k_free, lds_char v_now, lds_char v_free) __attribute__((always_inline)) {
            fetched();
            __syncthreads();                                 // these tiles have arrived, the others have been read
            keep_places();
            if (t + 1 < ntiles) {
                load_k((t + 1) * kKeys + 32, k_free);
                load_v((t + 1) * kKeys, v_free);
            }
            pass(2 * t, k_now, v_now);
            pass(2 * t + 1, k_now + 32 * ROW, v_now + 32 * ROW);
        };
        load_k(0, s_k1);
        load_k(32, s_k0);
        load_v(0, s_v0);
        fetched();
        __syncthreads();
        begin_with(0, s_k1);
        for (int t = 0;;) {
            two_blocks(t, s_k0, s_k1, s_v0, s_v1);
            if (++t >= ntiles) break;
            two_blocks(t, s_k1, s_k0, s_v1, s_v0);
            if (++t >= ntiles) break;
        }
        v_last = ((mine - 1) & 2 ? s_v1 : s_v0) + ((mine - 1) & 1) * 32 * ROW;   // (one of the last two tiles, which are still there)
    }
    // The wave's last block; its logits are in x.  The last one that rows see they see in part.  Values that a row does not see
    // have probability 0, but 0 times an infinity or NaN is not 0: where the block holds such values, they are taken as zeros, which
    // leaves all other sums as they would be without them, and then added key by key to the rows that see the key.
    if (SPLIT ? wave < mine : mine > 0) {
        const int b = SPLIT ? wave + (mine - 1 - wave) / STEP * STEP : mine - 1;
        frag pf[2];
        float sum[2];
        probabilities(x, pf, sum);
        settle(x, pf, sum);
        bool spoiled = false;
#pragma unroll
        for (int i = 0; i < ROW * 32 / 1024; ++i) {
            const pu32x4 y = *reinterpret_cast<const __attribute__((address_space(3))) pu32x4*>(v_last + own + i * 1024 + lane * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) spoiled |= (y[e] & T::kExp) == T::kExp || (y[e] >> 16 & T::kExp) == T::kExp;
        }
        if (b < mine - 1 || !__any(spoiled)) {
#pragma unroll
            for (int i = 0; i < NV; ++i) acc[i % ND] = mma32(v_frag(v_last, i), pf[i / ND], acc[i % ND]);
        } else {
            // the values' finite elements, or (of one key of 16) the others; zeros in their place
            typedef __attribute__((ext_vector_type(8))) unsigned short bits8;
            auto elements = [&](frag vf, int key) __attribute__((always_inline)) {
                const bits8 y = __builtin_bit_cast(bits8, vf);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool odd = (y[e] & T::kExp) == T::kExp;
                    vf[e] = (key < 0 ? !odd : odd && 8 * (e / 4) + 4 * h2 + e % 4 == key) ? vf[e] : (elem)0.f;
                }
                return vf;
            };
#pragma unroll
            for (int i = 0; i < NV; ++i) acc[i % ND] = mma32(elements(v_frag(v_last, i), -1), pf[i / ND], acc[i % ND]);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll 1
                for (int key = 0; key < 16; ++key)
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        const pfx16 y = mma32(elements(v_frag(v_last, j * ND + i), key), pf[j], acc[i]);
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][r] = b * 32 + 16 * j + key <= row ? y[r] : acc[i][r];
                    }
        }
    }
    const float sum = lsum + other_half(lsum);
    typedef __attribute__((ext_vector_type(4))) elem elem4;
    if constexpr (SPLIT) {
        // The waves' sums joined, a thread an eighth of a row.
        constexpr int OWN = D / 8;
        static_assert(WAVES == 4 && TILE >= 2 * 32 * D * 4, "two waves' sums in a buffer");
        __shared__ float s_m[WAVES][32], s_l[WAVES][32];
        // (the buffers of the blocks, four floats of a row permuted so that the rows of a write meet all banks)
        auto sums = [&](int w, int line, int four) __attribute__((always_inline)) {
            return reinterpret_cast<float4*>((w & 2 ? m_v0 : m_k0) + (w & 1) * 32 * D * 4) + line * (D / 4) + (four ^ (line & (D / 4 - 1)));
        };
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4)
                *sums(wave, n32, 8 * i + 2 * r4 + h2) = make_float4(acc[i][4 * r4], acc[i][4 * r4 + 1], acc[i][4 * r4 + 2], acc[i][4 * r4 + 3]);
        if (h2 == 0) {
            s_m[wave][n32] = m;
            s_l[wave][n32] = sum;
        }
        __syncthreads();
        const int at = tid / 8, d0 = tid % 8 * 4;            // columns d0 .. d0 + 3 of every 32
        if (row0 + at >= len) return;
        float M = s_m[0][at], total = 0.f, w[WAVES];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) M = fmaxf(M, s_m[i][at]);
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            w[i] = __builtin_amdgcn_exp2f(s_m[i][at] - M);
            total += s_l[i][at] * w[i];
        }
        const float inv = 1.f / total;
        elem* o = reinterpret_cast<elem*>(A.out) + ((int64_t)(begin + row0 + at) * A.Hq + hq) * D + d0;
#pragma unroll
        for (int c = 0; c < OWN / 4; ++c) {
            float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                const float4 x = *sums(i, at, 8 * c + tid % 8);
                y[0] += x.x * w[i];
                y[1] += x.y * w[i];
                y[2] += x.z * w[i];
                y[3] += x.w * w[i];
            }
            elem4 z;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = (elem)in_range<T>(y[e] * inv);
            *reinterpret_cast<elem4*>(o + 32 * c) = z;
        }
        if (A.lse && tid % 8 == 0)
            A.lse[(int64_t)hq * A.T + begin + row0 + at] = (M - T::kShift + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
    } else {
        if (row >= len) return;
        const float inv = 1.f / sum;
        elem* o = reinterpret_cast<elem*>(A.out) + ((int64_t)(begin + row) * A.Hq + hq) * D + 4 * h2;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                elem4 y;
#pragma unroll
                for (int r = 0; r < 4; ++r) y[r] = (elem)in_range<T>(acc[i][4 * r4 + r] * inv);
                *reinterpret_cast<elem4*>(o + 32 * i + 8 * r4) = y;
            }
        if (A.lse && h2 == 0)
            A.lse[(int64_t)hq * A.T + begin + row] = (m - T::kShift + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
}

}  // namespace

// Calls whose row tiles would leave compute units idle take the form that splits a row's keys over four waves: it has four
// times the workgroups, of a quarter of the steps each, and four times the fetches and starts.  Which is faster goes by the
// rows of all heads (512 workgroups, two per compute unit, at 16384) and, beyond that, by how many steps the longest tile
// has, which the mean length stands for; prompts of under four row tiles have nothing to split.  Whole rows / split, us (bf16): 4
// heads x 512 tokens 14.7 / 8.5, x 2048 39 / 17, x 8192 138 / 98, x 12000 213 / 197; 32 heads x 128 8.4 / 6.4, x 512 15.0 / 10.8, x
// 700 17.5 / 19.0, x 1024 24.4 / 24.7; 12 heads x 2500 48 / 38; 4 heads x four of 2000 40 / 34; 32 heads x eight of 64 7.7 / 8.8, x
// four of 200 10.6 / 16.1; 20 heads of 64 x 800 14.1 / 8.4, x 1600 24.3 / 15.9.
bool split_keys(int64_t T, int B, int Hq) {
    const int64_t rows = T * Hq, mean = T / B;
    return (rows <= 16384 && mean >= 128) || (rows <= 32768 && mean >= 1200) || (rows <= 49152 && mean >= 8192);
}

hipError_t launch_prompt(int dtype, int D, PromptArgs A, hipStream_t st) {
    A.scale2 = (float)(1.4426950408889634 / std::sqrt((double)D));
    const bool split = split_keys(A.T, A.B, A.Hq);
    const int rows = split ? 32 : kWaves * 32;
    A.ranks = (int)(A.T / rows) + A.B;                       // every prompt has at most one tile that is not full
    const int64_t groups = (int64_t)A.ranks * A.Hq;
    if (groups >= (int64_t)1 << 24) return hipErrorInvalidValue;   // (2^32 threads; the entry refuses such calls)
    auto launch = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)groups), dim3(kWaves * 64), 0, st, A); };
    auto form = [&](auto wide, auto narrow) { split ? launch(narrow) : launch(wide); };
    if (dtype == 0) D == 128 ? form(prompt_attn<p_bf16, 128, false>, prompt_attn<p_bf16, 128, true>) : form(prompt_attn<p_bf16, 64, false>, prompt_attn<p_bf16, 64, true>);
    else if (dtype == 2) D == 128 ? form(prompt_attn<p_f16, 128, false>, prompt_attn<p_f16, 128, true>) : form(prompt_attn<p_f16, 64, false>, prompt_attn<p_f16, 64, true>);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace snapkv
