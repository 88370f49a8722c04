// Attention of one new token per sequence over paged rows, plain or microscaled, of prefixes that groups of sequences share and of
// the sequences' own.
//
//   out[b, h] = sum_j softmax_j(q[b, h] . k_j / sqrt(D)) v_j,   lse[b, h] = log sum_j exp(q[b, h] . k_j / sqrt(D)),
//
// j over the rows of the prefix of b's group and then over b's own: one pass with the running maximum and sum of each part, and
// the parts joined.  A prefix is met by the query heads of all its sequences that read one KV head, as the columns of the same
// products, in tiles of 16, 32, 64 or 128 (one width for all groups, by their average), so its rows are read once for as many of them.  Rows of caches in 8 or 4 bits become
// bfloat16 numbers (exactly: a code has at most 4 significant bits) between the load and the product; fp16 queries meet them in two
// bfloat16 parts.  (The matrix instructions that take codes and scales themselves keep about 14 bits of a product's sum: not used.)
//
// What bounds it, and what it reaches (us, this card copies at 5.1 TB/s): own rows and small tiles the rows' loads, 32 x 1 to 16384 rows
// of 8 bits 61 (4.6 TB/s), 8 x 16000 of 4 bits, 32 heads 125 (4.4), 131072 of 4 bits 38 (3.7, of which 5 to 6 are the join); wide tiles
// loads and products together, 131071 rows of 8 bits for 16 users 77 (70 with the loads alone), 32749 for 64 users and their own 84.
// One short sequence costs its two launches: 8.9.
//
// MFMA layout (16x16x32): lane l = 16 kg + n supplies row or column n and contraction elements 8 kg .. +7 of an operand; accumulator
// register r of lane l is row 4 kg + r, column n.  Which element of a head is which contraction element is free, as long as
// queries and keys agree: a lane has those that lie side by side in a row of codes (element_of).
//
//   logits^T = K Q^T, 32 keys a step, 16 after 16: a lane gets keys 4 kg .. +3 of both.  out^T = V^T P^T with P in two parts:
//     contraction elements 8 kg .. +7 are those keys, so P never moves.  V goes through LDS, its rows' 16-byte pieces permuted,
//     and comes back by the transposing read (16 lanes read four rows of 16 columns, a lane gets the four of one column).
//
// Tiles of 64 and 128 use 32x32x16 and round P once to the products' type (two parts for fp16 queries over codes): there the products
// count, and a second part would be half as many again.
#include "snapkv_attn.h"
#include "snapkv_sequence.h"
#include "snapkv_serve.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace snapkv {
namespace {

constexpr int kWaves = 4;

// Keys of a share of S: whole steps of all waves, so many that nchunk shares hold it, and at least `least`.
__device__ __forceinline__ int share_of(int S, int nchunk, int least) {
    const int c = (S + nchunk - 1) / nchunk;
    return max(least, (c + 127) / 128 * 128);
}
__device__ __forceinline__ int clamped(int64_t n, int64_t most) { return (int)(n < 0 ? 0 : (n > most ? most : n)); }

// T: the type of queries and outputs; CACHE 0: pages of that type, 1 e4m3, 2 e2m1 codes.
template <typename T, int CACHE> struct kind {
    typedef dec_bf16 mat;                             // of the products
    typedef __bf16 elem;
    static constexpr int kQ = 1;                      // parts of a query
    // Probabilities are taken 2^kShift times as large, and relative to a maximum that is moved, and the sums with it, once it is outgrown by
    // 2^kGrowth.  bf16: values reach from float32's largest to its smallest normal numbers.  2^16 of the largest have a finite sum so (while no maximum
    // is outgrown, 64 at least), and the smallest, 2^-126, keep 8 bits in a product with the largest probability.
    static constexpr float kShift = -16.f, kGrowth = 8.f;
};
template <> struct kind<dec_f16, 0> {
    typedef dec_f16 mat;
    typedef _Float16 elem;
    static constexpr int kQ = 1;
    static constexpr float kShift = 15.f, kGrowth = 0.f;   // (two fp16 parts of one keep 20 bits down to 2^-19 of the largest so)
};
template <int CACHE> struct kind<dec_f16, CACHE> {
    typedef dec_bf16 mat;
    typedef _Float16 elem;
    static constexpr int kQ = 2;
    static constexpr float kShift = -16.f, kGrowth = 8.f;
};

// The head's element that is contraction element j of lane group kg in product c.
template <int CACHE, int D> __device__ __forceinline__ constexpr int element_of(int kg, int c, int j) {
    return CACHE == 0 ? 32 * c + 8 * kg + j : D / 4 * kg + 8 * c + j;
}

// Eight values of codes (of 8 bits: both words, of 4: the first) under a scale byte, as bfloat16 numbers.
template <int CACHE> __device__ __forceinline__ uint4 values_of(unsigned w0, unsigned w1, unsigned s) {
    const float u = __uint_as_float(s << 23);
    if constexpr (CACHE == 1)
        return make_uint4(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, u, false)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, u, true)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, u, false)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, u, true)));
    else
        return make_uint4(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, u, 0)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, u, 1)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, u, 2)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, u, 3)));
}

// Bytes of a row of codes or elements.
template <int CACHE, int D> constexpr int row_bytes() { return CACHE == 0 ? 2 * D : (CACHE == 1 ? D : D / 2); }

// Eight of a query's elements as one operand, or the two operands whose sum they are (11 bits: the high part has 8).
template <typename T, int CACHE> __device__ __forceinline__ void query_operands(uint4 x, uint4* q) {
    if constexpr (kind<T, CACHE>::kQ == 1) {
        q[0] = x;
    } else {
        const df16x8 h = __builtin_bit_cast(df16x8, x);
        unsigned hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) split2(dec_bf16{}, (float)h[2 * i], (float)h[2 * i + 1], hi[i], lo[i]);
        q[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        q[1] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// What a workgroup has to do: keys begin .. end - 1 of the rows that `table` names, for the query heads row0 .. of rows of them,
// sequence by sequence from b0 on, that read KV head kvh (or, a wave each and so fewer waves a head, that and the next 2^shift - 1); its answer is
// partial `slot` of theirs, or (slot < 0) the whole.
struct Task {
    int b0, row0, rows, kvh, shift;
    const int32_t* table;
    int begin, end, slot;
};

// Where a key's row lies, in bytes of codes or elements of the pool (the row's scales lie a 32nd of that behind theirs, a 16th for 4-bit codes).
// The table is read some time before the place is used.
template <int ROW> struct Rows {
    struct Place {
        int entry, line;                               // of the table, and row within the page
    };
    const int32_t* table;
    unsigned token, magic;                             // bytes between the rows of a page; of the division by the page size
    uint64_t page_bytes;
    int last, page, shift, last_page;
    __device__ __forceinline__ Rows(const SharedArgs& A, const Task& W)
        : table(W.table), token((unsigned)A.Hkv * ROW), magic(A.page_magic), page_bytes((uint64_t)((unsigned)A.Hkv * ROW) * (unsigned)A.page),
          last(W.end - 1), page(A.page), shift(A.page_shift), last_page(A.last_page) {}
    __device__ __forceinline__ Place look_up(int key) const {
        const int r = min(key, last);                  // (behind the end: the last row again)
        const int pg = (int)(__umulhi((unsigned)r << 1, magic) >> shift);
        return Place{table[pg], r - pg * page};
    }
    __device__ __forceinline__ int64_t place(const Place& p) const {
        const unsigned at = (unsigned)min(max(p.entry, 0), last_page);
        return (int64_t)(at * page_bytes + (uint64_t)token * (unsigned)p.line);
    }
};

// LDS of a workgroup: a step's rows and places of each wave, the scales of 128 keys and values of all its KV heads, and behind the loop the waves' sums.
template <int D> union Shared {
    struct {
        char rows[kWaves][32 * 2 * D];
        int64_t places[kWaves][32];
        unsigned char scales[32 * kWaves * 2 * 4 * (D / 32)];
    } step;
    struct {
        float acc[kWaves][16][D + 4], m[kWaves][16], l[kWaves][16];
    } sum;
};
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) char* lds_char;

// Which of its row's 16-byte places in LDS holds a piece of a value row (the four rows of a transposing read are in different banks, and those
// of a write), and of a key row (those of eight lanes that read one piece each are).
// (Both permutations turn bits of the place by bits of the row: what rows apart by a multiple of a lane's rows differ by is a constant.)
template <int D> __device__ __forceinline__ constexpr int place_of(int row, int piece) {
    return piece ^ ((row & 3) << 1 | (D == 128 ? (row >> 2 & 1) << 3 | (row >> 3 & 1) : row >> 2 & 1));
}
template <int ROW> __device__ __forceinline__ constexpr int key_place_of(int row, int piece) {
    constexpr int PIECES = ROW / 16;
    return piece ^ (row / (PIECES < 8 ? 8 / PIECES : 1) & (PIECES - 1));
}

// 32 rows on their way from the pool through a wave's registers to its LDS: neighbouring lanes have neighbouring 16 bytes, which costs the
// least of the look-ups that the first cache does (8 x 16000 rows of 4 bits, 32 heads: 176 us with a row's pieces 16 lanes apart, as products take them).
// PAST: past the caches' lasting part, for rows that are whole lines and met once (8-bit rows: 8 x 16000, 32 heads 193 us without, 170 with, 6.3 TB/s; 32 sequences
// of 1 to 16384, 8 heads 70 / 61.5; of 4 bits, two heads' rows to a line, 125 / 136).
template <int CACHE, int D, bool PAST> struct Stage {
    static constexpr int ROW = row_bytes<CACHE, D>(), LPR = ROW / 16, RPI = 64 / LPR, N = 32 / RPI;   // lanes of a row; rows of a load; loads
    u32x4 w[N];
    // base: the lane's part of the pool's first row
    __device__ __forceinline__ void load(const char* base, const int64_t* at) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (PAST) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base + at[i]));
            else w[i] = *reinterpret_cast<const u32x4*>(base + at[i]);
        }
    }
    // A lane's places in LDS: of its first key's codes or elements, its first value's first piece.
    static __device__ __forceinline__ unsigned key_at(int lane) { return lane / LPR * ROW + key_place_of<ROW>(lane / LPR, lane % LPR) * 16; }
    static __device__ __forceinline__ unsigned value_at(int lane) { return lane / LPR * (2 * D) + place_of<D>(lane / LPR, lane % LPR * P) * 16; }
    static constexpr int P = D / 8 / LPR;              // pieces of a lane's values
    __device__ __forceinline__ void store_keys(char* rows, unsigned at) const {
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4*>(rows + (at ^ (unsigned)(key_place_of<ROW>(i * RPI, 0) * 16)) + i * RPI * ROW) = w[i];
    }
    // scales: of the lane's first row, `apart` bytes from one row's to the next's.
    __device__ __forceinline__ void store_values(char* rows, unsigned at, const unsigned char* scales, int apart) const {
        unsigned s[N];
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = CACHE ? scales[i * RPI * apart] : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            auto put = [&](int c, uint4 y) __attribute__((always_inline)) {
                *reinterpret_cast<uint4*>(rows + (at ^ (unsigned)(place_of<D>(i * RPI, c) * 16)) + i * RPI * (2 * D)) = y;
            };
            if constexpr (CACHE == 0) {
                put(0, make_uint4(w[i].x, w[i].y, w[i].z, w[i].w));
            } else if constexpr (CACHE == 1) {
                put(0, values_of<1>(w[i].x, w[i].y, s[i]));
                put(1, values_of<1>(w[i].z, w[i].w, s[i]));
            } else {
                put(0, values_of<2>(w[i].x, 0, s[i]));
                put(1, values_of<2>(w[i].y, 0, s[i]));
                put(2, values_of<2>(w[i].z, 0, s[i]));
                put(3, values_of<2>(w[i].w, 0, s[i]));
            }
        }
    }
};
// A lane's part of a key row, as the products take it: lane group kg has the elements element_of.
template <int CACHE, int D> struct Key {
    static constexpr int ROW = row_bytes<CACHE, D>(), WORDS = ROW / 16;
    unsigned w[WORDS], s;
    static __device__ __forceinline__ unsigned at(int row, int kg) {       // of the first piece
        return row * ROW + key_place_of<ROW>(row, CACHE == 0 ? kg : (WORDS >= 4 ? kg * (WORDS / 4) : kg / 2)) * 16 + (WORDS >= 4 ? 0 : (kg & 1) * 8);
    }
    // row: 0, or 16 for the row as many further on, which has the same permutation
    __device__ __forceinline__ void read(const char* rows, unsigned at, int row) {
#pragma unroll
        for (int i = 0; i < (WORDS + 3) / 4; ++i) {
            const char* p = rows + (at ^ (unsigned)(i * (CACHE == 0 ? 64 : 16))) + row * ROW;
            if constexpr (WORDS >= 4) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(p);
                w[4 * i] = x.x;
                w[4 * i + 1] = x.y;
                w[4 * i + 2] = x.z;
                w[4 * i + 3] = x.w;
            } else {
                const uint2 x = *reinterpret_cast<const uint2*>(p);
                w[0] = x.x;
                w[1] = x.y;
            }
        }
    }
    __device__ __forceinline__ uint4 operand(int c) const {
        if constexpr (CACHE == 0) return make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        else if constexpr (CACHE == 1) return values_of<1>(w[2 * c], w[2 * c + 1], s);
        else return values_of<2>(w[c], 0, s);
    }
};

// The largest x of the four lanes that have a query's keys.
__device__ __forceinline__ float across_groups(float x) {
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    const auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1]));
}

// The other half of the wave: lane l gets lane l ^ 32's value.
__device__ __forceinline__ float other_half(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float((threadIdx.x & 32) ? y[0] : y[1]);
}

template <typename T, int CACHE, int D, int NC, bool PAST = false>
__device__ __forceinline__ void attend(const SharedArgs& A, const Task& W, Shared<D>& s) {
    typedef kind<T, CACHE> K;
    typedef typename K::mat M;
    typedef typename K::elem elem;
    constexpr int NP = D / 32;        // products along a head
    constexpr int NB = D / 16;        // blocks of 16 output elements
    constexpr float kShift = K::kShift;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, kg = lane >> 4;
    const int heads = 1 << W.shift, kvh = W.kvh + (wave & (heads - 1)), part = wave >> W.shift;
    auto head_of = [&](int row, int kvh) { return ((int64_t)W.b0 + row / A.g) * A.Hq + (int64_t)kvh * A.g + row % A.g; };

    uint4 qf[NC][NP][K::kQ];
#pragma unroll
    for (int b = 0; b < NC; ++b) {
        const int row = W.row0 + 16 * b + n16;
        const char* q = A.q + (row < W.rows ? head_of(row, kvh) : 0) * (2 * D);
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row < W.rows) x = *reinterpret_cast<const uint4*>(q + 2 * element_of<CACHE, D>(kg, c, 0));
            query_operands<T, CACHE>(x, qf[b][c]);
        }
    }
    char* const sv = s.step.rows[wave];
    int64_t* const places = s.step.places[wave];
    const int tr = 4 * kg + (n16 >> 2);                // row and place of the lane's first transposing read
    unsigned tr_at = tr * (2 * D) + place_of<D>(tr, (n16 & 3) >> 1) * 16 + (n16 & 1) * 8;
    unsigned key_at = Stage<CACHE, D, PAST>::key_at(lane), value_at = Stage<CACHE, D, PAST>::value_at(lane), operand_at = Key<CACHE, D>::at(n16, kg);
    float m[NC], lsum[NC];
    dfx4 acc[NC][NB];
#pragma unroll
    for (int b = 0; b < NC; ++b) {
        m[b] = -3.4028235e38f;                         // (finite: logits of -infinity have probability 0 and not NaN)
        lsum[b] = 0.f;
#pragma unroll
        for (int i = 0; i < NB; ++i) acc[b][i] = dfx4{0.f, 0.f, 0.f, 0.f};
    }
    typedef Stage<CACHE, D, PAST> Rows32;
    constexpr int ROW = Rows32::ROW, LPR = Rows32::LPR;
    const int STEP = 32 * kWaves >> W.shift;
    const Rows<ROW> rows(A, W);
    const int lane_at = kvh * ROW + lane % LPR * 16;
    const char *kb = A.k + lane_at, *vb = A.v + lane_at;
    Rows32 kr, vr;
    typename Rows<ROW>::Place p{};
    // Places of a step's rows: lane l finds that of row l % 32, and gets those of the rows it loads.
    auto store_places = [&]() {
        places[lane & 31] = rows.place(p);
        asm volatile("" ::: "memory");                 // (a wave's LDS operations are done in order)
    };
    auto load_from = [&](Rows32& r, const char* base) {
        int64_t at[Rows32::N];
#pragma unroll
        for (int i = 0; i < Rows32::N; ++i) at[i] = places[i * Rows32::RPI + lane / LPR];
        asm volatile("" ::: "memory");
        r.load(base, at);
        __builtin_amdgcn_sched_barrier(0);
    };
    const float rest = K::kGrowth / A.scale2;
    // Scales of 128 rows at a time: a lane fetches those of all the workgroup's KV heads of one key or value row at once (a line of the first cache
    // has up to 32 heads' scales; fetched by every head for itself they cost as much as the codes), and LDS hands them out.
    // With one KV head the rows that a wave fetches scales of are those it meets, and nothing is to be waited for.
    constexpr int NS = D / 32;
    const int apart = 2 * (NS << W.shift);             // bytes from a row's scales to the next's: keys', values'
    unsigned char* const mine = s.step.scales + (32 * wave + (lane & 31)) * apart + (lane >> 5) * (apart / 2);
    const unsigned char* const sb = CACHE ? (lane < 32 ? A.k_scales : A.v_scales) + W.kvh * NS : nullptr;
    u32x4 sr{};
    typename Rows<ROW>::Place sp{};
    auto load_scales = [&]() {
        const unsigned char* from = sb + (rows.place(sp) >> (CACHE == 1 ? 5 : 4));
        if (apart == 32) sr = *reinterpret_cast<const u32x4*>(from);
        else if (apart == 16) sr.xy = *reinterpret_cast<const u32x2*>(from);
        else if (apart == 8) sr.x = *reinterpret_cast<const unsigned*>(from);
        else sr.x = *reinterpret_cast<const unsigned short*>(from);
    };
    auto store_scales = [&]() {
        if (apart == 32) *reinterpret_cast<u32x4*>(mine) = sr;
        else if (apart == 16) *reinterpret_cast<u32x2*>(mine) = sr.xy;
        else if (apart == 8) *reinterpret_cast<unsigned*>(mine) = sr.x;
        else *reinterpret_cast<unsigned short*>(mine) = (unsigned short)sr.x;
    };
    int key = W.begin + 32 * part, block = W.begin + 32 * wave + (lane & 31);
    // (waves that share scales take the same number of steps)
    const int stop = CACHE != 0 && W.shift > 0 ? W.end + 32 * part : W.end;
    if (key < stop) {
        p = rows.look_up(key + (lane & 31));
        if constexpr (CACHE != 0) {
            sp = rows.look_up(block);
            load_scales();
            sp = rows.look_up(block + 32 * kWaves);
        }
        store_places();
        // (loads are waited for in their order: the same as in the loop, or its waits are longer)
        p = rows.look_up(key + STEP + (lane & 31));
        __builtin_amdgcn_sched_barrier(0);
        load_from(kr, kb);
        load_from(vr, vb);
    }
    for (int round = 0; key < stop; key += STEP, ++round) {
        const int among = round & (heads - 1);         // of the steps that 128 rows are
        if (CACHE != 0 && among == 0) {
            if (W.shift > 0) __syncthreads();          // (the ones before have been read)
            store_scales();
            if (W.shift > 0) __syncthreads();
            block += 32 * kWaves;
            load_scales();
            sp = rows.look_up(block + 32 * kWaves);
        }
        store_places();                                // of the next step
        p = rows.look_up(key + 2 * STEP + (lane & 31));
        __builtin_amdgcn_sched_barrier(0);
        Key<CACHE, D> kx, ky;
        // (sums of a place and a constant, made once in front of the loop, would take more registers than there are)
        asm volatile("" : "+v"(tr_at), "+v"(key_at), "+v"(value_at), "+v"(operand_at));
        kr.store_keys(sv, key_at);
        asm volatile("" ::: "memory");
        kx.read(sv, operand_at, 0);
        ky.read(sv, operand_at, 16);
        const unsigned char* const scales = s.step.scales + (among * STEP + 32 * part) * apart + (wave & (heads - 1)) * NS;
        if constexpr (CACHE != 0) {
            const unsigned char* own = scales + n16 * apart + kg * (D / 4) / 32;
            kx.s = own[0];
            ky.s = own[16 * apart];
        }
        load_from(kr, kb);
        dfx4 sx[NC], sy[NC];
#pragma unroll
        for (int b = 0; b < NC; ++b) sx[b] = sy[b] = dfx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NP; ++c) {
            const uint4 ox = kx.operand(c), oy = ky.operand(c);
#pragma unroll
            for (int b = 0; b < NC; ++b)
#pragma unroll
                for (int i = 0; i < K::kQ; ++i) {
                    sx[b] = mma(M{}, ox, qf[b][c][i], sx[b]);
                    sy[b] = mma(M{}, oy, qf[b][c][i], sy[b]);
                }
        }
        if (key + 32 > W.end) {                        // the last step
            const int k0 = key + 4 * kg;
#pragma unroll
            for (int b = 0; b < NC; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    sx[b][r] = k0 + r < W.end ? sx[b][r] : -INFINITY;
                    sy[b][r] = k0 + 16 + r < W.end ? sy[b][r] : -INFINITY;
                }
        }
        // m: in units of the logits before their scaling
        bool grown = false;
        float top[NC];
#pragma unroll
        for (int b = 0; b < NC; ++b) {
            top[b] = fmaxf(fmaxf(fmaxf(sx[b][0], sx[b][1]), fmaxf(sx[b][2], sx[b][3])), fmaxf(fmaxf(sy[b][0], sy[b][1]), fmaxf(sy[b][2], sy[b][3])));
            grown |= top[b] > m[b] + rest;
        }
        if (__any(grown)) {
#pragma unroll
            for (int b = 0; b < NC; ++b) {
                const float mn = fmaxf(m[b], across_groups(top[b]));
                const float alpha = __builtin_amdgcn_exp2f((m[b] - mn) * A.scale2);
                m[b] = mn;
                lsum[b] *= alpha;
#pragma unroll
                for (int i = 0; i < NB; ++i) acc[b][i] *= alpha;
            }
        }
        uint4 ph[NC], pl[NC];
#pragma unroll
        for (int b = 0; b < NC; ++b) {
            const float shift = kShift - m[b] * A.scale2;
            float e[8], sum[2];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sx[b][r], A.scale2, shift));
                e[4 + r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sy[b][r], A.scale2, shift));
            }
            sum[0] = e[0] + e[4];
            sum[1] = e[1] + e[5];
            sum[0] += e[2] + e[6];
            sum[1] += e[3] + e[7];
            lsum[b] += sum[0] + sum[1];
            split2(M{}, e[0], e[1], ph[b].x, pl[b].x);
            split2(M{}, e[2], e[3], ph[b].y, pl[b].y);
            split2(M{}, e[4], e[5], ph[b].z, pl[b].z);
            split2(M{}, e[6], e[7], ph[b].w, pl[b].w);
        }
        asm volatile("" ::: "memory");
        vr.store_values(sv, value_at, scales + apart / 2 + lane / LPR * apart + lane % LPR / (CACHE ? LPR / NS : 1), apart);
        asm volatile("" ::: "memory");
        load_from(vr, vb);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const lds_char from = (lds_char)sv + (tr_at ^ (unsigned)(i * 32));
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)from);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(from + 16 * 2 * D));
            const uint4 vt = __builtin_bit_cast(uint4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int b = 0; b < NC; ++b) {
                acc[b][i] = mma(M{}, vt, ph[b], acc[b][i]);
                acc[b][i] = mma(M{}, vt, pl[b], acc[b][i]);
            }
        }
        asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int b = 0; b < NC; ++b) m[b] = m[b] * A.scale2 - kShift;   // (probabilities are 2^(logit - that) now)
    __syncthreads();                                   // (all waves have read their values)
    constexpr int DT = D / 16;
    const int qi = tid >> 4, d0 = (tid & 15) * DT;
#pragma unroll
    for (int b = 0; b < NC; ++b) {
        if (b > 0) __syncthreads();                    // (the waves have read the block before)
        lsum[b] += __shfl_xor(lsum[b], 16);
        lsum[b] += __shfl_xor(lsum[b], 32);
#pragma unroll
        for (int i = 0; i < NB; ++i)
            *reinterpret_cast<float4*>(&s.sum.acc[wave][n16][16 * i + 4 * kg]) = make_float4(acc[b][i][0], acc[b][i][1], acc[b][i][2], acc[b][i][3]);
        if (kg == 0) {
            s.sum.m[wave][n16] = m[b];
            s.sum.l[wave][n16] = lsum[b];
        }
        __syncthreads();
        // 16 threads an item: a query head of one of the KV heads
        const int here = min(16, W.rows - W.row0 - 16 * b);
        for (int item = qi; item < heads * here; item += 16) {
            const int head = item / here, n = item - head * here, row = W.row0 + 16 * b + n;
            float most = s.sum.m[head][n];
            for (int w = head + heads; w < kWaves; w += heads) most = fmaxf(most, s.sum.m[w][n]);
            float Lq = 0.f, o[DT];
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] = 0.f;
            for (int w = head; w < kWaves; w += heads) {
                const float f = __builtin_amdgcn_exp2f(s.sum.m[w][n] - most);
                Lq += s.sum.l[w][n] * f;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] += s.sum.acc[w][n][d0 + d] * f;
            }
            const int64_t hq = head_of(row, W.kvh + head);
            if (W.slot < 0) {
                const float inv = Lq == 0.f ? 0.f : 1.f / Lq;      // (no rows; a sum that is NaN makes the row's answer NaN)
                elem* out = reinterpret_cast<elem*>(A.out) + hq * D + d0;
#pragma unroll
                for (int d = 0; d < DT; ++d) out[d] = (elem)(o[d] * inv);
                if (A.lse && (tid & 15) == 0)
                    A.lse[hq] = Lq == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(Lq)) * 0.6931471805599453f;
            } else {
                float* pa = A.part_acc + (hq * A.slots + W.slot) * D + d0;
#pragma unroll
                for (int d = 0; d < DT; ++d) pa[d] = o[d];
                if ((tid & 15) == 0) A.part_ml[hq * A.slots + W.slot] = make_float2(most, Lq);
            }
        }
    }
}

typedef __attribute__((ext_vector_type(8))) short frag;          // an operand's eight elements
typedef __attribute__((ext_vector_type(16))) float fx16;
__device__ __forceinline__ fx16 mma32(dec_bf16, frag a, frag b, fx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(dbf16x8, a), __builtin_bit_cast(dbf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ fx16 mma32(dec_f16, frag a, frag b, fx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(df16x8, a), __builtin_bit_cast(df16x8, b), c, 0, 0, 0);
}

// LDS of a workgroup that meets a prefix's rows with 64 or 128 query heads: two tiles each of keys and values, and behind the loop the
// waves' sums.
constexpr int kKeys = 64;      // keys of a tile
constexpr int kPlaces = 4 * kKeys;
template <int D> struct Wide {
    union {
        struct {
            char k[2][kKeys * 2 * D], v[2][kKeys * 2 * D];
        } tile;
        float acc[kWaves][32][D];
    };
    union {
        int64_t places[kPlaces];                      // of the rows around the tiles: row r's is number r % kPlaces
        struct {
            float m[kWaves][32], l[kWaves][32];
        } sum;
    };
};

// Rows of long prefixes go past the caches' lasting part (plain 131071 rows, 8 heads, 16 users 119 us without, 107 with; 64 users of 32749 rows 91 / 87).
constexpr int kPast = 2;       // (of a load into LDS: the bit for that)

// A lane's part of a tile on its way from the pool to LDS.  Plain rows go there by themselves, 16 bytes a lane at a time; codes pass
// through registers, a block of 32 of a key and a value row per thread (heads of 64: of one of them).
template <typename T, int CACHE, int D> struct Fetch;
template <typename T, int D> struct Fetch<T, 0, D> {
    static constexpr int PIECES = D / 8, RPL = 64 / PIECES, PER = kKeys / (RPL * kWaves);   // 16-byte pieces of a row; rows of a load; loads
    const char *kb, *vb;
    int first;                                        // row of the lane's first load
    __device__ __forceinline__ Fetch(const SharedArgs& A, const Task& W, int wave, int lane) {
        first = wave * RPL + lane / PIECES;           // (rows of the others have the same places)
        kb = A.k + W.kvh * (2 * D) + ((lane % PIECES) ^ (first & (PIECES - 1))) * 16;
        vb = A.v + W.kvh * (2 * D) + place_of<D>(first, lane % PIECES) * 16;
    }
    // Keys of rows from k on, values of rows from v on.
    __device__ __forceinline__ void start(const int64_t* places, int k, int v, char* to_k, char* to_v, int wave) {
        typedef __attribute__((address_space(1))) void* from;
        typedef __attribute__((address_space(3))) void* to;
        int64_t pk[PER], pv[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            pk[i] = places[(k + i * RPL * kWaves + first) & (kPlaces - 1)];
            pv[i] = places[(v + i * RPL * kWaves + first) & (kPlaces - 1)];
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            __builtin_amdgcn_global_load_lds((from)(kb + pk[i]), (to)(to_k + (i * kWaves + wave) * 1024), 16, 0, kPast);
            __builtin_amdgcn_global_load_lds((from)(vb + pv[i]), (to)(to_v + (i * kWaves + wave) * 1024), 16, 0, kPast);
        }
    }
    // (such loads write no register that the compiler would wait for, and a barrier alone does not wait)
    __device__ __forceinline__ void finish(char*, char*) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};
template <typename T, int CACHE, int D> struct Fetch {
    static constexpr int ROW = row_bytes<CACHE, D>(), BLOCKS = D / 32, N = D == 128 ? 2 : 1, W4 = CACHE == 1 ? 8 : 4;   // N: blocks of a thread; its words
    int key, block, tensor;
    const char* base[N];
    const unsigned char* scales[N];
    unsigned w[N][W4], s[N];
    __device__ __forceinline__ Fetch(const SharedArgs& A, const Task& W, int wave, int lane) {
        const int tid = wave * 64 + lane;
        tensor = N == 2 ? 0 : tid / (kKeys * BLOCKS);
        key = tid / BLOCKS % kKeys;
        block = tid % BLOCKS;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            base[n] = (tensor + n == 0 ? A.k : A.v) + W.kvh * ROW + block * (ROW / BLOCKS);
            scales[n] = (tensor + n == 0 ? A.k_scales : A.v_scales) + W.kvh * BLOCKS + block;
        }
    }
    __device__ __forceinline__ void start(const int64_t* places, int k, int v, char*, char*, int) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int64_t at = places[((tensor + n == 0 ? k : v) + key) & (kPlaces - 1)];
#pragma unroll
            for (int i = 0; i < W4 / 4; ++i) {
                u32x4 x;              // (4 bits: a block is all that a thread loads of its row; the halves of one of 8 bits would be fetched twice)
                if constexpr (CACHE == 2) x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(base[n] + at));
                else x = *reinterpret_cast<const u32x4*>(base[n] + at + 16 * i);
                w[n][4 * i] = x.x;
                w[n][4 * i + 1] = x.y;
                w[n][4 * i + 2] = x.z;
                w[n][4 * i + 3] = x.w;
            }
            s[n] = scales[n][at >> (CACHE == 1 ? 5 : 4)];
        }
    }
    __device__ __forceinline__ void finish(char* k, char* v) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bool is_k = tensor + n == 0;
            char* to = (is_k ? k : v) + key * (2 * D);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int piece = 4 * block + c, at = is_k ? piece ^ (key & (D / 8 - 1)) : place_of<D>(key, piece);
                *reinterpret_cast<uint4*>(to + at * 16) = values_of<CACHE>(w[n][c * (W4 / 4)], w[n][c * (W4 / 4) + (W4 / 4 - 1)], s[n]);
            }
        }
    }
};

// attend for up to 32 RB query heads in products of 32x32x16: lane l = 32 h + n supplies row or column n and contraction elements 8 h .. +7; register
// r of lane l is row 8 (r / 4) + 4 h + r % 4, column n.  RB waves have 32 query heads each, and each of the 4 / RB such sets every other block
// of 32 keys; all share the tiles in LDS.  The probabilities of a lane, 16 keys of one query head a block, enter the last product as they are (contraction
// element e stands for key 8 (e / 4) + 4 h + e % 4 of 16), rounded to its type once, or, fp16 queries over codes, whose products are in bfloat16, in two parts.
template <typename T, int CACHE, int D, int RB>
__device__ __forceinline__ void attend_wide(const SharedArgs& A, const Task& W, Wide<D>& s) {
    typedef kind<T, CACHE> K;
    typedef typename K::mat M;
    constexpr int KS = kWaves / RB;                   // waves that share the keys
    constexpr int NQ = D / 16, ND = D / 32;           // products along a head; blocks of 32 output elements
    constexpr bool kF16 = CACHE == 0 && std::is_same<T, dec_f16>::value;
    // exponent that probabilities are raised by, and the most that a lane's 16 may sum up to before its maximum is moved: 2^8 or 2^10 above it
    constexpr float kShift = kF16 ? 7.f : K::kShift, kMost = kF16 ? 32768.f : 0x1p-6f;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, h2 = lane >> 5, rb = wave % RB, ks = wave / RB;
    auto head_of = [&](int row) { return ((int64_t)W.b0 + row / A.g) * A.Hq + (int64_t)W.kvh * A.g + row % A.g; };
    const bool busy = W.row0 + 32 * rb < W.rows;      // the wave has query heads at all

    frag qf[NQ][K::kQ];
    {
        const int row = min(W.row0 + 32 * rb + n32, W.rows - 1);      // (behind the last: it again, and nothing is stored)
        const char* q = A.q + head_of(row) * (2 * D) + 16 * h2;
#pragma unroll
        for (int c = 0; c < NQ; ++c) {
            uint4 x[K::kQ];
            query_operands<T, CACHE>(*reinterpret_cast<const uint4*>(q + 32 * c), x);
#pragma unroll
            for (int i = 0; i < K::kQ; ++i) qf[c][i] = __builtin_bit_cast(frag, x[i]);
        }
    }
    float m = -3.4028235e38f, lsum = 0.f;             // (finite: logits of -infinity have probability 0 and not NaN)
    fx16 acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    const Rows<row_bytes<CACHE, D>()> rows(A, W);
    Fetch<T, CACHE, D> fetch(A, W, wave, lane);
    // a lane's places in a tile: its pieces of key row n32, and of the first value row that it transposes
    const int vr = 4 * h2 + (lane & 15) / 4;
    const unsigned k_at = n32 * (2 * D) + ((h2 ^ (n32 & (D / 8 - 1))) * 16);
    const unsigned v_at = vr * (2 * D) + place_of<D>(vr, 2 * ((lane >> 4) & 1) + (lane & 3) / 2) * 16 + (lane & 1) * 8;
    constexpr unsigned kTurn = D == 128 ? 16 : 0;     // (what rows 8 further down differ by)

    auto probabilities = [&](const fx16& x, float* e, float* sum) __attribute__((always_inline)) {
        const float shift = kShift - m;
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r] = __builtin_fmaf(x[r], A.scale2, shift);
#pragma unroll
        for (int r = 0; r < 16; ++r) e[r] = __builtin_amdgcn_exp2f(e[r]);
        sum[0] = e[0];
        sum[1] = e[1];
#pragma unroll
        for (int r = 2; r < 16; ++r) sum[r & 1] += e[r];
    };
    auto k_frag = [&](const char* sk, int c) __attribute__((always_inline)) { return *reinterpret_cast<const frag*>(sk + (k_at ^ (unsigned)(c * 32))); };
    auto v_frag = [&](const char* sv, int n) __attribute__((always_inline)) {      // 32 columns n % ND of 16 keys n / ND
        const unsigned at = (v_at ^ (unsigned)(n % ND * 64)) + n / ND * 16 * (2 * D);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)((lds_char)sv + at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)((lds_char)sv + (at ^ kTurn) + 8 * (2 * D)));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    fx16 x;                                           // logits of the wave's next block of keys
    auto product = [&](frag kf, int c) __attribute__((always_inline)) {
        fx16 z;
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
        for (int i = 0; i < K::kQ; ++i) x = mma32(M{}, kf, qf[c][i], c == 0 && i == 0 ? z : x);
    };
    auto hide = [&](int key) __attribute__((always_inline)) {                      // logits of keys behind the end
        if (key + 32 <= W.end) return;
        asm volatile("");                             // (a branch: 32 instructions otherwise)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (key + 8 * (r / 4) + 4 * h2 + r % 4 >= W.end) x[r] = -INFINITY;
    };
    // The softmax of the block whose logits are there, which only vector instructions do, then the products of the wave's next block's logits and
    // of this one's part of the output, which only matrix instructions do: the other wave of the SIMD is in the other half
    // meanwhile, and goes second.  Operands are read from LDS AHEAD products before their own.
    constexpr int NV = 2 * ND, AHEAD = 3;
    auto pass = [&](int next, const char* sk, const char* sv) __attribute__((always_inline)) {
        frag kf[NQ], vf[NV], pf[2][K::kQ];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) kf[i] = k_frag(sk, i);
        __builtin_amdgcn_sched_barrier(0);
        float e[16], sum[2];
        probabilities(x, e, sum);
        // A row's maximum is looked for, and its sums moved to it, only when they outgrow kMost.  (A row's two lanes have other halves of the keys.)
        const float both = sum[0] + sum[1];
        if (__any(both > kMost)) {
            float big = x[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) big = fmaxf(big, x[r]);
            const float others = other_half(both), top = fmaxf(big, other_half(big)) * A.scale2;
            const float mn = both > kMost || others > kMost ? fmaxf(m, top) : m;
            const float alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            lsum *= alpha;
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= alpha;
            probabilities(x, e, sum);
        }
        lsum += sum[0] + sum[1];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (K::kQ == 1) {
                typedef typename std::conditional<kF16, _Float16, __bf16>::type elem;
                __attribute__((ext_vector_type(8))) elem y;
#pragma unroll
                for (int r = 0; r < 8; ++r) y[r] = (elem)e[8 * j + r];
                pf[j][0] = __builtin_bit_cast(frag, y);
            } else {
                unsigned hi[4], lo[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) split2(dec_bf16{}, e[8 * j + 2 * r], e[8 * j + 2 * r + 1], hi[r], lo[r]);
                pf[j][0] = __builtin_bit_cast(frag, make_uint4(hi[0], hi[1], hi[2], hi[3]));
                pf[j][K::kQ - 1] = __builtin_bit_cast(frag, make_uint4(lo[0], lo[1], lo[2], lo[3]));
            }
        }
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (i + AHEAD < NQ) kf[i + AHEAD] = k_frag(sk, i + AHEAD);
            else vf[i + AHEAD - NQ] = v_frag(sv, i + AHEAD - NQ);
            product(kf[i], i);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i + AHEAD < NV) vf[i + AHEAD] = v_frag(sv, i + AHEAD);
#pragma unroll
            for (int n = 0; n < K::kQ; ++n) acc[i % ND] = mma32(M{}, vf[i], pf[i / ND][n], acc[i % ND]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        hide(next);
    };
    // Keys are a block of every wave set ahead of values: tile t of V is keys 64 t on, that of K keys 64 t + EARLY on, whose logits are taken meanwhile.
    // The next tiles arrive in the other two buffers.
    constexpr int EARLY = 32 * KS;
    const int tiles = (W.end - W.begin + kKeys - 1) / kKeys;
    // Places: a thread finds one of the first 256 rows, and 64 more for every tile, two tiles ahead, are shared out to the waves (the page is looked
    // up yet a tile before).  A lane that looked up the rows it loads did as much for that as for the softmax.
    s.places[(W.begin + tid) & (kPlaces - 1)] = rows.place(rows.look_up(W.begin + tid));
    auto page = rows.look_up(W.begin + 4 * kKeys + 16 * wave + (lane & 15));
    __syncthreads();
    fetch.start(s.places, W.begin, W.begin, s.tile.k[1], s.tile.v[0], wave);
    fetch.finish(s.tile.k[1], s.tile.v[0]);
    fetch.start(s.places, W.begin + EARLY, W.begin, s.tile.k[0], s.tile.v[0], wave);
    __syncthreads();
    if (busy) {
        const char* sk = s.tile.k[1] + (KS == 1 ? 0 : ks) * 32 * (2 * D);
#pragma unroll
        for (int i = 0; i < NQ; ++i) product(k_frag(sk, i), i);
        hide(W.begin + (KS == 1 ? 0 : ks) * 32);
    }
    fetch.finish(s.tile.k[0], s.tile.v[0]);
    __syncthreads();
    auto tile = [&](int t, int now) __attribute__((always_inline)) {
        const int key = W.begin + t * kKeys;
        char *k_now = s.tile.k[now], *v_now = s.tile.v[now], *k_next = s.tile.k[now ^ 1], *v_next = s.tile.v[now ^ 1];
        if (t + 1 < tiles) {
            fetch.start(s.places, key + kKeys + EARLY, key + kKeys, k_next, v_next, wave);
            // (rows of tile t + 4 take the places of those of tile t, which all have read)
            s.places[(key + 4 * kKeys + 16 * wave + (lane & 15)) & (kPlaces - 1)] = rows.place(page);
            page = rows.look_up(key + 5 * kKeys + 16 * wave + (lane & 15));
        }
        if (busy) {
#pragma unroll
            for (int i = 0; i < 2 / KS; ++i) {
                const int b = KS == 1 ? i : ks;
                if (key + 32 * b < W.end) pass(key + 32 * b + EARLY, k_now + 32 * b * (2 * D), v_now + 32 * b * (2 * D));
            }
        }
        if (t + 1 < tiles) fetch.finish(k_next, v_next);
        __syncthreads();                              // the next tiles have arrived, these have been read
    };
    for (int t = 0; t < tiles; t += 2) {
        tile(t, 0);
        if (t + 1 < tiles) tile(t + 1, 1);
    }
    // The waves' sums (four floats permuted, so that the rows of a write meet all banks), and the answer, 16 bytes of a row a lane.
    auto at = [&](int w, int line, int four) { return reinterpret_cast<float4*>(&s.acc[w][line][0]) + (four ^ (line & (D / 4 - 1))); };
    const float l = lsum + other_half(lsum);
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *at(wave, n32, 8 * i + 2 * r + h2) = make_float4(acc[i][4 * r], acc[i][4 * r + 1], acc[i][4 * r + 2], acc[i][4 * r + 3]);
    if (h2 == 0) {
        s.sum.m[wave][n32] = m - kShift;              // (probabilities are 2^(logit - that) now)
        s.sum.l[wave][n32] = l;
    }
    __syncthreads();
    constexpr int PER = D / 4;                        // threads of a row
    for (int line = tid / PER; line < 32 * RB; line += kWaves * 64 / PER) {
        const int row = W.row0 + line;
        if (row >= W.rows) break;
        const int w = line / 32, n = line % 32, four = tid % PER;
        float4 o = *at(w, n, four);
        float M = s.sum.m[w][n], L = s.sum.l[w][n];
        if constexpr (KS == 2) {
            const float M1 = s.sum.m[w + RB][n], top = fmaxf(M, M1), f0 = __builtin_amdgcn_exp2f(M - top), f1 = __builtin_amdgcn_exp2f(M1 - top);
            const float4 o1 = *at(w + RB, n, four);
            o = make_float4(o.x * f0 + o1.x * f1, o.y * f0 + o1.y * f1, o.z * f0 + o1.z * f1, o.w * f0 + o1.w * f1);
            L = L * f0 + s.sum.l[w + RB][n] * f1;
            M = top;
        }
        const int64_t to = head_of(row) * A.slots + W.slot;
        *reinterpret_cast<float4*>(A.part_acc + to * D + four * 4) = o;
        if (four == 0) A.part_ml[to] = make_float2(M, L);
    }
}

// The share of a sequence's own rows that workgroup i of those for them takes; false: none.
template <int CACHE, bool SHARED> __device__ __forceinline__ bool own_task(const SharedArgs& A, unsigned i, Task& W) {
    // A share's heads run on one XCD (workgroup i runs on XCD i % 8), which then reads whole lines of all heads; a sequence has
    // an odd number of places, so that the first shares, which are all that short sequences have, do not meet on a few XCDs.
    const int shift = CACHE ? A.head_shift : 0, sets = A.Hkv >> shift;
    W.shift = shift;
    W.kvh = (i % sets) << shift;
    int chunk = i / sets;
    if (A.by_xcd) {
        W.kvh = (i / 8 % sets) << shift;
        chunk = i / (8 * sets) * 8 + i % 8;
    }
    W.b0 = chunk / A.places;
    chunk %= A.places;
    if (chunk >= A.nchunk || W.b0 >= A.B) return false;
    const int S = clamped(A.lens[W.b0], A.max_len);
    const int share = share_of(S, A.nchunk, A.least);
    W.begin = chunk * share;
    if (W.begin >= S && (SHARED || chunk > 0)) return false;
    W.end = W.begin + share < S ? W.begin + share : S;
    W.row0 = 0;
    W.rows = A.g;
    W.table = A.table + (int64_t)W.b0 * A.table_stride;
    W.slot = !SHARED && S <= share ? -1 : A.prefix_chunks + chunk;
    return true;
}

// The share of a prefix and the tile of its query heads that workgroup i of those for prefixes takes.  Group i's tiles have the places
// from first(i) = i + floor(cu[i] g / R) on, R query heads a tile: rows / R rounded up is at most one more than the difference
// of the floors, so nobody counts through the groups before.
template <int R> __device__ __forceinline__ bool prefix_task(const SharedArgs& A, unsigned i, int lane, Task& W) {
    // the tiles of a share run together, and on one XCD where there are shares for all
    const unsigned units = (unsigned)A.Hkv * A.tiles;
    int chunk = i / units;
    unsigned j = i % units;
    if (A.prefix_by_xcd) {
        chunk = i / (8 * units) * 8 + i % 8;
        j = i / 8 % units;
    }
    // (from one head and share to the next the tiles are turned: places without a tile would else meet on a few of the chip's parts, which
    // get workgroups in turn whether they return at once or not)
    const unsigned unit = (A.prefix_by_xcd ? i / 8 : i) / A.tiles;
    const int tile = (j + unit + unit / 4) % A.tiles;
    W.kvh = j / A.tiles;
    W.shift = 0;
    if (chunk >= A.prefix_chunks) return false;
    auto at = [&](int i) { return A.cu ? clamped(A.cu[i], A.B) : (i == 0 ? 0 : A.B); };
    auto first = [&](int i) { return i + (int)((int64_t)at(i) * A.g / R); };
    int lo = 0;                                        // the last group whose places begin at or before the tile's
    for (int width = A.G; width > 1;) {                // (it is among lo .. lo + width - 1)
        const int w = (width + 63) / 64;
        const int k = __popcll(__ballot(lane * w < width && first(lo + lane * w) <= tile));
        const int n = k > 0 ? k - 1 : 0;
        lo += n * w;
        width = min(w, width - n * w);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    W.b0 = at(lo);
    W.rows = (at(lo + 1) - W.b0) * A.g;
    W.row0 = (tile - first(lo)) * R;
    if (W.row0 < 0 || W.row0 >= W.rows) return false;
    const int P = clamped(A.prefix_lens[lo], A.max_prefix);
    const int share = share_of(P, A.prefix_chunks, A.prefix_least);
    W.begin = chunk * share;
    if (W.begin >= P) return false;
    W.end = W.begin + share < P ? W.begin + share : P;
    W.table = A.prefix_table + (int64_t)lo * A.prefix_stride;
    W.slot = chunk;
    return true;
}

template <typename T, int CACHE, int D, bool PAST>
__global__ __launch_bounds__(kWaves * 64, D == 64 ? 4 : 3) void cached_attn(const SharedArgs A) {
    __shared__ __align__(256) Shared<D> s;
    Task W;
    if (own_task<CACHE, false>(A, blockIdx.x, W)) attend<T, CACHE, D, 1, PAST>(A, W, s);
}

// R: query heads of a tile.
template <typename T, int CACHE, int D, int R>
__global__ __launch_bounds__(kWaves * 64, R == 16 ? (D == 64 ? 4 : 3) : 2) void shared_attn(const SharedArgs A) {
    constexpr bool kWide = R > 32;
    __shared__ __align__(256) union {
        Shared<D> own;
        typename std::conditional<kWide, Wide<D>, Shared<D>>::type prefix;
    } s;
    Task W;
    if (blockIdx.x >= A.prefix_groups) {
        if (own_task<CACHE, true>(A, blockIdx.x - A.prefix_groups, W)) attend<T, CACHE, D, 1, CACHE == 0>(A, W, s.own);
    } else if (prefix_task<R>(A, blockIdx.x, threadIdx.x & 63, W)) {
        if constexpr (kWide) attend_wide<T, CACHE, D, R / 32>(A, W, s.prefix);
        else attend<T, CACHE, D, R / 16>(A, W, s.prefix);
    }
}

// Joins the partials of a query head: a workgroup for each, its threads four elements of every 8th (heads of 64: 16th) partial, or, with 1024 threads,
// of every 32nd (64th), eight in flight at a time, the first ones before the largest maximum is known.
template <typename T, int CACHE, int D, bool SHARED, int THREADS>
__global__ __launch_bounds__(THREADS) void cached_join(const SharedArgs A) {
    typedef typename kind<T, CACHE>::elem elem;
    constexpr int LANES = D / 4, PARTS = THREADS / LANES, WAVES = THREADS / 64, BATCH = 8;
    const int64_t hq = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = (int)(hq / A.Hq), part = tid / LANES;
    const int S = clamped(A.lens[b], A.max_len);
    const int share = share_of(S, A.nchunk, A.least);
    int n = (S + share - 1) / share, before = 0;
    if (SHARED) {
        int G = 0;                                     // b's group
        bool in = true;
        if (A.cu) {
            G = sequence_of(A.cu, A.G, b, lane);
            in = G < A.G && A.cu[G] <= b;              // (before the first and behind the last: none)
        }
        if (in) {
            const int P = clamped(A.prefix_lens[G], A.max_prefix);
            const int ps = share_of(P, A.prefix_chunks, A.prefix_least);
            before = (P + ps - 1) / ps;
        }
        n += before;
    } else if (n <= 1) {
        return;
    }
    const float2* ml = A.part_ml + hq * A.slots;
    const float* pa = A.part_acc + hq * A.slots * D + tid % LANES * 4;
    float2 p[BATCH];
    float4 x[BATCH];
    auto fetch = [&](int first) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int at = first + i * PARTS + part, s = at < before ? at : A.prefix_chunks + (at - before);
            p[i] = make_float2(-3.4028235e38f, 0.f);
            x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at < n) {
                p[i] = ml[s];
                x[i] = *reinterpret_cast<const float4*>(pa + (int64_t)s * D);
            }
        }
    };
    fetch(0);
    float M = -3.4028235e38f;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) M = fmaxf(M, p[i].x);
    for (int i = PARTS * BATCH + tid; i < n; i += THREADS) M = fmaxf(M, ml[i < before ? i : A.prefix_chunks + (i - before)].x);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    __shared__ float s_m[WAVES], s_l[PARTS], s_o[PARTS][D];
    if (lane == 0) s_m[wave] = M;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) M = fmaxf(M, s_m[w]);
    float Lq = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int first = 0;;) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float f = __builtin_amdgcn_exp2f(p[i].x - M);
            Lq += p[i].y * f;
            o = make_float4(o.x + x[i].x * f, o.y + x[i].y * f, o.z + x[i].z * f, o.w + x[i].w * f);
        }
        first += PARTS * BATCH;
        if (first >= n) break;
        fetch(first);
    }
    *reinterpret_cast<float4*>(&s_o[part][tid % LANES * 4]) = o;
    if (tid % LANES == 0) s_l[part] = Lq;
    __syncthreads();
    if (tid >= D) return;
    float y = 0.f;
    Lq = 0.f;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        y += s_o[i][tid];
        Lq += s_l[i];
    }
    y = Lq == 0.f ? 0.f : y / Lq;
    // (probabilities that were rounded up can carry a mean of numbers near the type's largest past it; infinities stay, and over codes means beyond
    // fp16's range)
    constexpr bool kHalf = std::is_same<T, dec_f16>::value;
    constexpr float kLargest = kHalf ? 65504.f : 3.3895314e38f;
    if (!(kHalf && CACHE != 0) && __builtin_fabsf(y) < INFINITY) y = __builtin_amdgcn_fmed3f(y, -kLargest, kLargest);
    reinterpret_cast<elem*>(A.out)[hq * D + tid] = (elem)y;
    if (A.lse && tid == 0) A.lse[hq] = Lq == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(Lq)) * 0.6931471805599453f;
}

}  // namespace

// Sequences that can be long or many (keys of all KV heads, from here on) have shares of 512 keys, where as many shares may be (below), and, over codes,
// workgroups that take four KV heads together, a wave each (or two): one fetch of scales for all, and whole lines of 4-bit codes.  Microseconds with one / two / four
// heads: 8 x 16000 rows, 32 heads, 4 bits 152 / 129 / 126, 8 bits 215 / 197 / 193; 131072 rows, 8 heads, 4 bits 43 / 39 / 40, 8 bits 70 / 65 / 61; 32
// sequences of 1 to 16384 rows, 8 heads, 8 bits 73 / 71 / 70.  Fewer keys: 8 x 4000 rows of 4 bits, 8 heads 16.8 / 17.8 / 20.9, 2 x 30000 22.4 / 22.0 / 24.5.
constexpr int64_t kManyKeys = 1 << 20;

// Shares of a sequence's own rows: as many as give 1024 workgroups if all sequences are as long as they may be, of 128 to 1024 keys,
// but no more than 16384 of all sequences and KV heads, or seven a sequence: where that is fewer, shares are longer (128 sequences of up to 131072 rows, 8 KV
// heads: 16 of 8192, though over codes a workgroup takes four heads' shares); a sequence of up to 512 rows is not cut.  Shares of a prefix, of
// 128 keys at least and no more than 256, go by the longest prefix there may be and the groups' average size: below.
SharedPlan shared_plan(int B, int G, int Hq, int Hkv, int D, int64_t max_prefix, int64_t max_len) {
    SharedPlan P{};
    const int g = Hq / Hkv;
    const int64_t pairs = (int64_t)B * Hkv, keys = pairs * max_len;
    int64_t chunk = std::max<int64_t>(128, (keys / 1024 + 127) / 128 * 128);
    chunk = std::min<int64_t>(chunk, keys >= kManyKeys ? 512 : 1024);
    if (max_len <= 512) chunk = 512;
    P.nchunk = (int)std::min((max_len + chunk - 1) / chunk, std::max<int64_t>(7, 16384 / pairs));
    P.least = P.nchunk == 1 || pairs > 128 ? 512 : (pairs > 64 ? 256 : 128);
    if (G > 0) {
        const int64_t rows = ((int64_t)B * g + G - 1) / G;    // of a group, on the average
        P.columns = rows <= 16 ? 16 : (rows <= 32 ? 32 : (rows <= 64 ? 64 : 128));
        P.tiles = (int)(G - 1 + ((int64_t)B * g + P.columns - 1) / P.columns);
        const int64_t units = (rows + P.columns - 1) / P.columns * G * Hkv;   // (as many tiles as groups of the average size have)
        // Shares, for so many workgroups with all tiles and KV heads, are dealt to the 8 XCDs in turn: as many for each, since of 12 four
        // would get two and four one.  Tiles of 64 or 128 have two workgroups a compute unit and no more, and fewer where the sequences' own
        // rows are many (own keys over the prefixes', a prefix's once a tile, all as long as they may be).
        // Microseconds by shares, 8 KV heads.  Tiles of 128: 128 users of 20011 rows 8 / 12 / 16: 94 / 93 / 79; 160 of 16001 8 / 10 / 13 / 16: 97 / 130 / 112 / 104; 256 of
        // 16001 4 / 6 / 8 / 12 / 16: 171 / 152 / 123 / 154 / 138; 64 of 32749 16 / 24 / 32 with one own row or two: 79 / 71 / 66, with half as many own keys as
        // prefix keys: 82 / 74 / 78, as many: 86 / 83 / 91, twice: 96 / 107 / 119.  Of 32: 8 users of 32749 32 / 64 / 128: 32.0 / 34.5 / 43.4.  Of 16: 4 of 131071, 8 bits, 32 / 64 / 128: 66 / 69 / 71;
        // 5 groups of 4, 16001 rows, 8 / 16 / 25: 86 / 76 / 81.  Heads of 64, 20 of them, 3 groups, 8 / 16 / 18: 30.0 / 28.5 / 29.3.  Of 66 sizes of all kinds, many of
        // which shaped the rule, it is within 6 % of the best count tried at 54, within 8 % at 60; the worst is 20 % (6 groups of 16 users, 12007 rows: 8 shares 96, 6 of
        // them 80), for a reason that was not found.
        const int64_t met = units * max_prefix;
        const int64_t most = P.columns == 16 ? 512 * (128 / D) : (P.columns == 32 ? 256 * (128 / D) : (20 * keys < 9 * met ? 512 : (2 * keys < 3 * met ? 384 : 256)));
        int64_t shares = (most + units - 1) / units;
        if (units < 128) {
            shares = std::max<int64_t>(8, (most / units + 4) / 8 * 8);
            while (P.columns > 32 && shares > 8 && shares * units > 512) shares -= 8;
        }
        P.prefix_chunks = (int)std::max<int64_t>(1, std::min<int64_t>({256, (max_prefix + 127) / 128, shares}));
        P.prefix_least = 128;
    }
    P.slots = P.prefix_chunks + P.nchunk;
    const size_t heads = (size_t)B * Hq;
    P.acc_bytes = (heads * P.slots * D * sizeof(float) + 255) & ~(size_t)255;
    P.bytes = P.slots <= 1 ? 0 : P.acc_bytes + heads * P.slots * sizeof(float2);
    return P;
}

hipError_t launch_shared(int dtype, int cache, int D, SharedArgs A, void* workspace, hipStream_t st) {
    const SharedPlan P = shared_plan(A.B, A.G, A.Hq, A.Hkv, D, A.max_prefix, A.max_len);
    A.nchunk = P.nchunk;
    A.least = P.least;
    A.prefix_chunks = P.prefix_chunks;
    A.prefix_least = P.prefix_least;
    A.tiles = P.tiles;
    A.slots = P.slots;
    // r / page for 0 <= r < 2^31: with 2^(l-1) < page <= 2^l, ceil(2^(31+l) / page) fits 32 bits and its product's error stays
    // below one part in r; 2 r times that is shifted by 32 and l
    int l = 0;
    while (l < 31 && (1ll << l) < A.page) ++l;
    A.page_magic = (unsigned)(((1ull << (31 + l)) + A.page - 1) / A.page);
    A.page_shift = l;
    A.last_page = (int)(A.pages - 1);
    A.scale2 = (float)(1.4426950408889634 / std::sqrt((double)D));
    A.part_acc = static_cast<float*>(workspace);
    A.part_ml = reinterpret_cast<float2*>(static_cast<char*>(workspace) + P.acc_bytes);
    const bool many = (int64_t)A.B * A.Hkv * A.max_len >= kManyKeys;
    A.head_shift = cache != 0 && many ? (A.Hkv % 4 == 0 ? 2 : (A.Hkv % 2 == 0 ? 1 : 0)) : 0;
    A.by_xcd = (int64_t)P.nchunk * A.B >= 8;
    A.places = A.by_xcd ? P.nchunk | 1 : P.nchunk;
    int64_t units = (int64_t)A.places * A.B;
    if (A.by_xcd) units = (units + 7) / 8 * 8;
    A.prefix_by_xcd = P.prefix_chunks >= 8;
    A.prefix_groups = (unsigned)((A.prefix_by_xcd ? (P.prefix_chunks + 7) / 8 * 8 : P.prefix_chunks) * (int64_t)P.tiles * A.Hkv);
    const dim3 grid((unsigned)(A.prefix_groups + units * (A.Hkv >> A.head_shift))), block(kWaves * 64), heads((unsigned)((int64_t)A.B * A.Hq));
    // (256 partials of 32 heads: a step over 131072 rows of 4 bits 38.7 us with 256 threads a head, 37.6 with 1024; 65 of 512 heads, 131071 rows of 8
    // bits, 73.3 / 75.7)
    auto join = [&](auto few, auto many) {
        if (P.slots > 64 && heads.x <= 128) hipLaunchKernelGGL(many, heads, dim3(1024), 0, st, A);
        else hipLaunchKernelGGL(few, heads, block, 0, st, A);
    };
    auto form = [&](auto t, auto c, auto d) {
        typedef decltype(t) T;
        constexpr int C = decltype(c)::value, DD = decltype(d)::value;
        if (A.G == 0) {
            if constexpr (C != 0) {
                if (C == 1 && DD == 128 && many) hipLaunchKernelGGL((cached_attn<T, C, DD, C == 1 && DD == 128>), grid, block, 0, st, A);
                else hipLaunchKernelGGL((cached_attn<T, C, DD, false>), grid, block, 0, st, A);
                if (P.slots > 1) join(cached_join<T, C, DD, false, 256>, cached_join<T, C, DD, false, 1024>);
            }
            return;
        }
        if (P.columns == 16) hipLaunchKernelGGL((shared_attn<T, C, DD, 16>), grid, block, 0, st, A);
        else if (P.columns == 32) hipLaunchKernelGGL((shared_attn<T, C, DD, 32>), grid, block, 0, st, A);
        else if (P.columns == 64) hipLaunchKernelGGL((shared_attn<T, C, DD, 64>), grid, block, 0, st, A);
        else hipLaunchKernelGGL((shared_attn<T, C, DD, 128>), grid, block, 0, st, A);
        join(cached_join<T, C, DD, true, 256>, cached_join<T, C, DD, true, 1024>);
    };
    auto of = [&](auto t, auto c) {
        if (D == 128) form(t, c, std::integral_constant<int, 128>{});
        else form(t, c, std::integral_constant<int, 64>{});
    };
    auto with = [&](auto t) {
        if (cache == 0) of(t, std::integral_constant<int, 0>{});
        else if (cache == 1) of(t, std::integral_constant<int, 1>{});
        else of(t, std::integral_constant<int, 2>{});
    };
    if (dtype == 0) with(dec_bf16{});
    else if (dtype == 2) with(dec_f16{});
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace snapkv
