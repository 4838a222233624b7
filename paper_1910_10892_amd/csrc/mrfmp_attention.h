// Shared by the attention's kernels, forward and backward: the problem on the device, products of 32 x 32 x 16 on the matrix unit for the three
// element types, and tiles of rows in LDS.
//
// Products: an operand of 32 rows (columns) and 16 entries along the sum is 8 entries a lane: lane l has row l % 32 and, of the sum, entries that it
// shares with no lane of the other half.  Which of the 16 these are does not matter as long as both operands agree.  The result's lane l
// has column l % 32 and the rows 8 (e / 4) + 4 (l / 32) + e % 4 for e = 0 .. 15 -- so entries 8 t .. 8 t + 7 are, as they are, an operand of the next product
// whose sum runs over those rows: rows 16 t + 4 half + {0, 1, 2, 3, 8, 9, 10, 11}.  Scores (keys x queries) so become an operand
// of probabilities x values in registers, and the other operand is read in the same order of keys.  In 16 bits a product is one instruction, in 32
// bits eight of 32 x 32 x 2.
#pragma once

#include "mrfmp_learn.h"

typedef float mrf_acc __attribute__((ext_vector_type(16)));
template <class T> struct MrfFrag { typedef T type __attribute__((ext_vector_type(8))); };

__device__ inline mrf_acc mrf_mma(const MrfFrag<mrf_bf16>::type &a, const MrfFrag<mrf_bf16>::type &b, const mrf_acc &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline mrf_acc mrf_mma(const MrfFrag<mrf_f16>::type &a, const MrfFrag<mrf_f16>::type &b, const mrf_acc &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ inline mrf_acc mrf_mma(const MrfFrag<float>::type &a, const MrfFrag<float>::type &b, mrf_acc c)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// Sums over many tiles.  In 32 bits a tile's product is a sum of its own, and these are added in 64 bits (a conversion and an addition an entry and tile, and twice the registers: 4
// sequences of 2,048, 16 heads of 64, forward 549 -> 607 us, both passes 2,640 -> 2,930; placed one by one between the matrix instructions of the next block, 612 and 2,980).  Terms
// of one sign and size are rounded the same way each time: 32,768 of them, each added to all before it, were off by 2e-4 of their sum.  In 16 bits a matrix instruction adds 16
// terms at once to what it has summed, and the terms' own roundings (2^-9 or 2^-12 of each) are more than that leaves.
typedef double mrf_long_acc __attribute__((ext_vector_type(16)));
template <class T> struct MrfSum { typedef mrf_acc type; };
template <> struct MrfSum<float> { typedef mrf_long_acc type; };

__device__ inline int mrf_acc_row(int e, int half) { return 8 * (e / 4) + 4 * half + e % 4; }

template <class T> __device__ inline typename MrfFrag<T>::type mrf_acc_frag(const mrf_acc &c, int t)
{
    typename MrfFrag<T>::type f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = mrf_from_f32<T>(c[8 * t + j]);
    return f;
}

// Entries moved down by `bytes` (the same in all lanes), where `mine`, with 0 behind them
template <int WORDS, class Words> __device__ inline void mrf_move_down(Words &w, int bytes, bool mine)
{
#pragma unroll
    for (int by = WORDS / 2; by >= 1; by /= 2) {
        const bool go = mine && (bytes / 4 & by);
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = go ? (j + by < WORDS ? w[j + by < WORDS ? j + by : 0] : 0u) : w[j];
    }
    const bool go = mine && (bytes & 2);
#pragma unroll
    for (int j = 0; j < WORDS; ++j) w[j] = go ? __builtin_amdgcn_alignbit(j + 1 < WORDS ? w[j + 1 < WORDS ? j + 1 : 0] : 0u, w[j], 16) : w[j];
}

// PER entries from d on of a row of D that starts at `row`, 0 behind its end and where it is not `there`.  Nothing is left out by a branch: what is not
// there is read from the row's start (its end) instead, so `row` has to be a row at any rate.
template <int PER, class T> __device__ inline void mrf_load_part(const T *row, int d, int D, bool there, T (&v)[PER])
{
    typedef T vec __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
    constexpr int WORDS = PER * (int)sizeof(T) / 4;
    if (D >= PER) {      // a row's last chunk, where it is no whole one: its last PER entries, moved down
        const vec x = *(const vec *)(row + min(d, D - PER));
        unsigned w[WORDS];
        __builtin_memcpy(w, &x, sizeof(w));
        if (D % PER) mrf_move_down<WORDS>(w, (PER - D % PER) * (int)sizeof(T), d + PER > D);
        there = there && d < D;
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = there ? w[j] : 0u;
        __builtin_memcpy(v, w, sizeof(w));
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const T x = row[d + j < D ? d + j : D - 1];
            v[j] = there && d + j < D ? x : (T)0.0f;
        }
        __builtin_amdgcn_sched_barrier(0);      // (the loads of one part at a time: all at once would take the registers that the sums need)
    }
}

template <class T> __device__ inline typename MrfFrag<T>::type mrf_load8(const T *row, int d, int D, bool there)
{
    T v[8];
    mrf_load_part<8>(row, d, D, there, v);
    typename MrfFrag<T>::type f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = v[j];
    return f;
}

// keeps a branch that all lanes take together: its instructions would otherwise be carried out, and their results left, by every tile that needs none of them
__device__ inline void mrf_stay_branch() { asm volatile(""); }

// N steps use(n, operands(n)): the operands of GROUP steps are on their way from LDS while the GROUP before is multiplied.  (In the compiler's own order a product waits
// for its operand's whole way, three times what it takes itself.)
template <int N, int GROUP, class Get, class Use> __device__ inline void mrf_ahead(const Get &get, const Use &use)
{
    static_assert(N % GROUP == 0, "whole groups");
    if constexpr (GROUP == 1) {      // (32 bits: a step takes longer than its operand's way)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            use(n, get(n));
            __builtin_amdgcn_sched_barrier(0);
        }
        return;
    }
    decltype(get(0)) f[2][GROUP];
#pragma unroll
    for (int i = 0; i < GROUP; ++i) f[0][i] = get(i);
#pragma unroll
    for (int g = 0; g < N / GROUP; ++g) {
        if (g + 1 < N / GROUP) {
#pragma unroll
            for (int i = 0; i < GROUP; ++i) f[(g + 1) & 1][i] = get((g + 1) * GROUP + i);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < GROUP; ++i) use(g * GROUP + i, f[g & 1][i]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Which rows of a result, of 32, lie in [from, to): a word for each lane, and for entry e all bits or none of them (an operation; a comparison, with its mask in
// scalar registers, takes three).
__device__ inline unsigned mrf_rows_between(int from, int to, int half)
{
    from = min(max(from, 0), 32);
    to = min(max(to, 0), 32);
    const unsigned below = to == 32 ? ~0u : (1u << to) - 1u, first = from == 32 ? ~0u : (1u << from) - 1u;
    return (below & ~first) >> (4 * half);
}
__device__ inline unsigned mrf_row_bits(unsigned rows, int e) { return (unsigned)__builtin_amdgcn_sbfe((int)rows, 8 * (e / 4) + e % 4, 1); }
__device__ inline float mrf_keep(unsigned bits, float x) { return __builtin_bit_cast(float, bits & __builtin_bit_cast(unsigned, x)); }
__device__ inline float mrf_keep_or_lowest(unsigned bits, float x)      // (-infinity where not)
{
    return __builtin_bit_cast(float, (bits & __builtin_bit_cast(unsigned, x)) | (~bits & 0xff800000u));
}

struct MrfAttnParams {
    int B, Q, K, Hq, Hk, G, D;
    float scale, c;                               // c = scale log2(e)
    const void *q, *k, *v;
    long long qs[3], ks[3], vs[3];
    long long first, last, offset;
    const int *offsets, *q_lengths, *k_lengths;
    const float *table;
    const int *bucket_of;
    long long map_offset, n_offsets;
    int n_buckets, heads_last;
    void *out;
    float *lse;
    float *part;                                  // of keys divided among `splits`: maximum and sum [splits][rows][2], then [splits][rows][D]
    int splits;
    // backward
    const void *dout;
    void *dq, *dk, *dv;
    float *delta;                                 // [B][Hq][Q]
    int shares;                                   // parts of the heads that share keys, one workgroup each:
    float *share;                                 // [shares][dk, dv][B][K][Hk][D], if more than one
    float *lines, *partial, *dtable;              // [B][Hq][strips][line], [Hq][n_buckets][parts]
    int strips, line;                             // strips of 32 keys; entries of a line
    int parts;
    long long pieces;
};

// What holds for a sequence: queries and keys that there are, and i + lo <= j <= i + hi for the keys j of query i
struct MrfAttnBatch {
    int nq, nk, lo, hi;
    long long map;      // place in the map of j - i = 0
    __device__ inline MrfAttnBatch(const MrfAttnParams &P, int b)
    {
        nq = P.Q;
        nk = P.K;
        if (P.q_lengths) nq = min(max(P.q_lengths[b], 0), P.Q);
        if (P.k_lengths) nk = min(max(P.k_lengths[b], 0), P.K);
        const long long o = P.offset + (P.offsets ? P.offsets[b] : 0);
        const long long most = P.K, least = -(long long)P.Q - 1;
        long long l = o + P.first, h = o + P.last;
        lo = (int)(l < least ? least : l > most ? most : l);
        hi = (int)(h < least ? least : h > most ? most : h);
        map = -o - P.map_offset;
    }
    // keys that queries i0 .. i1 may see: [from, to)
    __device__ inline int from(int i0) const { return max(i0 + lo, 0); }
    __device__ inline int to(int i1) const { return min(i1 + hi + 1, nk); }
};

// the bucket of j - i = d; a bucket's value of head h, times log2(e).  From MRF_ATTN_LEAST down a value leaves its pairs out: a row with nothing else would have a
// log-sum-exp of that size, whose 32 bits cannot tell its probabilities apart (nor from NaN, at the type's lowest value).
constexpr float MRF_ATTN_LEAST = -1048576.0f;
__device__ inline int mrf_attn_bucket(const MrfAttnParams &P, const MrfAttnBatch &s, long long d)
{
    long long at = s.map + d;
    at = at < 0 ? 0 : at >= P.n_offsets ? P.n_offsets - 1 : at;
    const int b = P.bucket_of[at];
    return b < 0 ? 0 : b >= P.n_buckets ? P.n_buckets - 1 : b;
}
__device__ inline float mrf_attn_level(const MrfAttnParams &P, int h, int bucket)
{
    const float value = P.table[P.heads_last ? (size_t)bucket * P.Hq + h : (size_t)h * P.n_buckets + bucket];
    return value <= MRF_ATTN_LEAST ? -INFINITY : value * 1.44269504088896340736f;
}
__device__ inline float mrf_attn_bias(const MrfAttnParams &P, const MrfAttnBatch &s, int h, long long d)
{
    return mrf_attn_level(P, h, mrf_attn_bucket(P, s, d));
}

// The bias along a tile: its values at N offsets in a row, and whether these are all of one bucket -- as most are, far from the queries: then there is nothing to look up
// for each pair.  Threads 0 .. N - 1 fetch, then put; all may ask behind the next barrier.  The buckets of a tile are fetched a tile before its values, which would otherwise
// wait for them.
template <int N> struct MrfLine {
    static constexpr int WAVES = (N + 63) / 64;
    float value[2][N];
    int same[2][WAVES];
    struct Next { int bucket; float value; int same; };
    // buckets of the offsets from `first` on
    __device__ inline void ahead(const MrfAttnParams &P, const MrfAttnBatch &s, long long first, Next &n) const
    {
        if ((int)threadIdx.x < N) n.bucket = mrf_attn_bucket(P, s, first + (int)threadIdx.x);
    }
    // values of those, and buckets of the offsets from `following` on
    __device__ inline void fetch(const MrfAttnParams &P, const MrfAttnBatch &s, int h, long long following, Next &n) const
    {
        if ((int)threadIdx.x < N) {
            const int other = __builtin_amdgcn_readfirstlane(n.bucket);
            n.value = mrf_attn_level(P, h, n.bucket);
            n.same = __any(n.bucket != other) ? -1 : other;
        }
        ahead(P, s, following, n);
    }
    __device__ inline void put(int buf, const Next &n)
    {
        if ((int)threadIdx.x < N) {
            value[buf][threadIdx.x] = n.value;
            if ((threadIdx.x & 63) == 0) same[buf][threadIdx.x >> 6] = n.same;
        }
    }
    __device__ inline bool flat(int buf) const
    {
        const int first = same[buf][0];
        bool all = first >= 0;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) all = all && same[buf][w] == first;
        return __builtin_amdgcn_readfirstlane(all ? 1 : 0) != 0;
    }
};

// Rows of a tensor in LDS: ROWS of DP entries.  A thread moves chunks of 16 bytes, which wait in its registers between the load and the store.  In 16 bits chunk c
// of row r lies at place c ^ swap(r): 16 rows' chunks c (an operand along the rows), and four rows' stretches of 32 entries (one across them), then
// fall on all banks.  (With rows 16 bytes longer instead, half of the reads' cycles were conflicts.)  In 32 bits rows are 16 bytes longer: an operand across them
// is read entry by entry, from places that are known when it is compiled.
template <class T, int DP, int ROWS, int NT> struct MrfRows {
    static constexpr int PER = 16 / (int)sizeof(T), LD = sizeof(T) == 2 ? DP : DP + PER, CPR = DP / PER, CHUNKS = ROWS * CPR, N = (CHUNKS + NT - 1) / NT;
    typedef T vec __attribute__((ext_vector_type(PER)));
    typedef T uvec __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
    vec r[N];

    static __device__ inline int swap(int row)
    {
        if constexpr (CPR >= 16) return (row & 3) << 2 | (row >> 2 & 3);
        else if constexpr (CPR == 8) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
        else return row >> 2 & 3;
    }
    static __device__ inline int place(int row, int chunk)
    {
        if constexpr (sizeof(T) == 4) return row * LD + chunk * PER;
        else return row * LD + (chunk ^ swap(row)) * PER;
    }

    int there;      // rows that there are, or -1 where all of the tile is as it was loaded
    int entries;

    // rows from `at` on, `rows` (1 at least) of them; of a row D entries; the others are 0.  (Chunks that are not there are read from elsewhere in the tensor, a row's
    // last one that is no whole one as its last PER entries, and put right only when they are stored: nothing waits for a load before that.  Entries one by one are 2 to 5
    // times slower: 47 sequences of 41 queries and 739 keys, 35 heads of 103, 576 us and 286.)
    __device__ __forceinline__ void load(const T *at, long long stride, int rows, int D)
    {
        static_assert(CHUNKS % NT == 0, "chunks of a tile");
        there = -1;
        entries = D;
        if (D >= PER) {
            if (rows < ROWS || D < DP) there = rows;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = (int)threadIdx.x + n * NT, row = c / (DP / PER), d = c % (DP / PER) * PER;
                const uvec u = *(const uvec *)(at + min(row, rows - 1) * stride + min(d, D - PER));
#pragma unroll
                for (int j = 0; j < PER; ++j) r[n][j] = u[j];
            }
        } else {
            int thread = threadIdx.x;
            asm volatile("" : "+v"(thread));      // (what follows from it is not worked out ahead: it would take the registers of tiles that do not come here)
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = thread + n * NT, row = c / (DP / PER), d = c % (DP / PER) * PER;
                T v[PER];
                mrf_load_part<PER>(at + (row < rows ? row : 0) * stride, d, D, row < rows, v);
#pragma unroll
                for (int j = 0; j < PER; ++j) r[n][j] = v[j];
            }
        }
    }
    __device__ __forceinline__ void store(T *lds)
    {
        if (there >= 0) {
            mrf_stay_branch();
            typedef unsigned words __attribute__((ext_vector_type(4)));
            if (entries % PER) {
                mrf_stay_branch();
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    words w = __builtin_bit_cast(words, r[n]);
                    mrf_move_down<4>(w, (PER - entries % PER) * (int)sizeof(T), ((int)threadIdx.x + n * NT) % (DP / PER) * PER + PER > entries);
                    r[n] = __builtin_bit_cast(vec, w);
                }
            }
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = (int)threadIdx.x + n * NT, row = c / (DP / PER), d = c % (DP / PER) * PER;
                const bool in = row < there && d < entries;
                words w = __builtin_bit_cast(words, r[n]);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = in ? w[j] : 0u;
                r[n] = __builtin_bit_cast(vec, w);
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int c = (int)threadIdx.x + n * NT, row = c / (DP / PER), d = c % (DP / PER) * PER;
            *(vec *)(lds + place(row, d / PER)) = r[n];
        }
    }
};

// Where a lane's parts of the operands lie, in elements: worked out once, moved from one of the two tiles in LDS to the other, and otherwise only the constant part of an
// address changes.
template <class T, int DP, int LD> struct MrfPlaces {
    static constexpr bool SMALL = sizeof(T) == 2;
    static constexpr int A = SMALL ? DP / 16 : 1, C = SMALL ? DP / 32 : 1;
    typedef typename MrfFrag<T>::type frag;
    int a[A], c[C][2];

    template <class Rows> __device__ inline void init()
    {
        const int lane = threadIdx.x & 63, half = lane >> 5;
        if constexpr (SMALL) {
#pragma unroll
            for (int n = 0; n < A; ++n) a[n] = Rows::place(lane & 31, 2 * n + half);
#pragma unroll
            for (int n = 0; n < C; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int at = 32 * n + (lane & 16) + 4 * (lane & 3);
                    c[n][x] = Rows::place(4 * half + (lane >> 2 & 3) + 8 * x, at / 8) + at % 8;
                }
        } else {
            a[0] = Rows::place(lane & 31, 2 * half);
            c[0][0] = 4 * half * LD + (lane & 31);
        }
    }
    __device__ inline void move(int by)
    {
#pragma unroll
        for (int n = 0; n < A; ++n) a[n] += by;
#pragma unroll
        for (int n = 0; n < C; ++n) {
            c[n][0] += by;
            if constexpr (SMALL) c[n][1] += by;
        }
    }
    // operand whose 32 rows are the tile's rows (of `lds`, a multiple of 16 rows on), and whose sum runs over entries 16 n ..
    __device__ inline frag along(const T *lds, int n) const
    {
        if constexpr (SMALL) {
            return *(const frag *)(lds + a[n]);
        } else {
            typedef float vec __attribute__((ext_vector_type(4)));
            const vec x = *(const vec *)(lds + a[0] + 16 * n), y = *(const vec *)(lds + a[0] + 16 * n + 4);
            frag f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = x[j], f[4 + j] = y[j];
            return f;
        }
    }
    // operand whose 32 rows are entries 32 n .., and whose sum runs over rows 4 half + {0 .. 3, 8 .. 11}
    __device__ inline frag across(const T *lds, int n) const
    {
        if constexpr (SMALL) {
            // the transposing read: of 16 lanes, four each point at a row's 16 entries, and each gets the four rows' values of one entry
            typedef short v4 __attribute__((ext_vector_type(4)));
            typedef short v8 __attribute__((ext_vector_type(8)));
            const v4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4 *)(lds + c[n][0]));
            const v4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4 *)(lds + c[n][1]));
            const v8 xy = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(frag, xy);
        } else {
            frag f;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = lds[c[0][0] + 32 * n + (8 * (j / 4) + j % 4) * LD];
            return f;
        }
    }
};

// A sum of many terms: what an addition rounds off (`lost`) is taken off the next term
__device__ inline void mrf_add(float &sum, float &lost, float term)
{
    const float more = term - lost, all = sum + more;
    lost = (all - sum) - more;
    sum = all;
}

// Probabilities are at most 1, and most of many keys far below: for a product in MRF_F16 they are taken times 2^15, where all that matter keep their digits
// (2^-14, the least number with all of them, would be a probability already with 16,384 keys).
template <class T> constexpr float mrf_attn_shift() { return 0.0f; }
template <> constexpr float mrf_attn_shift<mrf_f16>() { return 15.0f; }
template <class T> constexpr float mrf_attn_unshift() { return 1.0f; }
template <> constexpr float mrf_attn_unshift<mrf_f16>() { return 0x1p-15f; }

// sum (maximum) of the two halves of a wavefront, in both
__device__ inline float mrf_halves_sum(float v) { return mrf_xor32_f32(v, true); }
__device__ inline float mrf_halves_max(float v)
{
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const unsigned u0 = s[0], u1 = s[1];
    return fmaxf(__builtin_bit_cast(float, u0), __builtin_bit_cast(float, u1));
}

// What goes into a product in MRF_F16 and has no bound of its own (dS: gradients of any size, over any number of keys) is taken times a power of two,
// a lane's own, as its column of the product is: the largest one that leaves its largest value so far in range.  What was summed follows where it
// falls.  Other types have the range of 32 bits.
template <class T> struct MrfRange {
    float f = 1.0f, top = 0.0f;      // the factor; values up to `top` are in range with it
    template <class Sum, int N> __device__ inline void fit(mrf_acc &x, Sum (&sums)[N])
    {
        if constexpr (sizeof(T) == 2 && mrf_attn_shift<T>() != 0.0f) {
            float big = 0.0f;
#pragma unroll
            for (int e = 0; e < 16; ++e) big = fmaxf(big, fabsf(x[e]));
            big = mrf_halves_max(big);
            if (__any(big > top)) {
                if (big > top) {
                    int ex = __builtin_amdgcn_frexp_expf(big);      // big < 2^ex
                    ex = ex < -100 ? -100 : ex > 120 ? 120 : ex;
                    const float g = ldexpf(1.0f, 15 - ex), r = top > 0.0f ? g / f : 0.0f;
                    f = g;
                    top = ldexpf(1.0f, ex);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int e = 0; e < 16; ++e) sums[n][e] *= r;
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= f;
        }
    }
    __device__ inline float undo() const { return 1.0f / f; }
};

// In 32 bits: what a tile of 32 rows at `rows` adds to the sums, f being its other operand (parts 0 and 1 of 16 rows)
template <int DP, class Places, int N> __device__ inline void mrf_add_block(const Places &places, const float *rows, int ld, const MrfFrag<float>::type (&f)[2], mrf_long_acc (&sums)[N])
{
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
        mrf_acc x;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.0f;
#pragma unroll
        for (int y = 0; y < 2; ++y) x = mrf_mma(places.across(rows + 16 * y * ld, d), f[y], x);
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[d][e] += x[e];
    }
}

// entries d .. d + 3 of a row of D
template <class T> __device__ inline void mrf_store4(T *row, int d, int D, const float (&v)[4])
{
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (d + 4 <= D) {
        vec x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = mrf_from_f32<T>(v[j]);
        *(vec *)(row + d) = x;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) row[d + j] = mrf_from_f32<T>(v[j]);
    }
}

namespace mrf_host {
int attention_check(const mrf_attention *a, MrfAttnParams &P);

// Rows of queries go together where there are few on one head of keys, and the keys are then divided so that there are enough workgroups.
struct AttnPlan { bool pack; int splits; unsigned grid; };

// The kernels in 32 bits (MRF_ATTENTION_F32) and those of the backward pass for heads of more than 64 entries in 16 bits (MRF_ATTENTION_128) are translation units of
// their own: their sums are held in the accumulation registers, there being no room for them in the others.
int attention_forward_f32(const MrfAttnParams &P, const AttnPlan &plan, hipStream_t st);
int attention_backward_f32(const MrfAttnParams &P, hipStream_t st);
int attention_backward_128(const MrfAttnParams &P, int type, hipStream_t st);
}
