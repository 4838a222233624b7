// Rows of a matrix held in registers: layouts, loads, stores and reductions, for the layer norm and the policy loss.
//
// MrfRow: a row of C columns is spread over TL lanes, each of which holds CH chunks of V neighbouring columns: chunk i of lane l are
// the columns (l + TL i) V ...  A wavefront so holds 64 / TL rows, or a workgroup one (TL = 256, 1024).  The loads and stores of a chunk
// take one instruction at any address (the hardware asks for no alignment of vectors): a row's last chunk, where it is not full,
// reads on into the next row, except at the end of the matrix, and what is not the row's is masked; it is written in two or three
// smaller pieces.  TL is the smallest that keeps a lane's part at about a dozen values: the steps across lanes, which every row
// pays, stay few, and there are still enough rows in flight.
//
// MrfTile: short rows, above all those whose ends do not fall on a chunk's (C % 4).  The 64 / TL rows of a wavefront are neighbours in memory, one piece of
// 16-byte chunks: it goes through LDS as such, and a lane takes its columns l, l + TL, ... of its row from there.  No piece of a chunk
// is read or written alone, and for up to 32 columns a lane has a whole row: no step across lanes at all.
#pragma once

#include "mrfmp_learn.h"

template <class T, int V> struct MrfVec { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };

// Whether none of `rows` rows from the first-th on is among the last V of N: a chunk of V columns that starts inside of one ends inside of
// the matrix.
__device__ inline bool mrf_rows_fast(long long first, int rows, int V, long long N) { return first + rows + V <= N; }

template <int TL_, int V_, int CH_> struct MrfRow {
    static constexpr int TL = TL_, V = V_, CH = CH_, E = V_ * CH_, W = TL_ * V_ * CH_;

    static __device__ inline int column(int l, int i) { return (l + TL * i) * V; }

    // chunks as they lie in memory (a row on its way takes no more registers than it has to)
    template <class T> struct Raw { typename MrfVec<T, V>::type v[CH]; };

    // FAST: a row whose last chunk may read on (mrf_rows_fast).  The row starts `row` elements behind `at`, which all threads have in common.
    // Else nothing behind the row, and nothing at all where it is not `there`.
    template <bool FAST, class T> static __device__ inline void load(const T *at, unsigned row, bool there, int C, int l, Raw<T> &r)
    {
        typedef typename MrfVec<T, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            vec x;
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = (T)0.0f;
            if constexpr (FAST) {
                if (c < C) x = *(const vec *)(at + (row + (unsigned)c));
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (there && c + j < C) x[j] = at[row + (unsigned)(c + j)];
            }
            r.v[i] = x;
        }
    }

    // (columns from C on: `fill`)
    template <class T> static __device__ inline void convert(const Raw<T> &r, int C, int l, float (&v)[E], float fill)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = column(l, i) + j < C ? mrf_to_f32((T)r.v[i][j]) : fill;
    }

    // N values from the FROM-th on (indices known at compile time: the values stay in registers)
    template <class T, int N, int FROM> static __device__ inline void store_piece(T *at, const float (&v)[E])
    {
        typename MrfVec<T, N>::type x;
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = mrf_from_f32<T>(v[FROM + j]);
        *(typename MrfVec<T, N>::type *)at = x;
    }

    // the C % 4 columns that are left of a chunk, or of its second half
    template <class T, int FROM> static __device__ inline void store_rest(T *at, int C, const float (&v)[E])
    {
        if (C & 2) {
            store_piece<T, 2, FROM>(at, v);
            if (C & 1) store_piece<T, 1, FROM + 2>(at + 2, v);
        } else if (C & 1) {
            store_piece<T, 1, FROM>(at, v);
        }
    }

    template <class T, int I = 0> static __device__ inline void store(T *row, int C, int l, const float (&v)[E])
    {
        if constexpr (I < CH) {
            const int c = column(l, I);
            if (c + V <= C) {
                store_piece<T, V, I * V>(row + c, v);
            } else if (c < C) {
                if constexpr (V == 8) {
                    if (C & 4) {
                        store_piece<T, 4, I * V>(row + c, v);
                        store_rest<T, I * V + 4>(row + c + 4, C, v);
                    } else {
                        store_rest<T, I * V>(row + c, C, v);
                    }
                } else {
                    store_rest<T, I * V>(row + c, C, v);
                }
            }
            store<T, I + 1>(row, C, l, v);
        }
    }

    // parameters of the columns: fill where there are none
    static __device__ inline void load_columns(const float *at, int C, int l, float (&v)[E], float fill)
    {
        typedef typename MrfVec<float, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            vec x;
#pragma unroll
            for (int j = 0; j < V; ++j) x[j] = fill;
            if (at) {
                if (c + V <= C) {
                    x = *(const vec *)(at + c);
                } else if (c < C) {
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (c + j < C) x[j] = at[c + j];
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) v[i * V + j] = x[j];
        }
    }

    // v times the parameters of its columns, a chunk at a time
    static __device__ inline void scale_columns(const float *at, int C, int l, float (&v)[E])
    {
        typedef typename MrfVec<float, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            if (c + V <= C) {
                const vec x = *(const vec *)(at + c);
#pragma unroll
                for (int j = 0; j < V; ++j) v[i * V + j] *= x[j];
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < C) v[i * V + j] *= at[c + j];
            }
        }
    }

    // sum (minimum) over the row's lanes, in all of them.  Rows of more than a wavefront meet in `scratch` (one float per wavefront
    // of the workgroup), with a barrier: every thread calls it, and two calls in a row take different scratch.
    template <bool SUM> static __device__ inline float reduce(float v, float *scratch)
    {
        if constexpr (TL <= 64) {
            return SUM ? mrf_lanes_sum<TL>(v) : mrf_lanes_min<TL>(v);
        } else {
            v = SUM ? mrf_lanes_sum<64>(v) : mrf_lanes_min<64>(v);
            const int wv = threadIdx.x >> 6, first = wv & ~(TL / 64 - 1);
            if ((threadIdx.x & 63) == 0) scratch[wv] = v;
            __syncthreads();
            v = scratch[first];
#pragma unroll
            for (int w = 1; w < TL / 64; ++w) v = SUM ? v + scratch[first + w] : fminf(v, scratch[first + w]);
            return v;
        }
    }
    static __device__ inline float sum(float v, float *scratch) { return reduce<true>(v, scratch); }
    static __device__ inline float min(float v, float *scratch) { return reduce<false>(v, scratch); }

    // two sums at once, with one barrier
    static __device__ inline void sums(float &a, float &b, float2 *scratch)
    {
        if constexpr (TL <= 64) {
            a = mrf_lanes_sum<TL>(a);
            b = mrf_lanes_sum<TL>(b);
        } else {
            a = mrf_lanes_sum<64>(a);
            b = mrf_lanes_sum<64>(b);
            const int wv = threadIdx.x >> 6, first = wv & ~(TL / 64 - 1);
            if ((threadIdx.x & 63) == 0) scratch[wv] = make_float2(a, b);
            __syncthreads();
            a = scratch[first].x;
            b = scratch[first].y;
#pragma unroll
            for (int w = 1; w < TL / 64; ++w) {
                a += scratch[first + w].x;
                b += scratch[first + w].y;
            }
        }
    }
};


// 16 bytes at an address that is a multiple of A
template <int A> struct MrfChunk;
template <> struct MrfChunk<2> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct MrfChunk<4> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct MrfChunk<16> { typedef unsigned type __attribute__((ext_vector_type(4))); };

template <int TL_, int E_> struct MrfTile {
    static constexpr int TL = TL_, E = E_, W = TL_ * E_, ROWS = 64 / TL_;
    static constexpr int BYTES = 64 * E_ * 4;      // of LDS for a wavefront, whatever the type

    static __device__ inline int column(int l, int e) { return l + TL * e; }

    // `rows` (up to ROWS) rows from `at` on into this wavefront's LDS, zeros for the others
    template <class T> static __device__ inline void fetch(const T *at, int rows, int C, T *lds)
    {
        typedef typename MrfChunk<sizeof(T)>::type chunk;
        typedef typename MrfChunk<16>::type quad;
        constexpr int PER = 16 / (int)sizeof(T), NI = (E + PER - 1) / PER;
        const int lane = threadIdx.x & 63, n = ROWS * C;
        if (rows == ROWS) {
            const int chunks = n / PER;      // (64 / TL rows of any length are whole chunks)
            quad r[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (lane + 64 * i < chunks) r[i] = *(const chunk *)(at + (unsigned)(lane + 64 * i) * PER);
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (lane + 64 * i < chunks) ((quad *)lds)[lane + 64 * i] = r[i];
        } else {
            for (int k = lane; k < n; k += 64) lds[k] = k < rows * C ? at[k] : (T)0.0f;
        }
    }

    // the lane's columns of row `g` of the tile; columns from C on: `fill`
    template <class T> static __device__ inline void take(const T *lds, int g, int C, int l, float (&v)[E], float fill)
    {
        const T *row = lds + g * C + l;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = mrf_to_f32(row[TL * e]);
            v[e] = column(l, e) < C ? x : fill;
        }
    }

    template <class T> static __device__ inline void put(T *lds, int g, int C, int l, const float (&v)[E])
    {
        T *row = lds + g * C + l;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (column(l, e) < C) row[TL * e] = mrf_from_f32<T>(v[e]);
    }

    template <class T> static __device__ inline void flush(T *at, int rows, int C, const T *lds)
    {
        typedef typename MrfChunk<sizeof(T)>::type chunk;
        typedef typename MrfChunk<16>::type quad;
        constexpr int PER = 16 / (int)sizeof(T), NI = (E + PER - 1) / PER;
        const int lane = threadIdx.x & 63, n = ROWS * C;
        if (rows == ROWS) {
            const int chunks = n / PER;
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (lane + 64 * i < chunks) *(chunk *)(at + (unsigned)(lane + 64 * i) * PER) = ((const quad *)lds)[lane + 64 * i];
        } else {
            for (int k = lane; k < rows * C; k += 64) at[k] = lds[k];
        }
    }

    static __device__ inline void load_columns(const float *at, int C, int l, float (&v)[E], float fill)
    {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = at && column(l, e) < C ? at[column(l, e)] : fill;
    }

    static __device__ inline float sum(float v) { return mrf_lanes_sum<TL>(v); }
    static __device__ inline float min(float v) { return mrf_lanes_min<TL>(v); }
};

// F(TL, E), shortest rows first
#define MRF_TILES(F) \
    F(1, 8) F(1, 12) F(1, 16) F(1, 20) F(1, 24) F(1, 28) F(1, 32) F(2, 20) F(2, 24) F(2, 28) F(2, 32) F(4, 20) F(4, 24) F(4, 28) F(4, 32) \
    F(8, 20) F(8, 24) F(8, 28) F(8, 32)
constexpr int MRF_TILES_LONGEST = 256;
