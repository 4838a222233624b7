// Rows of a matrix held in registers: layouts, loads, stores and reductions, for the layer norm and the policy loss.
//
// A row of C columns is spread over TL lanes, each of which holds CH chunks of V neighbouring columns: chunk i of lane l are the columns
// (l + TL i) V ...  A wavefront so holds 64 / TL rows, or a workgroup one (TL = 256, 1024).  V = 4 (8 for long rows of 16-bit elements)
// where the rows allow loads of that many elements, 1 otherwise.  TL is the smallest that keeps a lane's part at about a dozen
// values: the steps across lanes, which every row pays, stay few, and there are still enough rows in flight.
#pragma once

#include "mrfmp_learn.h"

template <class T, int V> struct MrfVec { typedef T type __attribute__((ext_vector_type(V))); };
template <class T> struct MrfVec<T, 1> { typedef T type; };

template <int TL_, int V_, int CH_> struct MrfRow {
    static constexpr int TL = TL_, V = V_, CH = CH_, E = V_ * CH_, W = TL_ * V_ * CH_;

    static __device__ inline int column(int l, int i) { return (l + TL * i) * V; }

    // (columns from C on: `fill`)
    template <class T> static __device__ inline void load(const T *row, int C, int l, float (&v)[E], float fill)
    {
        typedef typename MrfVec<T, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            if (c < C) {
                if constexpr (V == 1) {
                    v[i] = mrf_to_f32(row[c]);
                } else {
                    const vec x = *(const vec *)(row + c);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[i * V + j] = mrf_to_f32((T)x[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[i * V + j] = fill;
            }
        }
    }

    // the same without conversion to 32 bits (fewer registers while a row is on its way)
    template <class T> struct Raw { typename MrfVec<T, V>::type v[CH]; };
    template <class T> static __device__ inline void load_raw(const T *row, int C, int l, Raw<T> &r)
    {
        typedef typename MrfVec<T, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            if (c < C) r.v[i] = *(const vec *)(row + c);
        }
    }
    template <class T> static __device__ inline void convert(const Raw<T> &r, int C, int l, float (&v)[E], float fill)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const bool in = column(l, i) < C;
            if constexpr (V == 1) {
                v[i] = in ? mrf_to_f32(r.v[i]) : fill;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[i * V + j] = in ? mrf_to_f32((T)r.v[i][j]) : fill;
            }
        }
    }

    template <class T> static __device__ inline void store(T *row, int C, int l, const float (&v)[E])
    {
        typedef typename MrfVec<T, V>::type vec;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = column(l, i);
            if (c < C) {
                if constexpr (V == 1) {
                    row[c] = mrf_from_f32<T>(v[i]);
                } else {
                    vec x;
#pragma unroll
                    for (int j = 0; j < V; ++j) x[j] = mrf_from_f32<T>(v[i * V + j]);
                    *(vec *)(row + c) = x;
                }
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
};

// The layouts, shortest rows first: MRF_ROWS_*(F) stands for F(TL, V, CH) for each.
#define MRF_ROWS_8(F) \
    F(64, 8, 1) F(64, 8, 2) F(64, 8, 3) F(64, 8, 4) F(256, 8, 2) F(256, 8, 3) F(256, 8, 4) F(1024, 8, 2) F(1024, 8, 3) F(1024, 8, 4)
#define MRF_ROWS_4(F) \
    F(4, 4, 1) F(8, 4, 1) F(8, 4, 2) F(8, 4, 3) F(16, 4, 2) F(16, 4, 3) F(16, 4, 4) F(64, 4, 2) F(64, 4, 3) F(64, 4, 4) F(64, 4, 6) F(64, 4, 8) \
    F(256, 4, 4) F(256, 4, 6) F(256, 4, 8) F(1024, 4, 4) F(1024, 4, 6) F(1024, 4, 8)
#define MRF_ROWS_1(F) \
    F(4, 1, 1) F(4, 1, 2) F(4, 1, 3) F(4, 1, 4) F(8, 1, 3) F(8, 1, 4) F(8, 1, 5) F(8, 1, 6) F(8, 1, 7) F(8, 1, 8) F(16, 1, 5) F(16, 1, 6) F(16, 1, 7) F(16, 1, 8) \
    F(32, 1, 5) F(32, 1, 6) F(32, 1, 7) F(32, 1, 8) F(64, 1, 6) F(64, 1, 8) F(64, 1, 12) F(64, 1, 16) F(64, 1, 24) F(64, 1, 32) \
    F(256, 1, 12) F(256, 1, 16) F(256, 1, 24) F(256, 1, 32) F(1024, 1, 12) F(1024, 1, 16) F(1024, 1, 24) F(1024, 1, 32)
constexpr int MRF_ROWS_LONGEST = 32768;      // columns; longer rows are read several times

namespace mrf_host {
// elements per access that rows of C columns starting at these addresses allow, 4 at most; `bytes` of an element of each array
inline int row_vector(int C, const void *const *at, const int *bytes, int n)
{
    if (C % 4) return 1;
    for (int i = 0; i < n; ++i)
        if (at[i] && ((uintptr_t)at[i] % (4 * (size_t)bytes[i]))) return 1;
    return 4;
}
// the same for 8 elements of 16 bits (arrays of 32 bits beside them take two accesses of 16 bytes)
inline bool row_vector_8(int C, const void *const *at, int n)
{
    if (C % 8) return false;
    for (int i = 0; i < n; ++i)
        if (at[i] && ((uintptr_t)at[i] % 16)) return false;
    return true;
}
}  // namespace mrf_host
