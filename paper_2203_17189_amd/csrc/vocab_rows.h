// A row of a vocabulary's logits in the registers of a workgroup: rows of any alignment and length, read in 16-byte
// pieces.  The elements in front of the row's first 16-byte boundary and behind its last whole piece (fewer than a piece
// each) go to single lanes.
#pragma once
#include "common.h"

namespace t5mi {

template <typename T> struct RowVec;
template <> struct RowVec<bf16> { typedef bf16x8 type; };
template <> struct RowVec<float> { typedef f32x4 type; };

template <typename T>
struct RowSplit {
  static constexpr int EPV = 16 / sizeof(T);
  int head, pieces, tail;
  // row: element pointer; V >= 1 elements
  __device__ __forceinline__ RowSplit(const T* row, int V) {
    const int off = (int)(((uintptr_t)row & 15) / sizeof(T));
    head = off ? EPV - off : 0;
    if (head > V) head = V;
    pieces = (V - head) / EPV;
    tail = V - head - pieces * EPV;
  }
  // The single element of thread t of nt (>= 16): its index, or -1.
  __device__ __forceinline__ int single(int t, int nt, int V) const {
    if (t < head) return t;
    const int q = t - (nt - EPV);
    return q >= 0 && q < tail ? V - tail + q : -1;
  }
};

}  // namespace t5mi
