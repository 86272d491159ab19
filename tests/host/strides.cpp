// strides.cpp -- rows_meet of kv_strides.h, for arrays that start `apart` values from each other.
#include "kv_strides.h"

extern "C" int meet(int64_t apart, int64_t a_row, int64_t a_head, int64_t a_heads, int64_t b_row, int64_t b_head,
                    int64_t b_heads, int64_t n, int64_t dim) {
  const int64_t a = (int64_t)1 << 50;
  return p2p::rows_meet({(const void*)a, a_row, a_head, a_heads}, {(const void*)(a + 2 * apart), b_row, b_head, b_heads}, n,
                        dim);
}
