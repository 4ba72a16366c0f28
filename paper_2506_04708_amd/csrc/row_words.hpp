// row_words.hpp -- 16 bytes of a row of logits at once, wherever the row begins: rows of an odd vocabulary, and tensors that
// begin inside another one, are aligned like their elements and no better.  (The hardware reads and writes such words in one piece.)
#pragma once
#include <stdint.h>

namespace stand {

template <int ES> struct RowWords;   // by the bytes of an element
template <> struct RowWords<2> { typedef uint32_t type __attribute__((vector_size(16), aligned(2))); };
template <> struct RowWords<4> { typedef uint32_t type __attribute__((vector_size(16), aligned(4))); };

}  // namespace stand
