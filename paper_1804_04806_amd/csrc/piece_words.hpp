// Which words of memory a piece of a row is made of, where rows are read word by word.  No more than arithmetic: the host's compilers take it too.
#pragma once
#include <cstdint>

namespace ucd {
namespace attention {

// Reads behind a buffer's end give 0.
constexpr uint32_t kOut = 0x80000000u;

// Word w of a piece of `have` bytes that begins `at` bytes behind a base: its offset from the multiple of 4 bytes at or below the base, which is `odd` bytes
// behind that.  Words begin at multiples of 4 bytes, so that one with an element of the row is on that element's page whatever stands beside it in the word.
// Tokens end `bytes` behind the base.  A piece of nothing has no words, also where its begin lies within one.
constexpr uint32_t piece_word(uint32_t at, uint32_t odd, uint32_t have, uint32_t bytes, int w)
{
    const uint32_t begin = at + odd, word = (begin & ~3u) + 4u * (uint32_t)w;
    return have != 0 && at < bytes && word < begin + have ? word : kOut;
}

}  // namespace attention
}  // namespace ucd
