// The words that tiles of 64 tokens read of tensors (B, L, heads, width) whose rows are read word by word: offsets in bytes from the tensor's first element,
// as piece_word gives them for every piece of 16 bytes.  Each has to begin at a multiple of 4 bytes and hold an element of its own row, and every element of
// the rows that are there has to be in a word.
#include <algorithm>
#include <cstdio>
#include <vector>

#include "piece_words.hpp"

using namespace ucd::attention;

// address: the tensor's first byte modulo 4.  Returns the number of faults.
static long look(long B, long L, long heads, long width, long gap, int size, int address, int cols, bool reversed)
{
    const long per = 16 / size, stride = (heads * width + gap) * size, words = size == 4 ? 4 : 5;
    const long end = (((B - 1) * L + L - 1) * stride) + heads * width * size;      // behind the last element
    long faults = 0;
    for (long b = 0; b < B; ++b)
        for (long head = 0; head < heads; ++head)
            for (long t0 = 0; t0 < L; t0 += 64) {
                const long base = (b * L + t0) * stride + head * width * size, tokens = std::min(64l, L - t0);
                const uint32_t odd = (uint32_t)((address + base) & 3), bytes = (uint32_t)(tokens * stride);
                for (long r = 0; r < 64; ++r)
                    for (long c = 0; c < cols; c += per) {
                        const long token = reversed ? 63 - r : r, have = std::max(0l, std::min(per, width - c));
                        const uint32_t at = (uint32_t)(token * stride) + (uint32_t)(c * size);
                        std::vector<char> seen((size_t)(have * size), 0);
                        for (int w = 0; w < words; ++w) {
                            const uint32_t o = piece_word(at, odd, (uint32_t)(have * size), bytes, w);
                            if (o >= kOut) continue;
                            const long from = base - (long)odd + (long)o, row = base + token * stride, first = row + c * size;
                            const bool real = token < tokens && from + 4 > row && from < row + width * size && from < end;
                            if (!real || (address + from) % 4 != 0) ++faults;
                            for (long i = 0; i < have * size; ++i)
                                if (from <= first + i && first + i < from + 4) seen[i] = 1;
                        }
                        if (token < tokens) faults += std::count(seen.begin(), seen.end(), 0);
                    }
            }
    return faults;
}

int main()
{
    long B, L, heads, width, gap;
    int size, address, cols, reversed;
    while (scanf("%ld %ld %ld %ld %ld %d %d %d %d", &B, &L, &heads, &width, &gap, &size, &address, &cols, &reversed) == 9)
        printf("%ld\n", look(B, L, heads, width, gap, size, address, cols, reversed != 0));
    return 0;
}
