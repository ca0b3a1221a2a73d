// The paged 8-bit cache's arithmetic on lengths, starts and pages, shared by its kernels and by host programs that walk it: which rows of a call belong to
// a sequence, which of its positions a table can hold, and how the attention of one token a sequence is cut into chunks.  Whatever
// the device arrays hold, what comes out stays inside the call's rows and the table.
#pragma once

#include <stddef.h>

#ifdef __HIP__
#define RCP_BOTH __host__ __device__ inline __attribute__((always_inline))
#else
#define RCP_BOTH inline
#endif

namespace rcp {

constexpr int KV8_MOST_TOKENS = 1 << 24;  // of a table's row, and rows of a call
constexpr int KV8_MOST_SEQUENCES = 1024;

RCP_BOTH int kv8_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The new tokens of sequence b: rows first .. first + count - 1 of the call, the first of them at position pos (below 0: more
// new tokens than the sequence is long) of a sequence of `length` tokens.
struct Kv8Run {
    int first, count, pos, length;
};

RCP_BOTH Kv8Run kv8_run(const int* starts, const int* lengths, int b, int rows)
{
    Kv8Run r;
    r.length = kv8_clamp(lengths[b], 0, KV8_MOST_TOKENS);
    if (starts == nullptr) {
        r.first = b;
        r.count = 1;
    } else {
        r.first = kv8_clamp(starts[b], 0, rows);
        r.count = kv8_clamp(starts[b + 1], r.first, rows) - r.first;
    }
    r.pos = r.length - r.count;
    return r;
}

// Pages that the new tokens of a run fall into, of a table that holds `capacity` tokens a sequence: [first_page, first_page + pages)
struct Kv8Pages {
    int first_page, pages;
};

RCP_BOTH Kv8Pages kv8_pages(const Kv8Run& r, int capacity, int shift)
{
    const int lo = r.pos < 0 ? 0 : r.pos, hi = r.length < capacity ? r.length : capacity;
    if (r.count == 0 || hi <= lo) return {0, 0};
    return {lo >> shift, ((hi - 1) >> shift) - (lo >> shift) + 1};
}

// No call has more (sequence, page) pairs to write: a run of n tokens touches at most (n + page - 2) / page + 1 pages.
RCP_BOTH long long kv8_most_pages(int rows, int sequences, int shift)
{
    return (static_cast<long long>(rows) >> shift) + 2LL * sequences;
}

// Tokens per chunk of the attention of one token a sequence: the fewest, in whole tiles of 64, with which `total` cached tokens (below 2^31) of
// `sequences` sequences make at most `chunks` chunks (chunks >= 2 * sequences): sum ceil(n / C) <= total / C + sequences.
RCP_BOTH int kv8_chunk_tokens(int total, int sequences, int chunks)
{
    const unsigned room = static_cast<unsigned>(chunks - sequences);
    const unsigned c = (static_cast<unsigned>(total) + room - 1) / room;
    return c <= 64 ? 64 : static_cast<int>((c + 63) / 64 * 64);
}

// chunks of a sequence: an empty one has one too, which writes zeros
RCP_BOTH int kv8_chunks(int tokens, int per_chunk)
{
    return tokens <= 0 ? 1 : static_cast<int>((static_cast<unsigned>(tokens) + static_cast<unsigned>(per_chunk) - 1) / static_cast<unsigned>(per_chunk));
}

// The sequence whose run holds row t, -1 if none does: the last b with starts[b] <= t.  Ends for any contents of `starts`.
RCP_BOTH int kv8_sequence_of(const int* starts, int sequences, int t, int rows)
{
    int lo = 0, hi = sequences - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int first = kv8_clamp(starts[lo], 0, rows), end = kv8_clamp(starts[lo + 1], first, rows);
    return t >= first && t < end ? lo : -1;
}

}  // namespace rcp
