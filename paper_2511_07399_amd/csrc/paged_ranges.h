// Which keys the rows of a ragged batch see, and which key tiles a run of rows visits.  Without dependencies: the kernels and the
// host use it.
#pragma once

namespace sdv2 {

// Tokens of a sequence whose kv_len the device array states: no more than its row of the page table holds, and not under zero.
constexpr int tokens_of(int kv_len, int table_stride, int page_shift) {
    const long long most = (long long)table_stride << page_shift;
    return kv_len < 0 ? 0 : kv_len > most ? (int)most : kv_len;
}

// Keys that a row may see: j < end, and j >= low or j < sink.
struct RowKeys {
    int end, low, sink;
};
struct MaskArgs {
    int block;                // 0: all keys; B: those of the row's block of B tokens and before
    int window, sink;         // 0: no window; else the last `window` keys up to the end, and the first `sink`
    float scale_log2e;        // softmax scale times log2 e (and the keys' scale)
};
// Row i of n new tokens of a sequence of kv_len >= 0 tokens.
constexpr RowKeys row_keys(const MaskArgs& m, int i, int n, int kv_len) {
    const int p = kv_len - n + i;
    int end = kv_len;
    if (m.block > 0) {
        const long long behind = ((long long)(p / m.block) + 1) * m.block;
        end = p < 0 ? 0 : behind < kv_len ? (int)behind : kv_len;
    }
    const int low = m.window > 0 && end > m.window ? end - m.window : 0;
    return RowKeys{end, low, m.window > 0 ? (m.sink < low ? m.sink : low) : 0};
}
constexpr bool sees(const RowKeys& k, int j) { return (j < k.end) & ((j >= k.low) | (j < k.sink)); }

// The key tiles that a run of rows sees, in order: those of the sink, then those from the window on.
struct Visited {
    int sink_tiles, skip;     // tile number n is tile n where n < sink_tiles, n + skip from there on
    int count;
    int e_first, low_last, sink_first;      // which tiles need no mask: see whole()
};
// Tiles of KT keys of rows first_token .. last_token of n.
template <int KT>
constexpr Visited visited_tiles(const MaskArgs& m, int first_token, int last_token, int n, int kv_len) {
    const RowKeys a = row_keys(m, first_token, n, kv_len), b = row_keys(m, last_token, n, kv_len);
    const int low_tile = a.low / KT, end_tile = (int)((unsigned)(b.end + KT - 1) / KT), sink_tiles = (a.sink + KT - 1) / KT;
    const int skip = sink_tiles < low_tile ? low_tile - sink_tiles : 0;
    return Visited{sink_tiles, skip, end_tile > skip ? end_tile - skip : 0, a.end, b.low, a.sink};
}
constexpr int tile_of(const Visited& v, int n) { return n < v.sink_tiles ? n : n + v.skip; }
// Whether every row sees all keys first .. end - 1 (pages aside).
constexpr bool whole(const Visited& v, int first, int end) { return end <= v.e_first && (first >= v.low_last || end <= v.sink_first); }

}  // namespace sdv2
