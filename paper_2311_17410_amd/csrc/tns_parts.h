// Lists of the attention that are cut into parts where blocks of `1 << part` rows end (counted from row 0): where they end, and which workgroup joins one of
// many parts.  Plain arithmetic, that a test builds for the host.
#pragma once
#include <cstdint>

namespace tns {

constexpr int kMany = 256;              // lists of more parts are joined by workgroups of their own

constexpr int64_t parts_end(int64_t list_end, int part, int64_t blocks) {
    const int64_t end = (list_end + ((int64_t)1 << part) - 1) >> part;
    return end < blocks ? end : blocks;
}
constexpr bool is_many(int64_t first, int64_t end) { return end - first > kMany; }

// A list of more than kMany parts, the first in block b, has one in each of the blocks b + 1 .. b + kMany: one of them has a number that is a multiple of
// kMany, and its first row is the list's (that of block b may be another one's).  The first such block stands for the list; they are
// places 0, 1, ... for those who look for lists to join: blocks kMany, 2 kMany, ...
constexpr int64_t place_of(int64_t first) { return first / kMany; }
constexpr int64_t many_places(int64_t blocks) { return blocks > 0 ? (blocks - 1) / kMany : 0; }
// The list of many parts that the place stands for, and its parts' blocks; -1 if there is none.
template <typename Lists>
constexpr int64_t many_at(int64_t place, int part, int64_t blocks, const Lists& lists, int64_t& first, int64_t& end) {
    const int64_t row = ((place + 1) * kMany) << part;
    if (row >= lists.total()) return -1;
    const int64_t list = lists.find(row);
    first = lists.edge(list) >> part;
    end = parts_end(lists.edge(list + 1), part, blocks);
    return is_many(first, end) && place_of(first) == place ? list : -1;
}

}  // namespace tns
