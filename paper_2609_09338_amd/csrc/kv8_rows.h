// The rows whose queries an append forms (kv8_append.hip), a group of `per` rows a wavefront.
// Rows before the first sequence and behind the last are neither read nor written.
#pragma once

namespace osp {

struct QueryRows {
  int first, end;
};
// `total` rows of which the sequences have [cu_first, cu_end).
constexpr QueryRows query_rows(int total, int cu_first, int cu_end) {
  return {cu_first > 0 ? cu_first : 0, cu_end < total ? cu_end : total};
}
// Whether group `i`, the rows from i * per on, has any of them.
constexpr bool group_has_rows(QueryRows q, int i, int per) {
  return q.first < q.end && (long)i * per < q.end && ((long)i + 1) * per > q.first;
}
constexpr bool has_row(QueryRows q, int row) { return row >= q.first && row < q.end; }
// The row that is read for a row of such a group: the nearest of them.
constexpr int row_read(QueryRows q, int row) { return row < q.first ? q.first : row < q.end ? row : q.end - 1; }

}  // namespace osp
