// Which pages of a cache hold which sequence.  Host code only: plain counting, no GPU call.
#include "mes_internal.h"

#include <algorithm>
#include <new>
#include <vector>

struct mes_pages {
  int n_pages, page_tokens, max_seqs, max_seq_pages, unused;
  std::vector<int32_t> holders;                  // of every page: sequences that hold it
  std::vector<std::vector<int32_t>> pages;       // of every sequence
  std::vector<int32_t> length;
  int lowest;                                    // no page below it is free
};

namespace mes {
namespace {

mes_pages* make(int n_pages, int page_tokens, int max_seqs, int max_seq_pages) {
  mes_pages* p = new mes_pages;
  try {
    p->n_pages = n_pages;
    p->page_tokens = page_tokens;
    p->max_seqs = max_seqs;
    p->max_seq_pages = max_seq_pages;
    p->unused = n_pages;
    p->lowest = 0;
    p->holders.assign(n_pages, 0);
    p->length.assign(max_seqs, 0);
    p->pages.resize(max_seqs);
  } catch (...) {
    delete p;
    throw;
  }
  return p;
}

int take(mes_pages* p) {
  while (p->holders[p->lowest]) ++p->lowest;
  p->holders[p->lowest] = 1;
  --p->unused;
  return p->lowest;
}

void drop(mes_pages* p, int page) {
  if (--p->holders[page]) return;
  ++p->unused;
  p->lowest = std::min(p->lowest, page);
}

// room for `n` pages, at least doubling, so that growing page by page stays cheap; may throw, before anything is changed
void make_room(std::vector<int32_t>& v, int64_t n) {
  if ((int64_t)v.capacity() < n) v.reserve(std::max<size_t>((size_t)n, 2 * v.capacity()));
}

bool is_seq(const mes_pages* p, int s) { return s >= 0 && s < p->max_seqs; }

// pages of `tokens` tokens (tokens fits 64 bits: a length plus an int)
int64_t pages_of(const mes_pages* p, int64_t tokens) { return (tokens + p->page_tokens - 1) / p->page_tokens; }

}  // namespace
}  // namespace mes

using namespace mes;

extern "C" {

mes_status mes_pages_create(int n_pages, int page_tokens, int max_seqs, int max_seq_pages, mes_pages** out) {
  if (!out) return fail(MES_ERR_NULL, "mes_pages_create: out is null");
  *out = nullptr;
  if (n_pages < 1 || max_seqs < 1 || max_seq_pages < 1) return fail(MES_ERR_SHAPE, "mes_pages_create: n_pages, max_seqs and max_seq_pages must be positive");
  if (page_tokens < 1) return fail(MES_ERR_SHAPE, "mes_pages_create: page_tokens must be positive (got %d)", page_tokens);
  if ((int64_t)max_seq_pages * page_tokens > 0x7fffffff) return fail(MES_ERR_SHAPE, "mes_pages_create: a sequence of %d pages of %d tokens is too long", max_seq_pages, page_tokens);
  try {
    *out = make(n_pages, page_tokens, max_seqs, max_seq_pages);
  } catch (...) {
    return fail(MES_ERR_DEVICE, "mes_pages_create: out of host memory");
  }
  return MES_OK;
}

void mes_pages_destroy(mes_pages* p) { delete p; }

mes_status mes_pages_grow(mes_pages* p, const int32_t* seqs, const int32_t* n_tokens, int n, int32_t* copy_src, int32_t* copy_dst,
                          int* n_copies) {
  if (!p || !n_copies || (n > 0 && (!seqs || !n_tokens || !copy_src || !copy_dst))) return fail(MES_ERR_NULL, "mes_pages_grow: null pointer");
  *n_copies = 0;
  if (n < 0 || n > p->max_seqs) return fail(MES_ERR_SHAPE, "mes_pages_grow: n = %d outside [0, %d]", n, p->max_seqs);
  // what it takes, before anything is changed.  A last page that m of the growing sequences hold and nobody else does is
  // copied m - 1 times: the last of them keeps it.  Counted by taking their holds off while looking, and putting them back.
  int64_t need = 0;
  mes_status st = MES_OK;
  int seen = 0;
  for (; seen < n && st == MES_OK; ++seen) {
    const int s = seqs[seen];
    if (!is_seq(p, s)) { st = fail(MES_ERR_SHAPE, "mes_pages_grow: sequence %d outside [0, %d)", s, p->max_seqs); break; }
    if (p->length[s] < 0) { st = fail(MES_ERR_SHAPE, "mes_pages_grow: sequence %d given twice", s); break; }
    if (n_tokens[seen] < 0) { st = fail(MES_ERR_SHAPE, "mes_pages_grow: n_tokens[%d] is negative", seen); break; }
    const int64_t after = (int64_t)p->length[s] + n_tokens[seen];
    if (pages_of(p, after) > p->max_seq_pages) { st = fail(MES_ERR_SHAPE, "mes_pages_grow: sequence %d outgrows its %d pages", s, p->max_seq_pages); break; }
    need += pages_of(p, after) - (int64_t)p->pages[s].size();
    const bool partial = n_tokens[seen] > 0 && p->length[s] % p->page_tokens;
    if (partial && p->holders[p->pages[s].back()] > 1) {
      ++need;
      --p->holders[p->pages[s].back()];
      copy_src[(*n_copies)++] = p->pages[s].back();
    }
    p->length[s] = ~p->length[s];                      // seen
  }
  for (int i = 0; i < seen; ++i) p->length[seqs[i]] = ~p->length[seqs[i]];
  for (int i = 0; i < *n_copies; ++i) ++p->holders[copy_src[i]];
  *n_copies = 0;
  if (st) return st;
  if (need > p->unused) return fail(MES_ERR_PAGES, "mes_pages_grow: %lld pages are needed, %d are free", (long long)need, p->unused);
  try {
    for (int i = 0; i < n; ++i) make_room(p->pages[seqs[i]], pages_of(p, (int64_t)p->length[seqs[i]] + n_tokens[i]));
  } catch (...) {
    return fail(MES_ERR_DEVICE, "mes_pages_grow: out of host memory");
  }
  for (int i = 0; i < n; ++i) {
    const int s = seqs[i];
    std::vector<int32_t>& own = p->pages[s];
    if (n_tokens[i] > 0 && p->length[s] % p->page_tokens && p->holders[own.back()] > 1) {
      const int fresh = take(p);
      copy_src[*n_copies] = own.back();
      copy_dst[(*n_copies)++] = fresh;
      drop(p, own.back());
      own.back() = fresh;
    }
    p->length[s] += n_tokens[i];
    while ((int64_t)own.size() < pages_of(p, p->length[s])) own.push_back(take(p));
  }
  return MES_OK;
}

mes_status mes_pages_fork(mes_pages* p, int parent, int child, int n_tokens) {
  if (!p) return fail(MES_ERR_NULL, "mes_pages_fork: null pointer");
  if (!is_seq(p, parent) || !is_seq(p, child) || parent == child) return fail(MES_ERR_SHAPE, "mes_pages_fork: sequences %d and %d must differ and lie in [0, %d)", parent, child, p->max_seqs);
  if (p->length[child]) return fail(MES_ERR_SHAPE, "mes_pages_fork: sequence %d is not empty", child);
  if (n_tokens < 0 || n_tokens > p->length[parent]) return fail(MES_ERR_SHAPE, "mes_pages_fork: %d tokens of a sequence of %d", n_tokens, p->length[parent]);
  const size_t m = (size_t)pages_of(p, n_tokens);
  try {
    make_room(p->pages[child], (int64_t)m);
  } catch (...) {
    return fail(MES_ERR_DEVICE, "mes_pages_fork: out of host memory");
  }
  p->pages[child].assign(p->pages[parent].begin(), p->pages[parent].begin() + m);
  for (int32_t page : p->pages[child]) ++p->holders[page];
  p->length[child] = n_tokens;
  return MES_OK;
}

mes_status mes_pages_free(mes_pages* p, int seq) {
  if (!p) return fail(MES_ERR_NULL, "mes_pages_free: null pointer");
  if (!is_seq(p, seq)) return fail(MES_ERR_SHAPE, "mes_pages_free: sequence %d outside [0, %d)", seq, p->max_seqs);
  for (int32_t page : p->pages[seq]) drop(p, page);
  p->pages[seq].clear();
  p->length[seq] = 0;
  return MES_OK;
}

mes_status mes_pages_compact(mes_pages* p, int32_t* copy_src, int32_t* copy_dst, int* n_copies) {
  if (!p || !copy_src || !copy_dst || !n_copies) return fail(MES_ERR_NULL, "mes_pages_compact: null pointer");
  *n_copies = 0;
  // holes below the number of pages in use are filled from the top; a page moves at most once, from above that line
  int low = 0, high = p->n_pages - 1;
  const int used = p->n_pages - p->unused;
  for (;;) {
    while (low < used && p->holders[low]) ++low;
    if (low >= used) break;
    while (!p->holders[high]) --high;
    copy_src[*n_copies] = high;
    copy_dst[(*n_copies)++] = low;
    p->holders[low] = p->holders[high];
    p->holders[high] = -low - 1;                       // moved there: read back below
    ++low;
    --high;
  }
  for (auto& own : p->pages)
    for (int32_t& page : own)
      if (p->holders[page] < 0) page = -p->holders[page] - 1;
  for (int i = 0; i < *n_copies; ++i) p->holders[copy_src[i]] = 0;
  p->lowest = 0;
  return MES_OK;
}

mes_status mes_pages_table(const mes_pages* p, const int32_t* seqs, int n, int32_t* table, int table_pages, int32_t* len) {
  if (!p || (n > 0 && (!seqs || !table))) return fail(MES_ERR_NULL, "mes_pages_table: null pointer");
  if (n < 0 || table_pages < 1) return fail(MES_ERR_SHAPE, "mes_pages_table: n = %d, table_pages = %d", n, table_pages);
  for (int i = 0; i < n; ++i) {
    if (!is_seq(p, seqs[i])) return fail(MES_ERR_SHAPE, "mes_pages_table: sequence %d outside [0, %d)", seqs[i], p->max_seqs);
    if ((int64_t)p->pages[seqs[i]].size() > table_pages) return fail(MES_ERR_SHAPE, "mes_pages_table: sequence %d has %zu pages, the table has room for %d", seqs[i], p->pages[seqs[i]].size(), table_pages);
  }
  for (int i = 0; i < n; ++i) {
    const std::vector<int32_t>& own = p->pages[seqs[i]];
    int32_t* row = table + (size_t)i * table_pages;
    std::fill(std::copy(own.begin(), own.end(), row), row + table_pages, 0);
    if (len) len[i] = p->length[seqs[i]];
  }
  return MES_OK;
}

int mes_pages_length(const mes_pages* p, int seq) { return p && is_seq(p, seq) ? p->length[seq] : -1; }
int mes_pages_unused(const mes_pages* p) { return p ? p->unused : -1; }

}  // extern "C"
