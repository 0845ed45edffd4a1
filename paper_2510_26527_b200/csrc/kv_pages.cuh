// What the calls on 4-bit caches share: the layout of a page, whose rows are whose, the codes of a token's head.
//
// A page is [kv_heads, page_tokens / 8] units of eight tokens: head_dim words of codes, then eight (scale, offset) pairs.  Units of keys
// hold their words by token: the lanes of a matrix instruction that stand for one key read 16 neighbouring bytes each.  Units of values
// hold them as the second product reads them: a lane's words (two tokens, head_dim / 64 groups of eight elements) are neighbours.
#pragma once

#include "launch.cuh"
#include "polyspec_kernels.cuh"

namespace polyspec {
namespace kv {

constexpr int kUnit = 8;                        // tokens of a unit
constexpr long long kMostTokens = 0x7fff0000;   // of a sequence: counters may run past its end by a CTA's step

__host__ __device__ constexpr int unit_bytes(int head_dim) { return 4 * head_dim + 4 * kUnit; }
inline size_t page_bytes(const polyspec_cache_pages& s, int kv_heads, int head_dim)
{
    return static_cast<size_t>(kv_heads) * (s.page_tokens / kUnit) * unit_bytes(head_dim);
}

// Word number of word w of token r in a unit.
__device__ __forceinline__ int key_word(int r, int w, int head_dim) { return r * (head_dim / 8) + w; }
__device__ __forceinline__ int value_word(int r, int w, int head_dim)
{
    return (8 * (w & 7) + r) * (head_dim / 64) + (w >> 3);
}

__device__ __forceinline__ void report(int32_t* status, polyspec_status what)
{
    if (status) atomicCAS(status, 0, static_cast<int>(what));
}

// One sequence's rows of a block and its cache: rows row0 .. row0 + n - 1 stand at slots base .. base + n - 1, of which the first
// `granted` are below len.  None is where base or len makes no sense, nor, of all rows between its row numbers, where n_rows does not; n is 0 where those make none.
struct SeqRows { int row0, n, granted, base, len; bool bad; };
__device__ __forceinline__ SeqRows seq_rows(const polyspec_cache_pages& s, const polyspec_block_rows& r, int b)
{
    SeqRows q = {0, 0, 0, 0, 0, false};
    const int row0 = r.rows_at[b], end = r.rows_at[b + 1], len = s.len[b];
    const int n = r.n_rows ? r.n_rows[b] : end - row0;
    const long long base = static_cast<long long>(r.base[b]) + (r.extra ? r.extra[b] : 0);
    if (row0 < 0 || end < row0 || end > r.rows) { q.bad = true; return q; }
    q.row0 = row0;
    q.n = n < 0 || n > end - row0 ? end - row0 : n;
    if (q.n != n || len < 0 || len > s.max_pages * s.page_tokens) { q.bad = true; return q; }
    q.len = len;
    if (base < 0) { q.bad = n > 0; return q; }                  // rows that stand nowhere attend to nothing
    q.granted = base >= len ? 0 : min(n, static_cast<int>(len - base));
    q.base = static_cast<int>(min(base, static_cast<long long>(len)));
    q.bad = q.granted < n;
    return q;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rows of heads: stride at least a row, a multiple of eight elements, 16-byte aligned.
inline bool rows_ok(const void* p, long long stride, int heads, int head_dim)
{
    return p && aligned16(p) && stride >= static_cast<long long>(heads) * head_dim && stride % 8 == 0;
}

inline polyspec_status check_state(const polyspec_cache_pages* s)
{
    if (!s || s->n_seqs < 1 || s->max_pages < 1 || s->n_pages < 1 || s->page_tokens < 1) return POLYSPEC_ERR_INVALID_ARG;
    if (!s->table || !s->len || !s->refs || !s->free_bits || !aligned4(s->table, s->len, s->refs, s->free_bits)) return POLYSPEC_ERR_INVALID_ARG;
    if (static_cast<long long>(s->max_pages) * s->page_tokens > kMostTokens || s->n_pages > (1 << 20)) return POLYSPEC_ERR_UNSUPPORTED;
    return s->page_tokens % kUnit || s->page_tokens > 32768 ? POLYSPEC_ERR_UNSUPPORTED : POLYSPEC_OK;
}

// (a sequence's rows times the heads of a group, which kernels count in 32 bits, would take 256 GB of queries to reach 2^31)
inline polyspec_status check_rows(const polyspec_block_rows* r)
{
    if (!r || !r->rows_at || !r->base || r->rows < 1 || !aligned4(r->rows_at, r->n_rows, r->base, r->extra)) return POLYSPEC_ERR_INVALID_ARG;
    return r->rows > (1 << 24) ? POLYSPEC_ERR_UNSUPPORTED : POLYSPEC_OK;
}

inline polyspec_status check_heads(int q_heads, int kv_heads, int head_dim)
{
    if (q_heads < 1 || kv_heads < 1 || head_dim < 1) return POLYSPEC_ERR_INVALID_ARG;
    if (q_heads % kv_heads || q_heads > 1024 || (head_dim != 64 && head_dim != 128)) return POLYSPEC_ERR_UNSUPPORTED;
    return POLYSPEC_OK;
}

}  // namespace kv
}  // namespace polyspec
