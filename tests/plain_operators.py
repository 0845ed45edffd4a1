"""Plain 64-bit statements of the 4-bit LM head, the sampling controls and the cache pages, for the tests of the kernels."""
import numpy as np
import torch


def head(hidden, codes, scales, zero_points):
    """(logits, sum of magnitudes) in float64: hidden [rows, d], codes [V, d] 0..15, scales and zero_points [V, groups]."""
    h = hidden.double().cpu()
    V, d = codes.shape
    group = d // scales.shape[1]
    z = torch.full(scales.shape, 8.0, dtype=torch.float64) if zero_points is None else (zero_points.cpu() & 15).double()
    w = (codes.cpu().double() - z.repeat_interleave(group, 1)) * scales.double().cpu().repeat_interleave(group, 1)
    return h @ w.t(), h.abs() @ w.abs().t()


def controls(logits, draft=None, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
             bias_tokens=None, bias_values=None, allowed=None, vocab_begin=0, vocab_size=None):
    """float64 result of the sampling controls on numpy arrays, the set of touched entries, and a bound on the magnitudes that
    the fp32 form adds up.  allowed [B, rows, V] bool."""
    z = np.asarray(logits, dtype=np.float64).copy()
    B, rows, V = z.shape
    touched = np.zeros(z.shape, dtype=bool)
    size = np.zeros(z.shape)
    for b in range(B):
        r = 1.0 if repetition is None else float(repetition[b])
        r = r if r > 0 else 1.0
        f = 0.0 if frequency is None else float(frequency[b])
        p = 0.0 if presence is None else float(presence[b])
        text = [] if history is None else [int(t) for t in history[b]]
        n = len(text) if history_len is None else min(max(int(history_len[b]), 0), len(text))
        m = 0 if prompt_len is None else min(max(int(prompt_len[b]), 0), n)
        for j in range(rows):
            said = text[m:n] + ([] if draft is None else [int(t) for t in draft[b][:j]])
            counts = {}
            for t in said:
                counts[t] = counts.get(t, 0) + 1
            for t in set(text[:m]) | set(counts):
                v = t - vocab_begin
                if t < 0 or not 0 <= v < V:
                    continue
                x = z[b, j, v]
                x = x / r if x > 0 else x * r
                size[b, j, v] += abs(x)
                c = counts.get(t, 0)
                if c:
                    x = x - f * c - p
                    size[b, j, v] += 2 * abs(f * c) + abs(p)
                z[b, j, v] = x
                touched[b, j, v] = True
            if bias_tokens is not None:
                for t, x in zip(bias_tokens[b], bias_values[b]):
                    v = int(t) - vocab_begin
                    if t >= 0 and 0 <= v < V:
                        z[b, j, v] += float(x)
                        size[b, j, v] += 2 * abs(float(x))
                        touched[b, j, v] = True
    if allowed is not None:
        z[~allowed] = -np.inf
        touched |= ~allowed
    return z, touched, size


def mask_words(allowed):
    """[..., V] bool -> [..., ceil(V/32)] int32."""
    V = allowed.shape[-1]
    W = (V + 31) // 32
    bits = np.zeros(allowed.shape[:-1] + (W * 32,), dtype=np.uint8)
    bits[..., :V] = allowed
    return np.packbits(bits, axis=-1, bitorder="little").view("<u4").view(np.int32).reshape(allowed.shape[:-1] + (W,))


class Pages:
    """The page tables as lists, one step at a time."""

    def __init__(self, n_seqs, max_pages, n_pages, page_tokens):
        self.P, self.max_pages, self.n_pages = page_tokens, max_pages, n_pages
        self.rows = [[] for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.refs = [0] * n_pages
        self.status = 0

    def need(self, tokens):
        return -(-tokens // self.P)

    def _drop(self, page):
        self.refs[page] -= 1

    def reserve(self, targets):
        """Returns the copies made, (from, to)."""
        free = [p for p in range(self.n_pages) if self.refs[p] == 0]
        shared = [c > 1 for c in self.refs]
        copies, spent, dropped = [], 0, []
        for b, want in enumerate(targets):
            if want <= self.len[b]:
                continue
            if want > self.max_pages * self.P:
                self.status = self.status or 6
                continue
            copy = self.len[b] % self.P != 0 and shared[self.rows[b][-1]]
            n = self.need(want) - len(self.rows[b]) + copy
            ok = n == 0 or spent + n <= len(free)
            if not ok:
                self.status = self.status or 8
                spent += n
                continue
            got = free[spent:spent + n]
            spent += n
            if copy:
                old, new = self.rows[b][-1], got.pop(0)
                self.rows[b][-1] = new
                dropped.append(old)
                self.refs[new] = 1
                copies.append((old, new))
            for p in got:
                self.refs[p] = 1
            self.rows[b] += got
            self.len[b] = want
        for p in dropped:
            self._drop(p)
        return copies

    def rollback(self, targets):
        for b, to in enumerate(targets):
            if 0 <= to < self.len[b]:
                for p in self.rows[b][self.need(to):]:
                    self._drop(p)
                self.rows[b] = self.rows[b][: self.need(to)]
                self.len[b] = to

    def fork(self, src, dst):
        before = list(self.len)
        for i, (s, d) in enumerate(zip(src, dst)):
            if s < 0 and d < 0:
                continue
            n = len(self.rows)
            if not (0 <= s < n and 0 <= d < n) or before[d] != 0 or s in dst or d in dst[:i]:
                self.status = self.status or 6
                continue
            self.rows[d], self.len[d] = list(self.rows[s]), self.len[s]
            for p in self.rows[d]:
                self.refs[p] += 1

    def compact(self):
        """Returns {old: new} of the moved pages."""
        live = [p for p in range(self.n_pages) if self.refs[p]]
        n = len(live)
        moves = dict(zip([p for p in live if p >= n], [p for p in range(n) if not self.refs[p]]))
        for old, new in moves.items():
            self.refs[new], self.refs[old] = self.refs[old], 0
        self.rows = [[moves.get(p, p) for p in row] for row in self.rows]
        return moves

    def arrays(self):
        table = np.full((len(self.rows), self.max_pages), -1, dtype=np.int32)
        for b, row in enumerate(self.rows):
            table[b, : len(row)] = row
        free = np.zeros((self.n_pages + 31) // 32 * 32, dtype=np.uint8)
        free[: self.n_pages] = [c == 0 for c in self.refs]
        return {"table": table, "len": np.array(self.len, dtype=np.int32), "refs": np.array(self.refs, dtype=np.int32),
                "free_bits": np.packbits(free, bitorder="little").view("<u4").view(np.int32)}
