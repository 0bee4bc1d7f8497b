"""Oracles of the operators around the attention, in 64 bits and plain loops: rotary append, logit edits, cache pages.

Test infrastructure only; shares nothing with the CUDA code.
"""
from __future__ import annotations

import collections

import numpy as np

PAGE = 16


# ------------------------------------------------------------------------------------------- rotary append
def axis_of_pair(axis_pairs, cyclic: bool):
    """Axis of each pair: blocks one after the other, or dealt out in turn to the axes that still have some left."""
    if not cyclic:
        return [a for a, n in enumerate(axis_pairs) for _ in range(n)]
    taken, out = [0] * len(axis_pairs), []
    while len(out) < sum(axis_pairs):
        for a, n in enumerate(axis_pairs):
            if taken[a] < n:
                taken[a] += 1
                out.append(a)
    return out


def rotate(x, pos, inv_freq, axis_pairs, cyclic, adjacent, factor):
    """``x`` float64 ``[T, H, D]``, ``pos`` ``[axes, T]``, ``inv_freq`` of 24 bits each.  Returns the rotated array and the sum of the
    magnitudes of the two products that each element is the sum of (what its rounding errors scale with)."""
    assert np.finfo(np.longdouble).nmant >= 63            # a position times a frequency has up to 32 + 24 bits: exact
    out, scale = x.copy(), np.abs(x)
    half = len(inv_freq)
    for p, axis in enumerate(axis_of_pair(axis_pairs, cyclic)):
        i, j = (2 * p, 2 * p + 1) if adjacent else (p, p + half)
        angle = np.asarray(pos[axis], dtype=np.longdouble) * np.longdouble(inv_freq[p])
        c, s = (factor * f(angle).astype(np.float64)[:, None] for f in (np.cos, np.sin))
        a, b = x[:, :, i], x[:, :, j]
        out[:, :, i], out[:, :, j] = a * c - b * s, b * c + a * s
        scale[:, :, i] = scale[:, :, j] = abs(factor) * (np.abs(a) + np.abs(b))
    return out, scale


def row_places(seq_lens, cu_q_lens, block_table, num_blocks):
    """For every row ``(position, page, slot)``; ``None`` for a row that is refused."""
    out = []
    for s in range(len(seq_lens)):
        n = cu_q_lens[s + 1] - cu_q_lens[s]
        for i in range(n):
            L = seq_lens[s]
            if L <= 0 or L > len(block_table[s]) * PAGE or n > L:
                out.append(None)
                continue
            pos = L - n + i
            page = block_table[s][pos // PAGE]
            out.append((pos, page, pos % PAGE) if 0 <= page < num_blocks else None)
    return out


# --------------------------------------------------------------------------------------------- logit edits
def adjust_logits(x, *, tokens=None, prompt_lens=None, total_lens=None, repetition=None, presence=None, frequency=None,
                  bias=None, mask=None, mask_rows=None):
    """``x`` float64 ``[rows, vocab]``; ``bias`` a list of ``(token, value)`` lists; ``mask`` boolean ``[masks, vocab]``.  Returns the edited
    array and the sum of the magnitudes of its terms."""
    rows, vocab = x.shape
    out, scale = x.copy(), np.abs(x)
    for r in range(rows):
        if tokens is not None:
            made, seen = {}, set()
            for i in range(int(total_lens[r])):
                t = int(tokens[r][i])
                if 0 <= t < vocab:
                    seen.add(t)
                    if i >= int(prompt_lens[r]):
                        made[t] = made.get(t, 0) + 1
            for t in seen:
                rep = 1.0 if repetition is None else float(repetition[r])
                out[r, t] = out[r, t] / rep if out[r, t] > 0 else out[r, t] * rep
                scale[r, t] = max(scale[r, t], abs(out[r, t]))
            for t, c in made.items():
                less = (0.0 if frequency is None else float(frequency[r])) * c + (0.0 if presence is None else float(presence[r]))
                out[r, t] -= less
                scale[r, t] += (0.0 if frequency is None else abs(float(frequency[r]))) * c + (0.0 if presence is None else abs(float(presence[r])))
        for t, b in dict(bias[r]).items() if bias is not None else ():
            if 0 <= t < vocab:
                out[r, t] += b
                scale[r, t] += abs(b)
        if mask is not None:
            m = r if mask_rows is None else int(mask_rows[r])
            if m >= 0:
                out[r, ~mask[m]] = -np.inf
    return out, scale


# --------------------------------------------------------------------------------------------- cache pages
class Pool:
    """The pool as Python lists; ``faults`` collects the codes of what was refused."""

    def __init__(self, num_seqs, max_blocks, num_blocks):
        self.table = [[-1] * max_blocks for _ in range(num_seqs)]
        self.lens = [0] * num_seqs
        self.refs = [0] * num_blocks
        self.max_blocks = max_blocks
        self.faults = []

    def _pages(self, n):
        return (n + PAGE - 1) // PAGE

    def _len_ok(self, n):
        return 0 <= n <= self.max_blocks * PAGE

    def _row(self, s):
        return 0 <= s < len(self.lens)

    def fork(self, parents, children):
        before, copied, named = list(self.lens), set(parents), set()
        for a, b in zip(parents, children):
            again = b in named
            named.add(b)
            if not (self._row(a) and self._row(b)) or b in copied or again or before[b] != 0 or not self._len_ok(self.lens[a]):
                self.faults.append("bounds")
                continue
            held = self.table[a][:self._pages(self.lens[a])]
            if any(not 0 <= p < len(self.refs) or self.refs[p] <= 0 for p in held):
                self.faults.append("bounds")
                continue
            self.table[b][:len(held)] = held
            self.lens[b] = self.lens[a]
            for p in held:
                self.refs[p] += 1

    def extend(self, new_rows):
        free = [p for p, n in enumerate(self.refs) if n <= 0]
        before, at, pairs = list(self.refs), 0, []
        for s, n in enumerate(new_rows):
            pairs.append((-1, -1))
            L = self.lens[s]
            if L < 0 or n < 0 or not self._len_ok(L + n):
                self.faults.append("bounds")
                continue
            if n == 0:
                continue
            split, have = False, self._pages(L)
            if L % PAGE:
                last = self.table[s][have - 1]
                if not 0 <= last < len(self.refs) or before[last] <= 0:
                    self.faults.append("bounds")
                    continue
                split = before[last] > 1
            need = self._pages(L + n) - have + split
            mine = free[at:at + need]
            at += need
            if need and at > len(free):
                self.faults.append("no pages")
                continue
            if split:
                pairs[-1] = (last, mine[0])
                self.refs[last] -= 1
                self.table[s][have - 1] = mine[0]
            for j, p in enumerate(mine[split:]):
                self.table[s][have + j] = p
            for p in mine:
                self.refs[p] = 1
            self.lens[s] = L + n
        return pairs

    def free(self, seqs, keep_lens=None):
        done = set()
        for i, s in enumerate(seqs):
            if s in done:
                continue
            done.add(s)
            keep = 0 if keep_lens is None else keep_lens[i]
            if not self._row(s) or not self._len_ok(self.lens[s]) or keep < 0:
                self.faults.append("bounds")
                continue
            if keep >= self.lens[s]:
                continue
            for j in range(self._pages(keep), self._pages(self.lens[s])):
                p, self.table[s][j] = self.table[s][j], -1
                if not 0 <= p < len(self.refs) or self.refs[p] <= 0:
                    self.faults.append("bounds")
                else:
                    self.refs[p] -= 1
            self.lens[s] = keep

    def compact(self):
        used = sum(n > 0 for n in self.refs)
        sources = [p for p, n in enumerate(self.refs) if n > 0 and p >= used]
        holes = [p for p, n in enumerate(self.refs) if n <= 0 and p < used]
        moves = dict(zip(sources, holes))
        page_map = [moves.get(p, p) if n > 0 else -1 for p, n in enumerate(self.refs)]
        refs = [0] * len(self.refs)
        for p, to in enumerate(page_map):
            if to >= 0:
                refs[to] = self.refs[p]
        table = [[-1] * self.max_blocks for _ in self.table]
        for row, out, L in zip(self.table, table, self.lens):
            if not self._len_ok(L):
                self.faults.append("bounds")
                continue
            for j, p in enumerate(row[:self._pages(L)]):
                out[j] = page_map[p] if 0 <= p < len(page_map) else -1
                if out[j] < 0:
                    self.faults.append("bounds")
        return table, refs, page_map, list(zip(sources, holes))


def copy_pages(cache, pairs):
    """``cache`` ``[pages, ...]``.  Pairs that depend on one another are not carried out; returns the copy and whether there were any."""
    live = [(s, d) for s, d in pairs if s >= 0 and d >= 0]
    sources, targets = collections.Counter(s for s, _ in live), collections.Counter(d for _, d in live)
    out, refused = cache.copy(), False
    for s, d in live:
        if s == d:
            continue
        # its destination is somebody else's destination or source, or its source is a destination (its own is another page)
        if max(s, d) >= len(cache) or targets[d] > 1 or sources[d] or targets[s]:
            refused = True
            continue
        out[d] = cache[s]
    return out, refused
