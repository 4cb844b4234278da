"""Plain host forms of the paged cache's operators, row by row in Python and 64 bits: what
the GPU tests compare with."""
import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


def e4m3_value(byte):
    """The value of every byte as a float of 4 exponent and 3 mantissa bits."""
    byte = np.asarray(byte, np.int64)
    sign, e, f = np.where(byte & 128, -1.0, 1.0), (byte >> 3) & 15, byte & 7
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (np.maximum(e, 1) - 10.0))
    return np.where((byte & 127) == 127, np.nan, sign * v)


GRID = np.sort(e4m3_value(np.arange(127)))


def nearest_e4m3(y):
    """To nearest, ties to the even mantissa."""
    a = np.abs(y)
    hi = np.minimum(np.searchsorted(GRID, a), 126)
    lo = np.maximum(hi - 1, 0)
    up = (GRID[hi] - a < a - GRID[lo]) | ((GRID[hi] - a == a - GRID[lo]) & (hi % 2 == 0))
    return np.copysign(np.where(up, GRID[hi], GRID[lo]), y)


def quantize(block, code):
    """(codes float64, scale float32) of a block of float32 values: every operation in float32."""
    block = np.asarray(block, np.float32)
    top = np.float32(TOP[code])
    if not np.isfinite(block).all():
        return np.zeros(block.shape), np.float32(np.nan)
    a = np.abs(block).max()
    if a < 2.0 ** -100:
        return np.zeros(block.shape), np.float32(0)
    y = np.clip(block * np.float32(top / a), -top, top).astype(np.float64)
    return (np.rint(y) if code == "int8" else nearest_e4m3(y)), np.float32(a / top)


def places(rows, d):
    """Places of element (row, dim) among a block's bytes: of keys, of values."""
    k, v = np.zeros((rows, d), np.int64), np.zeros((rows, d), np.int64)
    for j in range(rows):
        a, b, m = j // 32, j // 16 % 2, j % 16
        g, r = j // 4 % 4, j % 4
        for i in range(d):
            if d == 32:
                k[j, i] = ((a * 4 + i // 8) * 16 + m) * 16 + b * 8 + i % 8
            else:
                k[j, i] = ((((a * 2 + b) * (d // 64) + i // 64) * 4 + i // 16 % 4) * 16 + m) * 16 + i % 16
            v[j, i] = ((((a * (d // 32) + i // 32) * 4 + g) * 16 + i % 16) * 2 + i // 16 % 2) * 8 + b * 4 + r
    return k, v


def to_bytes(codes, code):
    if code == "int8":
        return (codes + 128).astype(np.uint8)
    table = {float(x): i for i, x in enumerate(e4m3_value(np.arange(127)))}
    flat = [table[abs(float(c))] | (128 if c < 0 else 0) for c in codes.reshape(-1)]
    return np.array(flat, np.uint8).reshape(codes.shape)


def from_bytes(raw, code):
    return raw.astype(np.float64) - 128 if code == "int8" else e4m3_value(raw)


def page_values(data, scale, rows, d, code):
    """(keys, values) [...][rows][d] of pages' bytes [...][2][rows d] and scales [...][2]."""
    pk, pv = places(rows, d)
    x = [from_bytes(np.asarray(data)[..., i, :], code)[..., p] * np.asarray(scale, np.float64)[..., i, None, None]
         for i, p in ((0, pk), (1, pv))]
    return x[0], x[1]


class Sequences:
    """The batch's sequences: tables, lengths, refs, tails and pages as the operators leave them."""

    def __init__(self, table, length, refs, page_rows):
        self.table, self.length, self.refs = (np.array(x, np.int64) for x in (table, length, refs))
        self.rows = page_rows

    def _serve(self, need):
        """Pages for need[b] >= 0 (-1: not asked): lowest free ones, slots in order."""
        free, first, out = [p for p in range(len(self.refs)) if self.refs[p] == 0], 0, []
        for n in need:
            ok = n >= 0 and (n == 0 or first + n <= len(free))
            out.append(free[first:first + n] if ok else None)
            first += max(n, 0)
        return out

    def _put(self, b, col, ids):
        for i, p in enumerate(ids):
            self.table[b, col + i] = p
            self.refs[p] = 1

    def take(self, count):
        need, cols = [], self.table.shape[1]
        for b, n in enumerate(count):
            start = max(self.length[b], 0)
            need.append(n if n >= 0 and start % self.rows == 0 and start // self.rows + n <= cols else -1)
        got = []
        for b, ids in enumerate(self._serve(need)):
            got.append(-1 if ids is None else len(ids))
            if ids is not None:
                start = max(self.length[b], 0)
                self._put(b, start // self.rows, ids)
                self.length[b] = start + len(ids) * self.rows
        return got

    def commit(self, path, path_len, n_new, window=0, sinks=0):
        """(full, moves): moves are (slot, position, new row), and self.filled (slot, column, page)."""
        rows, cols, kept, need = self.rows, self.table.shape[1], [], []
        for b, n in enumerate(self.length):
            good = 0
            for t in path[b][:max(path_len[b], 0)]:
                if not 0 <= t < n_new:
                    break
                good += 1
            kept.append(good)
            need.append((n + good) // rows - n // rows if n >= 0 and (n + good) // rows <= cols else -1)
        full, moves, self.filled = [], [], []
        served = self._serve(need)
        for b, ids in enumerate(served):
            n = self.length[b]
            full.append(0 if n < 0 else -1 if ids is None else len(ids))
            if n < 0 or ids is None:
                continue
            self._put(b, n // rows, ids)
            self.filled += [(b, n // rows + i, p) for i, p in enumerate(ids)]
            moves += [(b, n + i, path[b][i]) for i in range(kept[b])]
            self.length[b] = n + kept[b]
        if window:
            for b, ids in enumerate(served):
                if ids is None or self.length[b] < 0:
                    continue
                for c in range(cols):
                    p = self.table[b, c]
                    if c * rows >= sinks and (c + 1) * rows - 1 <= self.length[b] - window and p >= 0:
                        self.table[b, c] = -1
                        self.refs[p] -= 1
        return full, moves

    def fork(self, parents):
        copied = []
        for b, s in enumerate(parents):
            if s == b:
                continue
            kept = 0 <= s < len(parents) and parents[s] == s
            for c in range(self.table.shape[1]):
                now = self.table[s, c] if kept else -1
                for p, by in ((self.table[b, c], -1), (now, 1)):
                    if 0 <= p < len(self.refs):
                        self.refs[p] += by
                self.table[b, c] = now
            self.length[b] = self.length[s] if kept else -1
            if kept:
                copied.append((b, s))
        return copied

    def compact(self):
        """(pages in use, {from: to})"""
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        u = len(used)
        holes = [p for p in range(u) if self.refs[p] == 0]
        moves = dict(zip([p for p in used if p >= u], holes))
        for a, b in moves.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for b in range(self.table.shape[0]):
            for c in range(self.table.shape[1]):
                self.table[b, c] = moves.get(int(self.table[b, c]), self.table[b, c])
        return u, moves


def attention(q, table, length, pages, tails, fresh, rows, anc=None, window=0, sinks=0, scale=None):
    """(out, lse, S, vmax) in 64 bits.  q [B][T][H][D]; pages (keys, values) [P][G][rows][D]; tails
    [B][G][R][D]; fresh [B][T][G][D].  S is the largest sum of |q_i k_i| |scale| over seen rows."""
    b, t, h, d = q.shape
    g, ring, n_page = tails[0].shape[1], tails[0].shape[2], len(pages[0])
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, lse, big, vmax = np.zeros(q.shape), np.full((b, t, h), -np.inf), 0.0, 0.0
    for i in range(b):
        n = int(length[i])
        if n < 0:
            continue
        for j in range(t):
            mask = (2 << j) - 1 if anc is None else int(anc[i][j]) & ((1 << t) - 1)
            last = n + (j if anc is None else max(bin(mask).count("1") - 1, 0))
            where = []
            for p in range(n):
                if window and not (p > last - window or p < sinks):
                    continue
                if p < n // rows * rows:
                    if p // rows < table.shape[1] and 0 <= table[i, p // rows] < n_page:
                        where.append((0, table[i, p // rows], p % rows))
                else:
                    where.append((1, i, p % ring))
            where += [(2, i, x) for x in range(t) if mask >> x & 1]
            if not where:
                continue
            for kv in range(g):
                k, v = (np.stack([pages[w][a, kv, r] if s == 0 else tails[w][a, kv, r] if s == 1 else fresh[w][a, r, kv]
                                  for s, a, r in where]) for w in (0, 1))
                heads = slice(kv * (h // g), (kv + 1) * (h // g))
                x = q[i, j, heads] @ k.T * scale
                m = x.max(1, keepdims=True)
                e = np.exp(x - m)
                out[i, j, heads] = e @ v / e.sum(1, keepdims=True)
                lse[i, j, heads] = m[:, 0] + np.log(e.sum(1))
                big = max(big, (np.abs(q[i, j, heads]) @ np.abs(k).T).max() * abs(scale))
                vmax = max(vmax, np.abs(v).max())
    return out, lse, big, vmax
