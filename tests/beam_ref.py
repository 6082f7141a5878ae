"""Plain implementations that the beam-search and block-table kernels are tested against: scores in
64 bits, loops over rows, nothing of the library."""
import numpy as np

NORM_ALLOWED, NORM_FULL, NORM_NONE = 0, 1, 2


def log_sum_exp(x):
    """In 64 bits, from the definition; -inf for no terms."""
    if not len(x):
        return -np.inf
    if np.isnan(x).any():
        return np.nan
    m = x.max()
    if not np.isfinite(m):
        return m
    return m + np.log(np.exp(x - m).sum())


def row_scores(x, allowed, score, finished, eos, norm):
    """(tokens, scores in 64 bits) of one row's candidates."""
    if not score > -np.inf:
        return np.zeros(0, np.int64), np.zeros(0)
    if finished:
        return np.array([eos]), np.array([score], np.float64)
    tokens = np.flatnonzero(allowed)
    x = x.astype(np.float64)
    lse = 0.0 if norm == NORM_NONE else log_sum_exp(x[tokens] if norm == NORM_ALLOWED else x)
    with np.errstate(invalid="ignore"):
        s = score + (x[tokens] - lse)
    ok = s > -np.inf     # (False for NaN)
    return tokens[ok], s[ok]


def select(x, allowed, score, finished, eos, norm, n_req, n_out):
    """Per request the list of (score, beam, token), best first; x [rows, V] float, allowed bool."""
    K = len(x) // n_req
    V = x.shape[1]
    out = []
    for r in range(n_req):
        beams, tokens, scores = [], [], []
        for b in range(K):
            i = r * K + b
            t, s = row_scores(x[i], allowed[i], float(score[i]), bool(finished[i]), eos, norm)
            beams.append(np.full(len(t), b))
            tokens.append(t)
            scores.append(s)
        beams, tokens, scores = (np.concatenate(v) for v in (beams, tokens, scores))
        order = np.lexsort((beams * V + tokens, -scores))[:n_out]
        out.append([(scores[i], int(beams[i]), int(tokens[i])) for i in order])
    return out


def pack_mask(allowed):
    rows, V = allowed.shape
    W = (V + 31) // 32
    padded = np.zeros((rows, W * 32), bool)
    padded[:, :V] = allowed
    return np.packbits(padded, axis=1, bitorder="little").view(np.uint32)


def backtrack(token, parent):
    T, R, K = token.shape
    out = np.full((R, K, T), -1, np.int32)
    for r in range(R):
        for j in range(K):
            b, line = j, np.full(T, -1, np.int32)
            for t in range(T - 1, -1, -1):
                line[t] = token[t, r, b]
                b = parent[t, r, b]
                if not 0 <= b < K:
                    break
            else:
                out[r, j] = line
    return out


class Tables:
    """Block tables as lists, counts as a list; the lowest free block first, sequences in order."""

    def __init__(self, n_blocks, block, n_seq, max_blocks):
        self.n_blocks, self.block, self.max_blocks = n_blocks, block, max_blocks
        self.ref = [0] * n_blocks
        self.rows = [[] for _ in range(n_seq)]
        self.len = [0] * n_seq

    def free(self):
        return [b for b in range(self.n_blocks) if self.ref[b] == 0]

    def table(self):
        t = np.full((len(self.rows), self.max_blocks), -1, np.int32)
        for s, row in enumerate(self.rows):
            t[s, :len(row)] = row
        return t

    def blocks(self, n):
        return -(-n // self.block)

    def extend(self, new, n_tokens):
        n_free, free, want, at = len(self.free()), self.free(), 0, 0
        cu, slot, pos, seq, status = [0], [], [], [], []
        for s, n in enumerate(new):
            if n < 0 or self.len[s] + n > self.max_blocks * self.block:
                status.append(-1)
                cu.append(cu[-1])
                continue
            need = self.blocks(self.len[s] + n) - self.blocks(self.len[s])
            want += need
            at += n
            fits = n == 0 or (at <= n_tokens and (need == 0 or want <= n_free))
            status.append(0 if fits else -3)
            begin = cu[-1]
            cu.append(min(at, n_tokens))
            if fits:
                for _ in range(need):
                    b = free.pop(0)
                    self.rows[s].append(b)
                    self.ref[b] = 1
                self.len[s] += n
            for i in range(cu[-1] - begin):
                p = (self.len[s] - n if fits else self.len[s]) + i
                pos.append(p)
                seq.append(s)
                slot.append(self.rows[s][p // self.block] * self.block + p % self.block if fits else -1)
        rest = n_tokens - len(slot)
        return (np.array(cu, np.int32), np.array(slot + [-1] * rest, np.int64), np.array(pos + [-1] * rest, np.int32),
                np.array(seq + [-1] * rest, np.int32), np.array(status, np.int32))

    def shrink(self, keep):
        status = []
        for s, k in enumerate(keep):
            if not 0 <= k <= self.len[s]:
                status.append(-1)
                continue
            status.append(0)
            for b in self.rows[s][self.blocks(k):]:
                self.ref[b] -= 1
            del self.rows[s][self.blocks(k):]
            self.len[s] = int(k)
        return np.array(status, np.int32)

    def reorder(self, parent):
        """parent [R, K]; returns (copies [(src, dst, tokens)], copy_src, copy_dst, status)."""
        R, K = parent.shape
        rows, lens, wanted = [], [], []
        for r in range(R):
            seen = set()
            for j in range(K):
                p = parent[r, j]
                if not 0 <= p < K:
                    rows.append([])
                    lens.append(0)
                    continue
                rows.append(list(self.rows[r * K + p]))
                lens.append(self.len[r * K + p])
                if p in seen and lens[-1] % self.block:
                    wanted.append((len(rows) - 1, rows[-1].pop()))
                seen.add(p)
        for row in self.rows:
            for b in row:
                self.ref[b] -= 1
        for row in rows:
            for b in row:
                self.ref[b] += 1
        free, copies = self.free(), []
        n = R * K
        src, dst, status = (np.full(n, v, np.int32) for v in (-1, -1, 0))
        for i, b in wanted:
            if not free:
                status[i] = -3
                lens[i] = len(rows[i]) * self.block
                continue
            new = free.pop(0)
            rows[i].append(new)
            self.ref[new] = 1
            src[i], dst[i] = b, new
            copies.append((b, new, lens[i] % self.block))
        self.rows, self.len = rows, lens
        return copies, src, dst, status
