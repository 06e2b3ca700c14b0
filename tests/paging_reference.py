"""Plain forms of the operators on the cache's page lists and of the attentions
over shared and scored lists, for their tests.  Written from the definitions in
include/vsa2.h, one list entry, token and row after the other; nothing of the
library runs here."""
import math

import torch

import around_reference as ref

PAGE = ref.PAGE


def assign_reference(pool, table, refs, length, source=None, drop=None, count=None):
    """The state after the call, CPU tensors changed in place; returns room [batch]."""
    batch, m = table.shape
    pages = pool.shape[0]
    old = table.tolist()
    held = refs.tolist()
    is_page = lambda e: 0 <= e < pages
    new, keep, want = [], [], []
    for b in range(batch):
        src = b if source is None else int(source[b])
        n = min(max(int(length[b]), 0), PAGE * m) if 0 <= src < batch else 0
        first, num = (0, 0) if drop is None else (int(drop[b, 0]), max(int(drop[b, 1]), 0))
        row = [-1] * m
        for s in range(-(-n // PAGE)):
            at = s + (num if s >= first else 0)
            if at < m and is_page(old[src][at]):
                row[s] = old[src][at]
        new.append(row)
        keep.append(n)
        want.append(0 if count is None else max(int(count[b]), 0))
    for lists, one in ((old, -1), (new, 1)):
        for row in lists:
            for e in row:
                if is_page(e):
                    held[e] += one

    def take():
        for p in range(pages):
            if held[p] == 0:
                held[p] = 1
                return p
        return -1

    room = []
    for b in range(batch):
        n, row = keep[b], new[b]
        end = -(-n // PAGE)
        stuck = False
        if want[b] and n % PAGE:
            e = row[end - 1]
            if e < 0:
                stuck = True
            elif held[e] > 1:
                p = take()
                if p < 0:
                    stuck = True
                else:
                    pool[p] = pool[e]
                    held[e] -= 1
                    row[end - 1] = p
        last = min(m, -(-(n + want[b]) // PAGE))
        for s in range(end, last):
            row[s] = take()
        full = end
        while full < last and row[full] >= 0:
            full += 1
        room.append(0 if stuck else max(0, min(want[b], PAGE * full - n if full < last or last == m else want[b])))
    table.copy_(torch.tensor(new, dtype=table.dtype).view(batch, m))
    refs.copy_(torch.tensor(held, dtype=refs.dtype))
    return torch.tensor(room, dtype=torch.int32)


def copy_reference(src_pool, src_table, dst_pool, dst_table, index, start, count=None):
    """dst_pool (CPU, changed in place); every byte is read before any is written."""
    heads, D = dst_pool.shape[1], (dst_pool.shape[2] - 128) // 128
    source = src_pool.clone()
    batch, n = index.shape
    for b in range(batch):
        for i in range(n if count is None else min(max(int(count[b]), 0), n)):
            for h in range(heads):
                to = int(start[b]) + i
                page = ref.page_for(dst_table, b, h, to, dst_pool.shape[0])
                if page is None:
                    continue
                from_ = ref.page_for(src_table, b, h, int(index[b, i]), source.shape[0])
                a, z = ref.offsets(int(index[b, i]) % PAGE, D), ref.offsets(to % PAGE, D)
                for x in range(4):
                    dst_pool[page, h, z[x]] = (0 if x < 2 else 27) if from_ is None else source[from_, h, a[x]]
    return dst_pool


def rows_reference(pool, table, h, length, D):
    """{position: (k, v)} of KV head h's positions below length of one list [max_pages]."""
    lists = table[None] if table.dim() == 1 else table
    out = {}
    for pos in range(min(max(int(length), 0), lists.shape[-1] * PAGE)):
        x = ref.token_values(pool, lists, 0, h, pos, D)
        if x is not None:
            out[pos] = x
    return out


def softmax_reference(seen, q, score=lambda pos, x: x):
    """(o, lse, W = sum p |v|, largest sum |q k| / sqrt(D)) of one row over [(position, k, v)]."""
    D = q.shape[0]
    k, v = torch.stack([x[1] for x in seen]), torch.stack([x[2] for x in seen])
    pos = torch.tensor([x[0] for x in seen], dtype=torch.float64)
    y = score(pos, k @ q / math.sqrt(D))
    w = torch.softmax(y, 0)
    return w @ v, torch.logsumexp(y, 0), w @ v.abs(), (k.abs() @ q.abs()).max() / math.sqrt(D)


def shared_reference(prefix_pool, prefix_table, pool, table, q, prefix_length, length, count, causal):
    """(o, lse, W, largest sum |q k| / sqrt(D)) of q [batch, heads_q, n, D]."""
    batch, hq, n, D = q.shape
    heads, per = pool.shape[1], q.shape[0] // prefix_table.shape[0]
    group, most = hq // heads, table.shape[-1] * PAGE
    out = empty_rows(batch, hq, n, D)
    for b in range(batch):
        cnt = n if count is None else min(max(int(count[b]), 0), n)
        total = min(max(int(length[b]), 0), most)
        for h in range(heads):
            far = rows_reference(prefix_pool, prefix_table[b // per] if prefix_table.dim() == 2 else prefix_table[b // per, h:h + 1].expand(heads, -1)[None], h, int(prefix_length[b // per]), D)
            near = rows_reference(pool, table[b] if table.dim() == 2 else table[b, h:h + 1].expand(heads, -1)[None], h, total, D)
            for i in range(cnt):
                limit = total - (cnt - 1 - i) if causal else total
                seen = [(0, *x) for x in far.values()] + [(0, *x) for pos, x in near.items() if pos < limit]
                for y in range(h * group, (h + 1) * group):
                    put_row(out, b, y, i, seen, q[b, y, i].double())
    return out


def empty_rows(batch, hq, n, D):
    return (torch.zeros(batch, hq, n, D, dtype=torch.float64), torch.full((batch, hq, n), -math.inf, dtype=torch.float64),
            torch.zeros(batch, hq, n, D, dtype=torch.float64), torch.zeros(batch, hq, n, 1, dtype=torch.float64))


def put_row(out, b, y, i, seen, q, score=lambda pos, x: x):
    if seen:
        o, lse, w, big = softmax_reference(seen, q, score)
        out[0][b, y, i], out[1][b, y, i], out[2][b, y, i], out[3][b, y, i] = o, lse, w, big


def scored_reference(pool, table, q, length, count, causal, cap=0.0, slope=None, window=0, sink=0, span=None):
    """(o, lse, W, largest sum |q k| / sqrt(D)) of q [batch, heads_q, n, D]."""
    batch, hq, n, D = q.shape
    heads = pool.shape[1]
    group, most = hq // heads, table.shape[-1] * PAGE
    out = empty_rows(batch, hq, n, D)
    for b in range(batch):
        cnt = n if count is None else min(max(int(count[b]), 0), n)
        total = min(max(int(length[b]), 0), most)
        for h in range(heads):
            rows = rows_reference(pool, table[b] if table.dim() == 2 else table[b, h:h + 1].expand(heads, -1)[None], h, total, D)
            for i in range(cnt):
                at = total - cnt + i
                limit = at + 1 if causal else total

                def shown(pos):
                    near = (not window or pos > at - window) and (span is None or int(span[b, i, 0]) <= pos < int(span[b, i, 1]))
                    return pos < limit and (pos < sink or near)

                seen = [(pos, *x) for pos, x in rows.items() if shown(pos)]
                for y in range(h * group, (h + 1) * group):
                    def score(pos, x):
                        x = cap * torch.tanh(x / cap) if cap else x
                        return x if slope is None else x - slope[y].double() * (at - pos).abs()
                    put_row(out, b, y, i, seen, q[b, y, i].double(), score)
    return out
