"""Block tables, slot maps and free lists as plain Python: one sequence, one block, one entry at a time."""


class Caches:
    def __init__(self, pools, batch, max_blocks, page, free):
        """free: the pools' free blocks, the next one to be taken last."""
        self.table = [[[] for _ in range(batch)] for _ in range(pools)]
        self.free = [list(f) for f in free]
        self.pools, self.batch, self.max_blocks, self.page = pools, batch, max_blocks, page

    def plan(self, length, cached, pool=None, max_tokens=1 << 30):
        """order, place, pool_start, token_start, and per entry (slot, position, sequence)."""
        batch = len(length)
        pool = [0] * batch if pool is None else [int(g) for g in pool]
        part = [g if 0 <= g < self.pools else self.pools for g in pool]
        order = [b for g in range(self.pools + 1) for b in range(batch) if part[b] == g]
        where = {b: i for i, b in enumerate(order)}
        place = [where[b] for b in range(batch)]
        pool_start = [sum(p < g for p in part) for g in range(self.pools + 1)]
        token_start, entries, short = [0], [], set()
        for b in order:
            g = part[b]
            if g == self.pools:
                token_start.append(token_start[-1])
                continue
            table, have, want = self.table[g][b], int(cached[g][b]), int(length[b])
            if have < 0 or want < 0 or have > len(table) * self.page or want > self.max_blocks * self.page or want <= have:
                token_start.append(token_start[-1])
                continue
            need = max(0, -(-want // self.page) - len(table))
            if need and (g in short or need > len(self.free[g])):
                short.add(g)
            fits = token_start[-1] + want - have <= max_tokens
            planned = fits and not (need and g in short)
            if planned:
                table += [self.free[g].pop() for _ in range(need)]
            elif need:
                short.add(g)
            for position in range(have, want):
                slot = table[position // self.page] * self.page + position % self.page if planned else -1
                entries.append((slot, position, b))
            token_start.append(token_start[-1] + want - have)
        return order, place, pool_start, token_start, entries[:max_tokens]

    def release(self, keep):
        for g in range(self.pools):
            back = []
            for b in range(len(keep[g])):
                if keep[g][b] >= 0:
                    stay = -(-int(keep[g][b]) // self.page)
                    back += self.table[g][b][stay:]
                    del self.table[g][b][stay:]
            self.free[g] += back[::-1]
