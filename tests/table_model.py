"""What tkv_table_append does to a page table, token by token with lists."""
import numpy as np

PAGE = 64


class Table:
    def __init__(self, n_seqs, max_pages, p2, p4, free2=None, free4=None):
        self.max_pages, self.pool, self.lead = max_pages, (p2, p4), (0, p2)
        self.free = [list(free2) if free2 is not None else list(range(p2))[::-1],
                     list(free4) if free4 is not None else list(range(p2, p2 + p4))[::-1]]
        self.pages = [([], []) for _ in range(n_seqs)]
        self.count = [[0, 0] for _ in range(n_seqs)]

    def append(self, keep, lens, tags, channel_keys=False, max_work=1 << 30):
        """keep: [n_seqs, 2] or None; returns dict of outputs, or the name of what stands in the way."""
        n = len(self.pages)
        lens, tags = [int(x) for x in lens], np.asarray(tags)
        if any(x < 0 for x in lens) or sum(lens) > tags.size or any(t not in (2, 4) for t in tags[:sum(lens)]):
            return "refused"
        pages, count, free = [(list(a), list(b)) for a, b in self.pages], [list(c) for c in self.count], [list(f) for f in self.free]
        for b in reversed(range(n)):
            for w in range(2):
                if keep is not None:
                    count[b][w] = min(count[b][w], int(keep[b][w]))
                    if count[b][w] < 0:
                        return "refused"
                while len(pages[b][w]) * PAGE >= count[b][w] + PAGE:
                    free[w].append(pages[b][w].pop())
        positions, slots = np.full(tags.size, -1, np.int32), np.full(tags.size, -1, np.int32)
        work, where, at = [], {}, 0
        indptr = [0]
        short = False
        for b in range(n):
            held = sum(count[b])
            mine = tags[at:at + lens[b]]
            if channel_keys and ((mine == 2).sum() % 32 or count[b][0] % 32):
                return "refused"
            for w, bits in ((0, 2), (1, 4)):
                for i in np.flatnonzero(mine == bits):
                    place = count[b][w]
                    if place == PAGE * len(pages[b][w]):
                        if not free[w]:
                            short = True
                            pages[b][w].append(-5)
                        else:
                            pages[b][w].append(free[w].pop())
                    page = pages[b][w][-1]
                    key = (b, w, place // PAGE)
                    if key not in where:
                        where[key] = len(work)
                        work.append((page, np.full(PAGE, -1, np.int32)))
                    work[where[key]][1][place % PAGE] = at + i
                    slots[at + i] = page * PAGE + place % PAGE
                    count[b][w] += 1
            positions[at:at + lens[b]] = held + np.arange(lens[b])
            at += lens[b]
            indptr.append(at)
        wide = any(len(a) + len(b) > self.max_pages for a, b in pages) or len(work) > max_work
        if short or wide:
            return "exhausted" if short and not wide else ("capacity" if wide and not short else "both")
        self.pages, self.count, self.free = pages, count, free
        return {"indptr": np.array(indptr, np.int32), "positions": positions, "slots": slots,
                "work_pages": np.array([p for p, _ in work], np.int32), "work_src": np.array([s for _, s in work], np.int32).reshape(-1, PAGE)}

    def rows(self):
        out = np.full((len(self.pages), self.max_pages), -1, np.int32)
        for b, (x, y) in enumerate(self.pages):
            out[b, :len(x) + len(y)] = x + y
        return out
