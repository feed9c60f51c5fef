"""Block tables of requests on the host: the same rules with lists, one page at a time."""
from collections import deque


class Pool:
    def __init__(self, prefixes, drafts, width, page, ring):
        self.B, self.K, self.W, self.P = prefixes, drafts, width, page
        self.rows = [[[-1] * width for _ in range(drafts)] for _ in range(prefixes)]
        self.held = [(0, 0)] * prefixes
        self.free = deque(ring)

    def sets(self, state, draft, chosen):
        whole, held = state
        return set(range(0 if draft == chosen else whole, held))

    def advance(self, length, chosen, room):
        """(shared_len, served) of every request; the rows, held and free pages are brought on."""
        plan = []
        for b in range(self.B):
            a = min(max(chosen[b], 0), self.K - 1)
            want = (length[b] // self.P, -(-(length[b] + room) // self.P)) if length[b] > 0 else (0, 0)
            long = want[1] > self.W
            if long:
                want = self.held[b]
            gives = takes = 0
            for k in range(self.K):
                old, new = self.sets(self.held[b], k, a), self.sets(want, k, a)
                gives, takes = gives + len(old - new), takes + len(new - old)
            plan.append([a, want, -1 if long else 1, gives, takes])
        free = len(self.free) + sum(max(g - t, 0) for _, _, _, g, t in plan)
        needed = 0
        for b, q in enumerate(plan):
            more = q[4] - q[3]
            if more > 0:
                needed += more
                if needed > free:
                    q[1], q[2] = self.held[b], 0
        for b, (a, want, served, _, _) in enumerate(plan):
            if served < 1:
                continue
            for k in [a] + [k for k in range(self.K) if k != a]:
                for i in sorted(self.sets(self.held[b], k, a) - self.sets(want, k, a)):
                    self.free.append(self.rows[b][k][i])
        taken = {}
        for b, (a, want, served, _, _) in enumerate(plan):
            if served < 1:
                continue
            for k in [a] + [k for k in range(self.K) if k != a]:
                for i in sorted(self.sets(want, k, a) - self.sets(self.held[b], k, a)):
                    taken[b, k, i] = self.free.popleft()
        for b, (a, want, served, _, _) in enumerate(plan):
            if served < 1:
                continue
            old = [list(r) for r in self.rows[b]]
            for k in range(self.K):
                for i in range(self.W):
                    if i >= want[1]:
                        page = -1
                    elif i < want[0] or k == a:              # the chosen draft's
                        page = taken.get((b, a, i), old[a][i])
                    else:
                        page = taken.get((b, k, i), old[k][i])
                    self.rows[b][k][i] = page
            self.held[b] = want
        return [self.held[b][0] * self.P for b in range(self.B)], [q[2] for q in plan]
