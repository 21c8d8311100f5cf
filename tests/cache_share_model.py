"""How the cache attention deals out the keys of long tables, worked out on the
host from the constants of csrc/ei_cache.hip: every wave's run of steps and the
lists of parts that the second kernel joins."""
import os
import re
from dataclasses import dataclass, field

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                      "paper_2606_09508_amd", "csrc", "ei_cache.hip")


def _constants():
    text = open(SOURCE).read()

    def number(name):
        return int(re.search(rf"constexpr int {name} = (\d+);", text).group(1))
    out = {n: number(n) for n in ("kRows", "kKeys", "kCus", "kItemCost", "kShareLeast", "kThreads",
                                  "kShortKeys")}
    out["kShareGroups"] = int(re.search(r"constexpr int kShareGroups = (\d+) \* kCus;",
                                        text).group(1)) * out["kCus"]
    out["elder_share"] = tuple(int(x) for x in re.search(
        r"constexpr int elder_share\(int rt\) \{ return rt == 1 \? (\d+) : (\d+); \}", text).groups())
    return out


C = _constants()
WAVES = C["kThreads"] // 64


@dataclass
class Plan:
    """lengths: tokens of each sequence, its new[s] ones included; cols: of the table."""
    lengths: list
    new: list
    hq: int
    hkv: int
    page_len: int
    cols: int
    features: set = field(default_factory=set)

    def __post_init__(self):
        G, S = self.hq // self.hkv, len(self.new)
        tokens = sum(self.new)
        ragged = len(set(self.new)) > 1
        self.rt = 2 if tokens * G > C["kRows"] * S else 1
        tile = C["kRows"] * self.rt
        slots = tokens * G // tile + S if ragged else S * -(-tokens // S * G // tile)
        keys = self.cols * self.page_len
        assert keys > C["kShortKeys"], "a short table: a workgroup per item"
        cost = keys // C["kKeys"] + C["kItemCost"]
        waves = -(-slots * self.hkv * cost // C["kShareLeast"])
        self.groups = min(-(-waves // WAVES), C["kShareGroups"])
        self.workers = self.groups * WAVES
        self.steps = [-(-min(n, keys) // C["kKeys"]) for n in self.lengths]
        self.tiles = [-(-n * G // tile) for n in self.new]
        self._deal()

    def _cost(self, s):
        return (self.steps[s] + C["kItemCost"]) * self.tiles[s] * self.hkv

    def _deal(self):
        self.total = sum(self._cost(s) for s in range(len(self.new)))
        self.even = -(-self.total // self.workers)
        whole0 = self.steps[0] + C["kItemCost"]
        whole = self.total == self.even * self.workers and self.even % whole0 == 0
        full = self.workers == C["kShareGroups"] * WAVES
        self.elders = (self.workers // 2 if full and self.even > C["kShareLeast"] and not whole
                       else 0)
        self.elder = self.even + self.even // C["elder_share"][self.rt - 1]
        self.per = (-(-(self.total - self.elders * self.elder) // self.elders) if self.elders
                    else max(self.even, C["kShareLeast"]))
        self.features |= {f"rt{self.rt}"} | ({"elders"} if self.elders else set())
        if whole and full and self.even > C["kShareLeast"]:
            self.features.add("whole items")
        if max(self.tiles) > 1:
            self.features.add("tiles")

    def bound(self, w):
        return min(w, self.elders) * self.elder + max(w - self.elders, 0) * self.per

    def owner(self, u):
        rest = u - self.elders * self.elder
        return u // self.elder if rest < 0 else self.elders + rest // self.per

    def _find(self, u):
        start = 0
        for s in range(len(self.new)):
            if start + self._cost(s) > u:
                return s, start
            start += self._cost(s)
        return len(self.new), start

    def _run(self, s, start, u, end):
        """(item, its steps st0 .. st1 - 1, first unit of the next item, none, full)."""
        cost, steps = C["kItemCost"], self.steps[s]
        whole = steps + cost
        at = (u - start) % whole
        to = min(whole, at + end - u)
        st0, st1 = max(at - cost, 0), max(to - cost, 0)
        none = to < whole if steps == 0 else st0 == st1
        return ((u - start) // whole, st0, st1, u - at + whole, none, st0 == 0 and st1 == steps)

    def check(self):
        """Walks the waves' runs: every step of every item is taken once, no place
        for a part is used twice, and each list names its item's parts in the order
        of their keys.  Sets features, the most steps of a run and the most parts
        of an item."""
        seen, place, order, lists = set(), {}, {}, {}
        self.most_steps = self.most_parts = 1

        def take(s, r, slot, w0, group, joint):
            item, st0, st1, nxt, _, full = r
            steps = range(st0, st1) if self.steps[s] else [-1]
            for x in steps:
                assert (s, item, x) not in seen, "a step twice"
                seen.add((s, item, x))
            self.most_steps = max(self.most_steps, -(-len(steps) // (WAVES if joint else 1)))
            if full:
                return
            assert slot < 2 * self.workers and slot not in place, "a part's place twice"
            place[slot] = (s, item)
            order.setdefault((s, item), []).append(slot)
            if st0 == 0:
                assert w0 not in lists, "two lists of a wave"
                lists[w0] = ((s, item), self._list(nxt, slot, w0, group, joint))

        for group in range(self.groups):
            g0 = self.bound(group * WAVES)
            g1 = min(self.bound((group + 1) * WAVES), self.total)
            if g0 >= g1:
                continue
            s, start = self._find(g0)
            r = self._run(s, start, g0, g1)
            if g1 <= r[3]:
                self.features.add("joint")
                if not r[4]:
                    take(s, r, 2 * group * WAVES, group * WAVES, group, True)
                continue
            for w in range(group * WAVES, (group + 1) * WAVES):
                u0, u1 = self.bound(w), min(self.bound(w + 1), self.total)
                if u0 >= u1:
                    continue
                s, start = self._find(u0)
                u = u0
                while u < u1:
                    if u >= start + self._cost(s):
                        start += self._cost(s)
                        s += 1
                        continue
                    r = self._run(s, start, u, u1)
                    slot = 2 * w + (0 if u == u0 else 1)
                    u = r[3]
                    if not r[4]:
                        take(s, r, slot, w, group, False)
        want = {(s, i, x) for s in range(len(self.new)) for i in range(self.tiles[s] * self.hkv)
                for x in (range(self.steps[s]) if self.steps[s] else [-1])}
        assert seen == want, "steps left out"
        for key, parts in lists.values():
            assert order.pop(key) == parts, "a list that is not the parts in order"
            self.most_parts = max(self.most_parts, len(parts))
        assert not order, "parts without a list"
        return self

    def _list(self, nxt, slot, w0, group, joint):
        last = self.owner(nxt - 1)
        last_group = last // WAVES
        last_end = min(self.bound((last_group + 1) * WAVES), self.total)
        n_waves = 1 if joint else min((group + 1) * WAVES - 1, last) - w0 + 1
        out = [slot] + [2 * (w0 + p) for p in range(1, n_waves)]
        if last_group > group:
            joint_last = last_end <= nxt
            between = range(group + 1, last_group + (1 if joint_last else 0))
            out += [2 * WAVES * g for g in between]
            if between:
                self.features.add("groups in a list")
            if not joint_last:
                out += [2 * w for w in range(last_group * WAVES, last + 1)]
                self.features.add("waves after groups")
        return out


def _spread(n, lo, hi):
    return [lo + (hi - lo) * ((i * 7919) % n) // max(n - 1, 1) for i in range(n)]


# Launches that fill the chip: what each is there for, and its sequences (held
# tokens, new ones), heads, page length and the table's columns past the longest.
LARGE = {
    "long sequences, each over many workgroups":
        ({"rt1", "elders", "joint", "groups in a list", "waves after groups"},
         [20000, 9000, 30000, 12345], [1] * 4, 32, 8, 64, 1),
    "ragged sequences, several items a wave and several waves an item":
        ({"rt1", "elders", "joint", "groups in a list", "waves after groups"},
         [0, 131, 8000] + _spread(37, 300, 6000), [1] * 40, 32, 8, 64, 1),
    "drafted tokens, 32 rows":
        ({"rt2", "elders", "joint", "groups in a list", "waves after groups"},
         [16384, 9000, 12345, 16000, 8191, 14000], [4] * 6, 64, 8, 128, 1),
    "56 rows in two tiles":
        ({"rt2", "tiles", "elders", "joint", "groups in a list", "waves after groups"},
         [4000, 9001, 3333, 64, 7000], [7] * 5, 64, 8, 64, 1),
    "sequences of a length, whole items":
        ({"rt1", "whole items"}, [699] * 256, [1] * 256, 16, 8, 64, 30),
    "twice as many, two whole items a wave":
        ({"rt1", "whole items"}, [199] * 512, [1] * 512, 8, 8, 64, 40),
    "sequences of a length, no whole items":
        ({"rt1", "elders"}, [699] * 300, [1] * 300, 16, 8, 64, 30),
    "counts from none to many":
        ({"rt2", "tiles", "elders", "waves after groups"},
         _spread(60, 1, 3000), [(0, 1, 5, 0, 40, 2)[i % 6] for i in range(60)], 16, 4, 64, 1),
    "one KV head, runs of the least length":
        ({"rt1", "joint", "groups in a list"}, [40000, 7, 20000], [1] * 3, 8, 1, 128, 1),
}


def large(name):
    want, held, new, hq, hkv, page_len, spare = LARGE[name]
    lengths = [a + b for a, b in zip(held, new)]
    cols = max(-(-n // page_len) for n in lengths) + spare
    return want, Plan(lengths, new, hq, hkv, page_len, cols)
