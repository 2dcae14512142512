"""A CPU model of the global addresses that the 8-bit cache's kernels form (no GPU): for
seeded random descriptors, with the partitions, the item count and the workspace from
the library's own plan, every entry of the block tables, row, cache tile, partial state and
work-order slot that a work item touches lies inside its buffer; every block is folded and
every output row and state written exactly once; and the wide kernel's buffers are
never written while they are read.  The ranking by which workgroups find their items is
restated step by step (histogram, scan, ballots) against a sort."""
import numpy as np
import pytest

import paper_2405_11143_amd as pda

WAVE, WAVES, AT_ONCE, PICK_ITEMS, PICK_PAIRS = 64, 4, 768, 2304, 256


def inverse(G):
    return (65536 + G - 1) // G


def test_the_group_inverse_is_exact():
    for G in range(1, 17):
        for r in range(16 + 128):  # m0 + x of the wide kernel; up to 31 in the decode kernel
            assert r * inverse(G) >> 16 == r // G


# ------------------------------------------------------------------ attention --

def random_step(rng):
    G = int(rng.choice([1, 2, 3, 4, 5, 7, 8, 16]))
    Hkv = int(rng.randint(1, 5))
    n = int(rng.choice([1, 1, 2, 3, 5, 8, 9, 13, 32, 33, 47, 70, 150]))
    B = int(rng.randint(1, 6))
    D = int(rng.choice([64, 128]))
    tp = int(rng.choice([0, 16, 48, 80, 256, 4096]))
    longest = int(rng.choice([1, 16, 17, 70, 300, 1500, 5000] if tp != 16 else [1, 16, 17, 70, 300]))
    lens = rng.randint(-2, longest + 40, B)  # (clamped)
    lens[0] = longest
    mbps = -(-longest // 16) + int(rng.randint(0, 3))
    return dict(B=B, G=G, Hkv=Hkv, Hq=G * Hkv, n=n, D=D, lens=lens, longest=longest, mbps=mbps, tp=tp)


def plan(c):
    info = pda.pda_plan_fp8(pda.make_problem(c["B"], c["Hq"], c["Hkv"], c["D"], 999, c["mbps"], c["longest"], c["tp"],
                                             num_query_tokens=c["n"]))
    rows = c["n"] * c["G"]
    item_rows = 16 if rows <= 16 else 32 if rows <= 32 else 64 if rows <= 64 else 128
    tiles, P = -(-rows // item_rows), info["num_partitions"]
    items = P * c["B"] * c["Hkv"] * tiles
    slots = c["B"] * c["n"] * c["Hq"] * P if P > 1 else 0
    assert info["workspace_bytes"] == 4 * slots * (c["D"] + 2) + 4 * items  # the carving below is the library's
    assert P * info["partition_tokens"] >= c["longest"]
    return dict(Tp=info["partition_tokens"], P=P, tiles=tiles, item_rows=item_rows, items=items, slots=slots,
                bytes=info["workspace_bytes"])


class Written:
    """What a step writes: final rows, zero rows and partial states, each at most once."""

    def __init__(self, c, pl):
        self.c, self.pl = c, pl
        self.final = np.zeros(c["B"] * c["n"] * c["Hq"], int)
        self.state = np.zeros(max(pl["slots"], 1), int)

    def row(self, row, parts, p):
        D = self.c["D"]
        assert 0 <= row < len(self.final)
        if parts == 1:
            self.final[row] += 1
            return
        slot = row * self.pl["P"] + p
        assert 0 <= slot < self.pl["slots"] and p < self.pl["P"]
        for end in ((slot + 1) * D, self.pl["slots"] * D + slot + 1, self.pl["slots"] * (D + 1) + slot + 1):
            assert 4 * end <= self.pl["bytes"]  # its output, its maximum, its sum
        self.state[slot] += 1

    def check(self):
        """Every row is either written by pass 1 or merged from states that are all there."""
        c, pl = self.c, self.pl
        want_final, want_state = np.zeros_like(self.final), np.zeros_like(self.state)
        for b in range(c["B"]):
            L = min(max(int(c["lens"][b]), 0), c["longest"])
            for i in range(c["n"]):
                limit = L - c["n"] + 1 + i
                parts = -(-limit // pl["Tp"]) if limit > 0 else 0
                for h in range(c["Hq"]):
                    row = (b * c["n"] + i) * c["Hq"] + h
                    if parts <= 1:
                        want_final[row] = 1
                    else:
                        want_state[row * pl["P"]:row * pl["P"] + parts] = 1
        assert np.array_equal(self.final, want_final) and np.array_equal(self.state, want_state)


def out_row(c, b, g, r):
    i = r * inverse(c["G"]) >> 16
    return (b * c["n"] + i) * c["Hq"] + g * c["G"] + r - i * c["G"], i


def narrow_item(c, pl, wr, b, g, p):
    n, Tp, rows = c["n"], pl["Tp"], c["n"] * c["G"]
    L = min(max(int(c["lens"][b]), 0), c["longest"])
    limit_of = lambda r: L - n + 1 + out_row(c, b, g, r)[1]
    if p == 0 and L - n + 1 <= 0:
        for r in range(rows):
            if limit_of(r) <= 0:
                wr.row(out_row(c, b, g, r)[0], 1, 0)
    if L <= p * Tp:
        return
    for lane in range(16 * (1 if rows <= 16 else 2)):  # the query rows that lanes load
        assert 0 <= out_row(c, b, g, min(lane, rows - 1))[0] < c["B"] * n * c["Hq"]
    j0, j1 = p * Tp // 16, -(-min(L, (p + 1) * Tp) // 16)
    folded = np.zeros(j1 - j0, int)
    per = -(-(j1 - j0) // WAVES)
    for w in range(WAVES):
        wj0 = min(j1, j0 + w * per)
        wj1 = min(j1, wj0 + per)
        for jc in range(wj0, wj1, WAVE):
            cn = min(WAVE, wj1 - jc)
            assert jc + cn <= c["mbps"] and (jc + cn - 1) * 16 < L  # the entries read: all of them the context's
            held = {}

            def load(which, i):
                for x in range(2):
                    assert 0 <= min(i + x, cn - 1) < cn
                held[which] = [i + x if i + x < cn else None for x in range(2)]

            def fold(which):
                for x in held[which]:
                    if x is not None:
                        folded[jc + x - j0] += 1

            load(0, 0)
            for i in range(0, cn, 4):
                load(1, i + 2)
                fold(0)
                if i + 2 >= cn:
                    break
                load(0, i + 4)
                fold(1)
    assert (folded == 1).all()
    for r in range(rows):
        parts = -(-limit_of(r) // Tp) if limit_of(r) > 0 else 0
        if p < parts:
            wr.row(out_row(c, b, g, r)[0], parts, p)


def wide_item(c, pl, wr, item):
    n, G, Tp, tiles = c["n"], c["G"], pl["Tp"], pl["tiles"]
    W = pl["item_rows"] // 32
    HC = c["Hkv"] * tiles
    gc, b, p = item % HC, item // HC % c["B"], item // (HC * c["B"])
    g, rg = gc // tiles, gc % tiles
    L = min(max(int(c["lens"][b]), 0), c["longest"])
    wg0 = rg * W * 32
    rows = min(W * 32, n * G - wg0)
    i0 = wg0 // G
    m0 = wg0 - i0 * G
    assert rows > 0 and m0 < 16

    def at(x):
        i = (m0 + x) * inverse(G) >> 16
        return (b * n + i0 + i) * c["Hq"] + g * G + m0 + x - i * G, L - n + 1 + i0 + i

    if p == 0 and at(0)[1] <= 0:
        for x in range(rows):
            if at(x)[1] <= 0:
                wr.row(at(x)[0], 1, 0)
    t_pe = min((p + 1) * Tp, L)
    last = at(rows - 1)[1]
    if last <= p * Tp:
        return
    for w in range(W):
        for lane in range(32):
            assert 0 <= at(min(w * 32 + lane, rows - 1))[0] < c["B"] * n * c["Hq"]
    window, buffers, ahead = (1024, 3, True) if W == 4 else (256, 2, False)
    J0, J1 = p * Tp // 16, -(-min(last, t_pe) // 16)
    folded = np.zeros(J1 - J0, int)
    for jw in range(J0, J1, window):
        jwe = min(J1, jw + window)
        nsteps = -(-(jwe - jw) // 2)
        n_ids = -(-nsteps * 2 // WAVE) * WAVE
        assert n_ids <= window
        for x in (0, n_ids - 1):
            assert jw <= min(jw + x, jwe - 1) < min(c["mbps"], -(-L // 16))
        for step in wide_schedule(nsteps, buffers, ahead, n_ids):
            for blk in (2 * step, 2 * step + 1):
                if jw + blk < jwe:
                    folded[jw + blk - J0] += 1
    assert (folded == 1).all()
    for x in range(rows):
        row, limit = at(x)
        parts = -(-limit // Tp) if limit > 0 else 0
        if p < parts:
            wr.row(row, parts, p)


def wide_schedule(nsteps, buffers, ahead, n_ids):
    """The steps that a window folds, in order.  Checks that each finds its own tiles in its buffer (and, with scores
    formed ahead, the next one's), written before a barrier that comes before the read, with no write in between."""
    staged = buffers - 1
    epoch, wrote, reads = 0, {}, {}  # a buffer's (step, epoch of the write); epochs in which it was read
    raw, ids_from = None, None
    folds = []

    def issue(step):
        nonlocal raw, ids_from
        j = 2 * step
        if j % WAVE == 0:
            assert j + WAVE <= n_ids
            ids_from = j
        assert ids_from == j // WAVE * WAVE and j % WAVE + 1 < WAVE
        raw = step

    def commit(buffer, step):
        assert raw == step
        assert epoch not in reads.get(buffer, ()), "written while it may be read"
        wrote[buffer] = (step, epoch)

    def read(buffer, step):
        at, e = wrote[buffer]
        assert at == step and e < epoch, "not there yet"
        reads.setdefault(buffer, set()).add(epoch)

    for x in range(min(staged, nsteps)):
        issue(x)
        commit(x, x)
    if staged < nsteps:
        issue(staged)
    epoch += 1
    if ahead:
        read(0, 0)
    for step in range(nsteps):
        B = step % buffers
        if step > 0:
            epoch += 1
        if step + staged < nsteps:
            commit((B + staged) % buffers, step + staged)
        if step + buffers < nsteps:
            issue(step + buffers)
        read(B, step)
        folds.append(step)
        if ahead and step + 1 < nsteps:
            read((B + 1) % buffers, step + 1)
        elif ahead:  # (the scores of a step that is not there: not used; the buffer is not being written)
            reads.setdefault((B + 1) % buffers, set()).add(epoch)
    return folds


@pytest.mark.parametrize("seed", range(12))
def test_attention_steps(seed):
    rng = np.random.RandomState(seed)
    for _ in range(12):
        c = random_step(rng)
        pl = plan(c)
        wr = Written(c, pl)
        for item in range(pl["items"]):
            if pl["item_rows"] <= 32:
                H = c["Hkv"]
                assert pl["tiles"] == 1
                narrow_item(c, pl, wr, item // H % c["B"], item % H, item // (H * c["B"]))
            else:
                wide_item(c, pl, wr, item)
        wr.check()


def test_wide_schedules_of_every_length():
    for buffers, ahead, window in ((3, True, 1024), (2, False, 256)):
        for nsteps in list(range(1, 70)) + [window // 2 - 1, window // 2]:
            assert wide_schedule(nsteps, buffers, ahead, -(-2 * nsteps // WAVE) * WAVE) == list(range(nsteps))


# ------------------------------------------------------- items that are picked --

def pick_pair(lens, B, P, Tp, longest, pos):
    """pick_pair of pda_fp8_decode.hip, lane by lane."""
    threads = np.arange(256)
    cls = np.full(256, -1)
    for t in threads[:B * P]:
        p, b = divmod(int(t), B)
        L = min(max(int(lens[b]), 0), longest)
        tok = min(max(L - p * Tp, 0), Tp)
        cls[t] = 255 - min((tok + 15) // 16, 255)
    count = np.zeros(256, int)
    np.add.at(count, cls[cls >= 0], 1)
    found = []
    sums = count.reshape(64, 4).sum(1)
    before = sums.copy()
    o = 1
    while o < 64:
        before = before + np.where(np.arange(64) >= o, np.roll(before, o), 0)
        o *= 2
    before = before - sums
    for lane in range(64):
        at = before[lane]
        for e in range(4):
            v = count[4 * lane + e]
            if at <= pos < at + v:
                found.append((4 * lane + e, pos - at))
            at += v
    assert len(found) == 1
    c, place = found[0]
    hits = (cls == c).reshape(4, 64)
    pair = []
    for w in range(4):
        left = place - hits[:w].sum()
        for lane in range(64):
            if hits[w, lane] and left == hits[w, :lane].sum():
                pair.append(64 * w + lane)
    assert len(pair) == 1
    return pair[0]


def test_picked_pairs_are_the_sorted_ones():
    rng = np.random.RandomState(0)
    for trial in range(25):
        P = int(rng.randint(1, 9))
        B = int(rng.randint(1, 256 // P + 1)) if trial else 256 // P
        Tp = 16 * int(rng.choice([1, 5, 40, 300]))  # (past 255 blocks: one class)
        longest = P * Tp
        lens = rng.randint(-5, longest + 30, B)
        size = []
        for x in range(B * P):
            p, b = divmod(x, B)
            size.append(min((min(max(min(max(lens[b], 0), longest) - p * Tp, 0), Tp) + 15) // 16, 255))
        order = sorted(range(B * P), key=lambda x: (-size[x], x))
        assert [pick_pair(lens, B, P, Tp, longest, pos) for pos in range(B * P)] == order


# -------------------------------------------------------------- append and read --

def share(interleaved, R, D, u):
    shares = (D + 15) // 16
    if interleaved or R == 0:
        d0, d1 = 8 * u, 8 * (u + shares)
        return d0, d1, 2 if d1 < R else 1 if d0 < R else 0
    if u < R // 16:
        return 8 * u, R // 2 + 8 * u, 2
    d0 = R + 8 * (u - R // 16)
    return d0, d0 + 8 * (shares - R // 16), 0


def turns_read(interleaved, R, w):
    """Indices of the cosines that a share reads."""
    d0, d1, turned = w
    if not turned:
        return []
    if interleaved:
        return list(range(d0 // 2, d0 // 2 + 4)) + (list(range(d1 // 2, d1 // 2 + 4)) if turned == 2 else [])
    return list(range(d0, d0 + 8))


@pytest.mark.parametrize("seed", range(8))
def test_append(seed):
    rng = np.random.RandomState(seed)
    for _ in range(6):
        D = int(rng.choice([64, 128]))
        Hkv, Hq, with_q = int(rng.randint(1, 5)), 0, rng.rand() < 0.6
        Hq = Hkv * int(rng.randint(1, 9))
        n, B = int(rng.choice([1, 2, 3, 4, 5, 9, 23])), int(rng.randint(1, 4))
        R = 16 * int(rng.randint(0, D // 16 + 1)) if not with_q else 16 * int(rng.randint(1, D // 16 + 1))
        inter, NB = bool(rng.randint(2)), 50
        longest = int(rng.choice([1, 16, 40, 100]))
        mbps = -(-longest // 16)
        lens = rng.randint(-1, longest + 5, B)
        U, nq = D // 16, Hq if with_q else 0
        units = (nq + 2 * Hkv) * U
        for tokens in ([1] if n == 1 else [2, 4]):  # both of the kernel's, whichever a batch of this size would take
            every = tokens * units
            trips = -(-every // 256)
            threads = min(256, -(-(-(-every // trips)) // 64) * 64)
            assert threads % U == 0 and 0 < threads <= 256
            rows = nq + 2 * Hkv
            groups = (n - 1) // tokens + 1
            seen = set()
            for x in range(B * groups):
                b, i0 = x // groups, x % groups * tokens
                L = min(max(int(lens[b]), 0), longest)
                t0 = L - n + i0
                first, end = max(-t0, 0), min(tokens, n - i0)
                if first >= end:
                    continue
                assert end * (R // 2) <= tokens * (D // 2)  # turns
                for tr in range(threads // U):  # a row's U threads together
                    i, row = first, tr
                    while row >= rows:
                        row, i = row - rows, i + 1
                    while i < end:
                        which = 0 if row < nq else 1 if row < nq + Hkv else 2
                        h = row if which == 0 else row - nq if which == 1 else row - nq - Hkv
                        heads = Hq if which == 0 else Hkv
                        token = b * n + i0 + i
                        t = t0 + i
                        assert 0 <= t < L and 0 <= token < B * n and 0 <= h < heads
                        assert t // 16 < mbps
                        key = (which, token, h)
                        assert key not in seen
                        seen.add(key)
                        for u in range(U):
                            w = share(inter, R if which < 2 else 0, D, u)
                            assert w[0] + 8 <= D and w[1] + 8 <= D
                            assert all(0 <= z < R // 2 for z in turns_read(inter, R, w)) or which == 2
                            if which:
                                page, o = NB - 1, t % 16  # the last block: the largest offsets
                                tile = page * Hkv + h
                                for d in w[:2]:
                                    off = ((d // 64 * 4 + d // 8 % 4) * 16 + o) * 16 + d // 32 % 2 * 8 if which == 1 else \
                                        (((o // 2 % 2) * 4 + o // 4) * (D // 8) + d // 8) * 16 + o % 2 * 8
                                    assert tile * 16 * D + off + 8 <= NB * Hkv * 16 * D
                                assert tile * 32 + (0 if which == 1 else 16) + o < NB * Hkv * 32
                        row += threads // U
                        while row >= rows:
                            row, i = row - rows, i + 1
            want = {(which, b * n + i, h) for b in range(B) for i in range(n) if min(max(int(lens[b]), 0), longest) - n + i >= 0
                    for which in range(3) for h in range(nq if which == 0 else Hkv)}
            assert seen == want


@pytest.mark.parametrize("D", [64, 128])
def test_read(D):
    rng = np.random.RandomState(D)
    P = D // 8
    heads_at_once = 256 // (P * 16)
    assert heads_at_once >= 1
    for _ in range(40):
        B, Hkv = int(rng.randint(1, 5)), int(rng.randint(1, 6))
        longest = int(rng.choice([1, 16, 50, 90]))
        lens, first = rng.randint(-1, longest + 9, B), rng.randint(-20, longest + 10, B)
        start = np.cumsum(np.concatenate([[rng.randint(0, 3)], rng.randint(0, longest + 5, B)]))
        num_rows = int(rng.randint(0, start[-1] + 4))
        written = np.zeros(num_rows, int)
        blocks = -(-longest // 16)
        for bj in range(B * blocks):
            b, j = divmod(bj, blocks)
            L = min(max(int(lens[b]), 0), longest)
            row0 = int(start[b])
            end = min(L, int(first[b]) + int(start[b + 1]) - row0)
            lo, hi = max(16 * j, int(first[b])), min(16 * (j + 1), end)
            for o in range(16):
                t = 16 * j + o
                row = row0 + t - int(first[b])
                if t < lo or t >= hi or row < 0 or row >= num_rows:
                    continue
                assert 0 <= t < L and row0 <= row < start[b + 1]
                written[row] += 1
        want = np.zeros(num_rows, int)
        for b in range(B):
            for row in range(int(start[b]), min(int(start[b + 1]), num_rows)):
                want[row] = 0 <= first[b] + row - start[b] < min(max(int(lens[b]), 0), longest)
        assert np.array_equal(written, want)
        heads = sorted(g for sub in range(heads_at_once) for g in range(sub, Hkv, heads_at_once))
        assert heads == list(range(Hkv))
    for tid in range(256):  # a thread's 8 codes lie in their tile, its 16 bytes in the row
        c, o = tid % P, tid // P % 16
        assert ((c // 8 * 4 + c % 4) * 16 + o) * 16 + c // 4 % 2 * 8 + 8 <= 16 * D
        assert (((o // 2 % 2) * 4 + o // 4) * P + c) * 16 + o % 2 * 8 + 8 <= 16 * D
        assert tid // (P * 16) < heads_at_once


def test_rotary_rows():
    rng = np.random.RandomState(1)
    for _ in range(300):
        D = 8 * int(rng.randint(2, 65))
        R = 16 * int(rng.randint(1, D // 16 + 1))
        inter = bool(rng.randint(2))
        heads = int(rng.randint(1, 50))
        shares = (D + 15) // 16
        units = heads * shares
        trips = -(-units // 256)
        threads = min(256, -(-(-(-units // trips)) // 64) * 64)
        at_once = threads // shares
        assert at_once >= 1 and R // 2 <= 256
        seen = sorted(h for fr in range(at_once) for h in range(fr, heads, at_once))
        assert seen == list(range(heads))
        for u in range(shares):
            w = share(inter, R, D, u)
            assert all(0 <= z < R // 2 for z in turns_read(inter, R, w))
            assert w[0] + 8 <= D and (w[1] >= D or w[1] + 8 <= D)
            assert w[2] < 2 or w[1] < D
