"""The hand-over of tiles between the warps of the tensor-core paged attention kernel, run as a model on the CPU under
random interleavings: every ring entry holds its tile until the last reader is done with it, a wait by parity never
comes two phases late, and every run ends."""
import random
import re
from pathlib import Path

import pytest

SRC = (Path(__file__).resolve().parents[1] / "paper_2502_06282_b200" / "csrc" / "jk_paged_tc.cu").read_text()


def sizes(NR):
    """Ring depths and groups as the kernel's configuration states them."""
    def choice(name):
        text = re.search(r"static constexpr int %s = ([^;]+);" % name, SRC).group(1)
        for cond, value in re.findall(r"NR == (\d+) \? (\d+) :", text):
            if NR == int(cond):
                return int(value)
        return int(text.split(":")[-1])

    rows = choice("RW")
    groups = NR // rows
    return dict(info=int(re.search(r"#define PT_INFO (\d+)", SRC).group(1)), k=choice("KST"), v=choice("VST"),
                groups=groups, turns=4 // groups)


class Barrier:
    def __init__(self, count):
        self.count, self.pending, self.done = count, count, 0

    def arrive(self):
        self.pending -= 1
        if self.pending == 0:
            self.pending, self.done = self.count, self.done + 1

    def phase(self, n):
        """Wait for completion n (0-based) by its parity: what the hardware answers, checked for aliasing."""
        assert self.done <= n + 1, "a wait that comes two phases late"
        return self.done > n


def run(NR, units, seed):
    """units: list of (8-bit tiles, bf16 tiles) of the segments of one CTA."""
    rng = random.Random(seed)
    z = sizes(NR)
    KST, VST, INFO, NRG, NP = z["k"], z["v"], z["info"], z["groups"], z["turns"]
    B = lambda n, c: [Barrier(c) for _ in range(n)]
    k_full, k_empty, v_full, v_empty = B(KST, 1), B(KST, 1), B(VST, 1), B(VST, 1)
    info_full, w_full, w_empty = B(INFO, 1), B(8, 1), B(2, 1)
    s_full, s_empty = [B(2, 1) for _ in range(NP)], [B(2, NRG) for _ in range(NP)]
    p_full, p_empty = B(NP, NRG), B(NP, 1)
    q_full = Barrier(4)
    meet = Barrier(4)                                    # the groups' barrier between units
    info, k_slot, v_slot, w_buf = [None] * INFO, [None] * KST, [None] * VST, [None] * 2
    s_buf = [[None] * 2 for _ in range(NP)]
    p_buf = [[None] * NRG for _ in range(NP)]
    o_sum = {}                                           # (unit, turn) -> tiles added
    loads, s_pipe, o_pipe = [], [], []                   # copies in any order; products of an issuer in order
    tiles = []                                           # (number, unit, tile, wide)
    for u, (n8, n16) in enumerate(units):
        for t in range(n8 + n16):
            tiles.append((len(tiles), u, t, t >= n8))
    finished = []

    def producer(is_k):
        n_slots, empty, full, slots = (KST, k_empty, k_full, k_slot) if is_k else (VST, v_empty, v_full, v_slot)
        for tc, u, t, wide in tiles:
            if tc >= n_slots:
                yield lambda: empty[tc % n_slots].phase(tc // n_slots - 1)
            slots[tc % n_slots] = None                   # the copy may write from here on
            loads.append((slots, tc % n_slots, tc, full[tc % n_slots]))
            if is_k:
                yield None
                info[tc % INFO] = tc
                info_full[tc % INFO].arrive()

    def s_issuer():
        n, unit = [0] * NP, -1
        for tc, u, t, wide in tiles:
            if u != unit:
                unit = u
                yield lambda: q_full.phase(u)
            turn = t % NP
            cg, buf = n[turn], n[turn] & 1
            if cg >= 2:
                yield lambda: s_empty[turn][buf].phase((cg >> 1) - 1)
            yield lambda: k_full[tc % KST].phase(tc // KST)
            s_pipe.append(("s", tc, turn, buf))
            n[turn] += 1

    def o_issuer():
        n, w_n = [0] * NP, 0
        for tc, u, t, wide in tiles:
            turn = t % NP
            yield lambda: w_full[tc & 7].phase(tc >> 3)
            yield lambda: p_full[turn].phase(n[turn])
            o_pipe.append(("o", tc, u, turn, wide, w_n & 1))
            if not wide:
                w_n += 1
            n[turn] += 1

    def converter():
        w_n = 0
        for tc, u, t, wide in tiles:
            yield lambda: info_full[tc % INFO].phase(tc // INFO)
            assert info[tc % INFO] == tc
            yield lambda: v_full[tc % VST].phase(tc // VST)
            assert v_slot[tc % VST] == tc
            if not wide:
                if w_n >= 2:
                    yield lambda: w_empty[w_n & 1].phase((w_n >> 1) - 1)
                w_buf[w_n & 1] = None
                yield None
                w_buf[w_n & 1] = tc
                w_n += 1
            assert info[tc % INFO] == tc
            w_full[tc & 7].arrive()
            if not wide:
                v_empty[tc % VST].arrive()

    def softmax(grp):
        rg, turn = grp % NRG, grp // NRG
        cnt = 0
        for u, (n8, n16) in enumerate(units):
            meet.arrive()
            yield lambda: meet.phase(2 * u)
            q_full.arrive()
            meet.arrive()
            yield lambda: meet.phase(2 * u + 1)
            for tc, tu, t, wide in tiles:
                if tu != u or t % NP != turn:
                    continue
                yield lambda: info_full[tc % INFO].phase(tc // INFO)
                assert info[tc % INFO] == tc
                yield lambda: s_full[turn][cnt & 1].phase(cnt >> 1)
                assert s_buf[turn][cnt & 1] == tc
                if cnt > 0:
                    yield lambda: p_empty[turn].phase(cnt - 1)
                p_buf[turn][rg] = None
                yield None
                assert info[tc % INFO] == tc and s_buf[turn][cnt & 1] == tc
                p_buf[turn][rg] = tc
                s_empty[turn][cnt & 1].arrive()
                p_full[turn].arrive()
                cnt += 1
            if cnt > 0:
                yield lambda: p_empty[turn].phase(cnt - 1)
            assert o_sum.get((u, turn), []) == [tc for tc, tu, t, _ in tiles if tu == u and t % NP == turn]
        finished.append(grp)

    def product(op):
        if op[0] == "s":
            _, tc, turn, buf = op
            assert k_slot[tc % KST] == tc
            s_buf[turn][buf] = tc
            k_empty[tc % KST].arrive()
            s_full[turn][buf].arrive()
        else:
            _, tc, u, turn, wide, buf = op
            assert p_buf[turn] == [tc] * NRG
            assert (v_slot[tc % VST] if wide else w_buf[buf]) == tc
            o_sum.setdefault((u, turn), []).append(tc)
            p_empty[turn].arrive()
            (v_empty[tc % VST] if wide else w_empty[buf]).arrive()

    actors = {}
    for g in [producer(True), producer(False), s_issuer(), o_issuer(), converter()] + [softmax(i) for i in range(4)]:
        actors[len(actors)] = [g, None]
    # some actors run much slower than others in some runs
    weight = {a: rng.choice([1, 1, 8, 40]) for a in list(actors) + ["load", "s", "o"]}
    idle = 0
    while actors or loads or s_pipe or o_pipe:
        names = list(actors) + ["load"] * bool(loads) + ["s"] * bool(s_pipe) + ["o"] * bool(o_pipe)
        who = rng.choices(names, [weight[n] for n in names])[0]
        idle += 1
        assert idle < 200000, "nobody can go on"
        if who == "load":
            slots, i, tc, full = loads.pop(rng.randrange(len(loads)))
            slots[i] = tc
            full.arrive()
            idle = 0
        elif who in ("s", "o"):
            product((s_pipe if who == "s" else o_pipe).pop(0))
            idle = 0
        else:
            gen, cond = actors[who]
            if cond is not None and not cond():
                continue
            idle = 0
            try:
                actors[who][1] = next(gen)
            except StopIteration:
                del actors[who]
    assert sorted(finished) == [0, 1, 2, 3]


@pytest.mark.parametrize("NR", [16, 32, 64])
def test_tiles_change_hands_in_order(NR):
    rng = random.Random(NR)
    for seed in range(60):
        n = rng.randint(1, 5)
        run(NR, [(rng.choice([0, 1, 2, 7, 30]), rng.choice([1, 1, 2, 4])) for _ in range(n)], seed)
    # a share that ends inside a unit's pages, and one that begins in its tail
    run(NR, [(5, 0), (9, 1), (0, 3), (1, 0)], 99)


def test_the_model_sees_a_ring_that_is_too_short():
    """The same run with the tile descriptions' ring shortened has to fail."""
    global SRC
    kept = SRC
    try:
        SRC = re.sub(r"#define PT_INFO \d+", "#define PT_INFO 6", SRC)
        with pytest.raises(AssertionError):
            for seed in range(40):
                run(16, [(30, 2), (30, 2)], seed)
    finally:
        SRC = kept
