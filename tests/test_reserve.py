"""Room for tokens that the device writes (kv_session_reserve) on a metadata-only pool against the
pool model: no accepted token is lost to a cold copy that went stale (CPU only)."""

import copy

import numpy as np
import pytest

from oracle.pool_model import ERR_INVALID, ERR_STATE, ModelError, PoolModel
from test_host_runtime import _lib, _meta_pool, _random_call, _same, _snapshot


class Step:
    """Speculative steps of one session on a metadata-only pool, with what every page holds: a
    number that rises with each write, in the pages and in their cold copies."""

    def __init__(self, length, spill=False, stride=64):
        self.kv = _lib()
        self.pool = _meta_pool(self.kv, stride if not spill else stride // 4, 4 * stride, 2, stride)
        self.kv.kv_pool_set_spill(self.pool, spill)
        self.sid = self.kv.kv_session_create(self.pool, length)
        self.length = length
        self.now, self.hot_data, self.cold_data = 0, {}, {}
        self.want = {}

    def pages(self):
        _, _, hot, cold = self.kv.kv_session_info(self.pool, self.sid)
        return hot, cold

    def reserve(self, room, low=None, high=None):
        """Room behind the tokens held, of which the host may know bounds only."""
        before = self.pages()[0]
        end = (self.length if high is None else high) + room
        self.kv.kv_session_reserve(self.pool, self.sid, self.length if low is None else low, end)
        hot, _ = self.pages()
        assert len(hot) == -(-end // 16)
        for i in range(len(hot)):       # a new page holds nothing yet
            if i >= len(before):
                self.want[i] = self.now = self.now + 1
                (self.hot_data if hot[i] >= 0 else self.cold_data)[self.at(i)] = self.now
        for i in range(len(hot), len(before)):
            self.want.pop(i, None)

    def at(self, i):
        hot, cold = self.pages()
        return hot[i] if hot[i] >= 0 else cold[i]

    def accept(self, n):
        """The device's writes: pages only, no bookkeeping."""
        hot, _ = self.pages()
        for p in {t // 16 for t in range(self.length, self.length + n)}:
            self.now += 1
            self.want[p] = self.now
            (self.hot_data if hot[p] >= 0 else self.cold_data)[self.at(p)] = self.now
        self.length += n

    def evict_and_resume(self, lazy=False):
        hot, cold = self.pages()
        self.kv.kv_evict_session(self.pool, self.sid)
        after = self.pages()[1]
        for i, (h, c) in enumerate(zip(hot, cold)):
            if c < 0:                   # no valid copy: the eviction writes the page
                self.cold_data[after[i]] = self.hot_data.get(h)
        if lazy:
            self.kv.kv_resume_sessions_lazy(self.pool, [self.sid])
        else:
            self.kv.kv_resume_sessions(self.pool, [self.sid])
        new, cold = self.pages()
        for i, h in enumerate(new):
            if h >= 0:
                self.hot_data[h] = self.cold_data.get(cold[i])

    def promote(self, n):
        before, _ = self.pages()
        self.kv.kv_promote_pages(self.pool, n)
        new, cold = self.pages()
        for h, old, c in zip(new, before, cold):
            if h >= 0 and old < 0:
                self.hot_data[h] = self.cold_data.get(c)

    def check(self):
        hot, _ = self.pages()
        for i, want in self.want.items():
            got = (self.hot_data if hot[i] >= 0 else self.cold_data).get(self.at(i))
            assert got == want, "page %d holds write %s, its last one was %s" % (i, got, want)


@pytest.mark.parametrize("length,room,accepted", [(10, 6, 2), (100, 8, 0), (100, 64, 2), (16, 16, 0), (16, 16, 16),
                                                  (0, 8, 3), (15, 1, 1), (95, 33, 33), (31, 2, 1)])
def test_partly_accepted_drafts_survive_evictions(length, room, accepted):
    s = Step(length)
    for turn in range(4):
        s.reserve(room)
        s.accept(accepted)
        s.evict_and_resume()
        s.check()
    s.reserve(0)                        # the turn is over: room and its pages are given back
    hot, _ = s.pages()
    assert len(hot) == -(-s.length // 16)
    assert s.kv.kv_pool_stats(s.pool)["free_hot_pages"] == 64 - len(hot)
    s.kv.kv_session_extend(s.pool, s.sid, s.length + 1)      # a plain step goes on from there


@pytest.mark.parametrize("spill", [False, True])
@pytest.mark.parametrize("width", [1, 8, 64])
def test_random_turns_lose_nothing(width, spill):
    rng = np.random.default_rng(width)
    for trial in range(12):
        s = Step(int(rng.integers(0, 120)), spill)
        for turn in range(30):
            if s.length + width > 16 * 64:
                break
            s.reserve(int(rng.integers(1, width, endpoint=True)) if rng.random() < 0.3 else width)
            _, length, _, _ = s.kv.kv_session_info(s.pool, s.sid)
            s.accept(int(rng.integers(0, length - s.length, endpoint=True)))
            s.check()
            if rng.random() < 0.4:
                s.evict_and_resume(lazy=spill and rng.random() < 0.5)
                s.check()


def test_hand_worked():
    m = PoolModel(num_hot=10, num_cold=10, max_sessions=2, max_pages_per_session=6)
    a = m.create(20)
    m.reserve(a, 20, 70)                     # room for 50 drafts: pages 1 to 4
    assert m.row(a) == [0, 1, 2, 3, 4, -1] and m.sessions[a].seq_len == 70
    assert m.evict(a) == [(0, 0), (1, 1), (2, 2), (3, 3), (4, 4)]
    m.resume([a])
    m.reserve(a, 22, 40)                     # two were accepted: pages 1 and 2 may be written,
    assert m.row(a) == [0, 1, 2, -1, -1, -1]     # pages 3 and 4 are not needed
    assert m.sessions[a].cold == [0, -1, -1] and m.free_hot() == 7 and m.free_cold() == 9
    m.reserve(a, 32, 32)                     # nothing to write: page 2 goes, copies stay as they are
    assert m.sessions[a].cold == [0, -1] and m.sessions[a].seq_len == 32
    assert m.evict(a) == [(1, 1)] and m.cold_writes == 6
    m.resume([a])
    m.reserve(a, 32, 33)                     # behind a full page: only the new page
    assert m.sessions[a].cold == [0, 1, -1]
    m.reserve(a, 0, 33)                      # a lower bound of what it holds
    assert m.sessions[a].cold == [-1, -1, -1]


@pytest.mark.parametrize("seed,spill", [(0, False), (1, False), (2, True), (3, True)])
def test_random_sequences_follow_the_model(seed, spill):
    kv = _lib()
    nh, nc, ms, stride = (60, 45, 7, 9) if not spill else (20, 90, 7, 9)
    pool = _meta_pool(kv, nh, nc, ms, stride)
    kv.kv_pool_set_spill(pool, spill)
    model = PoolModel(nh, nc, ms, stride, spill=spill)
    rng = np.random.default_rng(200 + seed)
    done = refused = shorter = 0
    for step in range(2500):
        mine = rng.random() < 0.4
        if mine:
            sid = int(rng.integers(-1, ms + 1))
            length = model.sessions[sid].seq_len if 0 <= sid < ms else 0
            kept = int(rng.integers(-1, length + 2))
            new = int(rng.integers(max(kept - 2, 0), 16 * stride + 4))
            shorter += 0 <= kept <= new < length
            on_model = lambda m: m.reserve(sid, kept, new)                            # noqa: E731
            on_lib = lambda: kv.kv_session_reserve(pool, sid, kept, new)              # noqa: E731
        else:
            on_model, on_lib = _random_call(kv, pool, rng, nh, nc, ms, stride)
        before = _snapshot(kv, pool, ms)
        try:
            expect = on_model(model)
        except ModelError as e:
            refused += mine
            with pytest.raises(kv.KVError) as err:
                on_lib()
            assert err.value.status == e.code, (e, err.value)
            assert _snapshot(kv, pool, ms) == before
        else:
            done += mine
            assert on_lib() == expect
        _same(kv, pool, model, ms)
    assert done > 100 and refused > 100 and shorter > 50
    kv.kv_pool_destroy(pool)


def test_refusals_change_nothing():
    m = PoolModel(num_hot=2, num_cold=8, max_sessions=3, max_pages_per_session=4, spill=True)
    kv = _lib()
    pool = _meta_pool(kv, 2, 8, 3, 4)
    kv.kv_pool_set_spill(pool, True)
    for call in (lambda: m.import_cold(40, [5, 6, 7]), lambda: m.import_cold(40, [4, 6, 3]),
                 lambda: m.resume_lazy([0]),
                 lambda: kv.kv_session_import_cold(pool, 40, [5, 6, 7]),
                 lambda: kv.kv_session_import_cold(pool, 40, [4, 6, 3]),
                 lambda: kv.kv_resume_sessions_lazy(pool, [0])):
        call()
    for args, code in (((0, 30, 41), ERR_STATE),      # page 1 is shared with session 1
                       ((0, 20, 25), ERR_STATE), ((0, 41, 50), ERR_INVALID), ((0, -1, 10), ERR_INVALID),
                       ((0, 20, 19), ERR_INVALID), ((0, 40, 65), ERR_INVALID), ((1, 40, 41), ERR_STATE),
                       ((2, 0, 0), ERR_STATE), ((3, 0, 0), ERR_INVALID), ((-1, 0, 0), ERR_INVALID)):
        before, snap = copy.deepcopy(m.__dict__), _snapshot(kv, pool, 3)
        with pytest.raises(ModelError) as e:
            m.reserve(*args)
        assert e.value.code == code and m.__dict__ == before, args
        with pytest.raises(kv.KVError) as err:
            kv.kv_session_reserve(pool, *args)
        assert err.value.status == code and _snapshot(kv, pool, 3) == snap, args
    with pytest.raises(kv.KVError):
        kv.kv_session_reserve(0, 0, 0, 0)
    kv.kv_session_reserve(pool, 0, 40, 48)            # page 2 is this session's alone: written in place
    kv.kv_session_reserve(pool, 0, 30, 30)            # and let go; page 1, shared, takes no tokens
    assert kv.kv_session_info(pool, 0)[3] == [5, 6]
    kv.kv_pool_destroy(pool)


@pytest.mark.parametrize("spill", [False, True])
@pytest.mark.parametrize("width", [1, 8, 40])
def test_lengths_that_only_the_device_knows(width, spill):
    """The accepted counts reach the host every few steps: bounds of the length do between them."""
    rng = np.random.default_rng(90 + width)
    for trial in range(12):
        s = Step(int(rng.integers(0, 120)), spill)
        low = high = s.length
        for turn in range(30):
            if high + width > 16 * 64:
                break
            s.reserve(width, low, high)
            s.accept(int(rng.integers(0, width, endpoint=True)))
            high += width
            s.check()
            if rng.random() < 0.3:
                s.evict_and_resume(lazy=spill and rng.random() < 0.5)
                s.check()
            if rng.random() < 0.3:
                low = high = s.length


@pytest.mark.parametrize("width", [1, 8, 64])
def test_promotions_between_steps_lose_nothing(width):
    """Spilled pages are promoted before a step's room is made: the resident pages that the step
    writes have no cold copies that count as valid."""
    rng = np.random.default_rng(80 + width)
    promoted = 0
    for trial in range(12):
        s = Step(int(rng.integers(0, 120)), spill=True)
        for turn in range(30):
            if s.length + width > 16 * 64:
                break
            s.promote(int(rng.integers(0, 8)))
            s.check()
            s.reserve(width)
            s.accept(int(rng.integers(0, width, endpoint=True)))
            s.check()
            if rng.random() < 0.5:
                s.evict_and_resume(lazy=rng.random() < 0.8)
                s.check()
        promoted += s.kv.kv_pool_stats(s.pool)["promoted_pages"]
    assert promoted > 50
