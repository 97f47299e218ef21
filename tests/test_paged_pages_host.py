"""Which pages the owner of a paged cache gives to whom, without a GPU: its buffers lie in host memory, and of its calls only
the host's part happens."""
import pytest
import torch

from paper_2503_19950_amd import binding as B


class Host:
    """What stands in for the device: `recording` says whether a graph is being recorded."""
    recording = False

    def call(self, index, f, *args):
        if f is B._init_paged:
            return
        assert f is B._evict_paged
        cfg, cache, keep, recent, ws = args
        cfg, cache = cfg._obj, cache._obj
        keep = list(keep)
        if all(cache.n[b] <= keep[b] for b in range(cfg.B)):             # no launch
            st = f(*args, None)
            if st != B.LQ_OK:
                raise B.LogQuantError(st, f.__name__)
            return
        for b in range(cfg.B):
            if cache.n[b] > keep[b]:
                assert 0 <= recent <= keep[b] <= cache.pages[(1 - cache.cur[b]) * cfg.B + b] * cfg.page
                cache.n[b] = keep[b]
                cache.cur[b] ^= 1

    def no_recording(self, call):
        if self.recording:
            raise B.LogQuantError(B.LQ_ERR_STATE, call)


@pytest.fixture
def host(monkeypatch):
    h = Host()
    monkeypatch.setattr(B, "_cuda", lambda device: torch.device("cpu"))
    monkeypatch.setattr(B, "_on_device", h.call)
    monkeypatch.setattr(B.DeviceCachePaged, "_no_recording", lambda self, call: h.no_recording(call))
    return h


def make(rows=3, n_pages=12, weighted=True, max_pages=6):
    return B.DeviceCachePaged(B.make_config_paged(rows, 1, 1, 64, 32, "f16", n_pages, max_pages, weighted), "cpu")


def held(cache):
    return (list(cache.free), list(cache.uses), [[list(i) for i in half] for half in cache.ids], list(cache.pages), cache.shared,
            cache.counts(), list(cache.cur), cache.table.clone().tolist())


def consistent(cache):
    """Counts of names, free pages and the table say the same."""
    named = [i for half in cache.ids for ids in half for i in ids]
    assert cache.uses == [named.count(i) for i in range(cache.cfg.n_pages)]
    assert sorted(cache.free) == [i for i in range(cache.cfg.n_pages) if i not in named]
    assert cache.shared == sum(x > 1 for x in cache.uses)
    for half in range(2):
        for b, ids in enumerate(cache.ids[half]):
            assert cache.pages[half * cache.cfg.B + b] == len(ids)
            assert cache.table[half, b, :len(ids)].tolist() == ids


def with_a_left_prompt(n_pages=12):
    """Rows 0 and 1 read the two pages of a prompt; row 0 has been evicted from and holds 60 tokens in pages of its own."""
    cache = make(n_pages=n_pages)
    cache.reserve([64, 0, 0])
    prompt = list(cache.ids[0][0])
    cache.set_pages(1, prompt)
    cache.set_counts([64, 64, 0])
    cache.evict([40, 64, 64], 8)
    cache.reserve([64, 64, 0])
    cache.set_counts([60, 64, 0])
    consistent(cache)
    assert cache.ids[cache.cur[0] ^ 1][0] == prompt
    return cache, prompt


REFUSED = [dict(keep=[32, 64, 64], recent=33), dict(keep=[32, 64, 64], recent=-1), dict(keep=[-1, 64, 64], recent=0), dict(keep=[64, 64, -1], recent=0)]


@pytest.mark.parametrize("kw", REFUSED, ids=str)
def test_an_eviction_that_is_refused_changes_nothing(host, kw):
    for cache in (with_a_left_prompt()[0], make()):
        if not cache.n[0]:
            cache.reserve([64, 32, 0])
            cache.set_counts([64, 32, 0])
        before = held(cache)
        with pytest.raises(B.LogQuantError) as e:
            cache.evict(**kw)
        assert e.value.status == B.LQ_ERR_SHAPE and held(cache) == before


def test_an_eviction_in_a_recording_changes_nothing(host):
    cache, prompt = with_a_left_prompt()
    before = held(cache)
    host.recording = True
    with pytest.raises(B.LogQuantError) as e:
        cache.evict([32, 64, 64], 8)
    assert e.value.status == B.LQ_ERR_STATE and held(cache) == before
    host.recording = False
    cache.evict([32, 64, 64], 8)
    consistent(cache)
    assert not set(prompt) & set(cache.ids[cache.cur[0]][0]) and [cache.uses[i] for i in prompt] == [1, 1]


def test_an_eviction_that_the_pool_has_no_pages_for_changes_nothing(host):
    cache, prompt = with_a_left_prompt(n_pages=5)        # two of the prompt, two of row 0, one free
    assert len(cache.free) == 1
    before = held(cache)
    with pytest.raises(B.LogQuantError) as e:
        cache.evict([40, 64, 64], 8)
    assert e.value.status == B.LQ_ERR_CAPACITY and held(cache) == before
    cache.evict([32, 64, 64], 8)                         # one page is enough
    consistent(cache)


def test_pages_that_evictions_left_count_as_room_once_nothing_else_names_them(host):
    """Both readers of a prompt have been evicted from: what they left is shared by what they left alone."""
    cache = make(rows=2, n_pages=6)
    cache.reserve([64, 0])
    prompt = list(cache.ids[0][0])
    cache.set_pages(1, prompt)
    cache.set_counts([64, 64])
    cache.evict(40, 8)
    cache.reserve([64, 64])
    cache.set_counts([64, 64])
    assert not cache.free and [cache.uses[i] for i in prompt] == [2, 2]
    before = held(cache)
    with pytest.raises(B.LogQuantError):
        cache.evict([64, 40], 8)                         # row 0's still names them
    assert held(cache) == before
    with pytest.raises(B.LogQuantError):
        cache.evict(40, 8)                               # two pages for four
    assert held(cache) == before
    cache.evict(32, 8)                                   # two for two
    consistent(cache)
    assert sorted(cache.ids[0][0] + cache.ids[0][1]) == sorted(prompt)


def test_a_row_that_keeps_nothing_gives_back_what_others_read(host):
    cache, prompt = with_a_left_prompt()
    cache.evict([0, 64, 64])
    consistent(cache)
    assert cache.counts() == [0, 64, 0] and not cache.ids[cache.cur[0]][0] and [cache.uses[i] for i in prompt] == [1, 1]


def test_counts_that_no_page_holds_are_refused_before_pages_are_taken(host):
    cache = make()
    cache.reserve([32, 0, 0])
    cache.set_counts([40, 0, 0])
    before = held(cache)
    with pytest.raises(B.LogQuantError) as e:
        cache.evict(32)
    assert e.value.status == B.LQ_ERR_STATE and held(cache) == before
    plain = make(weighted=False)
    plain.reserve([64, 0, 0])
    plain.set_counts([64, 0, 0])
    before = held(plain)
    with pytest.raises(B.LogQuantError) as e:
        plain.evict(32)
    assert e.value.status == B.LQ_ERR_STATE and held(plain) == before


def test_reserved_spare_pages_are_ones_that_the_eviction_takes(host):
    """Pages for a recorded eviction are named before: the pages that the one before left are no such ones while another row reads
    them."""
    cache, prompt = with_a_left_prompt()
    cache.reserve([40, 0, 0], spare=True)
    consistent(cache)
    assert not set(prompt) & set(cache.ids[cache.cur[0] ^ 1][0])
    host.recording = True
    cache.evict([40, 64, 64], 8)
    host.recording = False
    consistent(cache)
    assert cache.counts() == [40, 64, 0]


def test_a_prompt_is_shared_on_after_one_of_its_readers_was_evicted_from(host):
    cache, prompt = with_a_left_prompt()
    cache.set_pages(2, prompt)                           # a new reader
    cache.set_counts([60, 64, 64])
    cache.set_pages(1, prompt + [cache.free.popitem()[0]])   # a reader names its pages again, and one more
    consistent(cache)
    assert [cache.uses[i] for i in prompt] == [3, 3]
    cache.evict([40, 64, 64], 8)                         # row 0 moves elsewhere
    consistent(cache)
    assert not set(prompt) & set(cache.ids[cache.cur[0]][0]) and [cache.uses[i] for i in prompt] == [2, 2]


def test_a_page_that_nobody_reads_any_more_is_not_named_before_it_is_given_back(host):
    cache, prompt = with_a_left_prompt()
    cache.release(1)
    before = held(cache)
    with pytest.raises(ValueError):
        cache.set_pages(2, prompt)
    assert held(cache) == before
    cache.release(0, spare=True)
    cache.set_pages(2, prompt)
    consistent(cache)


def test_places_are_no_positions_after_an_eviction(host):
    """A row that was evicted from holds fewer tokens than have come: keys are not turned by places any more."""
    cache = make()
    rope = B.Rope([1.0, 0.5], device="cpu")
    turn = lambda **kw: cache._turn(rope, None, 1, **kw)  # noqa: E731
    cache.reserve([96, 96, 96])
    cache.set_counts([64, 32, 0])
    assert turn()[1] is None
    cache.evict(40, 8)                                   # row 0
    with pytest.raises(ValueError):
        turn()
    with pytest.raises(ValueError):
        turn(n_new=[1, 1, 1])
    turn(n_new=[0, 1, 1])                                # it takes none
    assert cache._turn(None, None, 1) == (None, None) and cache.counts() == [40, 32, 0]
    other = cache.clone()
    with pytest.raises(ValueError):
        other._turn(rope, None, 1)
    cache.set_counts([64, 32, 0], [0, 0, 0])             # back to the tokens that were all there
    turn()
    cache.set_counts([39, 32, 0], [1, 0, 0])             # and on again, a token dropped
    with pytest.raises(ValueError):
        turn()
    cache.set_counts([0, 32, 0])                         # begins anew
    turn()
    other.release(0)
    other._turn(rope, None, 1)
    other.release(1)
    other.set_counts([0, 0, 0])
    assert not other.gaps
    cache.set_counts([64, 32, 0], [0, 0, 0])
    cache.evict([0, 32, 0])                              # an empty row whose next token is not the first
    with pytest.raises(ValueError):
        turn()


FAR = 2 ** 32                                            # what 32 bits would make 0 of


def test_numbers_beyond_32_bits_are_not_taken_modulo(host):
    cache = make()
    cache.reserve([64, 32, 0])
    cache.set_counts([64, 32, 0])
    before = held(cache)
    cache.evict(FAR)                                     # nobody has more
    cache.evict([FAR + 8, 2 ** 63, FAR], FAR + 4)
    assert held(cache) == before
    for kw in (dict(keep=40, recent=FAR), dict(keep=40, recent=FAR + 8), dict(keep=40, recent=-FAR), dict(keep=8 - FAR), dict(keep=[FAR + 40, 8 - FAR, 0])):
        with pytest.raises(B.LogQuantError) as e:
            cache.evict(**kw)
        assert e.value.status == B.LQ_ERR_SHAPE and held(cache) == before
    for counts, cur in (([FAR + 5, 0, 0], None), ([0, -FAR, 0], None), ([5, 0, 0], [FAR, 0, 0]), ([5, 0], None), ([5, 0, 0], [1])):
        with pytest.raises(ValueError):
            cache.set_counts(counts, cur)
        assert held(cache) == before
    cache.evict([40, FAR, FAR + 1], 8)
    assert cache.counts() == [40, 32, 0] and list(cache.cur) == [1, 0, 0]
    assert cache._how(0.0, FAR, None)._obj.window == 2 ** 31 - 1 and cache._how(0.0, -FAR, None)._obj.window == -1
    assert cache._how(0.0, 7, None)._obj.window == 7
    for values in ([FAR], [0, -FAR - 1], [2 ** 31]):
        with pytest.raises(ValueError):
            B._i32(values)
    assert list(B._i32([2 ** 31 - 1, -2 ** 31, True])) == [2 ** 31 - 1, -2 ** 31, 1] and B._i32(None) is None and len(B._i32([])) == 0


@pytest.mark.parametrize("row", [-1, -3, 3, 2 ** 31])
def test_rows_that_the_cache_does_not_have(host, row):
    cache = with_a_left_prompt()[0]
    before = held(cache)
    for spare in (False, True):
        with pytest.raises(ValueError):
            cache.set_pages(row, [cache.cfg.n_pages - 1], spare=spare)
        with pytest.raises(ValueError):
            cache.release(row, spare=spare)
    assert held(cache) == before
