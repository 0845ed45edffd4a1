"""Cache pages against the plain tables: every array equal after every call, and the contents of the pools with them."""
import ctypes
import random

import numpy as np
import pytest
import torch

from paper_2510_26527_b200 import binding, buildlib
from tests import plain_operators as plain

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    buildlib.build()
    binding.load_library()
    assert torch.cuda.is_available()


def _i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device=DEV)


class Both:
    """One state on the device and in plain lists, and pools of bytes beside them."""

    def __init__(self, n_seqs, max_pages, n_pages, page_tokens, pools=(), seed=0):
        self.pages = binding.CachePages.new(n_seqs, max_pages, n_pages, page_tokens, DEV)
        self.plain = plain.Pages(n_seqs, max_pages, n_pages, page_tokens)
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.pools = [torch.randint(0, 256, (planes, n_pages, size), generator=g, device=DEV, dtype=torch.int32).to(torch.uint8) for planes, size in pools]
        self.copies = [p.cpu().numpy().copy() for p in self.pools]

    def move(self, pairs):
        for p in self.copies:
            kept = {old: p[:, old].copy() for old, _ in pairs}
            for old, new in pairs:
                p[:, new] = kept[old]

    def reserve(self, targets, **kw):
        st = binding.polyspec_cache_reserve(self.pages, _i32(targets), pools=self.pools, **kw)
        self.move(self.plain.reserve(targets))
        self.check(st)

    def rollback(self, targets):
        st = binding.polyspec_cache_rollback(self.pages, _i32(targets))
        self.plain.rollback(targets)
        self.check(st)

    def fork(self, src, dst):
        st = binding.polyspec_cache_fork(self.pages, _i32(src), _i32(dst))
        self.plain.fork(src, dst)
        self.check(st)

    def compact(self):
        moved = torch.full((self.pages.n_pages,), -9, dtype=torch.int32, device=DEV)
        live = [c > 0 for c in self.plain.refs]
        binding.polyspec_cache_compact(self.pages, pools=self.pools, moved_to=moved)
        moves = self.plain.compact()
        self.move(list(moves.items()))
        self.check(None)
        assert moved.tolist() == [moves.get(p, p) if live[p] else -1 for p in range(self.pages.n_pages)]

    def check(self, status):
        torch.cuda.synchronize()
        if status is not None:
            assert int(status) == self.plain.status
        self.plain.status = 0
        for name, want in self.plain.arrays().items():
            got = getattr(self.pages, name).cpu().numpy()
            assert (got == want).all(), (name, np.argwhere(got != want)[:5])
        for got, want in zip(self.pools, self.copies):
            assert (got.cpu().numpy() == want).all()


@pytest.mark.parametrize("n_seqs,max_pages,n_pages,page_tokens,pools", [
    (1, 1, 1, 1, ()),
    (3, 4, 9, 1, ((1, 16),)),
    (5, 9, 40, 4, ((3, 48), (2, 2064))),
    (8, 20, 64, 16, ((2, 4096),)),
    (33, 17, 257, 3, ((1, 32), (1, 16), (2, 160))),
    (70, 40, 1500, 8, ((1, 2048),)),
])
@pytest.mark.parametrize("seed", [0, 1])
def test_random_histories(n_seqs, max_pages, n_pages, page_tokens, pools, seed):
    rng = random.Random(seed * 100 + n_seqs)
    both = Both(n_seqs, max_pages, n_pages, page_tokens, pools, seed)
    most = max_pages * page_tokens
    for step in range(60):
        what = rng.choice(["reserve", "reserve", "rollback", "fork", "compact"])
        n = both.plain.len
        if what == "reserve":
            both.reserve([x + rng.choice([0, 1, 2, page_tokens, rng.randrange(most + 2), -1]) if rng.random() < 0.6 else 0 for x in n])
        elif what == "rollback":
            both.rollback([rng.choice([-1, 0, x, x - 1, x // 2, x + 3, rng.randrange(most + 1)]) for x in n])
        elif what == "fork":
            k = rng.randrange(1, 2 * n_seqs + 1)
            src, dst = [rng.randrange(-1, n_seqs + 1) for _ in range(k)], [rng.randrange(-1, n_seqs + 1) for _ in range(k)]
            if rng.random() < 0.5:
                empty = [b for b in range(n_seqs) if n[b] == 0]
                full = [b for b in range(n_seqs) if n[b] > 0]
                if empty and full:
                    dst = empty[: rng.randrange(1, len(empty) + 1)]
                    src = [rng.choice(full) for _ in dst]
            both.fork(src, dst)
        else:
            both.compact()


def test_wide_pool_and_many_sequences():
    """More bitmap words than threads, more sequences than threads, needs that run past the pool."""
    both = Both(1500, 40, 40001, 2)
    rng = random.Random(5)
    both.reserve([rng.randrange(0, 81) for _ in range(1500)])
    both.rollback([rng.randrange(0, 81) for _ in range(1500)])
    both.reserve([80] * 1500)
    both.compact()
    both.rollback([0] * 700 + [-1] * 800)
    both.compact()
    both.fork([1400] * 690, list(range(690)))
    both.reserve([n + 1 for n in both.plain.len])


def test_copy_before_the_first_write_of_a_shared_page():
    both = Both(6, 4, 20, 4, ((2, 64),))
    both.reserve([6, 0, 0, 0, 0, 0])
    both.fork([0, 0, 0], [1, 2, 3])
    shared = both.plain.rows[0][1]
    both.reserve([0, 7, 9, 0, 0, 0])                       # two of the four write on: two copies, the others still share
    assert both.plain.refs[shared] == 2 and both.plain.rows[1][1] != shared
    both.reserve([7, 0, 0, 7, 0, 0])                       # both remaining holders at once: both copy, the page is free
    assert both.plain.refs[shared] == 0
    both.rollback([4, 4, 4, 4, 4, 4])
    both.fork([0], [4])
    both.reserve([0, 0, 0, 0, 5, 0])                       # a whole shared page is not copied
    assert both.plain.rows[4][0] == both.plain.rows[0][0]


def test_targets_from_the_state_itself_and_in_parts():
    both = Both(4, 8, 64, 4)
    both.reserve([3, 8, 0, 30])
    st = binding.polyspec_cache_reserve(both.pages, both.pages.len, plus=3)
    both.plain.reserve([n + 3 for n in both.plain.len])     # 33 tokens do not fit the table: reported
    both.check(st)
    extra = _i32([1, -2, 0, -1000])
    st = binding.polyspec_cache_rollback(both.pages, both.pages.len, extra, plus=-1)
    both.plain.rollback([n + e - 1 for n, e in zip(both.plain.len, [1, -2, 0, -1000])])
    both.check(st)


def test_broken_states_are_reported_and_skipped():
    both = Both(3, 4, 16, 4)
    both.reserve([9, 5, 2])
    both.pages.table[0, 1] = 99                             # no such page
    st = binding.polyspec_cache_rollback(both.pages, _i32([0, -1, -1]))
    torch.cuda.synchronize()
    assert int(st) == binding.ERR_BAD_INPUT_ON_DEVICE
    assert both.pages.len.tolist() == [0, 5, 2] and both.pages.refs.tolist()[:6] == [0, 1, 0, 1, 1, 1]
    both.pages.table[1, 1] = -1                             # a last page that is not there
    before = both.pages.table.clone()
    for call in (lambda: binding.polyspec_cache_reserve(both.pages, _i32([0, 6, 0])), lambda: binding.polyspec_cache_fork(both.pages, _i32([1]), _i32([0]))):
        st = call()
        torch.cuda.synchronize()
        assert int(st) == binding.ERR_BAD_INPUT_ON_DEVICE
        assert torch.equal(both.pages.table, before) and both.pages.len.tolist() == [0, 5, 2]
    both.pages.len[2] = 17                                  # more than the table holds
    for call in (lambda: binding.polyspec_cache_reserve(both.pages, _i32([0, 0, 30])), lambda: binding.polyspec_cache_rollback(both.pages, _i32([-1, -1, 1]))):
        st = call()
        torch.cuda.synchronize()
        assert int(st) == binding.ERR_BAD_INPUT_ON_DEVICE
    assert torch.equal(both.pages.table, before)


def test_bits_behind_the_last_page_are_not_pages():
    both = Both(2, 8, 37, 4)
    both.pages.free_bits[1] = -1                            # all 32 bits of a word that has five pages
    st = binding.polyspec_cache_reserve(both.pages, _i32([32, 32]))
    torch.cuda.synchronize()
    assert int(st) == 0 and both.pages.table.flatten().tolist() == list(range(16))
    small = Both(2, 40, 37, 1)
    small.pages.free_bits[1] = -1
    st = binding.polyspec_cache_reserve(small.pages, _i32([38, 37]))
    torch.cuda.synchronize()
    assert int(st) == binding.ERR_NO_PAGES and small.pages.len.tolist() == [0, 0]
    binding.polyspec_cache_reserve(small.pages, _i32([20, 17]))
    binding.polyspec_cache_compact(small.pages)
    torch.cuda.synchronize()
    assert small.pages.refs.tolist() == [1] * 37 and small.pages.free_bits.tolist() == [0, 0]


def test_compact_leaves_entries_behind_a_sequence_as_they_were():
    """Table words behind the pages a sequence holds are no entries, whatever free page they name."""
    both = Both(3, 8, 64, 4, ((2, 64),))
    both.reserve([12, 12, 12])                              # pages 0-2, 3-5, 6-8
    both.rollback([-1, 0, -1])                              # pages 3-5 are free: 6-8 move there
    stale = [63, 40, 7, 20, 6]                              # 7 and 6 are in use and move; the others are free
    both.pages.table[0, 3:] = _i32(stale)
    both.pages.workspace().fill_(0x5a)                      # what an earlier call may have left
    binding.polyspec_cache_compact(both.pages, pools=both.pools)
    both.move(list(both.plain.compact().items()))
    torch.cuda.synchronize()
    table = both.pages.table.tolist()
    assert table[0][:3] == [0, 1, 2] and table[2][:3] == [3, 4, 5]
    assert [table[0][3], table[0][4], table[0][6]] == [63, 40, 20]
    for got, want in zip(both.pools, both.copies):
        assert (got.cpu().numpy() == want).all()


def test_captured_cycle():
    both = Both(5, 8, 64, 4, ((2, 128),))
    both.reserve([10, 3, 0, 7, 7])
    both.fork([0], [2])
    base, acc = both.pages.len.clone(), _i32([0, 1, 2, 3, 5])
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    both.pages.workspace()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.polyspec_cache_reserve(both.pages, base, plus=5, pools=both.pools, device_status=status)
        binding.polyspec_cache_rollback(both.pages, base, acc, device_status=status)
        base.copy_(both.pages.len)
    for _ in range(3):
        now = list(both.plain.len)
        both.move(both.plain.reserve([n + 5 for n in now]))
        both.plain.rollback([n + a for n, a in zip(now, acc.tolist())])
        graph.replay()
        both.check(status)


def test_pool_offsets_past_32_bits():
    n_pages, size = 1100, 1 << 21
    pool = torch.zeros((2, n_pages, size), dtype=torch.uint8, device=DEV)          # 4.6 GB
    pages = binding.CachePages.new(2, 1100, n_pages, 1, DEV)
    binding.polyspec_cache_reserve(pages, _i32([1000, 100]))
    pool[1, 1099] = 7
    pool[1, 1098, -1] = 9
    binding.polyspec_cache_rollback(pages, _i32([998, 100]))
    binding.polyspec_cache_compact(pages, pools=[pool])
    torch.cuda.synchronize()
    assert pages.table[1, 98:].tolist()[:2] == [998, 999]
    assert int(pool[1, 998, -1]) == 9 and (pool[1, 999] == 7).all() and int(pool[1, 998].sum()) == 9


def test_compact_renames_no_word_behind_a_sequences_pages():
    """Whatever such a word names, pages that move included."""
    both = Both(4, 8, 64, 4, ((2, 64),))
    both.reserve([12, 12, 12, 0])                           # pages 0-2, 3-5, 6-8
    both.rollback([-1, 0, -1, -1])                          # 6-8 move to 3-5
    tails = {0: (3, [8, 7, 6, 63, 3]), 1: (0, [6, 8, 7, -1, 99, 6, 0, -7]), 2: (3, [6, 6, 7, 8, 5]), 3: (0, [8] * 8)}
    for b, (at, words) in tails.items():
        both.pages.table[b, at:] = _i32(words)
    binding.polyspec_cache_compact(both.pages, pools=both.pools)
    both.move(list(both.plain.compact().items()))
    torch.cuda.synchronize()
    table = both.pages.table.tolist()
    assert table[0][:3] == [0, 1, 2] and table[2][:3] == [3, 4, 5]
    for b, (at, words) in tails.items():
        assert table[b][at:] == words, b
    for got, want in zip(both.pools, both.copies):
        assert (got.cpu().numpy() == want).all()


@pytest.mark.parametrize("far", [1, 2, 31, 40, 700, 1100])
def test_reserve_reports_the_first_sequence_that_fails(far):
    """A shortage and an over-long target in one call: the lower sequence's status, in one warp, across warps and across rounds."""
    n = 1200
    for short, long_ in ((0, far), (far, 0), (n - 1 - far, n - 1), (n - 1, n - 1 - far)):
        pages = binding.CachePages.new(n, 4, 2, 4, DEV)
        targets = [0] * n
        targets[short], targets[long_] = 16, 17             # four pages where there are two; more than the table's sixteen tokens
        for _ in range(3):
            status = binding.polyspec_cache_reserve(pages, _i32(targets))
            assert int(status) == (binding.ERR_NO_PAGES if short < long_ else binding.ERR_BAD_INPUT_ON_DEVICE), (short, long_)
        assert int(pages.len.sum()) == 0


@pytest.mark.parametrize("given", [False, True])
def test_workspace_outlives_its_use_on_another_stream(given):
    """The state's workspace, allocated on one stream and used on another, is not handed out again before that use is over."""
    n_pages = 5003
    keep = [torch.empty(1, device=DEV)]
    side = torch.cuda.Stream()
    pages = binding.CachePages.new(3, 40, n_pages, 4, DEV)
    binding.polyspec_cache_reserve(pages, _i32([10, 20, 30]))
    size, at = pages.workspace().nbytes, pages.workspace().data_ptr()
    keep += [pages.table, pages.len, pages.refs, pages.free_bits]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(int(2e8))                         # a tenth of a second
        binding.polyspec_cache_compact(pages, stream=side if given else None)
    del pages
    again = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(4)]
    assert not side.query()
    assert at not in [x.data_ptr() for x in again]
    side.synchronize()


@pytest.mark.parametrize("how", ["current", "external", "raw"])
def test_a_state_outlives_an_external_stream_it_was_used_on(how, monkeypatch):
    """Nothing is recorded for a stream that is not torch's: the state may be dropped after the stream is gone."""
    recorded = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: recorded.append(stream))
    both = Both(3, 8, 64, 4)
    both.reserve([10, 20, 30])
    handle, cudart = ctypes.c_ulonglong(0), torch.cuda.cudart()
    assert int(cudart.cudaStreamCreate(ctypes.addressof(handle))) == 0
    torch.cuda.synchronize()
    external = torch.cuda.ExternalStream(handle.value)
    if how == "current":
        with torch.cuda.stream(external):
            binding.polyspec_cache_compact(both.pages)
    else:
        binding.polyspec_cache_compact(both.pages, stream=external if how == "external" else handle.value)
    both.plain.compact()
    both.check(None)
    assert int(cudart.cudaStreamDestroy(handle.value)) == 0
    assert recorded == []
    side = torch.cuda.Stream()
    binding.polyspec_cache_compact(both.pages, stream=side)
    both.check(None)
    assert recorded == [side]
