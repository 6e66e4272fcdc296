"""What the calls on branching sequences refuse, launch and count, without a GPU (see tests/recorder: the library's host
code against a HIP runtime that writes launches down)."""

import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

AT = 1 << 40                                             # an aligned address that nothing touches
KEEP, EMPTY = -1, -2


def _fed(on, kept):
    """Every head of a sequence holds as many kept pairs, and the host knows it."""
    return [["append", dict(on=on, counts=[max(row) + 128 for row in kept])], ["lengths", dict(on=on, kept=[n for row in kept for n in row])]]


def _run(configs, script):
    from tests import recorder
    out = subprocess.run([sys.executable, os.path.abspath(__file__), recorder._runtime(), recorder.LIB],
                         input=json.dumps([configs, script]), capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr
    return [(rc, [(recorder._readable(n), int(x), int(b)) for n, x, _, b in ls]) for rc, ls in json.loads(out.stdout)]


def _main():
    """Runs one script, [[op, args], ..] on the caches "a" and "b", and prints [[rc, launches], ..]."""
    rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)          # before the library: its names win
    lib = C.CDLL(sys.argv[2])

    class Config(C.Structure):
        _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                    ("window", C.c_int32), ("page_tokens", C.c_int32), ("tau", C.c_float), ("max_context", C.c_int32),
                    ("max_total_kept_tokens", C.c_int64)]

    configs, script = json.load(sys.stdin)
    handles, cfgs = {}, {}
    lib.spkv_cache_required_bytes.restype = C.c_size_t
    for name, config in zip("ab", configs):
        cfgs[name] = Config(**{**dict(batch=3, n_q_heads=32, n_kv_heads=8, head_dim=128, window=128, page_tokens=0, tau=0.5,
                                      max_context=1 << 16, max_total_kept_tokens=1 << 20), **config})
        handles[name] = C.c_void_p()
        need = lib.spkv_cache_required_bytes(C.byref(cfgs[name]))
        assert lib.spkv_cache_create(C.byref(cfgs[name]), C.c_void_p(AT), C.c_size_t(need), None, C.byref(handles[name])) == 0

    def ints(x):
        return None if x is None else (C.c_int32 * max(len(x), 1))(*x)

    def cu(counts):
        return None if counts is None else ints([sum(counts[:b]) for b in range(len(counts) + 1)])

    def taken():
        buf, got = C.create_string_buffer(1024), []
        while rt.rec_take(buf, 1024) >= 0:
            got.append(buf.value.decode().rsplit(" ", 3))
        return got

    taken()
    calls, ptr = [], C.c_void_p
    for op, a in script:
        who = handles.get(a.get("on", "a"))
        if op == "append":
            rc = lib.spkv_append(who, ptr(AT), ptr(AT), ptr(AT), cu(a["counts"]), None)
        elif op == "lengths":
            x = ints(a["kept"])
            rt.rec_device_bytes(x, C.c_size_t(4 * len(x)))
            rc = lib.spkv_cache_stats(who, (C.c_byte * 4096)(), None, None)
        elif op == "later":                               # what the next read-back of lengths finds
            x = ints(a["kept"])
            rt.rec_device_bytes(x, C.c_size_t(4 * len(x)))
            rc = 0
        elif op == "capture":
            rt.rec_capture(a["status"], 0)
            rc = 0
        elif op == "sync_error":                          # what waiting for a stream returns
            rt.rec_sync_error(a["error"])
            rc = 0
        elif op == "steps":
            n = C.c_int64()
            rc = lib.spkv_cache_safe_steps(who, None, C.byref(n))
            rc = n.value if rc == 0 else rc
        elif op == "fork":
            rc = lib.spkv_cache_fork(who, handles.get(a.get("of")), ints(a["source"]), None)
        elif op == "gather":
            rc = lib.spkv_cache_gather(who, ints(a.get("which")), a.get("n", 3), C.c_int64(a.get("rows", 10)), ptr(a.get("k", AT)),
                                       ptr(a.get("v", AT)), ptr(a.get("f", AT)), ptr(a.get("p", AT)), ptr(a.get("counts", AT)), None)
        elif op == "rows":
            rc = lib.spkv_append_rows(who, ptr(a.get("k", AT)), ptr(a.get("v", AT)), ptr(a.get("f", AT)), ptr(a.get("rows", AT)),
                                      a.get("n_rows", 100), cu(a["counts"]), None)
        elif op == "tree":
            rc = lib.spkv_score_tree(who, ptr(a.get("k", AT)), ptr(a.get("v", AT)), ptr(a.get("f", AT)), ptr(a.get("q", AT)),
                                     ptr(a.get("parents", AT)), cu(a["counts"]), ptr(a.get("out", AT)), ptr(a.get("lse", 0)),
                                     C.c_float(0.0), None)
        else:
            raise ValueError(op)
        calls.append([rc, taken()])
    json.dump(calls, sys.stdout)


FED = [["append", dict(counts=[9000, 50, 0])], ["lengths", dict(kept=[2000] * 8 + [0] * 16)]]


@pytest.mark.parametrize("bad", [dict(on="none"), dict(source=None), dict(source=[0, 3, 1]), dict(source=[-3, 0, 1])])
def test_forks_that_are_refused(bad):
    assert _run([{}], FED + [["fork", dict(source=[0, 0, 0], **bad) if "source" not in bad else bad]])[-1] == (-1, [])


@pytest.mark.parametrize("other", [dict(n_q_heads=16), dict(n_kv_heads=4), dict(head_dim=64), dict(window=64)])
def test_forks_from_caches_of_other_shapes(other):
    assert _run([{}, other], FED + [["fork", dict(of="b", source=[0, 0, 0])]])[-1] == (-1, [])


def test_launches_of_a_fork():
    def launches(source, of=None):
        rc, got = _run([{}, {}], FED + [["append", dict(on="b", counts=[9000, 50, 0])],
                                        ["lengths", dict(on="b", kept=[2000] * 8 + [0] * 16)], ["fork", dict(of=of, source=source)]])[-1]
        assert rc == 0
        return [n for n, _, _ in got]

    move, pages, assign = "spkv_fork_move", "spkv_fork_pages<128>", "spkv_fork_assign"
    assert launches([KEEP, 1, KEEP]) == []                   # nothing to do
    assert launches([1, 0, KEEP]) == [move]                  # pages change hands
    assert launches([EMPTY, EMPTY, 0]) == [move]
    assert launches([KEEP, KEEP, 0]) == [move, assign, pages]         # a copy, of many pages
    assert launches([KEEP, KEEP, 1]) == [move]               # of a sequence that is all window
    assert launches([2, 0, 0]) == [move, assign, pages]      # one takes the pages, one has copies
    assert launches([0, 1, 2], of="b") == [move, pages]      # of another cache always; into the pages at hand
    assert launches([KEEP, KEEP, 0], of="b") == [move, assign, pages]
    assert launches([1, EMPTY, 2], of="b") == [move]


def test_short_sequences_are_copied_in_one_launch():
    """Up to 64 workgroups of 128 KB each; not where a sequence that is replaced is a source, nor where only windows are copied."""
    def launches(kept, source, batch=3, **cfg):
        fed = [["append", dict(counts=[9000, 50] + [0] * (batch - 2))], ["lengths", dict(kept=[kept] * 8 + [0] * 8 * (batch - 1))]]
        return _run([dict(batch=batch, **cfg)], fed + [["fork", dict(source=source)]])[-1][1]
    few = lambda wide: [("spkv_fork_few<128>", wide, 256)]                    # noqa: E731
    assert launches(300, [KEEP, KEEP, 0]) == few(8)                           # 7 pages of 32 KB: 5, and 2 of the window
    assert launches(300, [KEEP, 0, EMPTY]) == few(4)
    assert launches(30 * 64, [KEEP, KEEP, 0]) == few(8)                       # 32 pages: four a workgroup
    assert [n for n, _, _ in launches(30 * 64 + 1, [KEEP, KEEP, 0])] == ["spkv_fork_move", "spkv_fork_pages<128>"]
    assert [n for n, _, _ in launches(300, [1, 0, 0])] == ["spkv_fork_move", "spkv_fork_pages<128>"]
    assert [n for n, _, _ in launches(300, [KEEP, KEEP, 1])] == ["spkv_fork_move"]
    assert launches(100, [KEEP] + [0] * 8, batch=9) == few(1)
    assert [n for n, _, _ in launches(100, [KEEP] + [0] * 9, batch=10)] == ["spkv_fork_move", "spkv_fork_pages<128>"]


def test_one_launch_only_where_the_pool_holds_what_goes_beside_what_comes():
    """The one launch gives pages back when the copies have theirs; a pool that holds the result, but not both at once, takes two."""
    move, pages, few = "spkv_fork_move", "spkv_fork_pages<128>", "spkv_fork_few<128>"

    def launches(cfg, kept, fork, other=None, other_kept=None):
        script = _fed("a", kept) + (_fed("b", other_kept) if other is not None else [])
        rc, got = _run([cfg] + ([other] if other is not None else []), script + [["fork", fork]])[-1]
        return rc, [n for n, _, _ in got]

    # one sequence ends, a short one is taken twice: 80 pages are in use in the end, 160 at once
    kept = [[300] * 8, [640] * 8, [0] * 8]                   # 5 and 10 pages a head, 120 in all; 40 are copied
    less = [[300] * 8, [500] * 8, [0] * 8]                   # (8 instead of 10: as many as the one launch gives back)
    turn = dict(source=[KEEP, EMPTY, 0])
    assert launches(dict(max_total_kept_tokens=7520), kept, turn) == (0, [move, pages])            # 118 + 24 pages
    assert launches(dict(max_total_kept_tokens=64 * (159 - 24)), kept, turn) == (0, [move, pages])
    assert launches(dict(max_total_kept_tokens=64 * (143 - 24)), less, turn) == (0, [move, pages])
    assert launches(dict(max_total_kept_tokens=64 * (144 - 24)), less, turn) == (0, [few])
    # two sequences that become others of another cache: one grows by as much as the other shrinks
    heads = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64)
    two = [[300] * 2, [900] * 2]                             # 5 and 15 pages a head, 40 in all
    near = [[300] * 2, [832] * 2]                            # 5 and 13
    swap = dict(source=[1, 0], of="b")
    move, pages, few = "spkv_fork_move", "spkv_fork_pages<64>", "spkv_fork_few<64>"
    assert launches(dict(heads, max_total_kept_tokens=64 * 38), two, swap, heads, two) == (0, [move, pages])      # 42 pages; 60 at once
    assert launches(dict(heads, max_total_kept_tokens=64 * 55), two, swap, heads, two) == (0, [move, pages])
    assert launches(dict(heads, max_total_kept_tokens=64 * 47), near, swap, heads, near) == (0, [move, pages])
    assert launches(dict(heads, max_total_kept_tokens=64 * 48), near, swap, heads, near) == (0, [few])
    # a slot given up for a sequence of as many pages
    one = dict(heads, n_q_heads=4, n_kv_heads=1)
    assert launches(dict(one, max_total_kept_tokens=640), [[700], [0]], dict(source=[EMPTY, 0], of="b"), one, [[700], [0]]) == (0, [move, pages])


def test_one_launch_only_where_it_gives_few_pages_back():
    """It does so with one thread a head; a head that gives up more than eight pages takes the two launches."""
    heads = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64)
    two, few = ["spkv_fork_move", "spkv_fork_pages<64>"], ["spkv_fork_few<64>"]

    def launches(kept, source):
        rc, got = _run([heads, heads], _fed("a", kept) + _fed("b", [[300] * 2, [0] * 2]) + [["fork", dict(source=source, of="b")]])[-1]
        assert rc == 0
        return [n for n, _, _ in got]

    assert launches([[59000] * 2, [0] * 2], [0, KEEP]) == two            # a short prompt in the place of a long conversation
    assert launches([[59000] * 2, [0] * 2], [EMPTY, 0]) == two           # or beside it
    assert launches([[59000] * 2, [0] * 2], [KEEP, 0]) == few            # nothing goes back
    assert launches([[13 * 64] * 2, [0] * 2], [0, KEEP]) == few          # 13 pages for 5
    assert launches([[0] * 2, [64, 13 * 64 + 1]], [KEEP, 0]) == two
    assert launches([[8 * 64] * 2, [0] * 2], [EMPTY, 0]) == few
    assert launches([[8 * 64, 8 * 64 + 1], [0] * 2], [EMPTY, 0]) == two


def test_a_few_pages_are_handed_out_by_the_copies():
    def launches(kept):
        return [n for n, _, _ in _run([{}], [["append", dict(counts=[9000, 50, 0])], ["lengths", dict(kept=[kept] * 8 + [0] * 16)],
                                             ["fork", dict(source=[KEEP, KEEP, 0])]])[-1][1]]
    assert launches(31 * 64) == ["spkv_fork_move", "spkv_fork_pages<128>"]
    assert launches(31 * 64 + 1) == ["spkv_fork_move", "spkv_fork_assign", "spkv_fork_pages<128>"]


def test_components_are_moved_side_by_side():
    """One workgroup row for each: a chain is one, sequences copied from one that stays are one each."""
    for source, n in (([KEEP, 0, 0], 2), ([1, 2, 0], 1), ([EMPTY, 0, 1], 1), ([EMPTY, EMPTY, EMPTY], 3)):
        assert _run([{}], FED + [["fork", dict(source=source)]])[-1][1][0][1] == n


def test_a_fork_under_capture_is_refused():
    got = _run([{}], FED + [["capture", dict(status=1)], ["fork", dict(source=[1, 0, KEEP])], ["fork", dict(source=[0, KEEP, 2])]])
    assert got[-2] == (-2, []) and got[-1] == (0, [])


def test_a_pool_that_cannot_hold_the_copies():
    """Judged by the exact lengths, and nothing launched: 2000 kept pairs are 32 pages a head."""
    small = dict(max_total_kept_tokens=64 * 8 * 40)          # 320 pages, and one for every pair: 344
    fed = [["append", dict(counts=[2128, 50, 0])], ["lengths", dict(kept=[2000] * 8 + [0] * 16)]]
    assert _run([small], fed + [["fork", dict(source=[KEEP, 0, KEEP])]])[-1] == (-3, [])
    assert _run([small], fed + [["fork", dict(source=[EMPTY, 0, KEEP])]])[-1][0] == 0
    got = _run([small], fed + [["later", dict(kept=[1000] * 8 + [0] * 16)], ["fork", dict(source=[KEEP, 0, KEEP])]])
    assert got[-1][0] == 0                                   # (it was the bound that did not fit)


def test_contexts_that_are_too_long():
    assert _run([dict(max_context=8000), {}], [["append", dict(on="b", counts=[9000, 50, 0])], ["fork", dict(of="b", source=[0, KEEP, KEEP])]])[-1] == (-3, [])
    assert _run([dict(max_context=8000), {}], [["append", dict(on="b", counts=[9000, 50, 0])], ["fork", dict(of="b", source=[1, 1, 2])]])[-1][0] == 0


def test_token_counts_follow_the_sequences():
    cfg = dict(max_context=10000)
    steps = ["steps", {}]
    got = _run([cfg], FED + [steps, ["fork", dict(source=[EMPTY, 0, KEEP])], steps, ["fork", dict(source=[KEEP, EMPTY, 1])], steps,
                             ["fork", dict(source=[EMPTY, EMPTY, EMPTY])], ["later", dict(kept=[0] * 24)], steps])
    assert [rc for rc, _ in got[2::2][:3]] == [1000] * 3 and got[-1][0] == 10000


@pytest.mark.parametrize("bad", [dict(on="none"), dict(n=-1), dict(n=4), dict(rows=-1), dict(rows=1 << 31), dict(which=[0, 1, 3]),
                                 dict(which=[0, -1, 1]), dict(k=AT + 8), dict(v=AT + 8), dict(f=AT + 4), dict(p=AT + 4), dict(counts=AT + 8),
                                 dict(n=513, which=[0] * 513)])
def test_gathers_that_are_refused(bad):
    assert _run([{}], FED + [["gather", bad]])[-1] == (-1, [])


def test_gathers_that_are_not():
    got = _run([{}], FED + [["gather", {}], ["gather", dict(n=5, which=[0, 0, 2, 1, 0], k=0, v=0, f=0, p=0)], ["gather", dict(n=0)],
                            ["gather", dict(rows=0)]])[2:]
    assert [(rc, [n for n, _, _ in ls]) for rc, ls in got] == [(0, ["spkv_gather_pairs<128>"])] * 2 + [(0, []), (0, ["spkv_gather_pairs<128>"])]


@pytest.mark.parametrize("bad,code", [
    (dict(on="none"), -1), (dict(k=0), -1), (dict(v=0), -1), (dict(f=0), -1), (dict(rows=0), -1), (dict(n_rows=0), -1), (dict(k=AT + 2), -1),
    (dict(rows=AT + 4), -1), (dict(counts=None), -1), (dict(counts=[1, 65, 0]), -1), (dict(counts=[1, -1, 0]), -1),
    (dict(counts=[0, 64, 0], on="b"), -3)])
def test_appends_of_rows_that_are_refused(bad, code):
    fed = FED + [["append", dict(on="b", counts=[0, 37, 0])]]
    assert _run([{}, dict(max_context=100)], fed + [["rows", {**dict(counts=[1, 2, 0]), **bad}]])[-1] == (code, [])


def test_appends_of_rows():
    got = _run([{}], FED + [["rows", dict(counts=[1, 64, 0])], ["rows", dict(counts=[0, 0, 0], k=0, rows=0)]])[2:]
    assert got == [(0, [("spkv_append_rows<128>", 24, 256)]), (0, [])]


@pytest.mark.parametrize("bad", [
    dict(on="none"), dict(counts=None), dict(counts=[0, 65, 0]), dict(counts=[3, -1, 1]), dict(k=0), dict(v=0), dict(q=0), dict(parents=0),
    dict(out=0), dict(k=AT + 8), dict(v=AT + 2), dict(f=AT + 4), dict(q=AT + 8), dict(parents=AT + 4), dict(out=AT + 8), dict(lse=AT + 4),
    dict(on="b", f=0, counts=[0, 21, 0])])
def test_trees_that_are_refused(bad):
    assert _run([{}, dict(window=20)], FED + [["tree", {**dict(counts=[1, 2, 0]), **bad}]])[-1] == (-1, [])


# half-pages of lists, columns: kernel.  Lists of nothing, short ones in ranges, long ones; 24 lists or 256.
def _tree(kept, n, batch=3, **kw):
    fed = [["append", dict(counts=[60000 if kept > 200 else kept + 128] + [3] * (batch - 1))], ["lengths", dict(kept=[kept] * 8 * batch)]]
    return _run([dict(batch=batch, **kw)], fed + [["tree", dict(counts=[n] + [1] * (batch - 1))]])[-1]


@pytest.mark.parametrize("n,kernel,threads", [(1, "few<128, 1, 4", 256), (4, "few<128, 1, 4", 256), (5, "few<128, 2, 4", 256), (8, "few<128, 2, 4", 256),
                                              (9, "split<128, 2", 128), (16, "split<128, 2", 128), (17, "split<128, 4", 256),
                                              (32, "split<128, 4", 256), (33, "split<128, 8", 512), (64, "split<128, 8", 512)])
def test_launches_of_a_tree(n, kernel, threads):
    """A workgroup as wide as the largest tree asks: the lists in ranges, and a join."""
    rc, got = _tree(2000, n)
    assert rc == 0 and len(got) == 2 and got[1][0].startswith("spkv_tree_merge<128, ")
    assert got[0][0] == f"spkv_tree_{kernel}, 0>" and got[0][2] == threads
    assert 200 <= got[0][1] <= 24 + 1024                  # ranges as many as a round of the chip, four at most


@pytest.mark.parametrize("n,kernel,threads,many,many_threads", [
    (4, "few<128, 1, 8", 512, "few<128, 1, 4", 256), (8, "few<128, 2, 8", 512, "few<128, 2, 4", 256),
    (16, "own_copies<128", 512, "split<128, 2", 128), (32, "split<128, 4", 256, "split<128, 4", 256), (64, "split<128, 8", 512, "split<128, 8", 512)])
def test_short_lists_take_one_launch(n, kernel, threads, many, many_threads):
    """Where whole lists take no longer than ranges of them and a join: one workgroup a list, whose results are final; of eight
    waves while there is one to a compute unit."""
    assert _tree(40, n, batch=24) == (0, [(f"spkv_tree_{kernel}, 1>", 192, threads)])
    assert _tree(40, n, batch=64, max_total_kept_tokens=1 << 22) == (0, [(f"spkv_tree_{many}, 1>", 512, many_threads)])


def test_launches_of_a_tree_over_long_lists():
    """33 to 64 columns take another kernel where the lists are long."""
    for n, kernel, threads, rounds in ((4, "few<128, 1, 4", 256, 4), (8, "few<128, 2, 4", 256, 4), (9, "own_copies<128", 512, 1),
                                       (16, "own_copies<128", 512, 1), (17, "split<128, 4", 256, 4), (64, "split<128, 8", 512, 4)):
        rc, got = _tree(20000, n)
        assert rc == 0 and [g[0].split("<")[0] for g in got][1:] == ["spkv_tree_merge"]
        assert got[0][0] == f"spkv_tree_{kernel}, 0>" and got[0][2] == threads
        assert 200 <= got[0][1] <= 256 * rounds + 24


def test_a_first_tree_after_a_prompt_is_not_captured():
    """It waits for the lengths, which a capture refuses; once they are known it may be."""
    prompt, tree = ["append", dict(counts=[9000, 50, 0])], ["tree", dict(counts=[4, 4, 4])]
    refused = [["capture", dict(status=1)], ["sync_error", dict(error=900)]]
    assert _run([{}], [prompt] + refused + [tree])[-1] == (-4, [])
    rc, launches = _run([{}], [prompt, ["lengths", dict(kept=[2000] * 8 + [0] * 16)]] + refused + [tree])[-1]
    assert rc == 0 and launches


def test_trees_that_are_empty():
    assert _run([{}], FED + [["tree", dict(counts=[0, 0, 0], k=0, q=0)]])[-1] == (0, [])
    assert _run([dict(window=20)], FED + [["tree", dict(counts=[20, 0, 3], f=0)]])[-1][0] == 0


def test_trees_of_many_pairs_take_several_launches():
    cfg = dict(batch=200, n_q_heads=8, n_kv_heads=4, head_dim=64, max_context=500, max_total_kept_tokens=100000)
    rc, got = _run([cfg], [["append", dict(counts=[5] * 200)], ["lengths", dict(kept=[0] * 800)], ["tree", dict(counts=[1] * 200)]])[-1]
    assert rc == 0 and [n.split("<")[0] for n, _, _ in got] == ["spkv_tree_few"] * 2
    # as many columns as there are, on as many pairs: what does not fit the partial results' room
    cfg = dict(batch=512, n_q_heads=512, n_kv_heads=32, head_dim=64, max_context=200, max_total_kept_tokens=1000)
    rc, got = _run([cfg], [["tree", dict(counts=[64] * 512)]])[-1]
    assert rc == 0 and len(got) >= 32
    rc, got = _run([cfg], [["tree", dict(counts=[64] + [0] * 511)]])[-1]
    assert rc == 0 and len(got) in (1, 2)


def test_another_device(monkeypatch):
    """Calls while another device than the cache's is the current one, caches of two devices, tensors that lie elsewhere."""
    import torch

    import paper_2605_14037_amd as spkv
    a, b = (object.__new__(spkv.SPKVCache) for _ in range(2))
    a.index, b.index = 1, 0
    a.cfg = b.cfg = spkv.SPKVConfig(1, 2, 1, 64, 128, 0, 0.5, 100, 100)
    a.lib = b.lib = None
    a.handle = b.handle = None
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        a._stream()
    with pytest.raises(ValueError, match="other: on cuda:0"):
        a.fork([0], b)
    with pytest.raises(ValueError, match="on cuda:1"):
        a.score_tree(*(torch.zeros(1, h, 64, dtype=torch.bfloat16) for h in (1, 1, 2)), torch.zeros(1, dtype=torch.int32), (C.c_int32 * 2)(0, 1))
    with pytest.raises(ValueError, match="out.0.*on cuda:1"):
        a.gather(out=[torch.zeros(1, 1, 3, 64)] * 2 + [torch.zeros(1, 1, 3)] * 2 + [torch.zeros(1, 1)])


if __name__ == "__main__":
    _main()
