"""What the calls over shared prompts refuse, and what they launch, without a GPU (see tests/recorder: the library's
host code against a HIP runtime that writes launches down)."""

import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

AT = 1 << 40                                             # an aligned address that nothing touches


def _run(prompts, cache, script):
    from tests import recorder
    out = subprocess.run([sys.executable, os.path.abspath(__file__), recorder._runtime(), recorder.LIB],
                         input=json.dumps([prompts, cache, script]), capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr
    return [(rc, [(recorder._readable(n), int(x), int(b)) for n, x, _, b in ls]) for rc, ls in json.loads(out.stdout)]


def _main():
    """Runs one script, [[op, args], ..] on the caches "p" (prompts) and "c", and prints [[rc, launches], ..]."""
    rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)          # before the library: its names win
    lib = C.CDLL(sys.argv[2])

    class Config(C.Structure):
        _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                    ("window", C.c_int32), ("page_tokens", C.c_int32), ("tau", C.c_float), ("max_context", C.c_int32),
                    ("max_total_kept_tokens", C.c_int64)]

    configs = json.load(sys.stdin)
    script, handles, cfgs = configs.pop(), {}, {}
    lib.spkv_cache_required_bytes.restype = lib.spkv_prefix_workspace_bytes.restype = C.c_size_t
    for name, config in zip("pc", configs):
        cfgs[name] = Config(**{**dict(n_q_heads=32, n_kv_heads=8, head_dim=128, window=128, page_tokens=0, tau=0.5,
                                      max_context=1 << 20, max_total_kept_tokens=1 << 23), **config})
        handles[name] = C.c_void_p()
        need = lib.spkv_cache_required_bytes(C.byref(cfgs[name]))
        assert lib.spkv_cache_create(C.byref(cfgs[name]), C.c_void_p(AT), C.c_size_t(need), None, C.byref(handles[name])) == 0

    def ints(x):
        return None if x is None else (C.c_int32 * len(x))(*x)

    def cu(counts):
        return None if counts is None else ints([sum(counts[:b]) for b in range(len(counts) + 1)])

    def taken():
        buf, got = C.create_string_buffer(1024), []
        while rt.rec_take(buf, 1024) >= 0:
            got.append(buf.value.decode().rsplit(" ", 3))
        return got

    taken()
    calls, ptr, zero = [], C.c_void_p, C.c_float(0.0)
    for op, a in script:
        who = {n: None if a.get(n) == "null" else handles[a.get(n, n)] for n in "pc"}
        ws = a.get("ws", AT)
        rows = sum(a["counts"]) if a.get("counts") else cfgs[a.get("c", "c") if a.get("c") != "null" else "c"].batch
        size = C.c_size_t(a.get("bytes", lib.spkv_prefix_workspace_bytes(handles["p"], C.c_int64(max(rows, 1)))))
        if op == "append":
            rc = lib.spkv_append(handles[a["to"]], ptr(AT), ptr(AT), ptr(AT), cu(a["counts"]), None)
        elif op == "lengths":
            x = ints(a["kept"])
            rt.rec_device_bytes(x, C.c_size_t(4 * len(x)))
            rc = lib.spkv_cache_stats(handles[a["of"]], (C.c_byte * 4096)(), None, None)
        elif op == "decode":
            rc = lib.spkv_decode_attention_shared(who["c"], who["p"], ints(a["member"]), ptr(a.get("q", AT)), ptr(a.get("out", AT)),
                                                  ptr(a.get("lse", 0)), zero, ptr(ws), size, None)
        else:
            rc = lib.spkv_prefix_attention(who["p"], who["c"], ints(a["member"]), ptr(a.get("q", AT)), cu(a.get("counts")),
                                           a.get("appended", 1), ptr(a.get("own", AT)), ptr(a.get("own_lse", AT)),
                                           ptr(a.get("out", AT)), ptr(a.get("lse", 0)), zero, ptr(ws), size, None)
        calls.append([rc, taken()])
    json.dump(calls, sys.stdout)


FED = [["append", dict(to="p", counts=[9000, 50])], ["lengths", dict(of="p", kept=[2000] * 8 + [0] * 8)],
       ["append", dict(to="c", counts=[40, 3, 7])], ["lengths", dict(of="c", kept=[0] * 24)]]


@pytest.mark.parametrize("op", ["decode", "join"])
@pytest.mark.parametrize("bad,code", [
    (dict(p="null"), -1), (dict(c="null"), -1), (dict(member=None), -1), (dict(member=[0, 2, 1]), -1), (dict(member=[0, -2, 1]), -1),
    (dict(q=0), -1), (dict(q=AT + 8), -1), (dict(out=0), -1), (dict(out=AT + 2), -1), (dict(lse=AT + 4), -1), (dict(ws=0), -1),
    (dict(ws=AT + 128), -1), (dict(bytes=0), -1), (dict(bytes=50000), -1), (dict(p="c", member=[0, 0, 0]), -1)])
def test_refusals(op, bad, code):
    args = {"member": [0, 1, -1], **bad}
    got = _run(dict(batch=2), dict(batch=3), FED + [[op, args]])[-1]
    assert got[0] == code and not any("prefix" in n for n, _, _ in got[1])


@pytest.mark.parametrize("bad,code", [
    (dict(own=0), -1), (dict(own_lse=0), -1), (dict(own=AT + 4), -1), (dict(own_lse=AT + 8), -1), (dict(counts=[1, 4, 1]), -2),
    (dict(counts=[41, 1, 1]), -2), (dict(counts=[1 << 24, 1 << 24, 1 << 24], appended=0), -1), (dict(counts=[2, -1, 1]), -1)])
def test_refusals_of_the_join(bad, code):
    assert _run(dict(batch=2), dict(batch=3), FED + [["join", dict(member=[0, 1, -1], **bad)]])[-1][0] == code


@pytest.mark.parametrize("other", [dict(n_q_heads=16), dict(n_kv_heads=4), dict(head_dim=64), dict(window=64)])
def test_caches_of_other_shapes(other):
    script = [["append", dict(to="p", counts=[9000, 50])], ["append", dict(to="c", counts=[4, 3, 7])], ["decode", dict(member=[0, 1, -1])]]
    assert _run(dict(batch=2), dict(batch=3, **other), script)[-1][0] == -1


def test_empty_sequences_and_empty_calls():
    script = [["append", dict(to="p", counts=[900])], ["append", dict(to="c", counts=[4, 0])]]
    got = _run(dict(batch=1), dict(batch=2), script + [["decode", dict(member=[0, 0])], ["join", dict(member=[0, 0], counts=[0, 0])],
                                                       ["join", dict(member=[0, 0], appended=0)]])
    assert got[2][0] == -2 and got[3] == (0, []) and got[4][0] == 0


def test_one_pass_over_the_lists_whatever_the_number_of_sequences():
    """A split and a merge launch; a workgroup as wide as the columns ask; no more workgroups than the chip holds."""
    few, split = "spkv_prefix_few<128, {}>", "spkv_prefix_split<128, {}>"
    for batch, name, waves in ((1, few.format(1), 4), (4, few.format(1), 4), (5, few.format(2), 4), (8, few.format(2), 4),
                               (9, split.format(2), 2), (16, split.format(2), 2), (17, split.format(4), 4),
                               (32, split.format(4), 4), (33, split.format(8), 8), (64, split.format(8), 8), (200, split.format(8), 8)):
        script = [["append", dict(to="p", counts=[60000])], ["lengths", dict(of="p", kept=[20000, 4000] * 4)],
                  ["append", dict(to="c", counts=[5] * batch)], ["lengths", dict(of="c", kept=[0] * 8 * batch)],
                  ["decode", dict(member=[0] * batch)]]
        rc, launches = _run(dict(batch=1), dict(batch=batch), script)[-1]
        mine = [x for x in launches if "prefix" in x[0]]
        assert rc == 0 and len(mine) == 2 and mine[1][0].startswith("spkv_prefix_merge<128"), launches
        assert mine[0][0] == name and mine[0][2] == 64 * waves
        own_items = (batch * 8 * 1 + waves - 1) // waves             # (40 tokens or fewer: one item a list)
        assert mine[0][1] - own_items <= 512


def test_prompts_without_tokens_are_not_visited():
    script = [["append", dict(to="p", counts=[0, 500])], ["append", dict(to="c", counts=[5] * 3)]]
    got = _run(dict(batch=2), dict(batch=3), script + [["join", dict(member=[0, -1, 0])], ["join", dict(member=[0, 1, 0])]])
    assert [n.split(",")[0] for n, _, _ in got[2][1]] == ["spkv_prefix_merge<128"]
    assert [n.split(",")[0] for n, _, _ in got[3][1]] == ["spkv_prefix_few<128", "spkv_prefix_merge<128"]


def test_own_lists_ride_in_the_prompts_launch_while_they_are_short():
    def launches(tokens, kept, options=()):
        script = [["append", dict(to="p", counts=[9000])], ["lengths", dict(of="p", kept=[2000] * 8)],
                  ["append", dict(to="c", counts=[tokens] * 2)], ["lengths", dict(of="c", kept=[kept] * 16)],
                  ["decode", dict(member=[0, 0])]]
        rc, got = _run(dict(batch=1), dict(batch=2), script)[-1]
        assert rc == 0
        return [n.split("<")[0] for n, _, _ in got if "copy" not in n]

    assert launches(5000, 60 * 32) == ["spkv_prefix_few", "spkv_prefix_merge"]
    assert launches(5000, 60 * 32 + 1) == ["spkv_decode_split", "spkv_decode_combine", "spkv_prefix_few", "spkv_prefix_merge"]


@pytest.mark.parametrize("asking,launches", [(1, 2), (64, 2), (65, 3)])
def test_rows_of_up_to_64_sequences_travel_with_the_launch(asking, launches):
    """More tokens a sequence: a table on the device, in a launch before, from more sequences with rows and a prompt on."""
    script = [["append", dict(to="p", counts=[9000])], ["append", dict(to="c", counts=[5] * 100)],
              ["join", dict(member=[0] * asking + [-1] * (100 - asking), counts=[3] * 100)],
              ["join", dict(member=[0] * 100, counts=[3] * asking + [0] * (100 - asking))],
              ["join", dict(member=[-1] * 100, counts=[3] * 100)]]
    *asked, none = _run(dict(batch=1), dict(batch=100), script)[2:]
    for rc, got in asked:
        assert rc == 0 and len(got) == launches and (got[0][0] == "spkv_prefix_rows") == (launches == 3), got
    assert none[0] == 0 and [n.split("<")[0] for n, _, _ in none[1]] == ["spkv_prefix_merge"]


if __name__ == "__main__":
    _main()
