"""The workspace of calls over shared prompts, without a GPU (see tests/recorder): the size for n rows serves every call of
at most n rows, and as well as that call's own size does."""

import ctypes as C
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

AT = 1 << 40                                             # an aligned address that nothing touches


def _run(heads, batch, calls, prompts=(60000,)):
    """[[op, rows, workspace for that many rows], ..] on a cache of `batch` sequences, the first behind the first prompt and so
    on: return code, size of the workspace and launches [(kernel, workgroups, threads of one), ..] of each."""
    from tests import recorder
    out = subprocess.run([sys.executable, os.path.abspath(__file__), recorder._runtime(), recorder.LIB],
                         input=json.dumps([heads, batch, calls, prompts]), capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr
    return [(rc, size, [(recorder._readable(n), int(x), int(t)) for n, x, _, t in ls]) for rc, size, ls in json.loads(out.stdout)]


def _ranges(call):
    """Return code and workgroups of the launch over the prompts' lists."""
    return call[0], [(n, x) for n, x, _ in call[2] if "spkv_prefix_few" in n or "spkv_prefix_split" in n]


def _main():
    rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)          # before the library: its names win
    lib = C.CDLL(sys.argv[2])
    i32, ptr = C.c_int32, C.c_void_p

    class Config(C.Structure):
        _fields_ = [("batch", i32), ("n_q_heads", i32), ("n_kv_heads", i32), ("head_dim", i32), ("window", i32),
                    ("page_tokens", i32), ("tau", C.c_float), ("max_context", i32), ("max_total_kept_tokens", C.c_int64)]

    heads, batch, calls, prompts = json.load(sys.stdin)
    lib.spkv_cache_required_bytes.restype = lib.spkv_prefix_workspace_bytes.restype = C.c_size_t

    def cache(n, counts):
        cfg = Config(n, heads, 8, 128, 128, 0, 0.5, 1 << 20, 1 << 23)
        h, need = ptr(), lib.spkv_cache_required_bytes(C.byref(cfg))
        assert lib.spkv_cache_create(C.byref(cfg), ptr(AT), C.c_size_t(need), None, C.byref(h)) == 0
        assert lib.spkv_append(h, ptr(AT), ptr(AT), ptr(AT), (i32 * (n + 1))(*[sum(counts[:b]) for b in range(n + 1)]), None) == 0
        kept = (i32 * (n * 8))(*[20000 if counts[0] > 1000 else 0] * (n * 8))
        rt.rec_device_bytes(kept, C.c_size_t(4 * len(kept)))
        lib.spkv_cache_stats(h, (C.c_byte * 4096)(), None, None)      # reads the lengths
        return h

    def taken():
        buf, got = C.create_string_buffer(1024), []
        while rt.rec_take(buf, 1024) >= 0:
            got.append(buf.value.decode().rsplit(" ", 3))
        return got

    p, c = cache(len(prompts), prompts), cache(batch, [5] * batch)
    member, zero, out = (i32 * batch)(*[b % len(prompts) for b in range(batch)]), C.c_float(0.0), []
    taken()
    for op, rows, of in calls:
        size = C.c_size_t(lib.spkv_prefix_workspace_bytes(p, C.c_int64(of)))
        if op == "join":                                  # one row of every sequence, the rest in the first
            rows -= batch - 1
            rc = lib.spkv_prefix_attention(p, c, member, ptr(AT), (i32 * (batch + 1))(*[0] + [rows + b for b in range(batch)]), 0, ptr(AT), ptr(AT),
                                           ptr(AT), None, zero, ptr(AT), size, None)
        else:
            assert rows == batch
            rc = lib.spkv_decode_attention_shared(c, p, member, ptr(AT), ptr(AT), None, zero, ptr(AT), size, None)
        out.append([rc, size.value, taken()])
    json.dump(out, sys.stdout)


ROWS = [1, 2, 7, 33, 100, 115, 200, 304, 334, 400, 457, 500, 511, 512, 513, 600, 1024, 2048, 3000, 4096]


@pytest.mark.parametrize("heads", [8, 32, 64, 128])
def test_the_size_for_more_rows_serves_fewer(heads):
    pairs = [(r, n) for n in ROWS for r in ROWS if r <= n]
    got = dict(zip(pairs, _run(heads, 1, [["join", r, n] for r, n in pairs])))
    for r, n in pairs:
        assert got[r, n][0] == 0 and got[r, n][1] >= got[r, r][1], (r, n)
        assert _ranges(got[r, n]) == _ranges(got[r, r]), (r, n)      # as many workgroups as with its own


@pytest.mark.parametrize("heads", [8, 32, 128])
@pytest.mark.parametrize("batch", [1, 100, 457, 512])
def test_a_decoding_step_in_a_workspace_for_questions(heads, batch):
    first, *others = _run(heads, batch, [["decode", batch, batch]] + [["decode", batch, n] for n in ROWS if n >= batch])
    assert first[0] == 0 and _ranges(first)[1][0][1] > 0
    assert [_ranges(x) for x in others] == [_ranges(first)] * len(others)


def test_less_than_one_range_is_refused():
    """Fewer ranges in a smaller workspace, down to one a list."""
    got = _run(32, 1, [["join", r, max(1, r // 8)] for r in (64, 65536)])
    assert got[0][0] == 0 and got[1][0] == -1


def _fit(rows, heads):
    """A launch has fewer than 2^32 threads: one of four elements of every output, rows filled up to workgroups of 256."""
    return rows * -(-heads // 8) * 256 < 1 << 32


@pytest.mark.parametrize("heads", [8, 24, 32, 128])
def test_more_rows_than_a_launch_holds(heads):
    most = ((1 << 24) - 1) // (heads // 8)
    assert _fit(most, heads) and not _fit(most + 1, heads)
    fits, more = _run(heads, 1, [["join", most, most], ["join", most + 1, most]])
    assert fits[0] == 0 and fits[1] > 0 and len(fits[2]) == 2 and all(x * t < 1 << 32 for _, x, t in fits[2])
    assert more[0] == -1 and more[2] == []
    assert _run(heads, 1, [["join", 1, most + 1]])[0][1] == 0          # no size either


def test_more_workgroups_than_a_launch_holds():
    """Many prompts, whose lists all have as many blocks of columns as the widest one."""
    rows = 1 << 21
    few, many = _run(32, 40, [["join", rows, rows]], prompts=[70] * 20)[0], _run(32, 40, [["join", rows, rows]], prompts=[70] * 40)[0]
    assert few[0] == 0 and all(x * t < 1 << 32 for _, x, t in few[2])
    assert many[0] == -1 and many[2] == []


if __name__ == "__main__":
    _main()
