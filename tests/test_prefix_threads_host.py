"""Threads that serve different caches behind one prompts' cache: its lengths are read back once, by one of them, while the
others wait.  Without a GPU: the library's host code against the recording runtime (see tests/recorder), with a copy
to the host that takes its time and launches that each thread may issue for itself."""

import ctypes as C
import os
import subprocess
import sys
import threading

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

SLOW = r"""
#include <atomic>
#include <cstdint>
#include <cstring>
#include <unistd.h>
struct Dim3 { uint32_t x, y, z; };
static std::atomic<int> reads{0};
static thread_local Dim3 grid, block;
static thread_local size_t shared;
static thread_local void* stream;
extern "C" {
int slow_reads() { return reads.load(); }
int hipMemcpy(void* to, const void*, size_t n, int) {
    reads.fetch_add(1);
    usleep(300000);
    memset(to, 0, n);
    return 0;
}
int __hipPushCallConfiguration(Dim3 g, Dim3 b, size_t n, void* s) { grid = g, block = b, shared = n, stream = s; return 0; }
int __hipPopCallConfiguration(Dim3* g, Dim3* b, size_t* n, void** s) { *g = grid, *b = block, *n = shared, *s = stream; return 0; }
int hipLaunchKernel(const void*, Dim3, Dim3, void**, size_t, void*) { return 0; }
}
"""
AT = 1 << 40                                             # an aligned address that nothing touches


def test_lengths_of_a_fresh_prompt_are_read_once(tmp_path):
    from tests import recorder
    source, slow = tmp_path / "slow.cpp", tmp_path / "slow.so"
    source.write_text(SLOW)
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-std=c++17", str(source), "-o", str(slow)], check=True)
    for decode in "01":
        out = subprocess.run([sys.executable, os.path.abspath(__file__), str(slow), recorder._runtime(), recorder.LIB, decode],
                             capture_output=True, text=True, timeout=120)
        assert out.returncode == 0, out.stderr
        assert out.stdout.split() == ["0"] * 6 + ["1"], out.stdout


def _main():
    """Six threads ask behind one fresh prompt: their return codes, then the read-backs."""
    slow = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)        # the first with a name wins
    C.CDLL(sys.argv[2], mode=C.RTLD_GLOBAL)
    lib = C.CDLL(sys.argv[3])
    i32, ptr = C.c_int32, C.c_void_p

    class Config(C.Structure):
        _fields_ = [("batch", i32), ("n_q_heads", i32), ("n_kv_heads", i32), ("head_dim", i32), ("window", i32),
                    ("page_tokens", i32), ("tau", C.c_float), ("max_context", i32), ("max_total_kept_tokens", C.c_int64)]

    lib.spkv_cache_required_bytes.restype = lib.spkv_prefix_workspace_bytes.restype = C.c_size_t

    def cache(tokens):
        cfg, h = Config(1, 32, 8, 128, 128, 0, 0.5, 1 << 20, 1 << 23), ptr()
        assert lib.spkv_cache_create(C.byref(cfg), ptr(AT), C.c_size_t(lib.spkv_cache_required_bytes(C.byref(cfg))), None, C.byref(h)) == 0
        assert lib.spkv_append(h, ptr(AT), ptr(AT), ptr(AT), (i32 * 2)(0, tokens), None) == 0
        return h

    own, prompt = [cache(5) for _ in range(6)], cache(60000)
    member, zero = (i32 * 1)(0), C.c_float(0.0)
    size = C.c_size_t(lib.spkv_prefix_workspace_bytes(prompt, C.c_int64(1)))
    start, codes, before = threading.Barrier(6), [None] * 6, slow.slow_reads()

    def serve(i):
        start.wait()
        if sys.argv[4] == "1":
            codes[i] = lib.spkv_decode_attention_shared(own[i], prompt, member, ptr(AT), ptr(AT), None, zero, ptr(AT), size, None)
        else:
            codes[i] = lib.spkv_prefix_attention(prompt, own[i], member, ptr(AT), None, 1, ptr(AT), ptr(AT), ptr(AT), None, zero,
                                                 ptr(AT), size, None)

    threads = [threading.Thread(target=serve, args=(i,)) for i in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    print(*codes, slow.slow_reads() - before)


if __name__ == "__main__":
    _main()
