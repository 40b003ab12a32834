"""CPU-only checks of the cache, attention and logits entry points: what the host refuses, and the arithmetic behind the kernels' addresses."""
import ctypes
import os
import subprocess
import tempfile

import pytest

from test_sanitizers import ENV, ROOT, SAN

FAKE = 0x10000000                                            # never dereferenced on the host


@pytest.fixture(scope="module")
def lib():
    from paper_2502_13652_amd import load_library
    return load_library()


def cache(**kw):
    from paper_2502_13652_amd.serving import _Cache
    a = dict(batch=2, layers=3, pages=40, page_size=16, kv_heads=2, head_dim=64, max_pages=8, dtype=1, k=FAKE, v=FAKE, page_table=FAKE, length=FAKE,
             refcount=FAKE, status=FAKE)
    a.update(kw)
    return _Cache(**a)


def attention(**kw):
    from paper_2502_13652_amd.serving import _Attention
    a = dict(q=FAKE, q_batch_stride=4 * 256, q_token_stride=256, out=FAKE, out_batch_stride=4 * 256, out_token_stride=256, lse=None, n_new=None,
             tokens=4, q_heads=4, layer=0, nodes=0, mask=None, scale=0.125)
    a.update(kw)
    return _Attention(**a)


def adjustments(**kw):
    from paper_2502_13652_amd.serving import _Adjustments
    return _Adjustments(**kw)


def test_cache_validation(lib):
    need = ctypes.c_size_t()
    ok = lambda **kw: lib.c2t_cache_workspace_bytes(ctypes.byref(cache(**kw)), ctypes.byref(need))
    assert ok() == 0 and need.value > 0 and ok(dtype=2, head_dim=256, page_size=256) == 0
    assert lib.c2t_cache_workspace_bytes(None, ctypes.byref(need)) == -1 and lib.c2t_cache_workspace_bytes(ctypes.byref(cache()), None) == -1
    for bad in (dict(batch=0), dict(layers=0), dict(pages=-1), dict(kv_heads=0), dict(max_pages=0), dict(dtype=3), dict(dtype=-1)) + \
            tuple({k: None} for k in ("k", "v", "page_table", "length", "refcount", "status")):
        assert ok(**bad) == -1, bad
    for big in (dict(dtype=0), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(page_size=0), dict(head_dim=32), dict(head_dim=96), dict(head_dim=512), dict(batch=4097),
                dict(kv_heads=1025), dict(layers=4097), dict(pages=1 << 27), dict(max_pages=(1 << 26) + 1), dict(k=FAKE + 8), dict(v=FAKE + 2)):
        assert ok(**big) == -2, big


def test_cache_calls_are_refused(lib):
    c = ctypes.byref(cache())
    for fn, args in ((lib.c2t_cache_reserve, (FAKE, FAKE, 1 << 20, None)), (lib.c2t_cache_write, (0, FAKE, FAKE, 512, 128, 4, None, None)),
                     (lib.c2t_cache_commit, (FAKE, 4, FAKE, None)), (lib.c2t_cache_truncate, (None, 0, None)), (lib.c2t_cache_fork, (FAKE, FAKE, 2, None))):
        assert fn(None, *args) == -1 and fn(ctypes.byref(cache(batch=0)), *args) == -1 and fn(ctypes.byref(cache(page_size=7)), *args) == -2
    assert lib.c2t_cache_reserve(c, None, FAKE, 1 << 20, None) == -1
    assert lib.c2t_cache_reserve(c, FAKE, None, 1 << 20, None) == -3
    assert lib.c2t_cache_reserve(c, FAKE, FAKE + 16, 1 << 20, None) == -3
    assert lib.c2t_cache_reserve(c, FAKE, FAKE, 8, None) == -3
    w = lib.c2t_cache_write
    assert w(c, 0, None, FAKE, 512, 128, 4, None, None) == -1 and w(c, 0, FAKE, None, 512, 128, 4, None, None) == -1
    assert w(c, 3, FAKE, FAKE, 512, 128, 4, None, None) == -1 and w(c, -1, FAKE, FAKE, 512, 128, 4, None, None) == -1
    assert w(c, 0, FAKE, FAKE, 512, 128, 0, None, None) == -1 and w(c, 0, FAKE, FAKE, 512, 120, 4, None, None) == -1
    assert w(c, 0, FAKE, FAKE, -8, 128, 4, None, None) == -1
    assert w(c, 0, FAKE + 4, FAKE, 512, 128, 4, None, None) == -2 and w(c, 0, FAKE, FAKE, 512, 132, 4, None, None) == -2
    assert w(c, 0, FAKE, FAKE, 516, 128, 4, None, None) == -2 and w(c, 0, FAKE, FAKE, 512, 1 << 41, 4, None, None) == -2
    assert w(c, 0, FAKE, FAKE, 512, 128, (1 << 24) + 1, None, None) == -2
    m = lib.c2t_cache_commit
    assert m(c, None, 4, FAKE, None) == -1 and m(c, FAKE, 4, None, None) == -1 and m(c, FAKE, 0, FAKE, None) == -1 and m(c, FAKE, 1026, FAKE, None) == -2
    assert lib.c2t_cache_truncate(c, None, -1, None) == -1
    f = lib.c2t_cache_fork
    assert f(c, None, FAKE, 1, None) == -1 and f(c, FAKE, None, 1, None) == -1 and f(c, FAKE, FAKE, 0, None) == -1 and f(c, FAKE, FAKE, 4097, None) == -2


def test_attention_is_refused(lib):
    c = ctypes.byref(cache())
    need = ctypes.c_size_t()
    size = lambda **kw: lib.c2t_attention_workspace_bytes(c, ctypes.byref(attention(**kw)), ctypes.byref(need))
    assert size() == 0 and need.value > 0
    assert lib.c2t_attention_workspace_bytes(c, None, ctypes.byref(need)) == -1 and lib.c2t_attention_workspace_bytes(c, ctypes.byref(attention()), None) == -1
    for bad in (dict(tokens=0), dict(q_heads=0), dict(q_heads=3), dict(nodes=-1), dict(nodes=5)):
        assert size(**bad) == -1, bad
    for big in (dict(nodes=1025, tokens=2000), dict(tokens=1 << 29), dict(tokens=1 << 27, q_heads=8)):
        assert size(**big) == -2, big
    many = cache(batch=4096, kv_heads=1024)                # more workgroups than a launch may have
    assert lib.c2t_attention_workspace_bytes(ctypes.byref(many), ctypes.byref(attention(q_heads=1024, tokens=800)), ctypes.byref(need)) == -2
    assert lib.c2t_cache_write(ctypes.byref(cache(kv_heads=1024)), 0, FAKE, FAKE, 0, 1 << 16, 1 << 22, None, None) == -2
    size()
    call = lambda ws=FAKE, n=None, **kw: lib.c2t_cache_attention(c, ctypes.byref(attention(**kw)), ws, need.value if n is None else n, None)
    for bad in (dict(q=None), dict(out=None), dict(layer=3), dict(layer=-1), dict(nodes=2), dict(mask=FAKE), dict(q_token_stride=248), dict(out_token_stride=0),
                dict(q_batch_stride=-8), dict(out_batch_stride=-8), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**bad) == -1, bad
    for big in (dict(q=FAKE + 8), dict(out=FAKE + 4), dict(q_token_stride=260), dict(q_batch_stride=1028), dict(out_token_stride=257), dict(out_batch_stride=4), dict(q_token_stride=1 << 41)):
        assert call(**big) == -2, big
    assert call(ws=None) == -3 and call(ws=FAKE + 128) == -3 and call(n=need.value - 1) == -3
    assert lib.c2t_cache_attention(None, ctypes.byref(attention()), FAKE, need.value, None) == -1 and lib.c2t_cache_attention(c, None, FAKE, need.value, None) == -1


def test_outputs_in_one_place_are_refused(lib):
    need = ctypes.c_size_t()
    c, one = cache(), cache(batch=1)
    assert lib.c2t_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(attention()), ctypes.byref(need)) == 0
    call = lambda c, **kw: lib.c2t_cache_attention(ctypes.byref(c), ctypes.byref(attention(**kw)), FAKE, need.value, None)
    for stride in (0, 8, 248):                               # sequences' rows on top of each other
        assert call(c, out_batch_stride=stride) == -1
    launched = (0, -5)                                       # (without a GPU a launch fails)
    import torch
    if not torch.cuda.is_available():
        assert call(one, out_batch_stride=0) in launched and call(c, out_batch_stride=256, out_token_stride=512) in launched and call(c, q_batch_stride=0) in launched


def test_adjustments_are_refused(lib):
    def call(t=None, batch=2, vocab=1000, nodes=4, dtype=1, tokens=FAKE, parent=FAKE, n_nodes=FAKE, logits=FAKE, stride=1000, out=FAKE, out_stride=1000):
        return lib.c2t_adjust_tree_logits(ctypes.byref(adjustments(**(t or {}))), batch, vocab, nodes, dtype, tokens, parent, n_nodes, logits, stride, out, out_stride, None)
    assert lib.c2t_adjust_tree_logits(None, 2, 1000, 4, 1, FAKE, FAKE, FAKE, FAKE, 1000, FAKE, 1000, None) == -1
    for bad in (dict(batch=0), dict(vocab=0), dict(nodes=-1), dict(dtype=7), dict(tokens=None), dict(parent=None), dict(n_nodes=None), dict(logits=None), dict(out=None),
                dict(stride=999), dict(out_stride=992), dict(out_stride=1008), dict(t=dict(tokens=FAKE, token_stride=5)), dict(t=dict(tokens=FAKE, n_tokens=FAKE)),
                dict(t=dict(bias=FAKE, bias_stride=4)), dict(t=dict(bias_tokens=FAKE, bias_stride=4)), dict(t=dict(bias=FAKE, bias_tokens=FAKE)),
                dict(t=dict(allowed=FAKE, allowed_row_stride=-1))):
        assert call(**bad) == -1, bad
    for big in (dict(dtype=2), dict(nodes=1025), dict(batch=65536), dict(vocab=(1 << 30) + 8, stride=1 << 31, out_stride=1 << 31), dict(logits=FAKE + 8), dict(out=FAKE + 2),
                dict(stride=1004, out=2 * FAKE), dict(out_stride=1004, out=2 * FAKE), dict(stride=1 << 41, out_stride=1 << 41),
                dict(t=dict(bias=FAKE, bias_tokens=FAKE, bias_stride=1025)), dict(t=dict(tokens=FAKE, n_tokens=FAKE, token_stride=(1 << 29) + 1)),
                dict(t=dict(allowed=FAKE, allowed_row_stride=1 << 41))):
        assert call(**big) == -2, big
    # of a context: its state is looked at last
    from test_library_abi import cfg
    need, ctx = ctypes.c_size_t(), ctypes.c_void_p()
    conf = cfg()
    assert lib.c2t_workspace_bytes(ctypes.byref(conf), ctypes.byref(need)) == 0
    assert lib.c2t_create(ctypes.byref(conf), ctypes.c_void_p(FAKE), need.value, ctypes.byref(ctx)) == 0
    t = adjustments()
    assert lib.c2t_adjust_logits(None, ctypes.byref(t), FAKE, 1000, FAKE, 1000, None) == -1
    assert lib.c2t_adjust_logits(ctx, None, FAKE, 1000, FAKE, 1000, None) == -1
    assert lib.c2t_adjust_logits(ctx, ctypes.byref(t), FAKE, 992, FAKE, 1000, None) == -1
    assert lib.c2t_adjust_logits(ctx, ctypes.byref(t), FAKE + 2, 1000, FAKE, 1000, None) == -2
    assert lib.c2t_adjust_logits(ctx, ctypes.byref(t), FAKE, 1000, FAKE, 1000, None) == -4      # before reset
    lib.c2t_destroy(ctx)


def test_two_threads_do_not_enqueue_between_each_others_kernels(monkeypatch):
    """A call of two kernels that share a workspace is enqueued whole, whichever thread makes it."""
    import threading
    import time
    import types

    import torch
    from paper_2502_13652_amd import PagedCache, serving
    inside, met = [], []

    def enqueue(*args):                                      # as ctypes does, it lets other threads run
        inside.append(args)
        time.sleep(0.002)
        met.append(len(inside))
        inside.pop()
        return 0
    monkeypatch.setattr(serving, "_launch", lambda device, stream, fn, *args: fn(*args))
    c = PagedCache.__new__(PagedCache)
    monkeypatch.setattr(serving, "load_library", lambda: types.SimpleNamespace(
        c2t_cache_workspace_bytes=lambda *a: 0, c2t_cache_truncate=enqueue, c2t_cache_attention=enqueue, c2t_attention_workspace_bytes=lambda *a: 0))
    monkeypatch.setattr(serving, "_whole", lambda *a: FAKE)
    monkeypatch.setattr(PagedCache, "_attention_workspace", lambda self, s, need: torch.zeros(1, dtype=torch.uint8))
    on_gpu = types.SimpleNamespace(is_cuda=True, dim=lambda: 5, dtype=torch.bfloat16, device=torch.device("cpu"), shape=(1, 4, 1, 16, 64))
    c._take(on_gpu, on_gpu, torch.zeros((2, 2), dtype=torch.int32), None, None)
    q = torch.zeros((2, 1, 1, 64), dtype=torch.bfloat16)

    def some(call):
        for _ in range(10):
            call()
    attend = lambda: c.attention(0, q, out=q)
    monkeypatch.setattr(PagedCache, "_attend", lambda self, a, workspace, need, *s: enqueue())
    threads = [threading.Thread(target=some, args=(f,)) for f in (attend, attend, c.truncate, c.truncate)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(met) == 40 and set(met) == {1}


def test_without_a_gpu_nothing_is_computed():
    import torch
    from paper_2502_13652_amd import PagedCache
    if not torch.cuda.is_available():
        with pytest.raises(RuntimeError, match="no CPU fallback"):
            PagedCache(1, 1, 4, 16, 1, 64, 2)
        with pytest.raises(ValueError):
            PagedCache.of_tensors(*[torch.zeros(1)] * 5)


def test_work_lists_and_addresses_of_the_paged_cache_under_sanitizers():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "paged_driver")
        r = subprocess.run(["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", "-o", exe, os.path.join(SAN, "paged_driver.cpp")],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert r.returncode == 0 and "paged driver ok" in r.stdout and "runtime error" not in r.stdout, r.stdout


def test_places_of_as_many_heads_as_there_may_be_under_sanitizers():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "heads_driver")
        r = subprocess.run(["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", "-o", exe, os.path.join(SAN, "heads_driver.cpp")],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert r.returncode == 0 and "heads driver ok" in r.stdout and "runtime error" not in r.stdout, r.stdout


def test_serving_entry_points_under_sanitizers():
    with tempfile.TemporaryDirectory() as d:
        exe = os.path.join(d, "serving_driver")
        r = subprocess.run(["hipcc", "-O1", "-g", "-std=c++17", "--offload-arch=gfx950",
                            "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                            "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                            "-Xarch_host", "-fno-sanitize-recover=all", "-o", exe,
                            os.path.join(SAN, "serving_driver.cpp"), os.path.join(ROOT, "paper_2502_13652_amd", "csrc", "c2t_lib.hip")],
                           stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout
        r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=ENV)
        assert r.returncode == 0 and "serving driver ok" in r.stdout and "runtime error" not in r.stdout and "AddressSanitizer" not in r.stdout, r.stdout


def test_the_header_and_the_binding_agree_on_the_counters():
    from paper_2502_13652_amd.serving import ATTENTION_COUNTERS
    with open(os.path.join(ROOT, "include", "c2t.h")) as f:
        assert "#define C2T_ATTENTION_COUNTERS %d\n" % ATTENTION_COUNTERS in f.read()


def readme_blocks():
    """The README's python examples."""
    with open(os.path.join(ROOT, "README.md")) as f:
        return [part.split("```")[0] for part in f.read().split("```python\n")[1:]]


def test_what_the_readme_imports_is_there():
    lines = [line for block in readme_blocks() for line in block.split("\n") if line.startswith(("import ", "from "))]
    assert len(lines) >= 2 and any("PagedCache" in line for line in lines)
    for line in lines:
        exec(line, {})
