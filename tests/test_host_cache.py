"""The entry points over a batch's K,V caches refuse bad arguments on the host, before any HIP call (no GPU here)."""
import ctypes as C
import os

import pytest
import torch

from paper_2407_14057_amd import binding as B

ONE = 4096                       # an aligned address that is never followed


def _cache(**change):
    c = dict(k=ONE, v=ONE, batch_stride=1000 * 128, row_stride=128, batch=3, capacity=1000, n_kv_heads=2, head_dim=64)
    c.update(change)
    return B.lazyllm_kv_cache(**c)


def _step(**change):
    s = dict(q=ONE, k_new=ONE, v_new=ONE, o=ONE, lengths=ONE, n_heads=4, q_len=2, max_len=900, prefix_len=100, prefix_k=ONE,
             prefix_v=ONE, prefix_stride=128)
    s.update(change)
    return B.lazyllm_step_attention(**s)


BAD_CACHES = [dict(head_dim=96), dict(head_dim=32), dict(n_kv_heads=0), dict(n_kv_heads=257), dict(batch=0), dict(batch=-1), dict(capacity=0),
              dict(batch=65536), dict(batch=60000, capacity=60000), dict(batch=1, capacity=(1 << 30) + 1)]
BAD_ROWS = [dict(k=0), dict(v=0), dict(k=ONE + 8), dict(v=ONE + 2), dict(row_stride=120), dict(row_stride=132), dict(row_stride=(1 << 24) + 8),
            dict(row_stride=0), dict(row_stride=-128), dict(batch_stride=1000 * 128 - 8), dict(batch_stride=1000 * 128 + 4), dict(batch_stride=0),
            dict(batch_stride=-1000 * 128), dict(batch_stride=1 << 50)]
BAD_STEPS = [dict(n_heads=0), dict(n_heads=3), dict(n_heads=258), dict(q_len=0), dict(q_len=65), dict(max_len=-1), dict(max_len=999),
             dict(max_len=0x7fffffff)]
BAD_POINTERS = [dict(q=0), dict(k_new=0), dict(v_new=0), dict(o=0), dict(lengths=0), dict(q=ONE + 8), dict(k_new=ONE + 4), dict(v_new=ONE + 2),
                dict(o=ONE + 8), dict(weight=ONE), dict(weight_out=ONE), dict(pos=ONE), dict(pos_new=ONE)]
BAD_PREFIXES = [dict(prefix_len=0), dict(prefix_len=-1), dict(prefix_k=0), dict(prefix_v=0), dict(prefix_k=ONE + 8), dict(prefix_v=ONE + 8),
                dict(prefix_len=(1 << 30) + 1), dict(prefix_stride=120), dict(prefix_stride=132), dict(prefix_stride=0), dict(prefix_stride=(1 << 24) + 8)]


def _attend(name, cache, step, ws=ONE, size=1 << 40):
    return getattr(B.lib(), name)(cache and C.byref(cache), step and C.byref(step), ws, size, None)


@pytest.mark.parametrize("name", ["lazyllm_op_cache_attention", "lazyllm_op_prefix_attention"])
def test_attention_refuses_bad_arguments(name):
    assert _attend(name, None, _step()) == B.LAZYLLM_EINVAL
    assert _attend(name, _cache(), None) == B.LAZYLLM_EINVAL
    for change in BAD_CACHES + BAD_ROWS:
        assert _attend(name, _cache(**change), _step()) == B.LAZYLLM_EINVAL, change
    for change in BAD_STEPS + BAD_POINTERS:
        assert _attend(name, _cache(), _step(**change)) == B.LAZYLLM_EINVAL, change
    assert _attend(name, _cache(), _step(), ws=None) == B.LAZYLLM_EINVAL
    assert _attend(name, _cache(), _step(), ws=ONE + 128) == B.LAZYLLM_EINVAL
    prefix = 100 if name == "lazyllm_op_prefix_attention" else 0
    for weights in (False, True):
        tables = dict(weight=ONE, weight_out=ONE) if weights else {}
        size = B.lazyllm_op_cache_attention_workspace_bytes(_cache(), 4, 2, 900, prefix, weights)
        assert size > 0
        assert _attend(name, _cache(), _step(**tables), size=size // 2) == B.LAZYLLM_ENOSPC
        assert _attend(name, _cache(), _step(**tables), size=0) == B.LAZYLLM_ENOSPC


def test_prefix_attention_refuses_bad_prefixes():
    for change in BAD_PREFIXES:
        assert _attend("lazyllm_op_prefix_attention", _cache(), _step(**change)) == B.LAZYLLM_EINVAL, change


def test_workspace_of_the_attention():
    size = B.lazyllm_op_cache_attention_workspace_bytes
    for change in BAD_CACHES:
        assert size(_cache(**change), 4, 2, 100) == 0, change
    for change in BAD_STEPS:
        s = _step(**change)
        assert size(_cache(), s.n_heads, s.q_len, s.max_len) == 0, change
    assert size(_cache(), 4, 2, 100, -1) == 0
    assert B.lib().lazyllm_op_cache_attention_workspace_bytes(None, 4, 2, 100, 0, 0) == 0
    assert size(_cache(), 4, 2, 900, 0, True) > size(_cache(), 4, 2, 900) > 0
    assert size(_cache(), 4, 2, 900, 5000) > size(_cache(), 4, 2, 900)
    assert size(_cache(), 4, 2, 100, (1 << 30) + 1) == 0
    # more workgroups than a launch can have
    assert size(_cache(batch=65535, capacity=20000, batch_stride=20000 * 128), 256, 64, 100) == 0
    many = _cache(batch=65535, capacity=20000, batch_stride=20000 * 128)
    assert _attend("lazyllm_op_cache_attention", many, _step(n_heads=256, q_len=64, max_len=100)) == B.LAZYLLM_EINVAL
    # sizes whose byte counts pass 32 bits
    long = _cache(batch=64, capacity=131072, batch_stride=1 << 30)
    assert size(long, 64, 64, 131072 - 64, 0, True) >= 64 * 64 * 64 * 131072 * 4


def _evict(cache=None, size=1 << 40, **change):
    a = dict(weight=ONE, pos=ONE, lengths=ONE, budget=500, sinks=4, recent=100, weight_out=ONE, pos_out=ONE, lengths_out=ONE, kept=None,
             status=None, workspace=ONE)
    a.update(change)
    return B.lib().lazyllm_op_cache_evict(C.byref(cache or _cache()), a["weight"], a["pos"], a["lengths"], a["budget"], a["sinks"], a["recent"],
                                          a["weight_out"], a["pos_out"], a["lengths_out"], a["kept"], a["status"], a["workspace"], size, None)


def test_eviction_refuses_bad_arguments():
    for change in BAD_CACHES + BAD_ROWS:
        assert _evict(_cache(**change)) == B.LAZYLLM_EINVAL, change
    assert _evict(_cache(batch=1, capacity=(1 << 24) + 1)) == B.LAZYLLM_EINVAL
    for name in ("weight", "pos", "lengths", "weight_out", "pos_out", "lengths_out", "workspace"):
        assert _evict(**{name: None}) == B.LAZYLLM_EINVAL, name
    for change in (dict(budget=0), dict(budget=-1), dict(sinks=-1), dict(recent=-1), dict(sinks=401), dict(budget=3, sinks=2, recent=2),
                   dict(sinks=0x7fffffff, recent=0x7fffffff), dict(workspace=ONE + 64)):
        assert _evict(**change) == B.LAZYLLM_EINVAL, change
    size = B.lazyllm_op_cache_evict_workspace_bytes(_cache(), 500)
    assert size > 0 and _evict(size=size - 1) == B.LAZYLLM_ENOSPC and _evict(size=0) == B.LAZYLLM_ENOSPC
    assert B.lazyllm_op_cache_evict_workspace_bytes(_cache(), 0) == 0
    assert B.lazyllm_op_cache_evict_workspace_bytes(_cache(head_dim=96), 10) == 0
    assert B.lazyllm_op_cache_evict_workspace_bytes(_cache(batch=1, capacity=(1 << 24) + 1), 10) == 0
    assert B.lib().lazyllm_op_cache_evict(None, ONE, ONE, ONE, 5, 0, 0, ONE, ONE, ONE, None, None, ONE, 1 << 30, None) == B.LAZYLLM_EINVAL


def test_prefix_of_another_shape_is_refused():
    k = torch.zeros(3, 20, 2, 64, dtype=torch.bfloat16)
    cache = B.make_kv_cache(k, torch.zeros_like(k))
    p = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for bad_k, bad_v in ((p[:0], p[:0]), (p[:, :1], p[:, :1]), (p, p[:4]), (p[0], p[0]), (p.transpose(0, 1), p.transpose(0, 1)), (p[..., ::2], p[..., ::2])):
        with pytest.raises(B.LazyLLMError) as e:
            B.lazyllm_op_prefix_attention(cache, bad_k, bad_v, k, k, k, k, 2, 1, 10, k, k)
        assert e.value.status == B.LAZYLLM_EINVAL


def test_descriptor_of_caches():
    k = torch.zeros(3, 20, 2, 64, dtype=torch.bfloat16)
    c = B.make_kv_cache(k, torch.zeros_like(k))
    assert (c.batch, c.capacity, c.n_kv_heads, c.head_dim, c.batch_stride, c.row_stride) == (3, 20, 2, 64, 20 * 128, 128)
    both = torch.zeros(3, 20, 2, 2, 64, dtype=torch.bfloat16)
    c = B.make_kv_cache(both[:, :, 0], both[:, :, 1])
    assert (c.batch_stride, c.row_stride, c.v - c.k) == (20 * 256, 256, 256)
    heads_first = torch.zeros(3, 2, 20, 64, dtype=torch.bfloat16).transpose(1, 2)
    for bad_k, bad_v in ((k.float(), k.float()), (k, k[:, :10]), (heads_first, heads_first), (k[0], k[0]), (k, both[:, :, 0]),
                         (k[..., ::2], k[..., ::2])):
        with pytest.raises(B.LazyLLMError) as e:
            B.make_kv_cache(bad_k, bad_v)
        assert e.value.status == B.LAZYLLM_EINVAL


def test_prefix_of_another_type_is_refused():
    k = torch.zeros(3, 20, 2, 64, dtype=torch.bfloat16)
    cache = B.make_kv_cache(k, k.clone())
    p = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    for bad_k, bad_v in ((p.half(), p.half()), (p, p.float())):
        with pytest.raises(B.LazyLLMError) as e:
            B.lazyllm_op_prefix_attention(cache, bad_k, bad_v, k, k, k, k, 2, 1, 10, k, k)
        assert e.value.status == B.LAZYLLM_EINVAL


def test_what_is_not_on_the_current_device_is_refused(monkeypatch):
    """Caches, workspace or stream of another device, or in host memory (-1); the library is not reached."""
    class On:                                            # stands for a tensor or a stream of a device
        def __init__(self, device):
            self.device_index, self.cuda_stream = device, 77

        def get_device(self):
            return self.device_index

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    cache = _cache()
    assert B._cache_stream(cache, On(1), On(1)) == 77                      # (a descriptor made by hand has no device)
    cache.device = 1
    assert B._cache_stream(cache, On(1), On(1)) == 77
    for where, ws, stream in ((0, 1, 1), (-1, 1, 1), (1, 0, 1), (1, -1, 1), (1, 1, 0), (0, 0, 0)):
        cache.device = where
        with pytest.raises(B.LazyLLMError) as e:
            B._cache_stream(cache, On(ws), On(stream))
        assert e.value.status == B.LAZYLLM_EINVAL
    k = torch.zeros(3, 20, 2, 64, dtype=torch.bfloat16)
    p, table = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 20)
    host = B.make_kv_cache(k, k.clone())
    assert host.device == -1
    for call in (lambda: B.lazyllm_op_cache_attention(host, k, k, k, table, 2, 1, 10, k, k),
                 lambda: B.lazyllm_op_prefix_attention(host, p, p, k, k, k, table, 2, 1, 10, k, k),
                 lambda: B.lazyllm_op_cache_evict(host, table, table, table, 5, 0, 0, table, table, table, k)):
        with pytest.raises(B.LazyLLMError) as e:
            call()
        assert e.value.status == B.LAZYLLM_EINVAL


class _Library:
    """Stands for the library: counts the calls that reach it."""

    def __init__(self, real):
        self.real, self.reached = real, 0

    def __getattr__(self, name):
        return self._reach if name.startswith("lazyllm_op_") else getattr(self.real, name)

    def _reach(self, *args):
        self.reached += 1
        return B.LAZYLLM_OK


class _Elsewhere(torch.Tensor):
    def get_device(self):
        return 3


def _operands(n_heads=4, q_len=2, batch=3, capacity=20, kvh=2, hd=64, budget=5, prefix=7):
    bf, i32 = torch.bfloat16, torch.int32
    k = torch.zeros(batch, capacity, kvh, hd, dtype=bf)
    t = dict(q=torch.zeros(batch, q_len, n_heads, hd, dtype=bf), k_new=torch.zeros(batch, q_len, kvh, hd, dtype=bf),
             v_new=torch.zeros(batch, q_len, kvh, hd, dtype=bf), o=torch.zeros(batch, q_len, n_heads, hd, dtype=bf),
             lengths=torch.zeros(batch, dtype=i32), weight=torch.zeros(batch, capacity), weight_out=torch.zeros(batch, capacity),
             pos_new=torch.zeros(batch, dtype=i32), pos=torch.zeros(batch, capacity, dtype=i32), status=torch.zeros(1, dtype=i32),
             pos_out=torch.zeros(batch, capacity, dtype=i32), lengths_out=torch.zeros(batch, dtype=i32),
             kept=torch.zeros(batch, budget, dtype=i32), prefix_k=torch.zeros(prefix, kvh, hd, dtype=bf),
             prefix_v=torch.zeros(prefix, kvh, hd, dtype=bf))
    return B.make_kv_cache(k, k.clone()), t


def _call(name, cache, t, ws, stream):
    if name == "evict":
        B.lazyllm_op_cache_evict(cache, t["weight"], t["pos"], t["lengths"], 5, 1, 1, t["weight_out"], t["pos_out"], t["lengths_out"], ws,
                                 kept=t["kept"], status=t["status"], stream=stream)
        return
    args = (t["q"], t["k_new"], t["v_new"], t["lengths"], 4, 2, 18, t["o"], ws)
    more = {k: t[k] for k in ("weight", "weight_out", "pos_new", "pos", "status")}
    if name == "prefix":
        B.lazyllm_op_prefix_attention(cache, t["prefix_k"], t["prefix_v"], *args, **more, stream=stream)
    else:
        B.lazyllm_op_cache_attention(cache, *args, **more, stream=stream)


OPERANDS = {"attention": ["q", "k_new", "v_new", "o", "lengths", "weight", "weight_out", "pos_new", "pos", "status"],
            "evict": ["weight", "pos", "lengths", "weight_out", "pos_out", "lengths_out", "kept", "status"]}
OPERANDS["prefix"] = OPERANDS["attention"] + ["prefix_k", "prefix_v"]


@pytest.mark.parametrize("name", list(OPERANDS))
def test_operands_of_another_device_type_size_or_layout_are_refused(name, monkeypatch):
    """Every tensor of a call, one at a time; the library, which gets addresses alone, is not reached."""
    library = _Library(B.lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)              # (where the tensors here are)
    monkeypatch.setattr(B, "_lib_handle", library)

    class Stream:
        device_index, cuda_stream = -1, 77

    ws = torch.zeros(4096, dtype=torch.uint8)
    cache, good = _operands()
    _call(name, cache, good, ws, Stream)
    assert library.reached == 1
    # stacked tables, and a status that is one of several, are as good; what may be left out may be left out
    for change in ([{"status": torch.zeros(4, dtype=torch.int32)}, {"status": None}, {"lengths": good["lengths"].view(1, 3)}] +
                   ([{"kept": None}] if name == "evict" else [{"weight": None, "weight_out": None}, {"pos": None, "pos_new": None}])):
        _call(name, cache, dict(good, **change), ws, Stream)
    reached = library.reached
    for operand in OPERANDS[name]:
        t = good[operand]
        bad = [t.as_subclass(_Elsewhere), t.to(torch.float64), t.to(torch.int64), t[:0]]
        if operand != "status":
            wide = torch.zeros(*t.shape[:-1], 2 * t.shape[-1], dtype=t.dtype)
            bad += [t[:-1], torch.cat([t, t]), wide, wide[..., ::2]]            # (the last: the right size, with gaps)
        for wrong in bad:
            with pytest.raises(B.LazyLLMError) as e:
                _call(name, cache, dict(good, **{operand: wrong}), ws, Stream)
            assert e.value.status == B.LAZYLLM_EINVAL, (operand, wrong.shape, wrong.dtype)
    for operand in ("q", "k_new", "v_new", "o", "lengths") if name != "evict" else OPERANDS[name][:6]:
        with pytest.raises(B.LazyLLMError) as e:                                # what has to be there
            _call(name, cache, dict(good, **{operand: None}), ws, Stream)
        assert e.value.status == B.LAZYLLM_EINVAL
    assert library.reached == reached


def test_layout_of_a_step():
    """The binding packs a step's members at once: in the order and with the sizes of the structure."""
    assert B._STEP_LAYOUT.size == C.sizeof(B.lazyllm_step_attention)
    s = B.lazyllm_step_attention.from_buffer_copy(B._STEP_LAYOUT.pack(*range(1, 18)))
    assert [getattr(s, name) for name, _ in s._fields_] == list(range(1, 18))


def test_step_of_the_readme_leaves_idle_requests_idle(monkeypatch):
    """The README's step, run on the host with calls that do nothing: a request whose length is negative takes no part in the
    next step either, the others have one token more."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        step = [block for block in f.read().split("```")[1::2] if "B.make_kv_cache(" in block]
    assert len(step) == 1
    calls = []

    class Calls:
        def __getattr__(self, name):
            calls.append(name)
            return lambda *args, **kwargs: 1

    lengths = torch.tensor([3, -1, 0, -7], dtype=torch.int32)
    monkeypatch.setattr(torch, "empty", lambda *args, **kwargs: None)
    names = ("k v n_heads max_len q k_new v_new o weight pos budget sinks recent evict_ws").split()
    exec(step[0], dict(dict.fromkeys(names), B=Calls(), torch=torch, lengths=lengths, position=lengths.clone()))
    assert "lazyllm_op_cache_attention" in calls and "lazyllm_op_cache_evict" in calls
    assert lengths.tolist() == [4, -1, 1, -7] and lengths.dtype == torch.int32


def _block(heads, rows, prefix):
    """Query rows that go over the prefix together, of `rows` (multiples of the heads of a group) of a K,V head."""
    n_heads, kvh, hd = heads
    group = n_heads // kvh
    assert rows % group == 0
    return B.lib().lazyllm_op_prefix_attention_block(C.byref(_cache(batch=rows // group, n_kv_heads=kvh, head_dim=hd, row_stride=kvh * hd)), n_heads,
                                                     1, prefix)


@pytest.mark.parametrize("heads,rows,prefix,direct,shared", [
    ((32, 8, 128), 256, 16000, 42.4, 47.6), ((32, 8, 128), 1024, 4000, 44.9, 46.8), ((32, 8, 128), 128, 32000, 57.4, 64.4),
    ((32, 8, 128), 128, 64453, 97.9, 107.1), ((32, 32, 128), 128, 20507, 130.0, 146.6), ((32, 32, 128), 64, 16000, 75.0, 117.1),
    ((32, 8, 128), 320, 17187, 55.7, 67.0), ((8, 1, 128), 2048, 16000, 41.8, 45.9), ((4, 4, 64), 256, 16000, 21.9, 30.7),
    ((4, 4, 64), 1024, 8789, 34.9, 35.7), ((32, 8, 128), 256, 32226, 86.5, 69.9), ((32, 8, 128), 512, 16113, 71.8, 65.2),
    ((32, 32, 128), 256, 8056, 93.7, 85.6), ((4, 4, 64), 256, 64453, 57.5, 50.3), ((4, 4, 64), 1024, 16113, 56.2, 46.6),
    ((64, 8, 64), 512, 10742, 40.7, 38.6), ((8, 1, 128), 2048, 26367, 62.6, 58.0), ((4, 4, 64), 192, 85937, 73.9, 61.2)])
def test_prefix_takes_the_form_that_was_measured_faster(heads, rows, prefix, direct, shared):
    """us of the two forms on an MI355X."""
    assert (_block(heads, rows, prefix) == 256) == (shared < direct)


def test_blocks_of_query_rows_behind_a_prefix():
    assert [_block((4, 4, 64), rows, 100) for rows in (1, 16, 17, 500)] == [16, 16, 32, 32]
    ask = B.lib().lazyllm_op_prefix_attention_block
    for change in BAD_CACHES:
        assert ask(C.byref(_cache(**change)), 4, 2, 100) == B.LAZYLLM_EINVAL, change
    for n_heads, q_len, prefix in ((0, 2, 100), (3, 2, 100), (4, 0, 100), (4, 65, 100), (4, 2, 0), (4, 2, -1), (4, 2, (1 << 30) + 1)):
        assert ask(C.byref(_cache()), n_heads, q_len, prefix) == B.LAZYLLM_EINVAL
    assert ask(None, 4, 2, 100) == B.LAZYLLM_EINVAL
    assert ask(C.byref(_cache()), 4, 2, 1 << 30) == 16                 # (12 rows; a block of 256 would be nearly empty)


def test_numbers_beyond_32_bits_are_refused(monkeypatch):
    """Cut to 32 bits, a bound or budget of 2^32 + 5 would be 5."""
    library = _Library(B.lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(B, "_lib_handle", library)

    class Stream:
        device_index, cuda_stream = -1, 77

    ws = torch.zeros(4096, dtype=torch.uint8)
    cache, t = _operands()
    far = (1 << 32) + 5
    tables = (t["weight"], t["pos"], t["lengths"])
    outs = (t["weight_out"], t["pos_out"], t["lengths_out"], ws)
    for call in (lambda: B.lazyllm_op_cache_attention(cache, t["q"], t["k_new"], t["v_new"], t["lengths"], 4, 2, far, t["o"], ws, stream=Stream),
                 lambda: B.lazyllm_op_cache_attention(cache, t["q"], t["k_new"], t["v_new"], t["lengths"], 4, 2, -far, t["o"], ws, stream=Stream),
                 lambda: B.lazyllm_op_cache_evict(cache, *tables, far, 1, 1, *outs, stream=Stream),
                 lambda: B.lazyllm_op_cache_evict(cache, *tables, 5, far, 1 - far, *outs, stream=Stream),
                 lambda: B.lazyllm_op_cache_evict(cache, *tables, 5, 1, far, *outs, stream=Stream),
                 lambda: B.lazyllm_op_cache_evict(cache, *tables, 5, 1, 1, *outs, status="text", stream=Stream)):
        with pytest.raises(B.LazyLLMError) as e:
            call()
        assert e.value.status == B.LAZYLLM_EINVAL
    assert library.reached == 0
