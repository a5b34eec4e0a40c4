"""Operator lists of a decoding tenant without a GPU: tensors that only look like ones on a GPU, to see what the lists refuse."""
import math

import pytest
import torch

from paper_2304_11745_amd import tokens as T


class Fake:
    """What an operator list asks of a tensor."""
    is_cuda = True

    def __init__(self, dtype, *shape, device="cuda:0"):
        self.dtype, self.shape, self.device = dtype, torch.Size(shape), torch.device(device)

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def pool(device="cuda:0", **other):
    u, i = torch.uint8, torch.int32
    t = dict(k_codes=(u, 4, 2, 32, 32), v_codes=(u, 4, 2, 1, 64, 16), k_scales=(i, 4, 2, 32, 1), v_scales=(i, 4, 2, 32, 1), page_table=(i, 3, 2))
    return [Fake(*spec, device=other.get(name, device)) for name, spec in t.items()]


@pytest.mark.parametrize("name", ["k_codes", "v_codes", "k_scales", "v_scales", "page_table"])
def test_the_tensors_of_a_cache_are_on_one_gpu(name):
    T.Cache(*pool())
    with pytest.raises(ValueError, match="one GPU"):
        T.Cache(*pool(**{name: "cuda:1"}))


def test_a_list_takes_a_cache_of_its_own_gpu_only():
    f, i = torch.float32, torch.int32
    here, there = T.Cache(*pool()), T.Cache(*pool("cuda:1"))
    start, start1 = Fake(i, 3), Fake(i, 3, device="cuda:1")
    qkv, out, kv = Fake(f, 3, 5, 8 * 64), Fake(f, 3, 5, 4 * 64), Fake(f, 3, 5, 4 * 64)
    T.OpList(f, 3).cache_attention(qkv, out, here, start, heads=4)
    T.OpList(f, 3).cache_read(kv, here, start)
    for bad in (lambda o: o.cache_write(qkv, there, start, heads=4), lambda o: o.cache_attention(qkv, out, there, start, heads=4),
                lambda o: o.cache_attention(qkv, out, here, start1, heads=4), lambda o: o.cache_read(kv, here, start1),
                lambda o: o.cache_read(kv, here, start, start1), lambda o: o.cache_read(kv, there, start1), lambda o: o.cache_read(kv, there, start)):
        with pytest.raises(ValueError, match="GPU"):
            bad(T.OpList(f, 3))


def lists(*devices):
    out = []
    for d in devices:
        o = T.OpList(torch.float32, 3)
        o.cache_read(Fake(torch.float32, 3, 5, 4 * 64, device=d), T.Cache(*pool(d)), Fake(torch.int32, 3, device=d))
        out.append(o)
    return out


def test_the_lists_of_a_session_are_on_one_gpu(monkeypatch):
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    with pytest.raises(ValueError, match="one GPU"):
        T.TokenSession(lists("cuda:0", "cuda:1"))


def test_lists_beside_other_tenants_are_on_the_sessions_gpu(monkeypatch):
    from paper_2304_11745_amd import harness
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="cuda:1"):
        harness.Session([], [], "cuda:0", extra=lists("cuda:1"))


def test_a_session_runs_on_its_own_gpu_whichever_is_current(monkeypatch):
    """Rounds and the release of a session; gacer_enqueue sees to it itself."""
    now, seen = [0], []

    class device:
        def __init__(self, d):
            self.d = torch.device(d).index

        def __enter__(self):
            self.before, now[0] = now[0], self.d

        def __exit__(self, *_):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda d=None: None)
    for call in ("gacer_run", "gacer_destroy"):
        monkeypatch.setattr(T.B, call, lambda *a, call=call: seen.append((call, now[0])) or 0)
    for gpu in (0, 1):
        for current in (0, 1):
            s, now[0], seen[:] = object.__new__(T.TokenSession), current, []
            s.device, s.ctx = torch.device("cuda", gpu), 1
            s.run()
            s.close()
            assert seen == [("gacer_run", gpu), ("gacer_destroy", gpu)] and now[0] == current
