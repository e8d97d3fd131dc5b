"""pipeline.PagedPrompt without a GPU: what it tells the allocator and what it keeps of the requests' lengths, over stand-ins for
its device tensors."""
from types import SimpleNamespace

import pytest
import torch

from test_pages_abi import V  # noqa: F401


class DeviceTensor:
    def __init__(self, *shape):
        self.shape, self.streams = shape, []

    def record_stream(self, s):
        self.streams.append(s)

    def numel(self):
        return 1 << 20

    def transpose(self, *a):
        return self


@pytest.fixture
def prompt(V, monkeypatch):
    """A prompt of two requests with room for 100 tokens whose library calls do nothing but can be made to fail."""
    from paper_2410_23317_amd import pipeline
    p = object.__new__(pipeline.PagedPrompt)
    p.max_len, p.tokens, p.chunk, p.before, p.workspace, p.device = 100, [0, 0], None, None, DeviceTensor(), torch.device("cpu")
    p.table, p.pages = DeviceTensor(), SimpleNamespace(arena=DeviceTensor(), shape=SimpleNamespace(L=1))
    p.calls, p.fail = [], False

    def call(name):
        def made(*a):
            if p.fail:
                raise ValueError(name)
            p.calls.append(name)
            return 0
        return made
    for name in ("vlc_pages_attn", "vlc_pages_read", "vlc_pages_attn_workspace_bytes"):
        monkeypatch.setattr(pipeline.V, name, call(name))
    monkeypatch.setattr(pipeline.V, "make_chunk", lambda table, max_new, max_len, lens: SimpleNamespace(
        tensors=(table, DeviceTensor()), lens=lens.tolist(), max_new=max_new, max_len=max_len))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "side")
    return p


def test_everything_a_call_works_on_is_recorded_on_its_stream(prompt):
    """What is dropped while another stream than the one it was made on works with it must not be handed out again before that."""
    prompt.begin_chunk([3, 5])
    lens = prompt.chunk.tensors[1]
    prompt.extend(0, 1, None, None, None, None, None)
    for t in (prompt.pages.arena, prompt.table, prompt.workspace, lens):
        assert "side" in t.streams
        t.streams.clear()
    prompt.read(DeviceTensor(2, 1, 1, 100, 64), DeviceTensor(2, 1, 1, 100, 64))
    for t in (prompt.pages.arena, prompt.table, lens):
        assert "side" in t.streams


def test_a_chunk_that_does_not_come_is_taken_back(prompt):
    """A refused extend() may be repeated; drop_chunk() leaves no counted positions behind, and the earlier chunk in force."""
    with pytest.raises(ValueError):
        prompt.drop_chunk()
    first = prompt.begin_chunk([3, 5])
    prompt.extend(0, 1, None, None, None, None, None)
    prompt.begin_chunk([10, 0])
    prompt.fail = True
    with pytest.raises(ValueError, match="vlc_pages"):
        prompt.extend(0, 1, None, None, None, None, None)
    assert prompt.tokens == [13, 5]                              # the same chunk again would be the same positions
    prompt.fail = False
    prompt.extend(0, 1, None, None, None, None, None)
    prompt.begin_chunk([1, 1])
    prompt.drop_chunk()
    assert prompt.tokens == [13, 5] and prompt.chunk.lens == [[13, 10], [5, 0]]
    with pytest.raises(ValueError):
        prompt.drop_chunk()                                      # that chunk's rows are in the pages
    prompt.begin_chunk([2, 0])
    assert prompt.chunk.lens == [[15, 2], [5, 0]] and prompt.chunk is not first
    with pytest.raises(ValueError):
        prompt.begin_chunk([100, 0])                             # refused: nothing changes
    assert prompt.tokens == [15, 5] and prompt.chunk.lens == [[15, 2], [5, 0]]
    prompt.drop_chunk()
    prompt.begin_chunk([1, 7])
    assert prompt.chunk.lens == [[14, 1], [12, 7]]


def test_tensors_that_do_not_fit_the_prompt_are_refused(prompt, monkeypatch):
    """A read that would leave tokens out, and a compression whose tensors, window or lengths are not the prompt's: the calls
    behind it take bare pointers."""
    from paper_2410_23317_amd import pipeline
    B, L, Hq, Hkv, d, m, tau = 2, 1, 4, 2, 64, 60, 8
    t = DeviceTensor
    path = SimpleNamespace(shape=SimpleNamespace(B=B, L=L, Hq=Hq, Hkv=Hkv, d=d, m=m, tau=tau, lens=None), score_from_stats=lambda *a: prompt.calls.append("score"),
                           topk_compact=lambda *a: prompt.calls.append("compact"), nnz=None, gamma=None, alpha=(1, 10), k=None, beta=None)
    monkeypatch.setattr(pipeline.V, "vlc_sparsity_allocate", lambda *a: prompt.calls.append("allocate"))
    q, kv = t(B, L, Hq, tau, d), t(B, L, Hkv, m, d)

    def compress(q=q, k=kv, v=kv):
        prompt.calls.clear()
        prompt.compress(path, q, None, k, v)
    with pytest.raises(ValueError, match="begin_chunk"):
        compress()
    prompt.begin_chunk([52, 52])
    with pytest.raises(ValueError, match="window"):
        compress()
    prompt.begin_chunk([8, 8])
    compress()
    assert prompt.calls == ["vlc_pages_read", "score", "allocate", "compact"]
    for kw in (dict(q=t(B, L, Hq, tau + 1, d)), dict(k=t(B, L, Hkv, m + 1, d)), dict(v=t(B, L, Hkv, m - 1, d)), dict(k=t(L, B, Hkv, m, d))):
        with pytest.raises(ValueError, match="shape"):
            compress(**kw)
    prompt.drop_chunk()
    for new in ([8, 7], [7, 8]):
        prompt.begin_chunk(new)
        with pytest.raises(ValueError, match="lens"):
            compress()
        prompt.drop_chunk()
    path.shape.lens = 4096
    for new in ([8, 7], [5, 6]):                                 # windows below the path's tau, as the pairs of lens say
        prompt.begin_chunk(new)
        compress()
        prompt.drop_chunk()
    prompt.begin_chunk([8, 7])
    compress()
    prompt.read(t(B, L, Hkv, 60, d), t(B, L, Hkv, 60, d))
    with pytest.raises(ValueError, match="59 rows"):
        prompt.read(t(B, L, Hkv, 59, d), t(B, L, Hkv, 59, d))
