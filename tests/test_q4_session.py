"""Session(kv_bits=4)'s staging rows: gone after the prefill that needed them, and, where sessions share them, each
prefill ordered behind the one before."""
import contextlib
import weakref

import numpy as np
import pytest
import torch

from paper_2608_08569_gb300 import _native as N
from paper_2608_08569_gb300.session import Session

DESC = N.CacheDesc(1, 2, 4, 2, 64, 64, torch.bfloat16)


class Stream:
    """What a prefill does on a stream, in order."""
    cuda_stream = 0

    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_event(self, event):
        self.log.append((self.name, "wait", event))

    def record_event(self):
        event = f"event {len(self.log)}"
        self.log.append((self.name, "record", event))
        return event


@pytest.fixture
def log(monkeypatch):
    """Calls of the binding are written down instead of made."""
    log = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(N, "voxzip_anchor_fuse_workspace_size", lambda *a: 256)
    monkeypatch.setattr(N, "voxzip_anchor_fuse", lambda *a, stream=None, **kw: log.append((stream and stream.name, "fuse", a[10])))
    monkeypatch.setattr(N, "voxzip_q4_pack", lambda desc, c, l0, lc, k, v, stream=None: log.append((stream and stream.name, "pack", k)))
    return log


def _prefill(s, **kw):
    k = torch.zeros(1, 2, 2, 8, 64, dtype=torch.bfloat16)
    s.prefill(k, k, None, None, None, None, torch.zeros(0, dtype=torch.int32), None, None, **kw)


def test_the_session_keeps_no_staging_rows_of_its_own(log):
    s = Session(DESC, (32,), 0.9, device="cpu", kv_bits=4)
    _prefill(s)
    assert [x[1] for x in log] == ["fuse", "pack"] and log[0][2] is log[1][2] and log[0][2].shape == DESC._rows
    rows = weakref.ref(log[0][2])
    log.clear()
    assert rows() is None and s.staging is None


def test_prefills_on_shared_staging_rows_take_turns(log):
    staging = dict(k=torch.zeros(DESC._rows, dtype=torch.bfloat16), v=torch.zeros(DESC._rows, dtype=torch.bfloat16))
    a, b = (Session(DESC, (32,), 0.9, device="cpu", kv_bits=4, staging=staging) for _ in range(2))
    _prefill(a, stream=Stream("A", log))
    _prefill(b, stream=Stream("B", log))
    assert [x[:2] for x in log] == [("A", "fuse"), ("A", "pack"), ("A", "record"),
                                    ("B", "wait"), ("B", "fuse"), ("B", "pack"), ("B", "record")]
    assert log[3][2] == log[2][2] and all(x[2] is staging["k"] for x in log if x[1] in ("fuse", "pack"))


def test_a_prefill_that_fails_between_its_launches_still_holds_the_next_one_back(log, monkeypatch):
    staging = dict(k=torch.zeros(DESC._rows, dtype=torch.bfloat16), v=torch.zeros(DESC._rows, dtype=torch.bfloat16))
    a, b = (Session(DESC, (32,), 0.9, device="cpu", kv_bits=4, staging=staging) for _ in range(2))
    with monkeypatch.context() as m:
        def refuse(*args, **kw):
            raise N.VoxZipError("voxzip_q4_pack", 3, "refused")
        m.setattr(N, "voxzip_q4_pack", refuse)
        with pytest.raises(N.VoxZipError):
            _prefill(a, stream=Stream("A", log))
    _prefill(b, stream=Stream("B", log))
    assert [x[:2] for x in log[:4]] == [("A", "fuse"), ("A", "record"), ("B", "wait"), ("B", "fuse")]


def test_a_plain_session_stages_nothing(log):
    s = Session(DESC, (32,), 0.9, device="cpu")
    _prefill(s)
    assert [x[1] for x in log] == ["fuse"] and log[0][2] is s.cache["k"]


@pytest.mark.parametrize("bits", [4, 16])
def test_what_a_prefill_allocates_belongs_to_its_stream(log, monkeypatch, bits):
    """torch hands a freed block to the next user of the stream that it was made on: memory of another stream may still
    be in use there, or go to its next user while the launches run."""
    s, a = Session(DESC, (32,), 0.9, device="cpu", kv_bits=bits), Stream("A", log)
    at, empty, made = [None], torch.empty, []

    @contextlib.contextmanager
    def on(stream):
        at.append(stream)
        yield
        at.pop()
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda *args, **kw: made.append(at[-1]) or empty(*args, **kw))
    _prefill(s, stream=a)
    assert made == [a] * (3 if bits == 4 else 1)  # the workspace, and staging rows of K and V


# ----------------------------------------------------------------------------- on the GPU

def _request(seed):
    from gpu_harness import make_inputs
    from paper_2608_08569_gb300 import workloads as W
    w = W.scaled(W.CONFIGS["short"], layers=2, steps=4, name="short_l2")
    inp = make_inputs(w, "cuda:0")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    k, v = (torch.randn(inp[x].shape, generator=g, device="cuda").to(w.dtype) for x in ("k_pre", "v_pre"))
    desc = N.CacheDesc(w.batch, w.layers, w.q_heads, w.kv_heads, w.head_dim, -(-w.capacity // 4) * 4, w.dtype)
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    sp = inp["spans"]
    return w, desc, (k, v, i32(w.in_len), i32([w.audio_begin] * w.batch), i32(w.audio_len), i32(sp.off), i32(sp.start),
                     i32(sp.end), i32(sp.groups))


@pytest.mark.gpu
@pytest.mark.parametrize("own_stream", [False, True])
def test_a_session_in_4_bits_holds_less_memory(own_stream):
    w, desc, prompt = _request(1)
    stream = torch.cuda.Stream() if own_stream else None
    torch.cuda.synchronize()
    held = []
    for bits in (16, 4):
        before = torch.cuda.memory_allocated()
        s = Session(desc, w.budget, w.gamma, kv_bits=bits)
        s.prefill(*prompt, stream=stream, read_back=False)
        torch.cuda.synchronize()
        held.append(torch.cuda.memory_allocated() - before)
        del s
    rows = desc._rows[0] * desc._rows[1] * desc._rows[2] * desc._rows[3]
    # 2 x 256 bytes a row against 2 x 72, beside scores, positions, lengths and stage 1's workspace on both sides
    assert held[0] - held[1] > 0.95 * rows * 2 * (256 - 72)


@pytest.mark.gpu
def test_sessions_on_two_streams_share_staging_rows(monkeypatch):
    """The first session's packing is held up while the second one's stage 1 could run."""
    prompts = [_request(s) for s in (1, 2)]
    w, desc, _ = prompts[0]
    want = []
    for _, _, prompt in prompts:
        s = Session(desc, w.budget, w.gamma, kv_bits=4)
        s.prefill(*prompt)
        want.append(s.cache)
    rows = lambda: torch.empty(desc._rows, dtype=desc.dtype, device="cuda")
    staging = dict(k=rows(), v=rows())
    got = [Session(desc, w.budget, w.gamma, kv_bits=4, staging=staging) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    pack = N.voxzip_q4_pack

    def late(*args, stream=None, **kw):
        if stream is streams[0]:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)  # about 10 ms
        pack(*args, stream=stream, **kw)
    monkeypatch.setattr(N, "voxzip_q4_pack", late)
    for s, (_, _, prompt), stream in zip(got, prompts, streams):
        s.prefill(*prompt, stream=stream, read_back=False)
    torch.cuda.synchronize()
    for s, c in zip(got, want):
        for name, t in c.items():
            assert torch.equal(t, s.cache[name]), name


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [4, 16])
def test_the_length_is_read_back_on_the_prefills_stream(bits):
    """On a stream that is still busy, a read on another one would see the cache before stage 1."""
    w, desc, prompt = _request(3)
    want = Session(desc, w.budget, w.gamma, kv_bits=bits)
    want.prefill(*prompt)
    s, stream = Session(desc, w.budget, w.gamma, kv_bits=bits), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)  # about 10 ms
    s.prefill(*prompt, stream=stream)
    assert s.n_max == want.n_max > 0
