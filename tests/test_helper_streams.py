"""With stream= given, a helper takes the memory of what it returns, and makes its copies, on that stream: memory of the
current stream may still be used by work queued there, and a copy made there is not ordered with the call. Run without a
GPU: the library and the streams are stand-ins that record where an allocation or a copy was made."""

import contextlib
import inspect
import weakref

import pytest
import torch

from paper_2606_07116_gb300 import offq as Q

STREAM = 0x5EED


class _Library:
    def __getattr__(self, name):
        return lambda *args: 64 if name.endswith("_workspace") or name.endswith("_bytes") else Q.OFFQ_OK


@pytest.fixture
def record(monkeypatch):
    """Allocations and copies, each with the streams that were entered around it."""
    entered, made = [], []

    @contextlib.contextmanager
    def on(stream, *_):
        entered.append(stream)
        yield
        entered.pop()

    empty, contiguous = torch.empty, torch.Tensor.contiguous
    monkeypatch.setattr(Q, "_on", on)
    monkeypatch.setattr(Q, "load_library", _Library)
    monkeypatch.setattr(Q, "_ptr", lambda t: 0)
    monkeypatch.setattr(Q, "_stream", lambda s: s)
    monkeypatch.setattr(Q.torch, "empty", lambda *a, **k: (made.append(("empty", list(entered))), empty(*a, **k))[1])
    monkeypatch.setattr(torch.Tensor, "contiguous", lambda t: t if t.is_contiguous() else
                        (made.append(("copy", list(entered))), contiguous(t))[1])
    Q._workspace_bytes.cache_clear()
    yield made
    Q._workspace_bytes.cache_clear()


def _attention_calls():
    x = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    cache = Q.kv4_cache(2, 2, 128, 16, device="cpu")
    slots, i32 = torch.zeros(3, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((3, 9), dtype=torch.int32)
    return {
        "rope_heads": (x,),
        "kv4_paged_write": (cache, x, x, slots, None, None, x),
        "kv4_paged_read": (cache, slots),
        "paged_attention": (x, cache, table[:, 7:], i32[:3], i32, 1, None, True),
        "prompt_attention": (x, x, x, i32, None, True, True),
    }


@pytest.mark.parametrize("name", list(_attention_calls()))
def test_attention_helpers_allocate_on_the_calls_stream(record, name):
    args = _attention_calls()[name]
    record.clear()
    getattr(Q, name)(*args, stream=STREAM)
    assert record and all(entered == [STREAM] for _, entered in record), record
    record.clear()
    getattr(Q, name)(*args)
    assert record and all(entered in ([], [None]) for _, entered in record)


@pytest.mark.parametrize("name", list(_attention_calls()))
def test_a_stream_given_by_position(record, name):
    """As the last of the positional arguments."""
    f = getattr(Q, name)
    bound = inspect.signature(f).bind(*_attention_calls()[name])
    bound.apply_defaults()
    bound.arguments["stream"] = STREAM
    record.clear()
    f(*bound.args)
    assert record and all(entered == [STREAM] for _, entered in record), record


def _linear_calls():
    """The helpers of the linears, the KV quantizers and the transform builder, with inputs that are copied where a
    helper takes such."""
    codes, f = torch.zeros((32, 64), dtype=torch.uint8), torch.zeros(2, dtype=torch.float32)
    x, kv = torch.zeros((2, 256)), torch.zeros((2, 1, 64))
    rot = torch.zeros((1, 64, 64)).transpose(1, 2)
    cols = torch.zeros((64, 4)).t()
    perm = torch.zeros(64, dtype=torch.int64)
    return {
        "quantize_act": (x, 128),
        "kv4_quantize": (kv,),
        "prepare_weight": (torch.zeros((128, 64)).t(), 128),
        "w4a4_linear": (codes, f, f, codes, f, f, 128),
        "quantize_act_group": (x, 128),
        "weight_group_sums": (codes, 32, 128),
        "w4a4_linear_group": (codes, f, f, codes, f, f),
        "kv4_quantize_rotated": (kv, rot),
        "rotate_heads": (kv, rot),
        "prepare_key_rotation": (rot,),
        "kv4_quantize_prepared": (kv, rot),
        "rotate_heads_prepared": (kv, rot),
        "kv4_quantize_reflected": (kv, rot),
        "rotate_heads_reflected": (kv, rot),
        "top1_tokens": (torch.zeros((2, 3, 64)),),
        "top1_direction": (cols,),
        "reflect_rows": (cols, perm.float()),
        "column_absmax": (cols,),
        "fuse_rotation": (cols, perm.float(), perm, 64),
    }


@pytest.mark.parametrize("name", list(_linear_calls()))
def test_other_helpers_allocate_on_the_calls_stream(record, name):
    args = _linear_calls()[name]
    record.clear()
    getattr(Q, name)(*args, stream=STREAM)
    assert record and all(entered == [STREAM] for _, entered in record), record


def test_no_helper_is_left_out():
    helpers = {n for n, f in vars(Q).items() if inspect.isfunction(f) and f.__module__ == Q.__name__
               and not n.startswith(("_", "offq_")) and "stream" in inspect.signature(f).parameters}
    assert helpers == set(_linear_calls()) | set(_attention_calls())


@pytest.mark.parametrize("name", list(_linear_calls()) + list(_attention_calls()))
def test_copies_live_until_the_call(monkeypatch, name):
    """A copy that only its address was taken of goes back to the allocator before the launch: another copy of the same
    call, or another thread, may be given its memory."""
    args = {**_linear_calls(), **_attention_calls()}[name]
    taken = []

    class Library:
        def __getattr__(self, function):
            def call(*_):
                if function.endswith(("_workspace", "_bytes")):
                    return 64
                assert all(ref() is not None for ref in taken), function
                return Q.OFFQ_OK
            return call

    monkeypatch.setattr(Q, "load_library", Library)
    monkeypatch.setattr(Q, "_ptr", lambda t: taken.append(weakref.ref(t)) if t is not None else None)
    monkeypatch.setattr(Q, "_stream", lambda s: s)
    getattr(Q, name)(*args)
    assert taken


def test_the_runtimes_own_handles_stand_for_the_default_stream(monkeypatch):
    """torch packs a stream's kind into its number, so the small handles 1 and 2 would be streams of its pools."""
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)
    assert [Q._on(h) for h in (0, 1, 2, STREAM)] == ["default"] * 3 + [STREAM]
