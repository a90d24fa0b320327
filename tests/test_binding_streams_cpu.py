"""What a call makes for itself when it is given a stream: on that stream, where the fills come before
the launch and a dropped workspace is not given out again before its end. No device is touched: the
tensors only say that they are on a GPU, and the launch is left out."""

import pytest
import torch

from paper_2609_04010_gb300 import binding as b


class OnGpu(torch.Tensor):
    is_cuda = True

    def record_stream(self, stream):
        self.used_on = getattr(self, "used_on", ()) + (stream,)


class Stream:
    device = torch.device("cpu")
    cuda_stream = 0


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32).as_subclass(OnGpu)


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16).as_subclass(OnGpu)


@pytest.fixture
def watched(monkeypatch):
    """The caller's stream, a stream to give, and [(tensor, the stream current when it was made)]."""
    caller, other = Stream(), Stream()
    now, made, launched = [caller], [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            now.append(self.stream)

        def __exit__(self, *_):
            now.pop()

    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    for name in ("zeros", "empty", "full", "empty_like"):
        def make(*args, _make=getattr(torch, name), **kwargs):
            kwargs.pop("device", None)
            made.append((_make(*args, **kwargs).as_subclass(OnGpu), now[-1]))
            return made[-1][0]
        monkeypatch.setattr(torch, name, make)

    def launch(what, *args, **kwargs):
        launched.append(now[-1])
    monkeypatch.setattr(b, "_call", launch)
    monkeypatch.setattr(b, "_raise", launch)
    return caller, other, made, launched


def rope():
    return dict(q=bf16(5, 4, 64), k=bf16(5, 2, 64), v=None, positions=i32(5),
                turns=torch.zeros(32, dtype=torch.int64).as_subclass(OnGpu))


def chunk():
    return dict(q=bf16(6, 4, 64), cache=(bf16(7, 2, 16, 64), bf16(7, 2, 16, 64)), page_table=i32(3, 5),
                row_start=i32(4), kv_len=i32(3))


def fork():
    return dict(parent=i32(3), kv_len=i32(3), page_table=i32(3, 5), shares=i32(9), free_pages=i32(9),
                free_count=i32(1), page_size=16)


@pytest.mark.parametrize("call,inputs,makes", [
    (b.rope_kv, rope, 2), (b.chunk_attention, chunk, 3), (b.fork_sequences, fork, 3)])
def test_what_a_call_makes_is_on_its_stream(watched, call, inputs, makes):
    caller, other, made, launched = watched
    given = inputs()
    made.clear()
    res = call(**given, stream=other)
    assert launched and len(made) >= makes and all(s is other for _, s in made)
    returned = res.values() if isinstance(res, dict) else res
    assert all(t.used_on == (caller,) for t in returned)
    # without one, on the caller's, and nothing is noted
    made.clear()
    res = call(**given)
    returned = res.values() if isinstance(res, dict) else res
    assert all(s is caller for _, s in made) and not any(hasattr(t, "used_on") for t in returned)


def test_what_a_call_is_given_is_kept_for_its_stream(monkeypatch):
    """The caller may drop the inputs when the call returns."""
    other = Stream()
    a = b.chunk_attn_args(**chunk(), out=bf16(6, 4, 64))
    ws = torch.zeros(256, dtype=torch.uint8).as_subclass(OnGpu)

    class Lib:
        def spec_chunk_attention(*_):
            return 0
    monkeypatch.setattr(b, "lib", lambda: Lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    b.chunk_attention_args(a, ws, other)
    assert all(t.used_on == (other,) for t in (*a.keep, ws))


def f32(*shape):
    return torch.zeros(shape).as_subclass(OnGpu)


def e4m3(*shape):
    return torch.zeros(shape, dtype=torch.uint8).view(torch.float8_e4m3fn).as_subclass(OnGpu)


EARLIER = {
    "verify_attention": lambda: (bf16(2, 3, 4, 64), bf16(7, 2, 16, 64), bf16(7, 2, 16, 64), i32(2, 3), i32(2)),
    "verify_attention_fp8": lambda: (bf16(2, 3, 4, 64), e4m3(7, 2, 2, 16, 64), f32(7, 2, 2), i32(2, 3), i32(2)),
    "accept_block": lambda: (f32(2, 3, 50), f32(2, 3, 50), i32(2, 3), f32(2), f32(2, 3)),
    "accept_block_filtered": lambda: (f32(2, 3, 50), f32(2, 3, 50), i32(2, 3), f32(2), i32(2), f32(2), f32(2, 3), 8),
    "sample_block": lambda: (f32(2, 3, 50), f32(2), f32(2, 3)),
    "accept_tree": lambda: (f32(2, 3, 50), i32(2, 3), i32(2, 3)),
    "build_tree": lambda: (f32(2, 3, 50), f32(2), i32(2), 2, 5),
    "lm_head_stats": lambda: (bf16(6, 64), bf16(256, 64), f32(2), 3),
    "map_slots": lambda: (i32(2), i32(2), i32(2, 3), 16, 7, i32(7), i32(1), 6),
    "adjust_logits": lambda: (f32(2, 3, 50),),
    "noise_tokens": lambda: (0, 5, 50),
    "philox_uniforms": lambda: (0, 5),
}


@pytest.mark.parametrize("name", sorted(EARLIER))
def test_the_other_calls_too(watched, name):
    caller, other, made, launched = watched
    given = EARLIER[name]()
    made.clear()
    launched.clear()
    getattr(b, name)(*given, stream=other)
    assert launched and made and all(s is other for _, s in made)


def test_every_call_that_allocates_is_covered():
    import inspect
    with_stream = {n for n, f in inspect.getmembers(b, inspect.isfunction)
                   if f.__module__ == b.__name__ and "stream" in inspect.signature(f).parameters
                   and not n.startswith("_") and not n.endswith("_args")}
    made_nothing = {"accept_block_noalloc", "append_kv_fp8", "commit_kv", "commit_tree_kv", "copy_pages", "read_device_status"}
    assert with_stream - made_nothing == set(EARLIER) | {"rope_kv", "chunk_attention", "fork_sequences"}
