"""The serving example says so when a call could not serve a sequence."""

import pytest

from test_gpu_serve_prompts import example

pytestmark = pytest.mark.gpu


def server(**kw):
    return example().Server(**dict(dict(batch=3, page_size=16, max_pages=8), **kw))


@pytest.mark.parametrize("eight_bit", [False, True])
def test_no_pages_left(eight_bit):
    s = server(num_pages=3, eight_bit=eight_bit)
    s.submit({0: list(range(30)), 1: list(range(40))})
    with pytest.raises(RuntimeError, match=r"no pages for new tokens: sequences \[1\]"):
        s.step()


def test_a_refused_fork():
    s = server(num_pages=3)
    s.submit({0: list(range(20))})
    s.step()
    with pytest.raises(RuntimeError, match=r"not forked: sequences \[2\]"):
        s.fork([0, 0, 0])


@pytest.mark.parametrize("eight_bit", [False, True])
def test_a_bad_page_in_the_attention(eight_bit):
    s = server(eight_bit=eight_bit)
    s.submit({0: list(range(20)), 1: list(range(3))})
    s.step()
    s.table[0, 0] = 10 ** 6
    s.submit({0: [1], 1: [2]})
    with pytest.raises(RuntimeError, match="attention: status 5, flags 4"):
        s.step()
    s.table[0, 0] = 1
    s.submit({0: [1], 1: [2]})
    assert s.step()[1] is not None


def test_one_workspace_for_all_steps():
    s = server()
    s.submit({0: list(range(90))})
    s.step(budget=60)
    ws = s.attn_ws
    s.step(budget=60)
    s.submit({0: [1], 1: [2]})
    s.step()
    assert s.attn_ws is ws
