"""Clipping into another list: an output that lies on a tensor another CTA has yet to read is refused before anything is enqueued,
in place and side by side are not."""
import random

import pytest
import torch

import paper_1905_04035_b200 as dst
from paper_1905_04035_b200 import binding
from paper_1905_04035_b200.build import build_library

AT = 0x100000             # never dereferenced
F32, BF16 = 0, 1


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return dst.load_library()


def tensors(items):
    a = (binding._Tensor * max(1, len(items)))()
    for c, (at, n, t) in zip(a, items):
        c.data, c.n, c.type = at, n, t
    return a


def refused(lib, ins, outs):
    """Whether the call is refused for the places of its tensors.  The last tensor is longer than any that is taken, so that no call
    gets as far as the device."""
    long = (AT << 20, (1 << 44) + 1, BF16)
    rc = lib.dst_clip(tensors(ins + [long]), tensors(outs + [long]), len(ins) + 1, AT - 256, None)
    assert rc in (1, 2)
    return rc == 1


def test_outputs_on_other_tensors_and_on_one_another_are_refused(lib):
    a, b = (AT, 100, F32), (AT + 400, 100, F32)
    far = [(AT + 4000 * i, 100, F32) for i in range(1, 400)]
    for ins, outs in (([a, b], [b, a]),                                            # in another order
                      ([a], [(AT + 4, 100, F32)]), ([(AT + 4, 100, F32)], [a]),    # shifted, either way
                      ([a], [(AT + 396, 100, F32)]), ([a], [(AT - 396, 100, F32)]),
                      ([a], [(AT + 2, 100, BF16)]), ([(AT, 100, BF16)], [(AT - 200, 100, F32)]),
                      ([a, b], [a, a]), ([a, b], [(AT + 9000, 100, F32), (AT + 9100, 100, F32)]),
                      ([a, a], [a, a]), ([a, a], [a, (AT + 9000, 100, F32)]),      # twice, and in place once
                      (far, far[:-1] + [(far[0][0] + 4, 100, F32)]), (far[::-1] + [a], far[::-1] + [(far[5][0] - 4, 100, F32)]),
                      (far, far[1:] + far[:1])):
        assert refused(lib, ins, outs), (ins[:2], outs[:2])


def test_what_holds_nothing_shares_nothing(lib):
    a, none = (AT, 0, F32), (AT, 0, BF16)
    assert lib.dst_clip(tensors([a, none, (None, 0, F32)]), tensors([none, none, none]), 3, AT - 256, None) == 0


def test_the_rule_is_that_of_comparing_every_pair(lib):
    rng = random.Random(5)
    seen = [0, 0]
    for _ in range(4000):
        n, spread = rng.randint(0, 6), rng.choice([6, 30, 200])
        ins = [(AT + 4 * rng.randrange(spread), rng.choice([0, 1, 2, 3]), rng.choice([F32, BF16])) for _ in range(n)]
        outs = [i if rng.random() < 0.5 else (AT + 4 * rng.randrange(spread), i[1], rng.choice([F32, BF16])) for i in ins]
        span = lambda t: (t[0], t[0] + t[1] * (4 if t[2] == F32 else 2))  # noqa: E731
        meet = lambda p, q: p[1] and q[1] and span(p)[0] < span(q)[1] and span(q)[0] < span(p)[1]  # noqa: E731
        want = any(meet(outs[j], outs[k]) for j in range(n) for k in range(j)) or any(
            meet(ins[k], outs[j]) and not (j == k and ins[k] == outs[j]) for j in range(n) for k in range(n))
        assert refused(lib, ins, outs) == bool(want), (ins, outs)
        seen[bool(want)] += 1
    assert min(seen) > 300


@pytest.mark.gpu
def test_the_binding_refuses_lists_that_share_memory_and_takes_those_that_do_not():
    buf = torch.arange(4000.0, device="cuda")
    clip = torch.tensor([1.0, 0.5], device="cuda")
    a, b = buf[:1000], buf[1000:2000]
    kept = buf.clone()
    for ins, outs in (([a, b], [b, a]), ([a], [buf[1:1001]]), ([buf[1:1001]], [a]), ([a, b], [buf[2000:3000], buf[999:1999]]), ([a, a], [a, buf[3000:]])):
        with pytest.raises((ValueError, dst.DstError)):
            dst.dst_clip(dst.TensorList(ins), clip, dst.TensorList(outs))
    torch.cuda.synchronize()
    assert torch.equal(buf, kept)
    dst.dst_clip(dst.TensorList([a, b, a]), clip, dst.TensorList([buf[2000:3000], b, buf[3000:]]))    # one in place, one read twice
    assert torch.equal(buf[2000:3000], kept[:1000] * 0.5) and torch.equal(buf[3000:], kept[:1000] * 0.5)
    assert torch.equal(b, kept[1000:2000] * 0.5) and torch.equal(a, kept[:1000])
    half = torch.zeros(1000, dtype=torch.bfloat16, device="cuda")
    dst.dst_clip(dst.TensorList([a, a]), clip, dst.TensorList([half, buf[2000:3000]]))
    assert torch.equal(half, (kept[:1000] * 0.5).bfloat16())
