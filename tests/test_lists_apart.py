"""Lists of tensors for clipping and AdamW whose memory overlaps are refused (host code on addresses; nothing is launched)."""
import struct

import pytest

F32, BF16 = 0, 1


def a_list(*tensors):
    """(address, elements, type) each, None for no tensor: what tensor_list makes of tensors."""
    rows = [(0, -1, -1) if t is None else t for t in tensors]
    return tuple(struct.pack(f"{len(rows)}{kind}", *(r[i] for r in rows)) for i, kind in enumerate("qqi"))


def apart(written, read, in_place=False):
    from paper_2505_11432_amd import binding as B
    return B._native.lists_apart(written, read, in_place)


def test_ranges():
    a, b = (4096, 10, F32), (4136, 10, F32)                 # the second begins where the first ends
    assert apart([a_list(a, b)], [])
    assert not apart([a_list(a, (4132, 1, F32))], []) and not apart([a_list((4132, 1, F32), a)], [])
    assert apart([a_list((4096, 10, BF16), (4116, 3, BF16))], []) and not apart([a_list((4096, 10, BF16), (4114, 3, BF16))], [])
    assert apart([], [a_list(a, a, a)])                     # what is only read may come again
    assert not apart([a_list(a)], [a_list(b, (4100, 1, BF16))]) and apart([a_list(a)], [a_list(b, b)])
    assert not apart([a_list((5000, 4, F32))], [a_list((4000, 1000, F32))])        # inside a long one that begins earlier
    assert not apart([a_list((5000, 4, F32)), a_list((4000, 1000, F32))], [])
    assert not apart([a_list(a)], [a_list((4000, 2, F32)), a_list((4090, 5, BF16))])
    # no tensor, an empty one, no list
    assert apart([a_list(None, (4096, 0, F32), a, (0, 0, BF16))], [a_list((4100, 0, F32), None)]) and apart([], []) and apart([a_list()], [])


def test_in_place():
    a, b = (4096, 10, F32), (8192, 10, F32)
    assert apart([a_list(a, b)], [a_list(a, b)], True) and not apart([a_list(a, b)], [a_list(a, b)], False)
    assert not apart([a_list(a, b)], [a_list(b, a)], True)          # another's place
    assert not apart([a_list(a, a)], [a_list(a, a)], True)          # one gradient twice: scaled twice, or once
    assert not apart([a_list((4100, 10, F32))], [a_list(a)], True)  # shifted
    assert not apart([a_list(None, b)], [a_list(a, a, b)], True) and apart([a_list(None, b)], [a_list(a, b)], True)


def test_refused_calls():
    from paper_2505_11432_amd import binding as B
    for bad in (([], []), ([], [], True, 1), (None, [], True), ([], 3, True), ([b"x"], [], True), ([(b"", b"", 3)], [], True), ([(b"", b"")], [], True)):
        with pytest.raises(TypeError):
            B._native.lists_apart(*bad)
    with pytest.raises(ValueError, match="one length"):
        B._native.lists_apart([(b"12345678", b"", b"")], [], True)


@pytest.mark.gpu
def test_refused_lists():
    import torch

    from paper_2505_11432_amd.optim import AdamW, GradClip
    buf = torch.ones((64,), device="cuda:0")
    a, b, both = buf[:10], buf[10:20], buf[5:15]
    GradClip([a, b], 1.0, out=[a, b]).clip()
    GradClip([a, both, a], 1.0).clip()                       # the norm alone
    for grads, out in (([a, a], [a, a]), ([a, b], [b, a]), ([a, both], [a, both]), ([a], [both])):
        with pytest.raises(AssertionError, match="memory"):
            GradClip(grads, 1.0, out=out)
    p, g, m, v, w = buf[:10], buf[10:20], buf[20:30], buf[30:40], buf[40:45].view(torch.bfloat16)
    AdamW([p], [g], [m], [v], weights=[w]).step()
    for lists in (([p, p], [g, g], [m, b], [v, buf[50:60]]), ([p], [p], [m], [v]), ([p], [g], [m], [m]), ([p], [g], [m], [buf[25:35]])):
        with pytest.raises(AssertionError, match="memory"):
            AdamW(*lists)
    with pytest.raises(AssertionError, match="memory"):
        AdamW([p], [g], [m], [v], weights=[buf[35:40].view(torch.bfloat16)])
    # the other refusals, of tensors that lie apart
    p, g, m, v = (torch.zeros((8, 8), device="cuda:0") for _ in range(4))
    for bad in (lambda: AdamW([p], [g[:4]], [m], [v]), lambda: AdamW([p], [g], [m.to(torch.bfloat16)], [v]), lambda: AdamW([p], [g], [m], [v[:4]]),
                lambda: AdamW([p], [g], [m], [v], weights=[torch.zeros((8, 8), device="cuda:0")]), lambda: AdamW([p.t()[:, :4]], [g], [m], [v]),
                lambda: AdamW([p], [g], [m], [v], lr=torch.zeros((2,), device="cuda:0")),
                lambda: AdamW([p], [g], [m], [v], step=torch.zeros((1,), device="cuda:0")), lambda: AdamW([p], [g], [m], [v]).step(coef=g)):
        with pytest.raises(AssertionError):
            bad()
