"""CPU: the definition of 8-bit caches that the GPU tests go by (tests/kv8_ref.py),
against torch's 8-bit floats and against itself."""
import math

import pytest
import torch

import kv8_ref as ref


def test_what_codes_stand_for():
    c = torch.arange(256, dtype=torch.uint8)
    want = c.view(torch.float8_e4m3fn).double()
    assert torch.equal(torch.nan_to_num(ref.VALUES[ref.E4M3], 1e9), torch.nan_to_num(want, 1e9))
    assert torch.equal(ref.VALUES[ref.I8], c.view(torch.int8).double())


@pytest.mark.parametrize("codes", [ref.E4M3, ref.I8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_codes_are_the_nearest(codes, dtype):
    g = torch.Generator().manual_seed(1)
    x = (torch.randn(300, 2, 48, generator=g) * torch.exp(2 * torch.randn(300, 2, 1, generator=g))).to(dtype)
    c, b = ref.coded(x, codes)
    v = ref.valued(c, b, codes)
    scale = 2.0 ** (b.double() - 127)
    most = ref.MOST[codes]
    top = x.double().abs().amax(-1)
    assert (top <= most * scale).all() and (top > most * scale / 2).all()  # the least power of two
    # A code stands for what is off by half of its last digit at most.
    step = scale if codes == ref.I8 else scale * 2.0 ** (torch.floor(torch.log2((x.double().abs() / scale[..., None])
                                                                              .clamp_min(2.0 ** -6))) - 3).amax(-1)
    off = (v - x.double()).abs()
    assert (off <= (step / 2)[..., None]).all()
    if codes == ref.E4M3:
        want = (x.double() / scale[..., None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
        assert torch.equal(c, want)
    # What is exact stays.
    assert torch.equal(ref.valued(*ref.coded(v, codes), codes), v)


def test_heads_at_the_borders():
    for codes, most in ((ref.E4M3, 448.0), (ref.I8, 127.0)):
        for e in (-126, -20, 0, 100):
            assert ref.scale_byte(most * 2.0 ** e, codes) == e + 127
            assert ref.scale_byte(math.nextafter(most * 2.0 ** e, math.inf), codes) == e + 128
        assert ref.scale_byte(0.0, codes) == 1
        assert ref.scale_byte(math.inf, codes) == ref.scale_byte(math.nan, codes) == 255
        x = torch.zeros(1, 1, 16)
        c, b = ref.coded(x, codes)
        assert (c == 0).all() and int(b) == 1
        x[0, 0, 3] = math.inf
        c, b = ref.coded(x, codes)
        assert (c == 0).all() and int(b) == 255 and torch.isnan(ref.valued(c, b, codes)).all()


def test_what_nodes_see():
    p = ref.trees(None, 3, [20, 9], [5, 4], 2, 1, 64, sinks=2)
    p.parents = [-1, 0, 0, 2, -1] + [-1, 0, 1, 2]
    see = [sorted(j for j, *_ in p.seen(0, 15 + i, 0)) for i in range(5)]
    ctx = list(range(15))
    assert see == [ctx + [15], ctx + [15, 16], ctx + [15, 17], ctx + [15, 17, 18], ctx + [19]]
    # A window of 2: positions 15, 16, 16, 17, 15 and the sinks.
    see = [sorted(j for j, *_ in p.seen(0, 15 + i, 2)) for i in range(5)]
    assert see == [[0, 1, 14, 15], [0, 1, 15, 16], [0, 1, 15, 17], [0, 1, 17, 18], [0, 1, 14, 19]]
    assert [sorted(j for j, *_ in p.seen(1, 5 + i, 3)) for i in range(4)] == \
        [[0, 1, 3, 4, 5], [0, 1, 4, 5, 6], [0, 1, 5, 6, 7], [0, 1, 6, 7, 8]]
