"""Element types that the attention calls' Python binding takes, on the host."""
import pytest

import paper_2601_20595_amd as csg

torch = pytest.importorskip("torch")


def test_a_tensor_of_another_type_is_refused():
    x = torch.zeros((4, 8, 128), dtype=torch.float16)
    p = torch.zeros(2, dtype=torch.int32)
    for dtype, other in (("bf16", torch.float16), ("f16", torch.bfloat16)):
        a = csg.DocAttn(8, 8, 128, dtype)
        c = csg.PagedCache(8, 8, 128, dtype, 4, 16, 1, 4)
        y = x.to(other)
        name = {"bf16": "bfloat16", "f16": "float16"}[dtype]
        with pytest.raises(ValueError, match="q must be %s" % name):
            a.forward(y, y, y, p, p, y, y)
        with pytest.raises(ValueError, match="k must be %s" % name):
            c.append(y, y, y, y, p, p, p[None])
        with pytest.raises(ValueError, match="q must be %s" % name):
            c.attn(y, y, y, p, p, p[None], y, None, p)


def test_bit_patterns_are_taken():
    # (what is refused then is the place: the host)
    for dtype in ("bf16", "f16"):
        with pytest.raises(ValueError, match="GPU"):
            x = torch.zeros((4, 8, 128), dtype=torch.int16)
            csg.DocAttn(8, 8, 128, dtype).forward(x, x, x, None, None, x, x)


@pytest.mark.parametrize("kind, good, bad", [("_INT32", torch.int32, torch.float32), ("_FLOAT32", torch.float32, torch.int32),
                                             ("_FLOAT64", torch.float64, torch.int64)])
def test_arrays_of_another_type_are_refused(kind, good, bad):
    for _ in range(2):  # also once the good one is known
        with pytest.raises(ValueError, match="GPU"):
            csg._arg(torch.zeros(3, dtype=good), 12, getattr(csg, kind), "x", 0)
        with pytest.raises(ValueError, match="x must be %s" % str(good).split(".")[1]):
            csg._arg(torch.zeros(3, dtype=bad), 12, getattr(csg, kind), "x", 0)
        with pytest.raises(ValueError, match="-byte elements"):
            csg._arg(torch.zeros(3, dtype=torch.int8), 12, getattr(csg, kind), "x", 0)
