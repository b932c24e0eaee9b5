"""Caps that hardly bend the scores: what remains of small scores, elementwise against fp64."""
import pytest

torch = pytest.importorskip("torch")
if torch.cuda.is_available():
    import test_gpu_cache
    from test_gpu_doc_attn import _run

pytestmark = pytest.mark.gpu

CAPS = [64.0, 65.0, 1e3, 1e6, 1e30]


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_documents(cap, dtype):
    _run(([100, 40], [150, 40], 4, 2, 128, True, [20, 0], cap, True), dtype)
    _run(([300], [300], 2, 2, 64, True, None, cap, False), dtype, sharp=4.0)


def test_scores_of_the_size_of_the_cap():
    _run(([150], [200], 4, 2, 128, True, None, 100.0, False), "bf16", sharp=60.0)
    _run(([150], [200], 4, 2, 64, True, None, 300.0, True), "f16", sharp=100.0)


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_cache(cap, dtype, monkeypatch):
    monkeypatch.setitem(test_gpu_cache.ATTN, "large cap", ([1, 4, 40], [333, 70, 200], 8, 2, 128, 32, [], cap, False))
    test_gpu_cache._attn_case("large cap", dtype)
