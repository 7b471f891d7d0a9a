"""GPU: the cases of test_gpu_attend_extremes.py through the chunk kernel (RS_ATTEND_FEW=0), on whole and on split key ranges."""
import pytest

import test_gpu_attend_extremes as E

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def chunk_kernel(monkeypatch):
    monkeypatch.setenv("RS_ATTEND_FEW", "0")


@pytest.mark.parametrize("kind", ["contiguous", "paged", "fp8"])
@pytest.mark.parametrize("held, rows", [(130, 130), (3000, 70), (1700, 33)])
def test_large_queries_and_keys(kind, held, rows):
    E.longer_requests(kind, held, rows)


@pytest.mark.parametrize("held, rows", [(100, 100), (400, 100), (3000, 70)])
@pytest.mark.parametrize("scale", E.SCALES)
def test_scales_of_the_callers(held, rows, scale):
    E.scaled(held, rows, scale)
