"""Tables of more requests than 64 KB of prefix sums hold, up to the most that a call takes, against the loop over requests."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

pytest.importorskip("torch")

from test_gpu_kv_tables import run  # noqa: E402


@pytest.mark.parametrize("B", [7679, 7680, 8193, 16384])
def test_many_requests(B):
    print(f"case tables B={B}", flush=True)
    rng = np.random.default_rng(B)
    kv_len = rng.integers(0, 60, B).tolist()
    n_new = (rng.integers(0, 5, B) * (rng.random(B) < 0.6)).tolist()
    need = sum(-(-(a + n) // 16) - -(-a // 16) for a, n in zip(kv_len, n_new))
    run(kv_len, n_new, 16, 5, sum(n_new) + 3, need - 7, B)
