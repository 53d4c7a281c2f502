"""fq_sample with numbers of 1 and more, which name the last entry with any weight, under each setting by itself."""
import numpy as np
import pytest

from test_gpu_sample import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("V", [1, 300, 2000, 32000, 128256])
@pytest.mark.parametrize("setting", [{}, {"temperature": 0.6}, {"temperature": 7.0}, {"top_p": 0.9}, {"top_p": 0.999}, {"min_p": 0.02},
                                     {"min_p": 1e-9}, {"top_k": 40}, {"top_k": 1500}, {"top_p": 0.95, "min_p": 0.01}])
def test_numbers_of_one_and_more(setting, V, half):
    rng = np.random.default_rng(V + len(setting))
    u = np.array([1.0, 5.0, 3e38, 1.0 - 2.0 ** -24], dtype=np.float32)
    for spread in (3.0, 0.3):
        x = rng.normal(0, spread, (4, V))
        x[:, -1] = -80.0  # weighs less than any unit, but for the hot temperature
        x[:, 0] = -20.0   # a few units
        run(x, u, half=half, **{k: [v] * 4 for k, v in setting.items()})
