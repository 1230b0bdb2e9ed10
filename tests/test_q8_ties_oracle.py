"""The 8-bit oracle at ties: half of a row's largest value is one whatever that is."""
import numpy as np

from oracle import q8_oracle as orc


def test_half_of_the_largest_goes_to_the_even_step():
    rng = np.random.default_rng(1)
    for top in (np.arange(128.0, 256.0), (1 + rng.random(2000)).astype(np.float32).astype(np.float64)):
        for scale in (1.0, 2.0 ** -90, 2.0 ** 60):
            t = top * scale
            q, _ = orc.rows8(np.stack([t, t / 2, -t / 2], 1))
            assert (q == [127, 64, -64]).all()
