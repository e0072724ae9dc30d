"""hydra.Rope on the host: what it keeps of its arguments."""
import numpy as np

from paper_2609_34318_amd import hydra


def test_given_frequencies_are_copied():
    """A program that writes the next layer's frequencies into the same array changes no Rope made before."""
    f = np.linspace(1.0, 0.1, 32)
    r = hydra.Rope(inv_freq=f)
    want = f.copy()
    f[:] = 7.0
    assert np.array_equal(r.inv_freq, want) and [r.c.inv_freq[j] for j in range(32)] == list(want)
    back = hydra.Rope(inv_freq=want[::-1])
    assert [back.c.inv_freq[j] for j in range(32)] == list(want[::-1])
