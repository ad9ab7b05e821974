"""The token mixing binding's first use from several threads: what it looks up once is
there whole or not at all."""
import torch

import paper_2308_15152_amd as pkg
from paper_2308_15152_amd import mixing


def test_nothing_is_seen_half_filled(monkeypatch):
    lib = pkg.load()
    seen = []

    class Library:
        """The library, which lets another thread look between two lookups."""

        def __getattr__(self, name):
            seen.append((len(mixing._calls), len(mixing._dtypes)))
            return getattr(lib, name)

    monkeypatch.setattr(mixing, "_calls", {})
    monkeypatch.setattr(pkg, "load", Library)
    mixing._start()
    assert len(seen) == len(mixing._calls) == 6
    assert all(calls == 0 and types == 3 for calls, types in seen)
    q = torch.zeros(1, 20, 2, 16)
    g = torch.zeros(1, 20, 2)
    assert pkg.delta_emu_forward_workspace(q, q, q, g, g) > 0
