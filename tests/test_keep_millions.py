"""The choice of the tokens that stay from millions of them: against a plain sort, in place and not, and how its time grows where so many
weights are alike that they go through memory for every digit."""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _say(msg):
    print(f"[gpu-case] {msg}", flush=True)
    sys.stdout.flush()


def _ints(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device=DEV)


def _stays(w, n, m, sink, recent):
    """Positions of one head's weights, NaN-free: the first, the last, of the rest the largest, ties lowest."""
    recent = min(recent, m)
    sink = min(sink, m - recent)
    between = np.arange(sink, n - recent)
    best = between[np.lexsort((between, -w[between]))[:m - sink - recent]]
    return np.sort(np.concatenate([np.arange(sink), best, np.arange(n - recent, n)]))


KINDS = {
    "spread": lambda rng, shape: np.exp(3 * rng.standard_normal(shape)),
    "equal": lambda rng, shape: np.full(shape, 0.25),
    "close": lambda rng, shape: (np.int32(0x3f000000) + rng.integers(0, 1 << 20, shape).astype(np.int32)).view(np.float32),
    "few": lambda rng, shape: rng.integers(0, 3, shape),
}


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [(1 << 20) - 1, 1 << 20, (1 << 20) + 1, 2500000])
def test_keep_of_millions(n, kind):
    from paper_2609_01925_amd import crisp as C
    _say(f"keep n={n} {kind}")
    rng = np.random.default_rng(n)
    width, lens, keep = n + 70, [n, 30000, 700], [n // 3, 29000, 100]
    w = KINDS[kind](rng, (3, 2, width)).astype(np.float32)
    cap, held = n // 3, [n - 9001, 30000, 10]
    out = torch.full(w.shape, 7.0, device=DEV)
    dev = torch.from_numpy(w).to(DEV)
    kept, count = C.crisp_cache_keep(dev, _ints(held), _ints(lens), _ints(keep), cap, 3, 100, out)
    again, _ = C.crisp_cache_keep(dev, _ints(held), _ints(lens), _ints(keep), cap, 3, 100, dev)
    assert torch.equal(kept, again) and count.tolist() == keep
    kept, out, dev = kept.cpu().numpy(), out.cpu().numpy(), dev.cpu().numpy()
    for s, m in enumerate(keep):
        for h in range(2):
            counted = np.where(np.arange(lens[s]) < held[s], w[s, h, :lens[s]], np.float32(0))
            want = _stays(counted, lens[s], m, 3, 100)
            assert (kept[s, h, :m] == want).all() and (kept[s, h, m:] == -1).all()
            assert (out[s, h, :m] == counted[want]).all() and (out[s, h, m:] == 7.0).all()
            assert (dev[s, h, :m] == counted[want]).all() and (dev[s, h, m:] == w[s, h, m:]).all()


def test_keep_time_of_equal_weights_grows_with_the_tokens():
    """Eight times the tokens, all of one weight, take no more than thirty times as long: eight times, and what the smaller call leaves idle, not
    the square's 64."""
    from paper_2609_01925_amd import crisp as C
    times = []
    for n in (1 << 20, 1 << 23):
        _say(f"keep n={n}, time of equal weights")
        w = torch.zeros(1, 4, n, device=DEV)
        ws, args = C.cache_keep_workspace(w), (w, _ints([n]), _ints([n]), _ints([1 << 19]), 1 << 19)
        best = float("inf")
        for _ in range(4):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            C.crisp_cache_keep(*args, ws=ws)
            end.record()
            end.synchronize()
            best = min(best, begin.elapsed_time(end))
        times.append(best)
    print(f"[gpu-case] {times[0]:.3f} ms of 2^20 tokens, {times[1]:.3f} ms of 2^23", flush=True)
    assert times[1] <= 30 * times[0], times
