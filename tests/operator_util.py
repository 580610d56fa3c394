"""Helpers of the tests of the layers and losses: buffers with guards, and element-by-element comparison."""
import numpy as np

GUARD = 64  # elements on both sides of a guarded tensor


def guarded(shape, dtype, shift=0, fill=-7.0):
    """A tensor of `shape` inside a larger buffer, `shift` elements off 16 bytes, and a check that the rest is untouched."""
    import torch
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * GUARD + shift,), fill, dtype=dtype, device="cuda:0")
    a = GUARD + shift

    def check():
        rest = torch.cat([buf[:a], buf[a + n:]])
        assert bool((rest == fill).all()), "written outside the tensor"
    return buf[a:a + n].view(shape), check


def put(a, dtype, shift=0):
    """The values of a numpy array on the GPU, `shift` elements off 16 bytes."""
    import torch
    a = np.asarray(a)
    t = torch.empty(a.size + shift, dtype=dtype, device="cuda:0")
    t[shift:].copy_(torch.from_numpy(np.ascontiguousarray(a)).reshape(-1).to(dtype))
    return t[shift:].view(a.shape)


def rounded(a, bf16):
    """The nearest values of the type, in 64 bits."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.float32)))
    return (t.to(torch.bfloat16) if bf16 else t).to(torch.float64).numpy()


def values(t):
    import torch
    return t.detach().to(torch.float64).cpu().numpy()


def close(name, got, want, tol):
    got, want, tol = np.asarray(got), np.asarray(want), np.broadcast_to(tol, np.shape(want))
    assert got.shape == want.shape, (name, got.shape, want.shape)
    if not got.size:
        return
    assert np.all(np.isfinite(got)), f"{name}: {np.sum(~np.isfinite(got))} values are not finite"
    over = np.abs(got - want) - tol
    i = np.unravel_index(np.argmax(over), over.shape)
    assert over[i] <= 0, f"{name}: at {i} got {got[i]:.9g}, want {want[i]:.9g}, off by {abs(got[i] - want[i]):.3g}, may {tol[i]:.3g}"
