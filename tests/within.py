"""Element by element comparison against fp64: half a step of the stored type around the exact value, and a slack for what the
fp32 arithmetic before the rounding may be off by, which the caller derives."""
import numpy as np

U = 2.0 ** -24      # half a step of fp32 relative to the value


def host64(x):
    import torch
    return x.detach().to(torch.float64).cpu().numpy()


def dev(a, dtype):
    """A device tensor of `dtype` ("f32" or "bf16") and its values in fp64."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    return t.cuda(), t.to(torch.float64).numpy()


def assert_within(name, got, ref, slack):
    import torch
    half = torch.finfo(got.dtype).eps / 2
    x = host64(got)
    ref, slack = np.asarray(ref, np.float64), np.broadcast_to(np.asarray(slack, np.float64), x.shape)
    assert x.shape == ref.shape, (name, x.shape, ref.shape)
    bound = half * (np.abs(ref) + slack) + slack + 1e-40     # below fp32's normal numbers steps are absolute
    off = np.abs(x - ref)
    bad = ~(off <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off / np.maximum(bound, 1e-300))), x.shape)
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} outside, worst at {i}: {x[i]!r} for {ref[i]!r}, bound {bound[i]!r}")


def guarded(shape, dtype, fill=-77.0, extra=3):
    """A buffer with `extra` rows more than `shape` has, and a view of the first ones: what is behind has to stay."""
    import torch
    whole = torch.full((shape[0] + extra, *shape[1:]), fill, dtype=dtype, device="cuda")
    return whole, whole[:shape[0]]


def assert_guard(whole, rows, fill=-77.0):
    assert bool((whole[rows:] == fill).all())
