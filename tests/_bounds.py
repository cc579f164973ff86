"""Element-by-element comparison within a bound, with a short report."""
import numpy as np


def assert_within(got, ref, tol, what=""):
    err = np.abs(np.asarray(got, np.float64) - ref)
    tol = np.broadcast_to(tol, err.shape)
    bad = ~(err <= tol)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, err / np.maximum(tol, 1e-300), -1)), err.shape)
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} outside; worst at {at}: got {np.asarray(got)[at]!r}, "
                             f"ref {np.broadcast_to(ref, err.shape)[at]!r}, off {err[at]:.3e}, bound {tol[at]:.3e}")
