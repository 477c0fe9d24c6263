"""CPU test of the norm of rows without columns: nothing to write but the statistics, which do not exist.  In a process of its own, on fake device
tensors (no GPU is used)."""
from tests.test_native_binding import run


def test_statistics():
    """Refused where they would be returned, never having been written, or left as they were; with them not wanted, Y is as empty as X."""
    out = run("""
with FakeTensorMode():
    x, v, w = new(5, 0), new(5, dtype=f32), new(0)
    for f in (lambda: binding.halo_layer_norm_fwd(x), lambda: binding.halo_layer_norm_fwd(x, w, kind="rms"),
              lambda: binding.halo_layer_norm_fwd(x, want_stats=False, mean=v), lambda: binding.halo_layer_norm_fwd(x, want_stats=False, rstd=v)):
        try:
            f()
            print("went through")
        except AssertionError as e:
            print("rows without columns" in str(e))
        except Exception as e:
            print("got as far as", type(e).__name__)
""")
    assert out.splitlines() == ["True"] * 4
