"""Host side of lessdec_state_select: what is refused before anything is launched.  No GPU."""
import ctypes as C

from paper_2402_09398_amd import binding

A = 0x10000                                                   # stands for a device pointer: no call below gets as far as reading it
STATE = ("k_cache", "v_cache", "acc", "pos", "psi", "H", "z", "n_seen", "pend_slot", "pend_v", "pend_psi")


def desc(**more):
    d = binding.Desc()
    d.batch, d.heads, d.head_dim, d.n_heavy, d.n_recent, d.rank, d.hidden, d.dtype = 4, 2, 64, 3, 4, 5, 64, binding.DTYPE_F16
    for name in STATE:
        setattr(d, name, A)
    for k, v in more.items():
        setattr(d, k, v)
    return d


def test_what_is_refused():
    call = binding.lib().lessdec_state_select
    assert call(None, A, None) == binding.EINVAL
    for more in ([dict(batch=0), dict(batch=4097), dict(heads=0), dict(head_dim=96), dict(n_heavy=-1), dict(n_heavy=0, n_recent=0), dict(rank=0),
                  dict(rank=65), dict(dtype=binding.DTYPE_BF16), dict(flags=64), dict(k_cache=A + 8), dict(acc=A + 4), dict(pos=A + 2)] +
                 [{name: None} for name in STATE]):
        assert call(C.byref(desc(**more)), A, None) == binding.EINVAL, more
    for source in (None, A + 2):
        assert call(C.byref(desc()), source, None) == binding.EINVAL
