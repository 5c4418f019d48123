"""Work memory that the binding does not hold on to, without a GPU (the stand-ins of test_binding_host.py)."""
import paper_2607_05272_amd.sim as binding
from test_binding_host import world   # noqa: F401


def test_large_work_memory_is_given_back_after_its_call(world):   # noqa: F811
    kept = world.call()
    small = world.sim._work.memory
    world.need = binding._KEEP + 1
    c = world.call()
    assert c.bytes == world.need and c.at != kept.at and any(c.held)      # there while the call is made
    assert world.made[-1]() is None                                       # and no longer
    assert world.sim._work.memory is small
    world.need = 64
    assert world.call().at == kept.at


def test_a_thread_holds_no_more_than_the_largest_that_is_kept(world):   # noqa: F811
    for need in (64, binding._KEEP, 1 << 16, 8 * binding._KEEP, 64):
        world.need = need
        assert any(world.call().held)
    assert sum(t().numel() for t in world.made if t() is not None) == binding._KEEP


def test_the_first_call_may_be_a_large_one(world):   # noqa: F811
    world.need = binding._KEEP + 1
    assert any(world.call().held) and getattr(world.sim._work, "memory", None) is None
