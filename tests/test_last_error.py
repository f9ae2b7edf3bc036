"""msd_last_error(NULL) from several threads (no GPU): a failure without a context can be
read on any thread, but for those of the msd_mx_* calls, which are the calling thread's."""
import os
import threading

import pytest

from paper_2505_14260_amd import msd

if not os.path.exists(msd.LIB_PATH):
    pytest.skip("libmsd.so not built", allow_module_level=True)

HEADS = msd.ModelDesc(2, 128, 4, 3, 64, 256, 512, 1e4, 1e-5)    # 4 heads over 3
VOCAB = msd.ModelDesc(2, 128, 4, 2, 64, 256, 300000, 1e4, 1e-5)   # past 262,144 tokens
LIMITS = msd.Limits(1, 256, 16, 64)


def on_a_thread(f):
    out = []
    t = threading.Thread(target=lambda: out.append(f()))
    t.start()
    t.join(60)
    assert out
    return out[0]


def fails(desc):
    """A failure without a context; its message as the calling thread reads it."""
    with pytest.raises(msd.MSDError):
        msd.msd_buffer_sizes(desc, LIMITS)
    return msd.msd_last_error(None)


def mx_fails(rows):
    with pytest.raises(msd.MSDError):
        msd.msd_mx_bytes(msd.Mx(None, None, rows, 64, 0, 1))
    return msd.msd_last_error(None)


def test_a_failure_is_read_on_another_thread():
    heads, vocab = on_a_thread(lambda: fails(HEADS)), None
    assert heads and on_a_thread(lambda: msd.msd_last_error(None)) == heads

    def after_one_of_its_own():
        nonlocal vocab
        own = fails(HEADS)
        vocab = on_a_thread(lambda: fails(VOCAB))
        return own, msd.msd_last_error(None)
    own, latest = on_a_thread(after_one_of_its_own)
    assert own == heads and latest == vocab != heads


def test_failures_of_operators_are_the_threads_own():
    def work():
        mine = mx_fails(-1)
        # what other threads do does not change it
        others = on_a_thread(lambda: fails(HEADS)), on_a_thread(lambda: (mx_fails(-1), fails(VOCAB)))
        still = msd.msd_last_error(None)
        # a later failure of this thread's that is no operator's does
        return mine, others, still, fails(VOCAB), msd.msd_last_error(None)
    mine, others, still, own, latest = on_a_thread(work)
    assert mine and still == mine and mine not in others
    assert own == latest != mine
    # nor does an operator's failure reach another thread
    heads = on_a_thread(lambda: fails(HEADS))
    on_a_thread(lambda: mx_fails(-1))
    assert on_a_thread(lambda: msd.msd_last_error(None)) == heads


def test_many_threads_at_once():
    """Each reads its own operator's message, and a whole one of the others'."""
    texts = {fails(HEADS), fails(VOCAB)}
    mine, wrong = on_a_thread(lambda: mx_fails(-1)), []

    def work(i):
        for _ in range(300):
            if i % 2:
                if mx_fails(-1) != mine:
                    wrong.append(i)
            elif fails(HEADS if i % 4 else VOCAB) not in texts:
                wrong.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not wrong and not any(t.is_alive() for t in threads)
