"""The first use of the worker's operators from two threads at once."""
import threading

import paper_2010_05888_amd as gf
from paper_2010_05888_amd import worker


def test_a_second_thread_sees_a_whole_table_or_makes_its_own(monkeypatch):
    """One thread is held after the first function that it looks up; another then asks for
    the last one."""
    lib, last = gf.load(), list(worker._SIGNATURES)[-1]
    got = []

    def second():
        try:
            got.append(worker._functions()[last])
        except BaseException as e:  # handed to the test's own thread
            got.append(e)

    class Held:
        looked_up = 0

        def __getattr__(self, name):
            Held.looked_up += 1
            if Held.looked_up == 2:
                other = threading.Thread(target=second)
                other.start()
                other.join()
            return getattr(lib, name)

    monkeypatch.setattr(worker, "_fn", {})
    monkeypatch.setattr(worker, "load", Held)
    table = worker._functions()
    assert len(got) == 1 and not isinstance(got[0], BaseException), got
    assert got[0].argtypes == worker._SIGNATURES[last][1]
    assert set(table) == set(worker._SIGNATURES) == set(worker._functions())
