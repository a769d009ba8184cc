"""CPU tests of what the binding refuses before a call reaches the library."""
import types

import pytest

import paper_2410_03065_amd as cake


def engine_on(device, model=(2, 8, 128)):
    eng = cake.Engine.__new__(cake.Engine)
    eng._dev_index, eng._q8_model = device, (*model, device)
    return eng


def described_by(eng):
    batch = cake.Q8Batch()
    batch.model = eng._q8_model
    return batch


def test_a_batch_on_another_device_is_refused():
    batch = described_by(engine_on(0))
    assert engine_on(0)._batch(batch) is batch
    with pytest.raises(cake.CakeError) as e:
        engine_on(1)._batch(batch)
    assert e.value.code == cake.E_INVAL
    with pytest.raises(cake.CakeError):
        engine_on(0, (2, 4, 128))._batch(batch)


@pytest.mark.parametrize("device,priority", [(1, 0), (0, -1)])
def test_a_compute_stream_of_another_device_or_priority_is_refused(device, priority):
    eng = engine_on(0)
    eng.dev = "cuda:0"
    stream = types.SimpleNamespace(device=types.SimpleNamespace(index=device), priority=priority, cuda_stream=0)
    with pytest.raises(cake.CakeError) as e:
        eng._take_streams(stream)
    assert e.value.code == cake.E_INVAL
