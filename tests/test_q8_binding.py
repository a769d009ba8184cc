"""CPU tests of what the binding refuses before a call reaches the library."""
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
