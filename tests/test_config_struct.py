"""A Config's C form is made once, belongs to that config alone, and changes nothing of
what a Config is."""
import copy
import dataclasses
import pickle

import torch

import paper_2503_10571_amd as radar


def _values(c):
    return [getattr(c, name) for name, _ in c._fields_]


def test_made_once_for_each_config():
    cfg = radar.Config(3, 8, 2, 64, 128, 16, 32, 4096, torch.float32, 5)
    names = [f.name for f in dataclasses.fields(cfg)]
    before, text = hash(cfg), repr(cfg)
    assert "_c" not in names and "_c" not in cfg.__dict__
    made = cfg._c
    assert cfg._c is made and _values(made) == _values(cfg.c_struct())
    assert (hash(cfg), repr(cfg), [f.name for f in dataclasses.fields(cfg)]) == (before, text, names)
    assert "_c" not in dataclasses.asdict(cfg)
    longer = dataclasses.replace(cfg, capacity=8192)
    assert longer._c.capacity == 8192 and cfg._c.capacity == 4096
    for same in (copy.copy(cfg), copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg))):
        assert same == cfg and hash(same) == before and _values(same._c) == _values(made)
