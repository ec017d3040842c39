"""A training step exchanges tables in the handle while it issues its launches (apply_work in csrc/train.cu).  What another thread may
issue meanwhile must not read those fields: the gated feed-forward block reads RowTables instead, which nothing writes after the
load.  Checked in the source, since the moment of an exchange cannot be hit on purpose."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_09261_b200", "csrc")
FILES = sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "gated_ff*")) + [os.path.join(CSRC, f) for f in ("dropout.cu", "blocknorm.cu")])


def _read(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def _exchanged():
    body = re.search(r"void apply_work\(.*?\n}\n", _read("train.cu"), re.S).group(0)
    return set(re.findall(r"\bh->(\w+)\s*=", body))


def test_the_exchanged_fields_are_found():
    assert {"tile_row0", "tile_rows", "pair_row0", "pair_rows", "n_tiles", "n_pairs", "wg_begin", "wg_mcount", "n_wg_chunks"} <= _exchanged()


@pytest.mark.parametrize("name", FILES)
def test_operators_read_no_field_that_a_step_exchanges(name):
    read = set(re.findall(r"\bh->(\w+)", _read(name)))
    assert not read & _exchanged(), read & _exchanged()


def test_the_fixed_tables_are_written_by_the_load_alone():
    for f in glob.glob(os.path.join(CSRC, "*.cu*")):
        name = os.path.basename(f)
        assert name == "partition.cu" or not re.search(r"all_rows(\.\w+)?\s*=[^=]|RowTables\s*&|&\s*\w+->all_rows", _read(name)), name
