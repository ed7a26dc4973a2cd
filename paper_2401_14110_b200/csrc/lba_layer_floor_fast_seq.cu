#define LBA_PROBLEM LinearProblem
#define LBA_QM lba::QM_FLOOR_FAST
#define LBA_ORD lba::ORD_SEQ
#include "lba_family.inc"
