// Class log probabilities of short rows, fp16 (a file a type: they compile side by side).
#define LOGPROB_ROWS_TYPE 2
#include "logprob_rows.cuh"
